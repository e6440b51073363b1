"""Columns of one buffer side by side: what a call reads in some and writes in others, as if they lay apart."""
import math

import pytest
import torch

from paper_2312_17530_amd import binding as b
from .test_gpu_training import BF16, F32, _head_case, _norm_case

pytestmark = pytest.mark.gpu


def _beside(x):
    """x and room of the same shape to its right, in one buffer."""
    both = torch.full((x.shape[0], 2 * x.shape[1]), math.nan, dtype=x.dtype, device="cuda")
    both[:, :x.shape[1]] = x
    return both[:, :x.shape[1]], both[:, x.shape[1]:]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(5, 64), (40, 301), (300, 1025), (3, 16400)])
def test_norm_beside_its_input(rows, cols, dtype):
    x, dy, gamma, beta = _norm_case(rows, cols, dtype, seed=cols)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    b.rsdgc_layer_norm(x, gamma, beta, 1e-5, y, mean, rstd)
    b.rsdgc_layer_norm_backward(dy, x, gamma, mean, rstd, dx, None, None, False, None)
    x2, y2 = _beside(x)
    b.rsdgc_layer_norm(x2, gamma, beta, 1e-5, y2)
    assert torch.equal(x2, x) and float((y2.float() - y.float()).abs().max()) <= 2.0 ** -7 * float(y.float().abs().max())
    dy2, dx2 = _beside(dy)
    b.rsdgc_layer_norm_backward(dy2, x, gamma, mean, rstd, dx2, None, None, False, None)
    assert torch.equal(dy2, dy) and float((dx2.float() - dx.float()).abs().max()) <= 2.0 ** -7 * float(dx.float().abs().max())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hidden", [64, 61])
@pytest.mark.parametrize("rows", [3, 40, 600])
def test_gradient_of_the_head_beside_its_input(rows, hidden, dtype):
    case = _head_case(rows, hidden, 200, dtype, seed=rows)
    size = b.rsdgc_head_workspace_bytes(dtype, rows, hidden, 200)
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    b.rsdgc_head_loss(case["x"], case["w"], case["target"], loss, lse, torch.empty(size, dtype=torch.uint8, device="cuda"))
    out = []
    x2, beside = _beside(case["x"])
    for x, dx in ((case["x"], torch.empty_like(case["x"])), (x2, beside), (x2.clone(memory_format=torch.contiguous_format), torch.empty_like(x2))):
        dw = torch.empty(200, hidden, device="cuda")
        b.rsdgc_head_loss_backward(x, case["w"], case["target"], lse, case["row_grad"], dx, dw, False, torch.empty(size, dtype=torch.uint8, device="cuda"))
        out.append((dx.clone(), dw))
    assert torch.equal(x2, case["x"])
    for dx, dw in out[1:]:
        # another alignment of x may take another form, whose roundings differ
        assert float((dx.double() - out[0][0].double()).norm()) <= (6e-3 if dtype == BF16 else 4e-5) * float(out[0][0].double().norm())
        assert float((dw.double() - out[0][1].double()).norm()) <= 4e-5 * float(out[0][1].double().norm())
