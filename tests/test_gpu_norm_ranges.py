"""Layer normalisation of more rows than one launch could take a workgroup each: a launch has less than 2^32 threads."""
import pytest
import torch

from paper_2312_17530_amd import binding as b

pytestmark = pytest.mark.gpu


def test_more_wide_rows_than_a_launch_has_workgroups():
    """Rows too wide for the registers, in place.  All but a few are the same, so that these and the few tell all."""
    rows, cols = (1 << 22) + 3, 16392
    need = rows * cols * 2
    if torch.cuda.mem_get_info()[0] + torch.cuda.memory_reserved() < need + (4 << 30):
        pytest.skip(f"{need >> 30} GiB of memory are needed")
    torch.cuda.empty_cache()
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    x.copy_(torch.randn(cols, generator=gen, device="cuda").bfloat16().expand(rows, cols))
    at = [0, 2047, 2048, 1 << 21, rows - 1]
    own = torch.randn(len(at), cols, generator=gen, device="cuda").bfloat16()
    x[at] = own
    row = x[1].double()
    want = torch.stack([row, *own.double()])
    want = (want - want.mean(1, keepdim=True)) / torch.sqrt(want.var(1, unbiased=False, keepdim=True) + 1e-5)
    mean, rstd = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    b.rsdgc_layer_norm(x, None, None, 1e-5, x, mean, rstd)
    # bfloat16's last rounding is 2^-9 of an element; float32's sums of 16392 terms are good to 2^-24 * 128
    for got, exact in zip([x[1], *x[at]], want):
        assert float((got.double() - exact).norm() / exact.norm()) <= 3e-3
    same = torch.ones(rows, dtype=torch.bool, device="cuda")
    same[at] = False
    for stat, exact in ((mean, row.mean()), (rstd, 1 / torch.sqrt(row.var(unbiased=False) + 1e-5))):
        assert bool((stat[same] == stat[1]).all()) and abs(float(stat[1] - exact)) <= 1e-5
    for first in range(0, rows, 1 << 20):
        part = x[first:first + (1 << 20)]
        assert bool(((part == x[1]).all(1) == same[first:first + (1 << 20)]).all())
    del x
    torch.cuda.empty_cache()
