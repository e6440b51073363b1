"""What the training operators refuse.  Arguments are checked before anything reaches the GPU, so this needs none: the addresses are
numbers, and no kernel is launched."""
import math
import os
import subprocess
import sys

import pytest
import torch

from paper_2312_17530_amd import binding as b

NAN = math.nan
X, W, Y, DX, DW, F, G, WS = (0x7000_0000_0000 + i * (1 << 36) for i in range(8))       # apart from each other


def _call(name, base, changes):
    args = dict(base)
    for k, v in changes.items():
        assert k in args, k
        args[k] = v
    return getattr(b.load(), name)(*args.values())


NORM = dict(dtype=1, rows=4, cols=64, x=X, ldx=64, gamma=F, beta=F + 4096, eps=1e-5, y=Y, ldy=64, mean=G, rstd=G + 4096, stream=None)
NORM_BACK = dict(dtype=1, rows=4, cols=64, dy=Y, lddy=64, x=X, ldx=64, gamma=F, mean=G, rstd=G + 4096, dx=DX, lddx=64, dgamma=DW, dbeta=DW + 4096,
                 accumulate=0, ws=WS, stream=None)
HEAD = dict(dtype=1, rows=4, hidden=64, vocab=100, x=X, ldx=64, w=W, ldw=64, target=F, loss=G, lse=G + 4096, ws=WS, stream=None)
HEAD_BACK = dict(dtype=1, rows=4, hidden=64, vocab=100, x=X, ldx=64, w=W, ldw=64, target=F, lse=G, row_grad=G + 4096, dx=DX, lddx=64, dw=DW,
                 accumulate=0, ws=WS, stream=None)
TAUGHT = dict(dtype=1, rows=4, hidden=64, vocab=100, x=X, ldx=64, w=W, ldw=64, top=8, idx=F, logit=F + 4096, t=2.0, loss=G, lse=G + 4096, ws=WS,
              stream=None)
TAUGHT_BACK = dict(dtype=1, rows=4, hidden=64, vocab=100, x=X, ldx=64, w=W, ldw=64, top=8, idx=F, logit=F + 4096, t=2.0, lse=G, row_grad=G + 4096,
                   dx=DX, lddx=64, dw=DW, accumulate=0, ws=WS, stream=None)

SIZES = [dict(dtype=2), dict(dtype=-1), dict(rows=-1), dict(ldx=63)]
HEADS = SIZES + [dict(rows=(1 << 30) + 1), dict(hidden=0), dict(hidden=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21), dict(vocab=0), dict(vocab=(1 << 26) + 1),
                 dict(ldw=63), dict(ldx=(1 << 20) + 1), dict(ldw=(1 << 20) + 1), dict(x=None), dict(w=None), dict(x=X + 1), dict(w=W + 1), dict(ws=None),
                 dict(ws=WS + 128), dict(lse=None), dict(lse=G + 4097)]
LOSS = [dict(loss=None), dict(loss=G + 2), dict(loss=X), dict(lse=W + 64), dict(loss=G, lse=G), dict(ws=X - 256), dict(ws=G)]
BACK = [dict(row_grad=None), dict(row_grad=G + 4098), dict(dx=None), dict(dx=DX + 1), dict(lddx=63), dict(dw=None), dict(dw=DW + 2), dict(dx=X),
        dict(dw=X), dict(dw=DX), dict(dx=W + 128), dict(dw=G + 4096 - 4), dict(ws=DW + 256), dict(ws=DX - 256)]
TOP = [dict(top=0), dict(top=-1), dict(top=1025), dict(idx=None), dict(logit=None), dict(idx=F + 2), dict(logit=F + 4097), dict(t=0.0), dict(t=-1.0),
       dict(t=NAN), dict(t=math.inf), dict(t=1e-60)]
NORMS = SIZES + [dict(cols=0), dict(cols=(1 << 24) + 1, ldx=1 << 25), dict(x=None), dict(x=X + 1), dict(gamma=F + 2)]

CASES = ([("rsdgc_layer_norm", NORM, c) for c in NORMS + [dict(eps=-1e-5), dict(eps=NAN), dict(eps=math.inf), dict(y=None), dict(y=Y + 1), dict(ldy=63),
                                                          dict(beta=F + 1), dict(mean=G + 2), dict(rstd=G + 3), dict(y=X + 64), dict(y=F - 128),
                                                          dict(mean=Y), dict(mean=G, rstd=G + 4), dict(y=X, ldy=128)]]
         + [("rsdgc_layer_norm_backward", NORM_BACK, c) for c in NORMS + [dict(dy=None), dict(mean=None), dict(rstd=None), dict(dx=None), dict(lddy=63),
                                                                          dict(lddx=63), dict(dx=DX + 1), dict(dgamma=DW + 2), dict(dbeta=DW + 1),
                                                                          dict(ws=None), dict(ws=WS + 8), dict(dx=X + 64), dict(dgamma=G),
                                                                          dict(dgamma=DW, dbeta=DW + 64), dict(ws=DX), dict(dx=G)]]
         + [("rsdgc_head_loss", HEAD, c) for c in HEADS + LOSS + [dict(target=None), dict(target=F + 2), dict(loss=F)]]
         + [("rsdgc_head_loss_backward", HEAD_BACK, c) for c in HEADS + BACK + [dict(target=None), dict(target=F + 1), dict(dw=F)]]
         + [("rsdgc_distill_loss", TAUGHT, c) for c in HEADS + LOSS + TOP + [dict(loss=F), dict(lse=F + 4096)]]
         + [("rsdgc_distill_loss_backward", TAUGHT_BACK, c) for c in HEADS + BACK + TOP + [dict(dx=F), dict(dw=F + 4096)]])


@pytest.mark.parametrize("name,base,changes", CASES, ids=[f"{n}-{i}-{'-'.join(c)}" for i, (n, _, c) in enumerate(CASES)])
def test_refused(name, base, changes):
    for dtype in ({1, 0} if "dtype" not in changes else {changes["dtype"]}):
        odd = [k for k, v in changes.items() if k in ("x", "w", "y", "dx") and isinstance(v, int) and v % 4 == 2]
        if dtype == 1 and odd:
            continue
        assert _call(name, base, {**changes, "dtype": dtype}) == b.RSDGC_EINVAL, (dtype, changes)


@pytest.mark.parametrize("name,base", [("rsdgc_head_loss_backward", HEAD_BACK), ("rsdgc_distill_loss_backward", TAUGHT_BACK)])
@pytest.mark.parametrize("stride", [(1 << 20) + 1, 1 << 23, 1 << 40])
@pytest.mark.parametrize("dtype", [0, 1])
def test_rows_of_dx_too_far_apart_are_refused(name, base, stride, dtype):
    assert _call(name, base, dict(dtype=dtype, lddx=stride)) == b.RSDGC_EINVAL


@pytest.mark.parametrize("name,base", [("rsdgc_layer_norm", NORM), ("rsdgc_head_loss", HEAD), ("rsdgc_distill_loss", TAUGHT)])
def test_no_rows_touch_nothing(name, base):
    # without rows no address of theirs is looked at, and nothing is launched
    gone = {k: None for k in ("x", "y", "target", "idx", "logit", "loss", "lse", "mean", "rstd") if k in base}
    assert _call(name, base, {"rows": 0, **gone}) == b.RSDGC_OK


def test_workspace_sizes():
    lib = b.load()
    for rows, cols in ((-1, 8), (8, 0), (8, (1 << 24) + 1)):
        assert lib.rsdgc_layer_norm_workspace_bytes(rows, cols) == 0
        with pytest.raises(b.RsdgcError):
            b.rsdgc_layer_norm_workspace_bytes(rows, cols)
    for args in ((2, 8, 8, 8, 0, 1), (0, -1, 8, 8, 0, 1), (0, 8, 0, 8, 0, 1), (0, 8, 8, 0, 0, 1), (0, 8, 8, 8, -1, 1), (0, 8, 8, 8, 1025, 1),
                 (0, 8, (1 << 20) + 1, 8, 0, 1), (0, 8, 8, (1 << 26) + 1, 0, 1), (0, (1 << 30) + 1, 8, 8, 0, 1)):
        assert lib.rsdgc_head_workspace_bytes(*args) == 0, args
    # every size in the range has a workspace, and one for both passes serves the losses alone
    for dtype in (0, 1):
        for rows in (0, 1, 8, 9, 33, 129, 161, 257, 385, 1025, 70000, 1 << 30):
            for hidden in (1, 3, 4, 127, 4096, 1 << 20):
                for vocab in (1, 255, 257, 65536, 1 << 26):
                    for top in (0, 1, 1024):
                        both, loss = (lib.rsdgc_head_workspace_bytes(dtype, rows, hidden, vocab, top, back) for back in (1, 0))
                        assert both >= loss > 0 and both % 256 == 0, (dtype, rows, hidden, vocab, top)



# widths up to the widest, in every form
WIDE = """
import sys
sys.path.insert(0, sys.argv[1])
from paper_2312_17530_amd import binding as b
from tests import test_training_refusals as t
for dtype in (0, 1):
    for rows in (1, 8, 9, 40, 64, 65, 300, 20000):
        for hidden in (131072, 131080, 1 << 20):
            for name, base in (("rsdgc_head_loss", t.HEAD), ("rsdgc_head_loss_backward", t.HEAD_BACK), ("rsdgc_distill_loss_backward", t.TAUGHT_BACK)):
                far = dict(dtype=dtype, rows=rows, hidden=hidden, vocab=1000, ldx=hidden, ldw=hidden, lddx=hidden)
                far |= {k: t.X + (i << 38) for i, k in enumerate(("x", "w", "dx", "dw", "ws", "target", "idx", "logit", "loss", "lse", "row_grad"))}
                changes = {k: v for k, v in far.items() if k in base}
                code = t._call(name, base, changes)
                assert code == b.RSDGC_EHIP, (name, changes, code)
print("all returned")
"""


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="the addresses are numbers: only where no kernel can be launched")
def test_the_widest_rows_return():
    """Accepted sizes come back with the launch's error where there is no GPU; in a process of its own, which a fault would end."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    proc = subprocess.run([sys.executable, "-c", WIDE, root], capture_output=True, text=True, timeout=300)
    assert proc.returncode == 0 and "all returned" in proc.stdout, (proc.returncode, proc.stderr[-2000:])


@pytest.mark.parametrize("name,base", [("rsdgc_distill_loss", TAUGHT), ("rsdgc_distill_loss_backward", TAUGHT_BACK)])
@pytest.mark.parametrize("t", [2e-39, 1e-45])
def test_a_temperature_without_a_reciprocal_is_refused(name, base, t):
    assert _call(name, base, dict(t=t)) == b.RSDGC_EINVAL


# Two matrices side by side in one buffer: 64 columns each, rows 128 elements apart
SIDE = [("rsdgc_layer_norm", NORM, "ldx", "x", "ldy", "y"), ("rsdgc_layer_norm_backward", NORM_BACK, "ldx", "x", "lddx", "dx"),
        ("rsdgc_layer_norm_backward", NORM_BACK, "lddy", "dy", "lddx", "dx"), ("rsdgc_head_loss_backward", HEAD_BACK, "ldx", "x", "lddx", "dx"),
        ("rsdgc_distill_loss_backward", TAUGHT_BACK, "ldx", "x", "lddx", "dx")]


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="the addresses are numbers: only where no kernel can be launched")
@pytest.mark.parametrize("name,base,ld_a,a,ld_b,b_", SIDE, ids=[f"{n}-{a}" for n, _, _, a, _, _ in SIDE])
@pytest.mark.parametrize("dtype", [0, 1])
def test_columns_of_one_buffer_side_by_side_are_taken(name, base, ld_a, a, ld_b, b_, dtype):
    size = 2 if dtype else 4
    for at in (64 * size, -64 * size, (128 - 64) * size):
        assert _call(name, base, {"dtype": dtype, ld_a: 128, ld_b: 128, a: X + 4096, b_: X + 4096 + at}) == b.RSDGC_EHIP, at
    # one element into each other, from either side, or rows of another length
    for at in (63 * size, -63 * size, 65 * size, -65 * size):
        assert _call(name, base, {"dtype": dtype, ld_a: 128, ld_b: 128, a: X + 4096, b_: X + 4096 + at}) == b.RSDGC_EINVAL, at
    assert _call(name, base, {"dtype": dtype, ld_a: 128, ld_b: 136, a: X + 4096, b_: X + 4096 + 64 * size}) == b.RSDGC_EINVAL
