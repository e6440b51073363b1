"""The head at the ends of what it accepts: numbers of tokens beyond what is taken together, widths and vocabularies beyond the usual,
gradients of losses of very different size.  The oracle is the formulas in 64 bits, on the GPU; tolerances as in test_gpu_training."""
import math

import pytest
import torch

from paper_2312_17530_amd import binding as b
from .test_gpu_training import BF16, F32, _close, _head_run

pytestmark = pytest.mark.gpu


def _case(rows, hidden, vocab, dtype, top=0, seed=0):
    """Inputs made on the GPU; one row in five has no answer, entries of a teacher name a token twice now and then."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def rand(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    w = rand(vocab, hidden).mul_(2 / math.sqrt(hidden)).to(dtype)
    case = dict(w=w, row_grad=0.01 * torch.rand(rows, generator=gen, device="cuda") - 0.002)
    x = rand(rows, hidden)
    if top == 0:
        target = torch.randint(vocab, (rows,), generator=gen, device="cuda")
        x[::2] += 3 * w[target[::2]].float()
        target[torch.rand(rows, generator=gen, device="cuda") < 0.2] = -1
        case["target"] = target.int()
    else:
        idx = torch.randint(vocab, (rows, top), generator=gen, device="cuda")
        x[::2] += w[idx[::2, 0]].float()
        idx[torch.rand(rows, generator=gen, device="cuda") < 0.2] = -1
        case["top_idx"], case["top_logit"] = idx.int(), 4 * rand(rows, top)
    case["x"] = x.to(dtype)
    return case


def _exact(case, t=1.0):
    """Results in 64 bits, and the gradients' terms without cancellation."""
    x, w, g = case["x"].double(), case["w"].double(), case["row_grad"].double()
    rows, vocab = x.shape[0], w.shape[0]
    logp = x @ w.t() / t
    lse = torch.logsumexp(logp, 1)
    logp -= lse[:, None]
    q = torch.zeros_like(logp)
    if "target" in case:
        idx, share = case["target"][:, None].long(), torch.ones(rows, 1, dtype=torch.float64, device="cuda")
        kept = (idx >= 0) & (idx < vocab)
    else:
        idx, logit = case["top_idx"].long(), case["top_logit"].double()
        kept = (idx >= 0) & (idx < vocab) & (logit > -math.inf)
        share = torch.softmax(torch.where(kept, logit / t, -math.inf), 1)
    q.scatter_add_(1, idx.clamp(0, vocab - 1), torch.where(kept, share, 0.0))
    has = kept.any(1)
    loss = torch.where(has, t * t * (torch.special.xlogy(q, q) - q * logp).sum(1), 0.0)
    g = torch.where(has, t * g, 0.0)[:, None]
    p = logp.exp_()
    d, both = (p - q) * g, (p + q) * g.abs()
    x = torch.where(has[:, None], x, 0.0)
    return dict(loss=loss, lse=lse, dx=d @ w, dw=d.t() @ x), dict(dx=both @ w.abs(), dw=both.t() @ x.abs())


def _check(tag, case, t=1.0):
    print("head", tag, flush=True)
    got, (want, terms) = _head_run(case, t), _exact(case, t)
    # the constants are derived for sums of up to 128^2 terms, whose errors grow with the root of their number
    longer = max(0.0, math.sqrt(max(case["x"].shape)) / 128 - 1)
    for k in got:
        more = longer * want[k].abs() + (terms[k] * (1 + longer) if k in terms else 0.0)
        _close(f"{tag} {k}", got[k], want[k].cpu(), case["x"].dtype if k == "dx" else F32, more.cpu())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("top", [0, 6])
@pytest.mark.parametrize("over", [1, 8, 9])
def test_a_few_tokens_more_than_are_taken_together(over, top, dtype):
    """16384 tokens go through the backward pass together; the rest of them, however few, are in the same form."""
    _check(f"16384 + {over} rows, top {top}, {dtype}", _case(16384 + over, 40, 300, dtype, top, seed=over), 2.0 if top else 1.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,hidden", [(1, 131080), (40, 131080), (20, 2056), (300, 131080)])
def test_wide_rows(rows, hidden, dtype):
    """Widths whose columns alone are more tiles of dx than the card has places for, and one whose vocabulary is cut into shares."""
    _check(f"{rows} rows of {hidden}, {dtype}", _case(rows, hidden, 203, dtype, seed=rows))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [30, 300])
def test_rows_as_far_apart_as_they_may_be(rows, dtype):
    """x, W and dx with 2^20 elements from one row to the next: the same bits as without gaps, and the gaps of dx as they were."""
    case = _case(rows, 48, 203, dtype, seed=rows)
    far = dict(case)
    for k in ("x", "w"):
        far[k] = torch.full((case[k].shape[0], 1 << 20), math.nan, dtype=dtype, device="cuda")[:, 512:560]
        far[k].copy_(case[k])
    out = torch.full((rows, 1 << 20), 7.0, dtype=dtype, device="cuda")
    dx = out[:, 64:112]
    want = _head_run(case)
    loss, lse, dw = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(203, 48, device="cuda")
    ws = torch.empty(b.rsdgc_head_workspace_bytes(dtype, rows, 48, 203), dtype=torch.uint8, device="cuda")
    b.rsdgc_head_loss(far["x"], far["w"], far["target"], loss, lse, ws)
    b.rsdgc_head_loss_backward(far["x"], far["w"], far["target"], lse, far["row_grad"], dx, dw, False, ws)
    for k, got in dict(loss=loss, lse=lse, dx=dx, dw=dw).items():
        assert torch.equal(got, want[k]), k
    assert bool((out[:, :64] == 7.0).all()) and bool((out[:, 112:] == 7.0).all())


@pytest.mark.parametrize("backward", [False, True])
def test_more_rows_behind_a_teacher_than_a_launch_has_waves(backward):
    """2^26 and a few tokens of width 1 over three words: a wave for each token would be 2^32 threads.  The tokens repeat, so that a few
    of them tell all."""
    rows, kinds = (1 << 26) + 5, 7
    small = _case(kinds, 1, 3, BF16, 1, seed=2)
    small["top_idx"][:, 0] = torch.tensor([0, 1, 2, -1, 2, 0, 1], device="cuda")
    at = torch.arange(rows, device="cuda", dtype=torch.int32) % kinds
    x, idx, logit, grad = (small[k].index_select(0, at) for k in ("x", "top_idx", "top_logit", "row_grad"))
    loss, lse = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    ws = torch.empty(b.rsdgc_head_workspace_bytes(BF16, rows, 1, 3, 1, backward), dtype=torch.uint8, device="cuda")
    want, _ = _exact(small, 2.0)
    b.rsdgc_distill_loss(x, small["w"], idx, logit, 2.0, loss, lse, ws)
    got = dict(loss=loss, lse=lse)
    if backward:
        got["dx"], dw = torch.empty_like(x), torch.empty(3, 1, device="cuda")
        b.rsdgc_distill_loss_backward(x, small["w"], idx, logit, 2.0, lse, grad, got["dx"], dw, False, ws)
        times = torch.bincount(at, minlength=kinds).double()
        d = want["dx"].new_tensor(0.0)
        for n in range(kinds):
            one = {k: small[k][n:n + 1] for k in ("x", "top_idx", "top_logit", "row_grad")}
            d = d + times[n] * _exact(one | dict(w=small["w"]), 2.0)[0]["dw"]
        # 16384 terms at a time, sqrt(16384) roundings of 2^-24, and 4096 sums of these one after another, much alike, so that their
        # roundings may all have one sign: half of 4096, the sum growing evenly
        assert float((dw.double() - d).norm()) <= (128 + 2048) * 2.0 ** -24 * float((times[:, None] * _rows_of(small)).abs().sum())
    for k, v in got.items():
        for n in range(kinds):
            mine = v.view(-1)[n::kinds]
            assert bool((mine == mine[0]).all()), (k, n)
        _close(k, v[:kinds], want[k].cpu(), BF16 if k == "dx" else F32)


def _rows_of(case):
    """|d| |x| of each token, summed over the vocabulary."""
    out = []
    for n in range(case["x"].shape[0]):
        one = {k: case[k][n:n + 1] for k in ("x", "top_idx", "top_logit", "row_grad")}
        out.append(_exact(one | dict(w=case["w"]), 2.0)[1]["dw"].sum())
    return torch.stack(out)[:, None]


def test_more_logits_than_a_launch_has_tiles():
    """65536 tokens over 8.4 million words of width 8, tiles of 256 x 256 and 512 threads: 2^32 threads and a few more.  64 of the tokens
    are compared."""
    rows, hidden, vocab = 65536, 8, (1 << 23) + 77
    size = b.rsdgc_head_workspace_bytes(BF16, rows, hidden, vocab, 0, False)
    if torch.cuda.mem_get_info()[0] + torch.cuda.memory_reserved() < size + (24 << 30):
        pytest.skip(f"{(size >> 30) + 24} GiB of memory are needed")
    torch.cuda.empty_cache()
    case = _case(rows, hidden, vocab, BF16, seed=3)
    loss, lse = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    b.rsdgc_head_loss(case["x"], case["w"], case["target"], loss, lse, torch.empty(size, dtype=torch.uint8, device="cuda"))
    at = torch.arange(0, rows, rows // 63, device="cuda")[:64]
    z = case["x"][at].double() @ case["w"].double().t()
    target = case["target"][at].long()
    want = torch.logsumexp(z, 1)
    _close("lse", lse[at], want.cpu(), F32)
    own = z[torch.arange(len(at), device="cuda"), target.clamp(min=0)]
    _close("loss", loss[at], torch.where(target >= 0, want - own, 0.0).cpu(), F32)
    del z
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t", [0.25, 1.0, 3.0])
@pytest.mark.parametrize("rows", [20, 900])
def test_teacher_logits_at_the_ends_of_float32(rows, t, dtype):
    """Entries at the type's lowest value count like any others, a row of nothing else is an even answer; the largest ones do not
    become infinite by the temperature."""
    case = _case(rows, 64, 200, dtype, 5, seed=rows)
    low, high = torch.finfo(F32).min, torch.finfo(F32).max
    case["top_idx"][:] = torch.tensor([3, 50, 7, 199, 120], device="cuda")
    case["top_logit"][0::4, 2:] = low                  # masked ones beside ordinary ones
    case["top_logit"][1::4] = low                      # nothing but masked ones
    case["top_logit"][2::4, 1:3] = high                # two share everything
    case["top_logit"][2::4, 3] = high * 0.75
    _check(f"{rows} rows, t {t}, {dtype}", case, t)


@pytest.mark.parametrize("rows", [20, 900])
def test_a_temperature_whose_square_is_beyond_float32(rows):
    """Logits that are almost nothing: rows without an answer have loss +0 all the same, the statistics are those of even words."""
    case = _case(rows, 64, 200, F32, 5, seed=rows)
    case["top_idx"][::3] = -1
    got, (want, _) = _head_run(case, 1e20), _exact(case, 1e20)
    none = (case["top_idx"] < 0).all(1)
    assert bool((got["loss"][none] == 0.0).all()) and not bool(torch.isnan(got["loss"]).any())
    _close("lse", got["lse"], want["lse"].cpu(), F32)
    assert bool((got["dx"][none] == 0.0).all())


@pytest.mark.parametrize("top", [0, 6])
@pytest.mark.parametrize("dtype,rows,hidden,vocab", [(BF16, 100, 64, 900), (BF16, 100, 61, 900), (BF16, 700, 64, 900), (BF16, 700, 61, 900), (BF16, 2100, 520, 5003), (F32, 700, 64, 900)])
def test_words_that_are_much_alike(dtype, rows, hidden, vocab, top):
    """Embeddings share a direction that is a hundred times what tells them apart.  A token's d sums up to nothing, so the shared part
    leaves dx but for the roundings of d, which count a hundredfold: as many of its bits as float32 results need."""
    case = _case(rows, hidden, vocab, dtype, top, seed=hidden)
    gen = torch.Generator(device="cuda").manual_seed(5)
    shared = torch.randn(hidden, generator=gen, device="cuda")
    case["w"].copy_(shared + 0.01 * torch.randn(vocab, hidden, generator=gen, device="cuda"))
    case["x"].copy_(torch.randn(rows, hidden, generator=gen, device="cuda"))
    _check(f"alike {rows}x{hidden}x{vocab} top {top} {dtype}", case, 2.0 if top else 1.0)


def _check_rows(tag, case, t=1.0, but=None):
    """Every token's loss, lse and dx against its own size, not that of the largest, and dw as a whole; but one token's, and dw then not."""
    print("head", tag, flush=True)
    got, (want, terms) = _head_run(case, t), _exact(case, t)
    kind = case["x"].dtype
    keep = torch.arange(case["x"].shape[0], device="cuda") != (-1 if but is None else but)
    for k in ("loss", "lse"):
        off, size = (got[k].double() - want[k]).abs()[keep], (want["lse"].abs() + want["loss"].abs())[keep]
        assert float((off / size).max()) <= 1e-5, (tag, k, float((off / size).max()))
    off = (got["dx"].double() - want["dx"]).norm(dim=1)
    may = {F32: 1e-5, BF16: 3e-3}[kind] * want["dx"].norm(dim=1) + 1e-5 * terms["dx"].norm(dim=1)
    worst = int(torch.where(keep, off - may, -math.inf).argmax())
    assert bool((off <= may)[keep].all()), f"{tag}: row {worst} of dx is {float(off[worst] / want['dx'][worst].norm()):.3g} off"
    if but is None:
        _close(f"{tag} dw", got["dw"], want["dw"].cpu(), F32, terms["dw"].cpu())


@pytest.mark.parametrize("top", [0, 6])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,hidden", [(20, 64), (700, 64), (700, 61), (16384 + 40, 24)])
def test_tokens_whose_gradients_differ_by_many_orders(rows, hidden, dtype, top):
    """row_grad from 1e-28 to 1: a token's row of dx does not know the others' gradients."""
    case = _case(rows, hidden, 300, dtype, top, seed=rows)
    gen = torch.Generator(device="cuda").manual_seed(6)
    case["row_grad"] = torch.pow(10.0, -28 * torch.rand(rows, generator=gen, device="cuda")) * (1 - 2 * (torch.rand(rows, generator=gen, device="cuda") < 0.3))
    _check_rows(f"gains {rows}x{hidden} top {top} {dtype}", case, 2.0 if top else 1.0)


@pytest.mark.parametrize("top", [0, 6])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("outlier", [1e4, 1e10])
@pytest.mark.parametrize("rows", [20, 700])
def test_a_token_with_a_channel_far_above_the_others(rows, outlier, dtype, top):
    """One token's channel that the matrix does not read: the other tokens' logits, losses and dx do not know of it."""
    case = _case(rows, 64, 300, dtype, top, seed=rows)
    case["w"][:, 0] = 0
    case["x"][5, 0] = outlier
    for k in ("target", "top_idx"):
        if k in case:
            case[k][5] = 7
    _check_rows(f"outlier {outlier} in {rows} top {top} {dtype}", case, 2.0 if top else 1.0, but=5)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,hidden,vocab,top,t", [(20, 1024, 5000, 64, 1.0), (24, 1021, 5000, 64, 1.0), (100, 2056, 700, 40, 1.0), (700, 1024, 5000, 64, 1.0), (1500, 4096, 2000, 64, 1.0),
                                                     (900, 301, 2000, 200, 0.5)])
def test_a_student_that_agrees_with_its_teacher(rows, hidden, vocab, top, t, dtype):
    """The teacher's logits are the student's own largest: the loss is a small difference, whose logits have to come from the same sums to
    cancel.  What cannot is the rounding of its terms, q log q and q log p, four of 2^-24."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    w = (torch.randn(vocab, hidden, generator=gen, device="cuda") / math.sqrt(hidden)).to(dtype)
    x = (4 * torch.randn(rows, hidden, generator=gen, device="cuda")).to(dtype)
    most = (x.double() @ w.double().t()).topk(top, 1)
    case = dict(x=x, w=w, top_idx=most.indices.int(), top_logit=most.values.float(), row_grad=torch.full((rows,), 1 / rows, device="cuda"))
    tag = f"agrees {rows}x{hidden}x{vocab} top {top} {dtype}"
    print("head", tag, flush=True)
    got, (want, terms) = _head_run(case, t), _exact(case, t)
    log_q = torch.log_softmax(case["top_logit"].double() / t, 1)
    log_p = most.values / t - want["lse"][:, None]
    parts = t * t * (log_q.exp() * (log_q.abs() + log_p.abs())).sum(1)
    off = (got["loss"].double() - want["loss"]).norm()
    assert off <= 1e-5 * want["loss"].norm() + 2.0 ** -22 * parts.norm(), (tag, float(off / want["loss"].norm()), float(off / parts.norm()))
    _close(f"{tag} lse", got["lse"], want["lse"].cpu(), F32)
    for k, kind in (("dx", dtype), ("dw", F32)):
        _close(f"{tag} {k}", got[k], want[k].cpu(), kind, terms[k].cpu())
