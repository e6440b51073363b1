"""Normalisation, head, losses and compressor together: a head is trained for some steps, and every step's gradients and losses are
compared with the formulas in 64 bits, at the parameters that the step had.

Tolerances: the operators' (float32 results 1e-5, bfloat16 results 3e-3 of the 2-norm), and on top what passes through a bfloat16
tensor between them: y (2^-9 relative) reaches losses, dx and all gradients, dy (2^-9, two of them with both losses, added in
bfloat16 once more) dx and the gradients of scale and shift.  At most four such roundings, independent of each other, each at most
2^-9 = 2e-3 of the 2-norm of what it reaches, where gradients cancel at most threefold: 4 * 2e-3 * 3 = 2.4e-2 for bfloat16;
float32 stays at 1e-5 times the same 12.  The passes hand lse on as float32: what one ulp of it moves a gradient by comes on top (a
token that is nearly sure of its answer has d = p - 1 of a thousandth, and an ulp of an lse of 15 is 1e-6 of p)."""
import math

import numpy as np
import pytest
import torch

from paper_2312_17530_amd import binding as b
from paper_2312_17530_amd.head_session import HeadSession

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
REL = {F32: 1.2e-4, BF16: 2.4e-2}


def _exact(head, x, target, top_idx, top_logit, share, ulps=0.0):
    """Loss per row, dx and the parameters' gradients of the mean loss, in 64 bits; the gradients with lse so many float32 ulps off."""
    n = x.shape[0]
    x = x.double().cpu().requires_grad_()
    gamma, beta = (t.double().cpu().clone().requires_grad_() for t in (head.gamma, head.beta))
    w = head.w.double().cpu()
    y = torch.nn.functional.layer_norm(x, (x.shape[1],), gamma, beta, head.eps)
    z = y.detach() @ w.t()
    loss, dz = torch.zeros(n, dtype=torch.float64), torch.zeros_like(z)
    part = share if target is not None and top_idx is not None else 1.0 if top_idx is not None else 0.0
    if target is not None:
        q = torch.nn.functional.one_hot(target.clamp(0).long().cpu(), w.shape[0]).double() * (target >= 0).double().cpu()[:, None]
        lse = torch.logsumexp(z, 1, keepdim=True)
        loss += (1 - part) * (q * (lse - z)).sum(1)
        dz += (1 - part) / n * (torch.exp(z - lse * (1 + ulps * 2.0 ** -23)) - q) * q.sum(1, keepdim=True)
    if top_idx is not None:
        t = head.temperature
        q = torch.zeros_like(z).scatter(1, top_idx.long().cpu(), torch.softmax(top_logit.double().cpu() / t, 1))
        lse = torch.logsumexp(z / t, 1, keepdim=True)
        loss += part * t * t * torch.where(q > 0, q * (torch.log(q.clamp(min=1e-300)) - (z / t - lse)), 0.0).sum(1)
        dz += part / n * t * (torch.exp(z / t - lse * (1 + ulps * 2.0 ** -23)) - q)
    y.backward(dz @ w)
    return [loss, x.grad, gamma.grad, beta.grad, dz.t() @ y.detach()]


def _near(tag, got, want, rel, moved=None):
    """moved: the result where lse is one float32 ulp off."""
    off, norm = float((got.detach().double().cpu() - want).norm()), float(want.norm())
    assert off <= rel * norm + (0.0 if moved is None else float((moved - want).norm())), f"{tag}: {off / norm:.3g} of the norm"


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("with_target,top", [(True, 0), (False, 5), (True, 5)])
def test_a_head_learns_through_the_compressor(dtype, with_target, top):
    rows, hidden, vocab = 96, 128, 350
    gen = torch.Generator().manual_seed(top + 2 * with_target)
    head = HeadSession(rows, hidden, vocab, dtype, ratio=0.2, top=top, temperature=2.0)
    head.set_weights(1 + 0.1 * torch.randn(hidden, generator=gen), 0.1 * torch.randn(hidden, generator=gen),
                     torch.randn(vocab, hidden, generator=gen) / math.sqrt(hidden))
    x = torch.randn(rows, hidden, generator=gen).to(dtype).cuda()
    target = torch.randint(0, vocab, (rows,), generator=gen).int().cuda() if with_target else None
    if with_target:
        target[::7] = -1
    top_idx = top_logit = None
    if top:
        top_idx = torch.stack([torch.randperm(vocab, generator=gen)[:top] for _ in range(rows)]).int().cuda()
        top_logit = (3 * torch.randn(rows, top, generator=gen)).cuda()
    means = []
    for step in range(6):
        want, moved = (_exact(head, x, target, top_idx, top_logit, 0.25, ulps) for ulps in (0.0, 1.0))
        loss, dx = head.step(x, target, top_idx, top_logit, share=0.25)
        for tag, got, value, other in zip(("loss", "dx", "dgamma", "dbeta", "dmatrix"), (loss, dx, head.dgamma, head.dbeta, head.dmatrix), want, moved):
            _near(f"step {step} {tag}", got, value, REL[dtype], other)
        means.append(float(loss.mean()))
        before = head.weights.clone()
        head.compress()
        sent = head.decompress(dense=torch.zeros_like(head.grad))
        head.apply(4.0)
        # the update is what was sent
        moved = before.double() - head.weights.double()
        assert float((moved - 4.0 * sent.double()).abs().max()) <= 2.0 ** -22 * float(before.abs().max() + 4 * sent.abs().max())
    assert all(later < earlier for earlier, later in zip(means, means[1:])), means


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_microbatches_add_up_and_evaluation_is_the_same_loss(dtype):
    rows, hidden, vocab = 70, 65, 129
    gen = torch.Generator().manual_seed(3)
    head = HeadSession(rows, hidden, vocab, dtype, ratio=0.2)
    head.set_weights(torch.ones(hidden), torch.zeros(hidden), torch.randn(vocab, hidden, generator=gen) / 8)
    x = torch.randn(rows, hidden, generator=gen).to(dtype).cuda()
    target = torch.randint(0, vocab, (rows,), generator=gen).int().cuda()
    loss, _ = head.step(x, target)
    whole, losses = head.grad.clone(), loss.clone()
    assert torch.equal(head.evaluate(x, target), losses)
    # two halves: their means count half each
    head.step(x[:35], target[:35])
    first = head.loss[:35].clone()
    head.step(x[35:], target[35:], accumulate=True)
    _near("losses", torch.cat([first, head.loss[:35]]), losses.double().cpu(), 1e-5)
    _near("gradients", head.grad / 2, whole.double().cpu(), REL[dtype])


def test_what_the_binding_refuses():
    x = torch.zeros(4, 16, dtype=BF16, device="cuda")
    w = torch.zeros(10, 16, dtype=BF16, device="cuda")
    f = lambda n: torch.zeros(n, device="cuda")  # noqa: E731
    target, idx = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, 3, dtype=torch.int32, device="cuda")
    ws = torch.empty(b.rsdgc_head_workspace_bytes(BF16, 4, 16, 10, 3), dtype=torch.uint8, device="cuda")
    refused = [
        lambda: b.rsdgc_layer_norm(x, f(15), None, 1e-5, x.clone()),                                  # too short
        lambda: b.rsdgc_layer_norm(x, x[0], None, 1e-5, x.clone()),                                   # scale not float32
        lambda: b.rsdgc_layer_norm(x, None, None, 1e-5, x.float()),                                   # another type
        lambda: b.rsdgc_layer_norm(x, None, None, 1e-5, x.clone().t()),                               # columns along rows
        lambda: b.rsdgc_layer_norm(x, None, None, -1.0, x.clone()),
        lambda: b.rsdgc_layer_norm(x.cpu(), None, None, 1e-5, x.clone()),
        lambda: b.rsdgc_layer_norm_backward(x, x, None, f(4), f(4), x.clone(), f(16), f(16), False, ws[:16]),   # no room
        lambda: b.rsdgc_layer_norm_backward(x, x, None, None, f(4), x.clone(), None, None, False, None),
        lambda: b.rsdgc_head_loss(x, w[:, :8], target, f(4), f(4), ws),
        lambda: b.rsdgc_head_loss(x, w.float(), target, f(4), f(4), ws),
        lambda: b.rsdgc_head_loss(x, w, target.long(), f(4), f(4), ws),
        lambda: b.rsdgc_head_loss(x, w, target[:3], f(4), f(4), ws),
        lambda: b.rsdgc_head_loss(x, w, target, f(3), f(4), ws),
        lambda: b.rsdgc_head_loss(x, w, target, f(4), f(4), ws[:256]),
        lambda: b.rsdgc_head_loss(x, w, target, f(4), f(4), None),
        lambda: b.rsdgc_head_loss_backward(x, w, target, f(4), f(4), x, f(160), False, ws),           # dx over x
        lambda: b.rsdgc_head_loss_backward(x, w, target, f(4), f(4), x.clone(), f(159), False, ws),
        lambda: b.rsdgc_head_loss_backward(x, w, target, None, f(4), x.clone(), f(160), False, ws),
        lambda: b.rsdgc_distill_loss(x, w, idx, f(12).view(4, 3), 0.0, f(4), f(4), ws),
        lambda: b.rsdgc_distill_loss(x, w, idx, f(12).view(4, 3), math.inf, f(4), f(4), ws),
        lambda: b.rsdgc_distill_loss(x, w, idx, f(16).view(4, 4), 1.0, f(4), f(4), ws),
        lambda: b.rsdgc_distill_loss(x, w, idx[:, :0], f(0).view(4, 0), 1.0, f(4), f(4), ws),
    ]
    for n, call in enumerate(refused):
        with pytest.raises(b.RsdgcError):
            call()
            print("not refused:", n)
    with pytest.raises(TypeError):
        b.rsdgc_layer_norm(x.half(), None, None, 1e-5, x.half())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("top", [0, 5])
def test_the_mean_over_the_rows_that_have_a_target(dtype, top):
    """row_grad = 1 / count: the gradients of the mean over the rows with a target, however much padding there is."""
    rows, hidden, vocab, share = 60, 64, 130, 0.25
    gen = torch.Generator().manual_seed(7)
    head = HeadSession(rows, hidden, vocab, dtype, ratio=0.2, top=top, temperature=2.0)
    head.set_weights(1 + 0.1 * torch.randn(hidden, generator=gen), 0.1 * torch.randn(hidden, generator=gen),
                     torch.randn(vocab, hidden, generator=gen) / math.sqrt(hidden))
    x = torch.randn(rows, hidden, generator=gen).to(dtype).cuda()
    target = torch.randint(0, vocab, (rows,), generator=gen).int().cuda()
    target[20:] = -1
    taught = {}
    if top:
        idx = torch.stack([torch.randperm(vocab, generator=gen)[:top] for _ in range(rows)]).int().cuda()
        taught = dict(top_idx=idx, top_logit=(3 * torch.randn(rows, top, generator=gen)).cuda(), share=share)
    has = (target >= 0).float()
    # the rows that have a target alone: their mean over 20 is the reference's mean over its rows
    kept = {k: v[:20] if k != "share" else v for k, v in taught.items()}
    args = (head, x[:20], target[:20], kept.get("top_idx"), kept.get("top_logit"), share)
    want, moved = (_exact(*args, ulps) for ulps in (0.0, 1.0))
    _, dx = head.step(x, target, row_grad=has / has.sum(), **taught)
    for tag, got, value, other in zip(("dx", "dgamma", "dbeta", "dmatrix"), (dx[:20], head.dgamma, head.dbeta, head.dmatrix), want[1:], moved[1:]):
        _near(tag, got, value, REL[dtype], other)
    assert float(dx[20:].float().abs().max()) == 0.0
