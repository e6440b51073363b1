"""The end of a language model's training step on one GPU, together with the compressor of its gradients: layer normalisation,
the vocabulary head under cross entropy, under distillation from a teacher's top logits, or under both, and the gradients of all
three parameters in the arena that ``compress`` reads.  Buffer plumbing like ``Session``: the arithmetic is the library's.  All
calls run on the current stream."""
from __future__ import annotations

from typing import Optional

import torch

from . import binding
from .session import Session


class HeadSession(Session):
    """Parameters: ``weights``, a float32 arena of three layers of the plan with the views ``gamma``, ``beta`` and ``matrix``
    (vocab x hidden); ``w`` is the matrix in the activations' type.

        head = HeadSession(rows=4096, hidden=2048, vocab=50021, ratio=0.01)
        head.set_weights(gamma, beta, matrix)
        loss, dx = head.step(x, target)                    # gradients are in head.grad, dx goes on to the layers below
        head.compress()                                    # what is sent to the other workers
        head.apply(eta)                                    # and what it does to the weights
    """

    def __init__(self, rows: int, hidden: int, vocab: int, dtype=torch.bfloat16, p: int = 3, alpha: float = 0.5, ratio: float = 0.01,
                 top: int = 0, temperature: float = 1.0, eps: float = 1e-5, device: str = "cuda:0", **session):
        super().__init__([(1, hidden), (1, hidden), (vocab, hidden)], p, alpha, [1.0, 1.0, ratio], device=device, **session)
        self.rows, self.hidden, self.vocab, self.dtype = rows, hidden, vocab, dtype
        self.top, self.temperature, self.eps = top, temperature, eps
        dev = self.device
        self.weights = torch.zeros_like(self.grad)
        self.gamma, self.beta, self.matrix = self._layers(self.weights)
        self.dgamma, self.dbeta, self.dmatrix = self._layers(self.grad)
        self.w = self.matrix if dtype == torch.float32 else torch.zeros(vocab, hidden, dtype=dtype, device=dev)
        self.gamma.fill_(1.0)
        # activations of one microbatch
        self.y, self.dy, self.dy_taught, self.dx = (torch.empty(rows, hidden, dtype=dtype, device=dev) for _ in range(4))
        self.mean, self.rstd, self.loss, self.loss_taught, self.lse, self.row_grad = (torch.empty(rows, device=dev) for _ in range(6))
        self.room = torch.empty(0, dtype=torch.uint8, device=dev)

    def _layers(self, arena):
        g, b, m = (arena[o:o + n] for o, n in zip(self.offsets, self.sizes))
        return g, b, m.view(self.vocab, self.hidden)

    def _make_room(self, n: int) -> None:
        need = max(binding.rsdgc_layer_norm_workspace_bytes(n, self.hidden),
                   binding.rsdgc_head_workspace_bytes(self.dtype, n, self.hidden, self.vocab, 0),
                   binding.rsdgc_head_workspace_bytes(self.dtype, n, self.hidden, self.vocab, self.top) if self.top else 0)
        if need > self.room.numel():
            self.room = torch.empty(need, dtype=torch.uint8, device=self.device)

    def set_weights(self, gamma, beta, matrix) -> None:
        for to, value in ((self.gamma, gamma), (self.beta, beta), (self.matrix, matrix)):
            to.copy_(torch.as_tensor(value))
        self._refresh()

    def _refresh(self) -> None:
        if self.w is not self.matrix:
            self.w.copy_(self.matrix)

    def evaluate(self, x, target):
        """Loss of each row, without gradients."""
        n = x.shape[0]
        self._make_room(n)
        binding.rsdgc_layer_norm(x, self.gamma, self.beta, self.eps, self.y[:n])
        binding.rsdgc_head_loss(self.y[:n], self.w, target, self.loss[:n], self.lse[:n], self.room)
        return self.loss[:n]

    def step(self, x, target=None, top_idx=None, top_logit=None, share: float = 0.5, accumulate: bool = False, row_grad=None):
        """One microbatch: (loss of each row, dx), the parameters' gradients into the arena (accumulate: on top of what is there).
        They are those of the sum of the rows' losses times ``row_grad`` (float32, one for each row; None: 1 / rows, the mean over
        all rows, in which one without a target counts as 0).  The mean over the rows that have a target:

            has = (target >= 0).float()
            head.step(x, target, row_grad=has / has.sum())

        With a target and a teacher's entries, `share` of the loss is the teacher's.  Both returned tensors are overwritten by the
        next call."""
        n = x.shape[0]
        taught = top_idx is not None
        assert 0 < n <= self.rows and (target is not None or taught) and (not taught or top_idx.shape[1] == self.top)
        part = share if taught and target is not None else 1.0 if taught else 0.0
        self._make_room(n)
        assert row_grad is None or (row_grad.shape == (n,) and row_grad.dtype == torch.float32)
        y, dy, dx, loss, lse, gain = (t[:n] for t in (self.y, self.dy, self.dx, self.loss, self.lse, self.row_grad))
        mean, rstd, room = self.mean[:n], self.rstd[:n], self.room
        binding.rsdgc_layer_norm(x, self.gamma, self.beta, self.eps, y, mean, rstd)
        if target is not None:
            binding.rsdgc_head_loss(y, self.w, target, loss, lse, room)
            self._gain(gain, row_grad, 1.0 - part)
            binding.rsdgc_head_loss_backward(y, self.w, target, lse, gain, dy, self.dmatrix, accumulate, room)
        if taught:
            both = target is not None
            of_teacher, dy_taught = (self.loss_taught[:n], self.dy_taught[:n]) if both else (loss, dy)
            binding.rsdgc_distill_loss(y, self.w, top_idx, top_logit, self.temperature, of_teacher, lse, room)
            self._gain(gain, row_grad, part)
            binding.rsdgc_distill_loss_backward(y, self.w, top_idx, top_logit, self.temperature, lse, gain, dy_taught,
                                                self.dmatrix, accumulate or both, room)
            if both:
                loss.mul_(1.0 - part).add_(of_teacher, alpha=part)
                dy.add_(dy_taught)
        binding.rsdgc_layer_norm_backward(dy, x, self.gamma, mean, rstd, dx, self.dgamma, self.dbeta, accumulate, room)
        return loss, dx

    @staticmethod
    def _gain(out, row_grad, part: float) -> None:
        if row_grad is None:
            out.fill_(part / out.numel())
        else:
            torch.mul(row_grad, part, out=out)

    def apply(self, eta: float, messages: Optional[list] = None) -> None:
        """weights -= eta * (sum of the messages, in order; own one if none are given)."""
        if messages is None:
            messages = [(self.out_idx, self.out_val, self.out_counts)]
        binding.rsdgc_apply(self.plan, messages, self.weights, eta, self.workspace)
        self._refresh()
