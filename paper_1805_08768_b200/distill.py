"""Distilled training of a client between two rounds: 4-bit layers and a teacher's largest logits.

Sparse Binary Compression makes what a client *sends* small.  This module is for the other half of a
round with a language model: weights arrive in 4-bit floating point and are multiplied as they are, a
teacher's knowledge arrives as the k largest logits of every position and the mass of all the others,
and the gradients that the loss against them gives are what the client's weight update is made of.

Everything that computes is the CUDA library's (``binding.sbc_fp4_*``, ``sbc_top_logits``,
``sbc_distill_*``); this module puts it behind torch's autograd and moves arguments.  Gradients are
first ones: differentiating them again raises.
``ToyDistillation`` is a small seeded model that runs all of it inside ``DelayedSGD``.
"""
from __future__ import annotations

from typing import List, NamedTuple, Optional, Sequence

import torch

from . import binding


class TeacherMessage(NamedTuple):
    """What a teacher sends for a batch of positions: 8 k + 4 bytes each."""
    values: torch.Tensor        # float32 [positions, k], descending
    indices: torch.Tensor       # int32 [positions, k]
    rest: torch.Tensor          # float32 [positions]: log of the others' mass
    temperature: float

    @property
    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in (self.values, self.indices, self.rest))


def _rows(t: torch.Tensor) -> torch.Tensor:
    """A matrix as the calls take one: contiguous along its rows, which do not overlap.  Transposes and
    broadcast values (what a sum's gradient is) are copied."""
    across, along = t.stride()
    return t if (along == 1 or t.shape[1] == 1) and (across >= t.shape[1] or t.shape[0] == 1) else t.contiguous()


def teach(logits: torch.Tensor, k: int, temperature: float = 1.0) -> TeacherMessage:
    """The message for a teacher's logits [positions, words]."""
    return TeacherMessage(*binding.sbc_top_logits(_rows(logits), k, temperature), temperature)


class _FirstOnly(torch.autograd.Function):
    """A gradient as it is, tied to what it was made of: differentiating it again raises.  (Kernels leave no
    trace, so without the tie it would pass for a constant, and only this part of a sum would be lost.)"""

    @staticmethod
    def forward(ctx, grad, *sources):
        return grad.view_as(grad)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("the library's operators have no second derivatives")


def _first_only(grad, *sources):
    """The tie is needed only where a graph of the gradients is asked for."""
    return _FirstOnly.apply(grad, *sources) if grad is not None and torch.is_grad_enabled() else grad


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, values, indices, rest, temperature, alpha, labels):
        flat = _rows(logits.detach())
        loss, stats = binding.sbc_distill_loss(flat, values, indices, rest, temperature, alpha, labels)
        ctx.save_for_backward(logits, flat, values, indices, rest, labels, stats)
        ctx.about = (temperature, alpha)
        return loss

    @staticmethod
    def backward(ctx, grad_loss):
        logits, flat, values, indices, rest, labels, stats = ctx.saved_tensors
        temperature, alpha = ctx.about
        grad = binding.sbc_distill_grad(flat, values, indices, stats, grad_loss.float().contiguous(), rest,
                                        temperature, alpha, labels)
        return _first_only(grad, logits, grad_loss), None, None, None, None, None, None


def distill_loss(logits: torch.Tensor, message: TeacherMessage, alpha: float = 1.0,
                 labels: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Loss per position (float32): alpha temperature^2 KL(teacher || student) over the sent words and one
    outcome for all others, plus (1 - alpha) cross entropy of ``labels`` (negative: none)."""
    return _DistillLoss.apply(logits, message.values, message.indices, message.rest, message.temperature, alpha, labels)


class _Fp4Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, format, tie):
        flat, master = _rows(x.detach().reshape(-1, x.shape[-1])), _rows(w.detach())
        # (an input that asks for gradients does so under no_grad, too; there is no tie then)
        need_x, need_w = (bool(tie) and needed for needed in ctx.needs_input_grad[:2])
        ctx.about = (x.shape, x.dtype, w.dtype, format)
        ctx.tie = tie
        if flat.shape[0] == 0:
            ctx.save_for_backward(w)
            return x.new_zeros(*x.shape[:-1], w.shape[0])
        # along the rows for this product; along the columns, still in 4 bits, for the backward ones
        x4, ctx.x4_t = binding.sbc_fp4_quantise_both(flat, format) if need_w else (binding.sbc_fp4_quantise(flat, format), None)
        w4, ctx.w4_t = (binding.sbc_fp4_quantise_both(master, format) if need_x
                        else (binding.sbc_fp4_quantise(master, format), None))
        return binding.sbc_fp4_product(x4, w4, x.dtype).view(*x.shape[:-1], w4.rows)

    @staticmethod
    def backward(ctx, dy):
        shape, x_dtype, w_dtype, format = ctx.about
        if dy.numel() == 0:
            (w,) = ctx.saved_tensors
            return dy.new_zeros(shape, dtype=x_dtype), torch.zeros_like(w), None, None
        sources = (dy, *ctx.tie)
        dy = _rows(dy.reshape(-1, dy.shape[-1]))
        need_x, need_w = ctx.needs_input_grad[0], ctx.needs_input_grad[1]
        dx = dw = None
        if need_x and need_w:
            dy4, dy4_t = binding.sbc_fp4_quantise_both(dy, format)
        else:
            dy4 = binding.sbc_fp4_quantise(dy, format) if need_x else None
            dy4_t = binding.sbc_fp4_quantise(dy, format, transposed=True) if need_w else None
        if need_x:
            dx = binding.sbc_fp4_product(dy4, ctx.w4_t, x_dtype).view(shape)
        if need_w:
            dw = binding.sbc_fp4_product(dy4_t, ctx.x4_t, w_dtype)
        return _first_only(dx, *sources), _first_only(dw, *sources), None, None


def fp4_linear(x: torch.Tensor, w: torch.Tensor, format: str = "e8m0") -> torch.Tensor:
    """x w^T with both sides, and in the backward pass the output's gradient, rounded to 4 bits along the
    axis that a product contracts; w [out, in] stays a master copy and gets a gradient in its own type."""
    if x.shape[-1] != w.shape[1]:
        raise ValueError(f"x has {x.shape[-1]} features, w takes {w.shape[1]}")
    # what was rounded to 4 bits is kept for the backward pass, not x itself: an empty tensor stands for both in _first_only
    # (in a list: it is no input of the product)
    tie = [_FirstOnly.apply(x.new_empty(0), x, w)] if torch.is_grad_enabled() and (x.requires_grad or w.requires_grad) else []
    return _Fp4Linear.apply(x, w, format, tie)


def fp4_apply(x: torch.Tensor, w: binding.Fp4Tensor) -> torch.Tensor:
    """x w^T for weights that are held in 4 bits (no gradients): a token or a batch."""
    flat = _rows(x.reshape(-1, x.shape[-1]))
    if flat.shape[0] == 0:
        return x.new_zeros(*x.shape[:-1], w.rows)
    y = binding.sbc_fp4_product(binding.sbc_fp4_quantise(flat, w.format), w, x.dtype)
    return y.view(*x.shape[:-1], w.rows)


class ToyDistillation:
    """A seeded word model's last two layers, learning on every client's shard from a teacher of the same
    shape whose weights the clients hold in 4 bits.  Feeds ``DelayedSGD``: ``weights`` and ``local_update``."""

    def __init__(self, n_clients: int, device: torch.device, in_dim: int = 96, hidden: int = 160, words: int = 300,
                 positions: int = 256, batch: int = 64, k: int = 16, temperature: float = 2.0, alpha: float = 0.9,
                 lr: float = 4.0, format: str = "e8m0", seed: int = 0):
        g = torch.Generator(device="cpu").manual_seed(seed)
        self.format, self.alpha, self.lr, self.batch = format, alpha, lr, batch
        teacher = [torch.randn(hidden, in_dim, generator=g) / in_dim ** 0.5, 4 * torch.randn(words, hidden, generator=g) / hidden ** 0.5]
        self.teacher = [binding.sbc_fp4_quantise(w.to(device), format) for w in teacher]
        self.weights = [(torch.randn(hidden, in_dim, generator=g) / in_dim ** 0.5).to(device),
                        torch.zeros(words, hidden, device=device)]
        self.x = [torch.randn(positions, in_dim, generator=g).to(device, torch.bfloat16) for _ in range(n_clients)]
        self.messages: List[TeacherMessage] = [teach(self.teach_logits(x), k, temperature) for x in self.x]
        self.labels = [m.indices[:, 0].long() for m in self.messages]
        self.cursor = [0] * n_clients

    def teach_logits(self, x: torch.Tensor) -> torch.Tensor:
        """The teacher's logits; one position or many."""
        return fp4_apply(torch.tanh(fp4_apply(x, self.teacher[0])), self.teacher[1])

    def _loss(self, params: Sequence[torch.Tensor], client: int, part: slice) -> torch.Tensor:
        m = self.messages[client]
        message = TeacherMessage(m.values[part], m.indices[part], m.rest[part], m.temperature)
        hidden = torch.tanh(fp4_linear(self.x[client][part], params[0], self.format))
        logits = fp4_linear(hidden, params[1], self.format)
        return distill_loss(logits, message, self.alpha, self.labels[client][part]).mean()

    def loss(self, params: Optional[Sequence[torch.Tensor]] = None) -> float:
        params = self.weights if params is None else params
        with torch.no_grad():
            return float(sum(self._loss(params, c, slice(None)) for c in range(len(self.x))) / len(self.x))

    def local_update(self, client: int, weights: Sequence[torch.Tensor], delay: int) -> List[torch.Tensor]:
        """``delay`` SGD iterations on the client's shard, starting from ``weights``; returns W_after - W."""
        params = [w.detach().clone().requires_grad_(True) for w in weights]
        for _ in range(delay):
            lo = self.cursor[client]
            self.cursor[client] = (lo + self.batch) % (self.x[client].shape[0] - self.batch + 1)
            grads = torch.autograd.grad(self._loss(params, client, slice(lo, lo + self.batch)), params)
            with torch.no_grad():
                for w, gr in zip(params, grads):
                    w -= self.lr * gr
        return [(w.detach() - w0).contiguous() for w, w0 in zip(params, weights)]
