"""A client's own layers: what it trains between two rounds, next to the 4-bit layers of ``distill``.

``layer_norm``, ``dropout``, ``gated`` and ``adapter`` put the CUDA library's calls (``binding.sbc_layer_norm``,
``sbc_dropout``, ``sbc_gated``, ``sbc_adapter`` and their gradients) behind torch's autograd; everything that
computes is the library's.  Gradients are first ones: differentiating them again raises.  ``AdaptedBlock`` is one
block of a language model made of them, with a low-rank adapter of every client beside a projection that all
clients share in 4 bits, and ``ToyAdapters`` trains such adapters inside ``DelayedSGD``: all clients at once, each
token with its own client's adapter.
"""
from __future__ import annotations

from typing import List, Optional, Sequence, Tuple

import torch

from . import binding
from .distill import TeacherMessage, _FirstOnly, _first_only, _rows, distill_loss, fp4_apply, fp4_linear, teach


def _flat(t: torch.Tensor) -> torch.Tensor:
    """A tensor as a matrix of its last dimension's rows."""
    return _rows(t.reshape(-1, t.shape[-1]))


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        flat = _flat(x.detach())
        w, b = (None if t is None else t.detach().contiguous() for t in (weight, bias))
        y, stats = binding.sbc_layer_norm(flat, w, b, eps)
        ctx.save_for_backward(x, weight, bias, flat, w, stats)
        return y.view(x.shape)

    @staticmethod
    def backward(ctx, dy):
        x, weight, bias, flat, w, stats = ctx.saved_tensors
        need_x, need_w, need_b = ctx.needs_input_grad[:3]
        kind = None if w is not None or bias is None else bias.dtype
        dx, dw, db = binding.sbc_layer_norm_grad(_flat(dy.to(flat.dtype)), flat, stats, w, need_x, need_w or need_b, weight_dtype=kind)
        sources = [t for t in (dy, x, weight, bias) if t is not None]
        return (_first_only(dx.view(x.shape), *sources) if need_x else None, _first_only(dw, *sources) if need_w else None,
                _first_only(db, *sources) if need_b else None, None)


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
               eps: float = 1e-5) -> torch.Tensor:
    """The last dimension of x normalised, times weight plus bias (float32 or of x's type, both alike)."""
    return _LayerNorm.apply(x, weight, bias, eps)


class DropoutNumbers:
    """The random numbers of a client's steps: a key, a step that lies on the GPU, and how many of the step's numbers
    its layers have taken so far.  A captured step draws anew in each replay if ``next_step`` is captured with it.

    A layer that its backward pass computes again (activation checkpointing) has to draw what its forward pass drew:
    ``take`` its numbers outside of what is computed again and give them to ``dropout`` as ``at``."""

    def __init__(self, seed: int, device: torch.device):
        self.rng = torch.tensor([int(seed) & ((1 << 63) - 1), 0], dtype=torch.int64, device=device)
        self.taken = 0

    def next_step(self) -> None:
        """Numbers that no step before had.  (A backward pass needs those of its forward pass: it comes first.)"""
        self.rng[1:].add_(1)
        self.taken = 0

    def take(self, elements: int) -> int:
        """Numbers for so many elements that no other layer of the step has; where they begin."""
        if torch._C._current_graph_task_id() != -1:
            # (what is computed again would take others than its forward pass did, and nothing else would tell)
            raise RuntimeError("numbers are taken in a backward pass: take them before the forward pass and give them to dropout as `at`")
        at, self.taken = self.taken, self.taken + (elements + 7) // 8
        return at


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, rng, at, tie):
        y = binding.sbc_dropout(_flat(x.detach()), p, rng, at, None if residual is None else _flat(residual.detach()))
        ctx.save_for_backward(rng)   # (changed in place before the backward pass, autograd raises); x itself is not kept
        ctx.about = (p, at, residual is not None, x.shape, x.dtype)
        ctx.tie = tie
        return y.view(x.shape)

    @staticmethod
    def backward(ctx, dy):
        (rng,) = ctx.saved_tensors
        p, at, added, shape, dtype = ctx.about
        dx = None
        if ctx.needs_input_grad[0]:
            dx = _first_only(binding.sbc_dropout(_flat(dy.to(dtype)), p, rng, at).view(shape), dy, *ctx.tie)
        return dx, dy if added and ctx.needs_input_grad[1] else None, None, None, None, None


def dropout(x: torch.Tensor, p: float, numbers: DropoutNumbers, residual: Optional[torch.Tensor] = None,
            at: Optional[int] = None) -> torch.Tensor:
    """residual + x, elements of x dropped with probability p and the others scaled up; neither a mask nor x is kept.
    ``at``: where x's numbers begin, from ``numbers.take(x.numel())`` before; None: they are taken here."""
    if residual is not None and (residual.shape != x.shape or residual.dtype != x.dtype):
        raise ValueError("the residual must have x's shape and type")
    # an empty tensor stands for x where a gradient's gradient is asked for (in a list: it is no input)
    tie = [_FirstOnly.apply(x.new_empty(0), x)] if torch.is_grad_enabled() and x.requires_grad else []
    return _Dropout.apply(x, residual, p, numbers.rng, numbers.take(x.numel()) if at is None else at, tie)


class _Gated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gate, up, act, keep):
        flat = _flat(x.detach())
        g, u = (_rows(w.detach().to(x.dtype)) for w in (gate, up))
        ctx.kinds = (gate.dtype, up.dtype)
        if not keep:
            ctx.save_for_backward(x, gate, up)
            return binding.sbc_gated(flat, g, u, act).view(*x.shape[:-1], g.shape[0])
        h, kept = binding.sbc_gated(flat, g, u, act, keep=True)
        ctx.save_for_backward(x, gate, up, flat, g, u, kept)
        return h.view(*x.shape[:-1], g.shape[0])

    @staticmethod
    def backward(ctx, dh):
        x, gate, up, flat, g, u, kept = ctx.saved_tensors
        need_x, need_g, need_u = ctx.needs_input_grad[:3]
        kind = torch.float32 if torch.float32 in ctx.kinds else x.dtype
        dx, dg, du = binding.sbc_gated_grad(_flat(dh.to(x.dtype)), flat, g, u, kept, need_x, need_g or need_u, kind)
        sources = (dh, x, gate, up)
        return (_first_only(dx.view(x.shape), *sources) if need_x else None, _first_only(dg.to(ctx.kinds[0]), *sources) if need_g else None,
                _first_only(du.to(ctx.kinds[1]), *sources) if need_u else None, None, None)


def gated(x: torch.Tensor, gate: torch.Tensor, up: torch.Tensor, act: str = "silu") -> torch.Tensor:
    """act(x gate^T) * (x up^T) for bfloat16 or float16 x; float32 weights stay master copies, are rounded to x's type
    for the products and get float32 gradients."""
    keep = torch.is_grad_enabled() and (x.requires_grad or gate.requires_grad or up.requires_grad)
    return _Gated.apply(x, gate, up, act, keep)


class _Adapter(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, base, down, up, ids, plan, scale, keep, status):
        flat, d, u = _flat(x.detach()), down.detach().contiguous(), up.detach().contiguous()
        shared = None if base is None else _flat(base.detach())
        ctx.keep, ctx.base = keep, None if base is None else base.shape
        if not keep:   # (at most the base asks for a gradient, which is the output's)
            return binding.sbc_adapter(flat, d, u, ids, scale, shared, plan, status=status).view(*x.shape[:-1], u.shape[2])
        y, kept = binding.sbc_adapter(flat, d, u, ids, scale, shared, plan, keep=True, status=status)
        ctx.save_for_backward(x, down, up, flat, d, u, kept.mid, kept.plan.room)
        ctx.about = (scale, kept.plan.tokens, kept.plan.count)
        return y.view(*x.shape[:-1], u.shape[2])

    @staticmethod
    def backward(ctx, dy):
        if not ctx.keep:
            return None, dy.reshape(ctx.base), None, None, None, None, None, None, None
        x, down, up, flat, d, u, mid, room = ctx.saved_tensors
        scale, tokens, count = ctx.about
        need_x, need_base, need_d, need_u = ctx.needs_input_grad[:4]
        kept = binding.AdapterKept(mid, binding.AdapterPlan(room, tokens, count))
        dx, dd, du = binding.sbc_adapter_grad(_flat(dy.to(flat.dtype)), flat, d, u, kept, scale, None, need_x, need_d or need_u)
        sources = (dy, x, down, up)
        return (_first_only(dx.view(x.shape), *sources) if need_x else None, dy.reshape(ctx.base) if need_base else None,
                _first_only(dd, *sources) if need_d else None, _first_only(du, *sources) if need_u else None, None, None, None, None, None)


def adapter(x: torch.Tensor, down: torch.Tensor, up: torch.Tensor, ids: Optional[torch.Tensor] = None, scale: float = 1.0,
            base: Optional[torch.Tensor] = None, plan: Optional[binding.AdapterPlan] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """base + scale (x down_i^T) up_i, i the adapter of the token (``ids``: int32, one per row of x, negative: none; or a
    ``plan`` of them, binding.sbc_adapter_plan, for all layers of a batch).  ``down`` [adapters, rank, in] and ``up``
    [adapters, rank, out] are float32 or of x's type.  An id that is no adapter's counts as none, and STATUS_RANGE is or-ed into
    ``status`` (int32 on the GPU, zeroed by the caller; with a plan, that of sbc_adapter_plan)."""
    keep = torch.is_grad_enabled() and any(t.requires_grad for t in (x, down, up))
    return _Adapter.apply(x, base, down, up, ids, plan, scale, keep, status)


class AdaptedBlock:
    """One block of a language model: x + dropout(projection(gated(norm(x)))), the projection shared by all clients in
    4 bits with every client's low-rank adapter beside it.  The block's own weights are fixed here; what a client
    trains, and sends, are its adapter's two factors."""

    def __init__(self, width: int, hidden: int, device: torch.device, p: float = 0.1, scale: float = 2.0, format: str = "e8m0",
                 act: str = "silu", dtype: torch.dtype = torch.bfloat16, seed: int = 0):
        g = torch.Generator(device="cpu").manual_seed(seed)
        self.norm = torch.ones(width, device=device), torch.zeros(width, device=device)
        self.gate = (torch.randn(hidden, width, generator=g) / width ** 0.5).to(device, dtype)
        self.up = (torch.randn(hidden, width, generator=g) / width ** 0.5).to(device, dtype)
        self.projection = (torch.randn(width, hidden, generator=g) / hidden ** 0.5).to(device)
        self.served = binding.sbc_fp4_quantise(self.projection, format)   # the same, as it is kept where nothing is trained
        self.p, self.scale, self.format, self.act = p, scale, format, act

    def factors(self, rank: int, seed: int = 0) -> List[torch.Tensor]:
        """A new adapter's factors, float32: down [rank, hidden], up [rank, width] of zeros."""
        hidden, width = self.gate.shape
        g = torch.Generator(device="cpu").manual_seed(seed)
        return [(torch.randn(rank, hidden, generator=g) / hidden ** 0.5).to(self.gate.device), torch.zeros(rank, width, device=self.gate.device)]

    def train(self, x: torch.Tensor, down: torch.Tensor, up: torch.Tensor, plan: binding.AdapterPlan, numbers: DropoutNumbers,
              at: Optional[int] = None) -> torch.Tensor:
        """Tokens of many clients, each with its client's adapter.  ``at``: as for ``dropout``."""
        h = gated(layer_norm(x, *self.norm), self.gate, self.up, self.act)
        y = adapter(h, down, up, None, self.scale, fp4_linear(h, self.projection, self.format), plan)
        return dropout(y, self.p, numbers, x, at)

    def serve(self, x: torch.Tensor, down: torch.Tensor, up: torch.Tensor, ids: torch.Tensor, status: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The next token of each of many requests, or whole prompts: nothing is dropped or kept.  ``status``: as for ``adapter``."""
        with torch.no_grad():
            h = gated(layer_norm(x, *self.norm), self.gate, self.up, self.act)
            return x + adapter(h, down, up, ids, self.scale, fp4_apply(h, self.served), status=status)


class ToyAdapters:
    """Clients that learn a teacher's logits by low-rank adapters alone.  Feeds ``DelayedSGD``: ``weights`` (one adapter, the
    server's) and ``local_updates``, which runs all clients' iterations of a round in one batch, or ``local_update`` for one client."""

    def __init__(self, n_clients: int, device: torch.device, width: int = 96, hidden: int = 160, words: int = 200, positions: int = 96,
                 rank: int = 4, k: int = 16, temperature: float = 2.0, lr: float = 4.0, seed: int = 0):
        g = torch.Generator(device="cpu").manual_seed(seed)
        self.block = AdaptedBlock(width, hidden, device, seed=seed + 1)
        self.weights = self.block.factors(rank, seed + 2)
        self.head = (4 * torch.randn(words, width, generator=g) / width ** 0.5).to(device)
        self.n_clients, self.lr, self.words = n_clients, lr, words
        self.x = torch.randn(n_clients * positions, width, generator=g).to(device, torch.bfloat16)
        self.ids = torch.arange(n_clients, device=device, dtype=torch.int32).repeat_interleave(positions)
        self.plan = binding.sbc_adapter_plan(self.ids, n_clients)
        self.positions, self.alone = positions, binding.sbc_adapter_plan(torch.zeros_like(self.ids[:positions]), 1)
        # the teacher: the same block with an adapter that is not known to the clients
        taught = [torch.randn(1, *w.shape, generator=g).to(device) / w.shape[1] ** 0.5 for w in self.weights]
        y = self.block.serve(self.x, taught[0], 4 * taught[1], torch.zeros_like(self.ids))
        self.message = teach(fp4_linear(y, self.head), k, temperature)
        self.numbers = DropoutNumbers(seed + 3, device)

    def _loss(self, y: torch.Tensor, message: Optional[TeacherMessage] = None) -> torch.Tensor:
        return distill_loss(fp4_linear(y, self.head), self.message if message is None else message)

    def loss(self, weights: Optional[Sequence[torch.Tensor]] = None) -> float:
        down, up = (w[None] for w in (self.weights if weights is None else weights))
        with torch.no_grad():
            return float(self._loss(self.block.serve(self.x, down, up, torch.zeros_like(self.ids))).mean())

    def _grads(self, x: torch.Tensor, message: TeacherMessage, plan: binding.AdapterPlan, down: torch.Tensor,
               up: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
        y = self.block.train(x, down, up, plan, self.numbers)
        loss = self._loss(y, message).view(plan.count, -1).mean(1).sum()
        grads = torch.autograd.grad(loss, (down, up))
        self.numbers.next_step()
        return grads

    def step(self, down: torch.Tensor, up: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
        """The gradients of all clients' adapters ([clients, rank, ...]) on their tokens."""
        return self._grads(self.x, self.message, self.plan, down, up)

    def _updates(self, step, clients: int, weights: Sequence[torch.Tensor], delay: int) -> List[List[torch.Tensor]]:
        params = [w.detach().repeat(clients, 1, 1).requires_grad_(True) for w in weights]   # (copies: one client's, too)
        for _ in range(delay):
            grads = step(*params)
            with torch.no_grad():
                for w, g in zip(params, grads):
                    w -= self.lr * g
        return [[(w[c].detach() - w0).contiguous() for w, w0 in zip(params, weights)] for c in range(clients)]

    def local_updates(self, weights: Sequence[torch.Tensor], delay: int) -> List[List[torch.Tensor]]:
        """``delay`` SGD iterations of every client from ``weights``, in one batch; returns W_after - W of each."""
        return self._updates(self.step, self.n_clients, weights, delay)

    def local_update(self, client: int, weights: Sequence[torch.Tensor], delay: int) -> List[torch.Tensor]:
        """The same for one client, on its tokens alone."""
        if not 0 <= client < self.n_clients:
            raise IndexError(f"client {client} of {self.n_clients}")
        rows = slice(client * self.positions, (client + 1) * self.positions)
        values, indices, rest, temperature = self.message
        message = TeacherMessage(values[rows], indices[rows], rest[rows], temperature)
        return self._updates(lambda down, up: self._grads(self.x[rows], message, self.alone, down, up), 1, weights, delay)[0]
