"""What the operators of a client's own layers do behind autograd, on the CPU: the library's calls are replaced by plain
computations, so what is tested is what the wrappers keep, ask for and hand on."""
import itertools

import pytest
import torch
from torch.utils.checkpoint import checkpoint

from paper_1805_08768_b200 import binding, block


def adapter(x, down, up, ids, scale=1.0, base=None, plan=None, keep=False, status=None):
    d, u = (t.double()[ids.clamp(min=0).long()] * (ids >= 0)[:, None, None] for t in (down, up))
    y = scale * torch.einsum("ti,tri,tro->to", x.double(), d, u)
    y = (y if base is None else y + base.double()).to(x.dtype)
    if not keep:
        return y
    return y, binding.AdapterKept(torch.zeros(1), binding.AdapterPlan(ids, x.shape[0], down.shape[0]))


@torch.enable_grad()   # (inside of a backward pass it is off)
def adapter_grad(dy, x, down, up, kept, scale, base, need_input, need_adapters):
    leaves = [t.detach().double().requires_grad_(True) for t in (x, down, up)]
    ids = kept.plan.room
    d, u = (t[ids.clamp(min=0).long()] * (ids >= 0)[:, None, None] for t in leaves[1:])
    grads = torch.autograd.grad(scale * torch.einsum("ti,tri,tro->to", leaves[0], d, u), leaves, dy.double())
    dx, dd, du = (g.to(t.dtype) for g, t in zip(grads, (x, down, up)))
    return dx if need_input else None, dd if need_adapters else None, du if need_adapters else None


@pytest.fixture
def plain(monkeypatch):
    monkeypatch.setattr(binding, "sbc_adapter", adapter)
    monkeypatch.setattr(binding, "sbc_adapter_grad", adapter_grad)


@pytest.mark.parametrize("asked", [a for a in itertools.product([False, True], repeat=4) if any(a)])
def test_adapter_gives_every_gradient_that_is_asked_for(plain, asked):
    """x, base, down and up each with or without: a base alone, too (fixed adapters beside a projection that is trained)."""
    g = torch.Generator().manual_seed(1)
    x, base = torch.randn(6, 4, generator=g), torch.randn(6, 5, generator=g)
    down, up = torch.randn(3, 2, 4, generator=g), torch.randn(3, 2, 5, generator=g)
    ids = torch.tensor([0, 2, -1, 1, 2, 0], dtype=torch.int32)
    dy = torch.randn(6, 5, generator=g)
    every = [t.clone().requires_grad_(True) for t in (x, base, down, up)]
    want = torch.autograd.grad(block.adapter(every[0], every[2], every[3], ids, 1.5, every[1]), every, dy)
    some = [t.clone().requires_grad_(a) for t, a in zip((x, base, down, up), asked)]
    y = block.adapter(some[0], some[2], some[3], ids, 1.5, some[1])
    assert torch.equal(y, adapter(x, down, up, ids, 1.5, base))
    leaves = [t for t, a in zip(some, asked) if a]
    got = torch.autograd.grad(y, leaves, dy)
    assert all(torch.equal(a, b) for a, b in zip(got, [w for w, a in zip(want, asked) if a]))
    assert torch.equal(want[1], dy)


@pytest.mark.parametrize("fixed", [False, True])
def test_adapter_takes_a_base_of_any_leading_dimensions(plain, fixed):
    """The base's rows are x's whatever dimensions they are in (what a projection of the flattened tokens gave), and so are its gradient's."""
    g = torch.Generator().manual_seed(1)
    x, base = torch.randn(2, 3, 4, generator=g), torch.randn(6, 5, generator=g).requires_grad_(True)
    down, up = torch.randn(3, 2, 4, generator=g).requires_grad_(not fixed), torch.randn(3, 2, 5, generator=g)
    y = block.adapter(x, down, up, torch.tensor([0, 2, -1, 1, 2, 0], dtype=torch.int32), 1.0, base)
    dy = torch.randn(y.shape, generator=g)
    (got,) = torch.autograd.grad(y, base, dy)
    assert torch.equal(got, dy.view(6, 5))


def drop(x, p, rng, at=0, residual=None):
    """(each place in the step's numbers keeps other elements)"""
    keep = (torch.arange(x.numel()) // 8 + at).view(x.shape) % 2 == 0
    y = x * keep
    return y if residual is None else y + residual


@pytest.mark.parametrize("reentrant", [False, True])
def test_dropout_that_is_computed_again(monkeypatch, reentrant):
    """Under activation checkpointing the forward pass runs twice: with numbers taken before, the second time draws the same;
    taking them there is refused, since the gradients would be another mask's."""
    monkeypatch.setattr(binding, "sbc_dropout", drop)
    x = torch.randn(3, 8, generator=torch.Generator().manual_seed(1)).requires_grad_(True)
    numbers = block.DropoutNumbers(1, torch.device("cpu"))
    numbers.take(8)
    at = numbers.take(x.numel())
    assert at == 1 and numbers.taken == 4
    (want,) = torch.autograd.grad((block.dropout(x, 0.5, numbers, at=at) ** 2).sum(), x)
    y = checkpoint(lambda t: block.dropout(t, 0.5, numbers, at=at) ** 2, x, use_reentrant=reentrant)
    y.sum().backward()
    assert torch.equal(x.grad, want) and numbers.taken == 4
    y = checkpoint(lambda t: block.dropout(t, 0.5, numbers) ** 2, x, use_reentrant=reentrant)
    with pytest.raises(RuntimeError, match="taken in a backward pass"):
        y.sum().backward()
    # outside of a backward pass numbers can be taken again
    assert numbers.take(1) == 7
