"""The distillation module on the GPU: autograd around the operators, and a federated toy run of all of them."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_1805_08768_b200 import binding as sbc
from paper_1805_08768_b200 import distill
from paper_1805_08768_b200.dsgd import DelayedSGD

DEV = torch.device("cuda:0")


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def rounded(x, fmt):
    return sbc.sbc_fp4_dequantise(sbc.sbc_fp4_quantise(x.contiguous(), fmt)).double()


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(1, 33, 7), (35, 650, 300), (130, 100, 257)])
def test_fp4_linear(shape, dtype, fmt):
    """Output and both gradients are products of the rounded factors: at most
    (cols / 64 + 4) 2^-22 sum |a b| from the sums, half a unit in the last place from the result's type."""
    tokens, inner, outer = shape
    x = torch.randn(tokens, inner, generator=gen(1), device=DEV).to(dtype).requires_grad_(True)
    w = torch.randn(outer, inner, generator=gen(2), device=DEV).requires_grad_(True)
    dy = torch.randn(tokens, outer, generator=gen(3), device=DEV).to(dtype)
    y = distill.fp4_linear(x, w, fmt)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    assert y.dtype == dtype and dx.dtype == dtype and dw.dtype == torch.float32
    x0, w0 = x.detach(), w.detach()
    for got, a, b, length in ((y, rounded(x0, fmt), rounded(w0, fmt), inner), (dx, rounded(dy, fmt), rounded(w0.t(), fmt), outer),
                              (dw, rounded(dy.t(), fmt), rounded(x0.t(), fmt), tokens)):
        want, size = a @ b.t(), a.abs() @ b.abs().t()
        unit = 2.0 ** -24 if got.dtype == torch.float32 else 2.0 ** -8
        allowed = (math.ceil(length / 64) + 4) * 2.0 ** -22 * size + unit * want.abs() + 1e-30
        assert bool(((got.double() - want).abs() <= allowed).all())


def test_fp4_linear_parts_and_shapes():
    x = torch.randn(2, 5, 64, generator=gen(1), device=DEV)
    w = torch.randn(48, 64, generator=gen(2), device=DEV)
    whole = distill.fp4_linear(x, w)
    assert whole.shape == (2, 5, 48)
    assert torch.equal(whole.view(10, 48), distill.fp4_linear(x.view(10, 64), w))
    assert torch.equal(whole, distill.fp4_apply(x, sbc.sbc_fp4_quantise(w)))
    a, b = x.clone().requires_grad_(True), w.clone().requires_grad_(True)
    dy = torch.randn(2, 5, 48, generator=gen(3), device=DEV)
    both = torch.autograd.grad(distill.fp4_linear(a, b), (a, b), dy)
    assert torch.equal(both[0], torch.autograd.grad(distill.fp4_linear(a, w), a, dy)[0])
    assert torch.equal(both[1], torch.autograd.grad(distill.fp4_linear(x, b), b, dy)[0])
    none = torch.empty(0, 64, device=DEV, requires_grad=True)
    y = distill.fp4_linear(none, b)
    assert y.shape == (0, 48)
    dx, dw = torch.autograd.grad(y.sum(), (none, b))
    assert dx.shape == (0, 64) and not bool(dw.any())
    with pytest.raises(ValueError):
        distill.fp4_linear(x, w[:, :63])


def test_loss_under_autograd_is_the_fused_call():
    z = (3 * torch.randn(12, 700, generator=gen(4), device=DEV)).requires_grad_(True)
    message = distill.teach(z.detach() + torch.randn(12, 700, generator=gen(5), device=DEV), 20, 2.0)
    labels = message.indices[:, 1].long()
    loss = distill.distill_loss(z, message, 0.7, labels)
    (grad,) = torch.autograd.grad(loss.mean(), z)
    want, want_grad = sbc.sbc_distill_loss_grad(z.detach(), message.values, message.indices, torch.full((12,), 1 / 12, device=DEV),
                                                message.rest, 2.0, 0.7, labels)
    assert torch.equal(loss, want) and torch.equal(grad, want_grad)
    (half,) = torch.autograd.grad(distill.distill_loss(z.t().contiguous().t(), message, 0.7, labels).mean(), z)
    assert torch.equal(half, grad)
    assert message.nbytes == 12 * (20 * 8 + 4)


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
def test_clients_learn_from_a_teacher_through_sparse_updates(fmt):
    toy = distill.ToyDistillation(3, DEV, format=fmt)
    before = toy.loss()
    run = DelayedSGD(toy.weights, 3, 0.02, 4, toy.local_update)
    for _ in range(25):
        run.round()
    run.check()
    after = toy.loss()
    assert math.isfinite(after) and after < 0.6 * before
    # a single position goes the same way as a batch
    one = toy.teach_logits(toy.x[0][:1])
    assert one.shape == (1, 300) and bool(torch.isfinite(one).all())


def test_toy_runs_repeat_exactly():
    results = []
    for _ in range(2):
        toy = distill.ToyDistillation(2, DEV, seed=3)
        updates = [u for c in range(2) for u in toy.local_update(c, toy.weights, 3)]
        results.append(updates)
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_second_derivatives_are_refused():
    """A gradient that is differentiated again raises, instead of leaving out these functions' part of a sum."""
    z = torch.randn(4, 200, generator=gen(1), device=DEV).requires_grad_(True)
    message = distill.teach(z.detach() + torch.randn(4, 200, generator=gen(2), device=DEV), 8)
    for logits in (z, z.t().contiguous().t()):
        for total in (lambda t: t.sum(), lambda t: t.square().sum()):
            loss = total(distill.distill_loss(logits, message)) + (z ** 2).sum()
            (plain,) = torch.autograd.grad(loss, z, retain_graph=True)
            (grad,) = torch.autograd.grad(loss, z, create_graph=True)
            assert torch.equal(grad, plain)             # asking for the graph alone changes nothing
            with pytest.raises(RuntimeError, match="second derivatives"):
                torch.autograd.grad(grad.square().sum(), z)
    x = torch.randn(6, 64, generator=gen(3), device=DEV).requires_grad_(True)
    w = torch.randn(10, 64, generator=gen(4), device=DEV).requires_grad_(True)
    for total in (lambda t: (t * t.detach()).sum(), lambda t: t.square().sum()):
        loss = total(distill.fp4_linear(x, w)) + (x ** 2).sum() + (w ** 2).sum()
        plain = torch.autograd.grad(loss, (x, w), retain_graph=True)
        grads = torch.autograd.grad(loss, (x, w), create_graph=True)
        assert all(torch.equal(a, b) for a, b in zip(grads, plain))
        for g, of in ((grads[0], w), (grads[1], x), (grads[0], x), (grads[1], w)):
            with pytest.raises(RuntimeError, match="second derivatives"):
                torch.autograd.grad(g.square().sum(), of, retain_graph=True)


def test_the_product_keeps_its_input_in_four_bits_only():
    """Nothing of the forward call holds on to x between the two passes."""
    w = torch.randn(32, 4096, generator=gen(4), device=DEV).requires_grad_(True)
    start = torch.randn(4096, 4096, generator=gen(3), device=DEV).requires_grad_(True)
    base = torch.cuda.memory_allocated()
    x = start + 1.0
    size = x.numel() * 4
    y = distill.fp4_linear(x, w)
    del x
    assert torch.cuda.memory_allocated() - base < size / 2
    (y * y).sum().backward()
    assert start.grad.shape == start.shape and w.grad.shape == w.shape


ORDERS = {"transposed": lambda t: t.t().contiguous().t(), "every second": lambda t: t.repeat_interleave(2, 1)[:, ::2],
          "padded": lambda t: torch.nn.functional.pad(t, (3, 2))[:, 3:-2], "one row": lambda t: t[:1].expand(t.shape),
          "one column": lambda t: t[:, :1].expand(t.shape), "one value": lambda t: t[:1, :1].expand(t.shape)}


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
@pytest.mark.parametrize("order", list(ORDERS))
@pytest.mark.parametrize("tokens", [1, 37])
def test_fp4_linear_of_any_order(order, tokens, fmt):
    """Inputs, weights and gradients that are transposes, slices or broadcast give what their copies give."""
    make = ORDERS[order]
    x = torch.randn(tokens, 70, generator=gen(1), device=DEV)
    w = torch.randn(45, 70, generator=gen(2), device=DEV)
    dy = torch.randn(tokens, 45, generator=gen(3), device=DEV)

    def call(x, w, dy):
        x, w = x.detach().requires_grad_(True), w.detach().requires_grad_(True)
        y = distill.fp4_linear(x, w, fmt)
        return (y, *torch.autograd.grad(y, (x, w), dy))

    for xs, ws, dys in ((make(x), w, dy), (x, make(w), dy), (x, w, make(dy)), (make(x), make(w), make(dy))):
        for a, b in zip(call(xs, ws, dys), call(xs.contiguous(), ws.contiguous(), dys.contiguous())):
            assert torch.equal(a, b)
    held = sbc.sbc_fp4_quantise(w, fmt)
    assert torch.equal(distill.fp4_apply(make(x), held), distill.fp4_apply(make(x).contiguous(), held))


@pytest.mark.parametrize("total", [lambda y: y.sum(), lambda y: y.mean(), lambda y: y.sum(0)[3], lambda y: y.mean(0).sum(), lambda y: y[:, 0].sum(),
                                   lambda y: (y.t() @ torch.ones(y.shape[0], 2, device=DEV)).sum(), lambda y: y.t().contiguous().sum()])
def test_fp4_linear_under_ordinary_reductions(total):
    """The gradient that autograd hands over, whatever its strides, against the same one as a matrix of its own."""
    x = torch.randn(2, 9, 64, generator=gen(1), device=DEV).requires_grad_(True)
    w = torch.randn(24, 64, generator=gen(2), device=DEV).requires_grad_(True)
    y = distill.fp4_linear(x, w)
    got = torch.autograd.grad(total(y.view(18, 24)), (x, w), retain_graph=True)
    leaf = y.detach().view(18, 24).clone().requires_grad_(True)
    (dy,) = torch.autograd.grad(total(leaf), leaf)
    want = torch.autograd.grad(y, (x, w), dy.contiguous().view(2, 9, 24))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("order", list(ORDERS))
def test_distill_loss_of_any_order(order):
    z = ORDERS[order](2 * torch.randn(10, 300, generator=gen(1), device=DEV))
    message = distill.teach(z, 12, 2.0)
    for a, b in zip(message[:3], distill.teach(z.contiguous(), 12, 2.0)[:3]):
        assert torch.equal(a, b)
    message = distill.teach(z + torch.randn(10, 300, generator=gen(2), device=DEV), 12, 2.0)
    results = []
    for logits in (z, z.contiguous()):
        logits = logits.detach().requires_grad_(True)
        loss = distill.distill_loss(logits, message)
        results.append((loss, *torch.autograd.grad(loss.sum(), logits)))
    (loss, grad), (want, want_grad) = results
    if order == "padded":    # such rows are read where they are and cut into vectors elsewhere: sums in another order
        delta = (300 / 256 + 64 + 4 * 30) * 2.0 ** -24
        assert bool(((loss - want).abs() <= 4 * delta * 2.0 ** 2).all())
        assert bool(((grad - want_grad).abs() <= 8 * delta + 2 * 2.0 ** -24 * want_grad.abs()).all())
    else:
        assert torch.equal(loss, want) and torch.equal(grad, want_grad)


def test_evaluation_rounds_one_way(monkeypatch):
    """Without gradients nothing is quantised along the columns, whatever the weights ask for."""
    x = torch.randn(5, 64, generator=gen(1), device=DEV)
    w = torch.randn(24, 64, generator=gen(2), device=DEV).requires_grad_(True)
    want = distill.fp4_linear(x, w).detach()
    monkeypatch.setattr(distill.binding, "sbc_fp4_quantise_both", None)
    with torch.no_grad():
        assert torch.equal(distill.fp4_linear(x, w), want)
    with torch.inference_mode():
        assert torch.equal(distill.fp4_linear(x, w), want)
    assert torch.equal(distill.fp4_linear(x, w.detach()), want)
