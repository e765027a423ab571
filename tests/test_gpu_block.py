"""The operators of a client's own layers behind autograd, and together: a block, and a federated toy run of adapters."""
import gc

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_1805_08768_b200 import binding as sbc
from paper_1805_08768_b200 import block, distill
from paper_1805_08768_b200.dsgd import DelayedSGD

DEV = torch.device("cuda:0")


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(*shape, seed, dtype=torch.float32):
    return torch.randn(*shape, generator=gen(seed), device=DEV).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_layer_norm_under_autograd(dtype):
    x = randn(3, 7, 70, seed=1, dtype=dtype).requires_grad_(True)
    w, b = randn(70, seed=2).requires_grad_(True), randn(70, seed=3).requires_grad_(True)
    dy = randn(3, 7, 70, seed=4, dtype=dtype)
    y = block.layer_norm(x, w, b, 1e-4)
    got = torch.autograd.grad(y, (x, w, b), dy)
    flat = x.detach().view(21, 70)
    want_y, stats = sbc.sbc_layer_norm(flat, w.detach(), b.detach(), 1e-4)
    want = sbc.sbc_layer_norm_grad(dy.view(21, 70), flat, stats, w.detach())
    assert torch.equal(y.view(21, 70), want_y) and all(torch.equal(a.view(c.shape), c) for a, c in zip(got, want))
    # any order of the input and of the gradient, and parts of the gradients
    xt = x.detach().transpose(0, 1).contiguous().transpose(0, 1).requires_grad_(True)
    y = block.layer_norm(xt, w, b, 1e-4)
    assert all(torch.equal(a, c) for a, c in zip(torch.autograd.grad(y, (xt, w, b), dy), got))
    (dx,) = torch.autograd.grad(block.layer_norm(x, w.detach(), b.detach(), 1e-4).sum(), x)
    assert dx.shape == x.shape
    assert torch.equal(torch.autograd.grad(block.layer_norm(x.detach(), w, b, 1e-4), w, dy)[0], got[1])
    assert block.layer_norm(x.detach()[:0], w, b).shape == (0, 7, 70)


def test_dropout_under_autograd():
    x, r = (randn(5, 33, seed=s).requires_grad_(True) for s in (1, 2))
    dy = randn(5, 33, seed=3)
    numbers = block.DropoutNumbers(11, DEV)
    y = block.dropout(x, 0.4, numbers, r)
    z = block.dropout(x, 0.4, numbers)
    assert numbers.taken == 2 * 21
    assert torch.equal(y.detach(), sbc.sbc_dropout(x.detach(), 0.4, numbers.rng, 0, r.detach()))
    assert torch.equal(z.detach(), sbc.sbc_dropout(x.detach(), 0.4, numbers.rng, 21))
    dx, dr = torch.autograd.grad(y, (x, r), dy)
    assert torch.equal(dx, sbc.sbc_dropout(dy, 0.4, numbers.rng, 0)) and torch.equal(dr, dy)
    # the backward pass needs its forward pass's numbers
    y = block.dropout(x, 0.4, numbers)
    numbers.next_step()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(y.sum(), x)
    assert not torch.equal(block.dropout(x.detach(), 0.4, numbers), z.detach())
    with pytest.raises(ValueError):
        block.dropout(x, 0.4, numbers, r[:2])


def test_dropout_keeps_nothing():
    """Between the passes there is the output and nothing else: the input's memory is free once its owner lets go of it."""
    numbers = block.DropoutNumbers(11, DEV)
    leaf = randn(1, 64, seed=1).requires_grad_(True)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    y = block.dropout(leaf.expand(1 << 14, 64) * 2.0, 0.5, numbers)   # (4 MB made and dropped, 4 MB out; a constant's product keeps no operand)
    assert torch.cuda.memory_allocated() - before < 5 << 20
    (grad,) = torch.autograd.grad(y.sum(), leaf)
    assert grad.shape == leaf.shape


@pytest.mark.parametrize("master", [torch.bfloat16, torch.float32])
def test_gated_under_autograd(master):
    x = randn(2, 25, 48, seed=1, dtype=torch.bfloat16).requires_grad_(True)
    g, u = (randn(72, 48, seed=s, dtype=master).requires_grad_(True) for s in (2, 3))
    dh = randn(2, 25, 72, seed=4, dtype=torch.bfloat16)
    h = block.gated(x, g, u, "gelu")
    got = torch.autograd.grad(h, (x, g, u), dh)
    flat, g0, u0 = x.detach().view(50, 48), g.detach().bfloat16(), u.detach().bfloat16()
    want_h, kept = sbc.sbc_gated(flat, g0, u0, "gelu", keep=True)
    want = sbc.sbc_gated_grad(dh.view(50, 72), flat, g0, u0, kept, grad_dtype=master)
    assert torch.equal(h.view(50, 72), want_h) and all(a.dtype == c.dtype and torch.equal(a.view(c.shape), c) for a, c in zip(got, want))
    with torch.no_grad():
        assert block.gated(x, g, u, "gelu").shape == (2, 25, 72)
    assert torch.equal(torch.autograd.grad(block.gated(x, g.detach(), u.detach(), "gelu"), x, dh)[0], got[0])
    assert torch.equal(torch.autograd.grad(block.gated(x.detach(), g, u.detach(), "gelu"), g, dh)[0], got[1])
    gt = g.detach().t().contiguous().t().requires_grad_(True)
    assert torch.equal(torch.autograd.grad(block.gated(x, gt, u, "gelu"), gt, dh)[0], got[1])


def test_adapter_under_autograd():
    x = randn(30, 40, seed=1, dtype=torch.bfloat16).requires_grad_(True)
    base = randn(30, 56, seed=2, dtype=torch.bfloat16).requires_grad_(True)
    down, up = randn(3, 5, 40, seed=3).requires_grad_(True), randn(3, 5, 56, seed=4).requires_grad_(True)
    ids = torch.randint(-1, 3, (30,), generator=gen(5), device=DEV, dtype=torch.int32)
    dy = randn(30, 56, seed=6, dtype=torch.bfloat16)
    y = block.adapter(x, down, up, ids, 1.5, base)
    got = torch.autograd.grad(y, (x, base, down, up), dy)
    want_y, kept = sbc.sbc_adapter(x.detach(), down.detach(), up.detach(), ids, 1.5, base.detach(), keep=True)
    want = sbc.sbc_adapter_grad(dy, x.detach(), down.detach(), up.detach(), kept, 1.5)
    assert torch.equal(y, want_y) and torch.equal(got[0], want[0]) and torch.equal(got[1], dy)
    assert torch.equal(got[2], want[1]) and torch.equal(got[3], want[2])
    plan = sbc.sbc_adapter_plan(ids, 3)
    again = torch.autograd.grad(block.adapter(x, down, up, None, 1.5, base, plan), (x, base, down, up), dy)
    assert all(torch.equal(a, c) for a, c in zip(again, got))
    # without the graph the few-token form answers
    with torch.no_grad():
        few = block.adapter(x, down, up, ids, 1.5, base)
    assert torch.equal(few, sbc.sbc_adapter(x.detach(), down.detach(), up.detach(), ids, 1.5, base.detach()))
    # factors that are shared by broadcasting get the sum of their copies' gradients
    one_d, one_u = randn(1, 5, 40, seed=7).requires_grad_(True), randn(1, 5, 56, seed=8).requires_grad_(True)
    dd, du = torch.autograd.grad(block.adapter(x, one_d.expand(3, 5, 40), one_u.expand(3, 5, 56), ids, 1.5), (one_d, one_u), dy)
    copies = [t.detach().expand(3, *t.shape[1:]).contiguous() for t in (one_d, one_u)]
    _, kept = sbc.sbc_adapter(x.detach(), *copies, ids, 1.5, keep=True)
    _, wd, wu = sbc.sbc_adapter_grad(dy, x.detach(), *copies, kept, 1.5)
    assert torch.allclose(dd, wd.sum(0, keepdim=True), rtol=1e-6, atol=1e-6) and torch.allclose(du, wu.sum(0, keepdim=True), rtol=1e-6, atol=1e-6)


def test_second_derivatives_raise():
    x = randn(40, 32, seed=1, dtype=torch.bfloat16).requires_grad_(True)
    w = randn(32, seed=2).requires_grad_(True)
    g = randn(48, 32, seed=3, dtype=torch.bfloat16).requires_grad_(True)
    d, u = randn(2, 4, 32, seed=4).requires_grad_(True), randn(2, 4, 32, seed=5).requires_grad_(True)
    ids = torch.zeros(40, dtype=torch.int32, device=DEV)
    numbers = block.DropoutNumbers(1, DEV)
    for make, leaf in ((lambda: block.layer_norm(x, w), x), (lambda: block.layer_norm(x, w), w), (lambda: block.gated(x, g, g), x),
                       (lambda: block.gated(x, g, g), g), (lambda: block.adapter(x, d, u, ids), d), (lambda: block.adapter(x, d, u, ids), x),
                       (lambda: block.dropout(x, 0.5, numbers), x)):
        y = make()
        (first,) = torch.autograd.grad((y.float() ** 2).sum(), leaf, create_graph=True)
        with pytest.raises(RuntimeError, match="second derivatives"):
            torch.autograd.grad(first.float().sum(), leaf)


def plain_block(b, x, down, up, ids, keep, dtype):
    """The block in torch's own operations and 64 bits; what the operators round is rounded (straight through for gradients)."""
    def rounded(t):
        return t + (t.detach().to(dtype).double() - t.detach())

    gate, lift = b.gate.double(), b.up.double()
    h = torch.nn.functional.layer_norm(x, x.shape[-1:], *(t.double() for t in b.norm))
    h = rounded(h)
    h = rounded(torch.nn.functional.silu(h @ gate.t()) * (h @ lift.t()))
    w = sbc.sbc_fp4_dequantise(sbc.sbc_fp4_quantise(b.projection, b.format)).double()
    h4 = sbc.sbc_fp4_dequantise(sbc.sbc_fp4_quantise(h.detach().to(dtype), b.format)).double()
    y = rounded((h + (h4 - h.detach())) @ w.t())
    mid = torch.einsum("tk,trk->tr", h, down[ids.long()])
    y = rounded(y + b.scale * torch.einsum("tr,tro->to", mid, up[ids.long()]))
    return rounded(x + y * keep)


def test_block_against_plain_operations():
    """The operators one after the other: output and adapter gradients against the same chain in 64 bits.

    Every value on the way is rounded as the operators round it, but a 64-bit value next to a rounding's border may fall on the
    other side; a few such steps of 2^-8 in a chain of six leave the whole (2-norm) within 2^-7, and the gradients, whose own
    roundings on the way down (dg, du, dy in 4 bits: the projection's input gradient is not asked for here) are the output
    gradient's in bfloat16, within 2^-6."""
    b = block.AdaptedBlock(96, 160, DEV, p=0.25, seed=3)
    tokens = 150
    x = randn(tokens, 96, seed=1, dtype=torch.bfloat16)
    ids = torch.randint(0, 4, (tokens,), generator=gen(2), device=DEV, dtype=torch.int32)
    down = (randn(4, 6, 160, seed=3) / 160 ** 0.5).requires_grad_(True)
    up = (randn(4, 6, 96, seed=4) * 0.3).requires_grad_(True)
    plan = sbc.sbc_adapter_plan(ids, 4)
    numbers = block.DropoutNumbers(5, DEV)
    y = b.train(x, down, up, plan, numbers)
    dy = randn(tokens, 96, seed=6, dtype=torch.bfloat16)
    got = torch.autograd.grad(y, (down, up), dy)
    keep = sbc.sbc_dropout(torch.ones(tokens, 96, device=DEV), 0.25, block.DropoutNumbers(5, DEV).rng).double()
    d64, u64 = (t.detach().double().requires_grad_(True) for t in (down, up))
    want_y = plain_block(b, x.double(), d64, u64, ids, keep, torch.bfloat16)
    want = torch.autograd.grad(want_y, (d64, u64), dy.double())
    assert float((y.double() - want_y).norm() / want_y.norm()) < 2.0 ** -7
    for a, c in zip(got, want):
        assert a.dtype == torch.float32 and float((a.double() - c).norm() / c.norm()) < 2.0 ** -6


def test_block_serves_tokens_as_it_serves_prompts():
    """Single tokens of many requests and the whole batch: the same numbers up to the order of sums (each result is one
    rounding of each of three operators from the other's: within three steps of the largest)."""
    b = block.AdaptedBlock(96, 160, DEV, seed=3)
    x = randn(130, 96, seed=1, dtype=torch.bfloat16)
    ids = torch.randint(-1, 5, (130,), generator=gen(2), device=DEV, dtype=torch.int32)
    down, up = randn(5, 6, 160, seed=3) / 160 ** 0.5, randn(5, 6, 96, seed=4) * 0.3
    whole = b.serve(x, down, up, ids)
    parts = torch.cat([b.serve(x[i:i + 13], down, up, ids[i:i + 13].contiguous()) for i in range(0, 130, 13)])
    step = 2.0 ** -7 * float(whole.abs().max())
    assert float((whole.double() - parts.double()).abs().max()) <= 3 * step


def test_training_step_in_a_graph():
    """Forward and backward of the block captured and replayed: each replay draws its own numbers, and gives what the eager
    step with those numbers gives."""
    toy = block.ToyAdapters(3, DEV)
    params = [w.detach().expand(3, *w.shape).contiguous() for w in toy.weights]
    params[1].normal_(generator=gen(1)).mul_(0.1)

    def grads():
        leaves = [p.detach().requires_grad_(True) for p in params]    # leaves of this pass's own
        return toy.step(*leaves)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        grads()
    torch.cuda.synchronize()
    gc.collect()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        held = grads()
    seen = []
    for _ in range(3):
        step = int(toy.numbers.rng[1])
        graph.replay()
        torch.cuda.synchronize()
        seen.append([t.clone() for t in held])
        toy.numbers.rng[1] = step
        assert all(torch.equal(a, c) for a, c in zip(grads(), seen[-1]))
        assert int(toy.numbers.rng[1]) == step + 1
    assert not torch.equal(seen[0][0], seen[1][0])


def test_federated_run_of_adapters():
    """Clients' adapters train inside the sparse binary method; every operator of the block is on the way.  (That gradients and
    updates are finite and arrive is tested, not how far a loss falls.)"""
    toy = block.ToyAdapters(3, DEV)
    run = DelayedSGD(toy.weights, 3, 0.05, 2, toy.local_update)
    before = [w.clone() for w in run.weights]
    for _ in range(3):
        run.round()
    run.check()
    for updates in run.last_updates:
        assert all(bool(torch.isfinite(u).all()) and float(u.abs().max()) > 0 for u in updates)
    assert all(not torch.equal(a, b) for a, b in zip(before, run.weights))
    assert toy.loss(run.weights) == toy.loss(run.weights)
    # clients differ: each has its own tokens and its own copy of the adapter
    first, second = run.last_updates[0], run.last_updates[1]
    assert not torch.equal(first[1], second[1])
    # one client alone gets what it gets beside the others
    alone = [w.detach()[None].clone().requires_grad_(True) for w in run.weights]
    y = toy.block.train(toy.x[:96], alone[0], alone[1], sbc.sbc_adapter_plan(torch.zeros(96, dtype=torch.int32, device=DEV), 1), block.DropoutNumbers(1, DEV))
    both = [w.detach()[None].expand(3, *w.shape).contiguous().requires_grad_(True) for w in run.weights]
    z = toy.block.train(toy.x, both[0], both[1], toy.plan, block.DropoutNumbers(1, DEV))
    assert float((y.double() - z[:96].double()).abs().max()) <= 3 * 2.0 ** -7 * float(y.abs().max())
