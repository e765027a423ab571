"""The gated feed-forward block on the GPU against plain computations in 64 bits.

Tolerances.  Products of two 16-bit values are exact in 32 bits; each of the n / 16 + 16 additions into a 32-bit sum of n
of them (those of eight warps' sums among them) may lose 2^-22 of a number no larger than sum |a b|.  The activations come from
an exponential that is off by (2 + 1.2 |z|) 2^-23 of itself, so by (8 + 2 |z|) 2^-23 of the value; their slopes are below 1.2.
What the backward pass multiplies (dg, du) is rounded to the type, half a step of each; so is every result.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_1805_08768_b200 import binding as sbc

DEV = torch.device("cuda:0")
STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25}
HALF = [torch.bfloat16, torch.float16]


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def act64(g, act):
    """(value, slope) in 64 bits"""
    if act == "relu":
        return g.clamp(min=0), (g > 0).double()
    if act == "gelu":
        p = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (g + 0.044715 * g ** 3))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)
    s = torch.sigmoid(g)
    return (s, s * (1 - s)) if act == "sigmoid" else (g * s, s * (1 + g * (1 - s)))


def problem(tokens, inner, hidden, dtype, seed=1):
    g = gen(seed)
    x = torch.randn(tokens, inner, generator=g, device=DEV).to(dtype)
    gate, up = ((torch.randn(hidden, inner, generator=g, device=DEV) / inner ** 0.5).to(dtype) for _ in range(2))
    return x, gate, up, (torch.randn(tokens, hidden, generator=g, device=DEV) * 0.5).to(dtype)


def lost(length):
    return (length / 16 + 16) * 2.0 ** -22


def projections(x, gate, up, act):
    """g and u, what they may be off by, and act(g) and its slope with what those may"""
    xs, gs, us = x.double(), gate.double(), up.double()
    g, u = xs @ gs.t(), xs @ us.t()
    eg, eu = (lost(x.shape[1]) * (xs.abs() @ w.abs().t()) for w in (gs, us))
    value, slope = act64(g, act)
    rel = (8 + 2 * g.abs()) * 2.0 ** -23
    ev = 1.2 * eg + rel * value.abs() + 1e-37
    es = 1.0 * eg + rel * (1 + g.abs())      # (second derivatives of the smooth ones are below 1)
    return g, u, eg, eu, value, ev, slope, es


def check_forward(h, x, gate, up, act):
    g, u, eg, eu, value, ev, _, _ = projections(x, gate, up, act)
    want = value * u
    allowed = ev * u.abs() + eu * value.abs() + ev * eu + 2.0 ** -23 * want.abs() + STEP[h.dtype] * want.abs() + TINY[h.dtype]
    assert bool(((h.double() - want).abs() <= allowed).all())


def check_backward(dx, dgate, dup, dh, x, gate, up, act):
    g, u, eg, eu, value, ev, slope, es = projections(x, gate, up, act)
    d = dh.double()
    dg, du = d * u * slope, d * value
    step = STEP[x.dtype]
    tiny = TINY[x.dtype]
    eg = d.abs() * (u.abs() * es + eu * slope.abs() + eu * es) + step * dg.abs() + tiny
    eu = d.abs() * ev + step * du.abs() + tiny
    if act == "relu":   # the slope jumps: where g is nearer to 0 than it may be off by, it may be either
        near = g.abs() <= lost(x.shape[1]) * (x.double().abs() @ gate.double().abs().t())
        eg = torch.where(near, (d * u).abs() * 1.01, eg)
    ws = gate.double(), up.double()
    if dx is not None:
        want = dg @ ws[0] + du @ ws[1]
        size = (dg.abs() + eg) @ ws[0].abs() + (du.abs() + eu) @ ws[1].abs()
        allowed = eg @ ws[0].abs() + eu @ ws[1].abs() + lost(2 * gate.shape[0]) * size + STEP[dx.dtype] * want.abs() + TINY[dx.dtype]
        off = (dx.double() - want).abs()
        assert bool((off <= allowed).all())
        # two independent roundings, each at most a step, so about 1 / sqrt(3) of one: in the mean square not more than a step
        if want.numel() > 1000 and act != "relu":
            assert float(off.norm() / want.norm()) < 1.2 * step
    for got, e, ee in ((dgate, dg, eg), (dup, du, eu)):
        if got is None:
            continue
        want = e.t() @ x.double()
        allowed = ee.t() @ x.double().abs() + lost(x.shape[0]) * ((e.abs() + ee).t() @ x.double().abs()) + STEP[got.dtype] * want.abs() + TINY[got.dtype]
        off = (got.double() - want).abs()
        assert bool((off <= allowed).all())
        if want.numel() > 1000 and act != "relu":
            assert float(off.norm() / want.norm()) < 1.2 * step


SHAPES = [(1, 1, 1), (1, 650, 2600), (3, 17, 9), (8, 64, 128), (9, 100, 40), (16, 4096, 64), (31, 96, 257), (32, 33, 65), (33, 64, 64), (64, 8, 3),
          (127, 130, 200), (128, 128, 128), (129, 650, 300), (257, 256, 640), (700, 1300, 129), (35, 2600, 650)]


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("shape", SHAPES)
def test_gated(shape, dtype):
    x, gate, up, dh = problem(*shape, dtype)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    check_forward(sbc.sbc_gated(x, gate, up, status=status), x, gate, up, "silu")
    h, kept = sbc.sbc_gated(x, gate, up, keep=True, status=status)
    check_forward(h, x, gate, up, "silu")
    dx, dgate, dup = sbc.sbc_gated_grad(dh, x, gate, up, kept, status=status)
    assert dx.dtype == dgate.dtype == dup.dtype == dtype and dx.shape == x.shape and dgate.shape == gate.shape
    check_backward(dx, dgate, dup, dh, x, gate, up, "silu")
    assert int(status) == 0


@pytest.mark.parametrize("act", list(sbc.ACTIVATIONS))
@pytest.mark.parametrize("tokens", [5, 150])
def test_gated_activations(act, tokens):
    x, gate, up, dh = problem(tokens, 96, 200, torch.bfloat16)
    x *= 4   # far into both tails
    check_forward(sbc.sbc_gated(x, gate, up, act), x, gate, up, act)
    h, kept = sbc.sbc_gated(x, gate, up, act, keep=True)
    check_forward(h, x, gate, up, act)
    check_backward(*sbc.sbc_gated_grad(dh, x, gate, up, kept), dh, x, gate, up, act)


@pytest.mark.parametrize("act", list(sbc.ACTIVATIONS))
@pytest.mark.parametrize("tokens", [5, 150])
def test_gated_far_tails(act, tokens):
    """Projections of 1e13 and more, of either sign: the activations are what they tend to, and no gradient becomes a NaN."""
    x, gate, up, dh = problem(tokens, 64, 96, torch.bfloat16)
    x = x * 1e14
    up = up * 1e-14
    h, kept = sbc.sbc_gated(x, gate, up, act, keep=True)
    assert bool(torch.isfinite(h).all()) and bool(torch.isfinite(kept).all()) and bool(torch.isfinite(sbc.sbc_gated(x, gate, up, act)).all())
    g = x.double() @ gate.double().t()
    far = g.abs() > 1e12
    limit = torch.where(g > 0, 1.0 if act == "sigmoid" else g, 0.0)
    assert bool(((kept[:, :, 1].double() - limit).abs() <= 2.0 ** -15 * limit.abs())[far].all())
    assert all(bool(torch.isfinite(t).all()) for t in sbc.sbc_gated_grad(dh, x, gate, up, kept))


def test_gated_gradients_of_32_bits_and_parts():
    x, gate, up, dh = problem(300, 130, 260, torch.bfloat16)
    h, kept = sbc.sbc_gated(x, gate, up, keep=True)
    both = sbc.sbc_gated_grad(dh, x, gate, up, kept, grad_dtype=torch.float32)
    assert both[1].dtype == both[2].dtype == torch.float32
    check_backward(*both, dh, x, gate, up, "silu")
    only = sbc.sbc_gated_grad(dh, x, gate, up, kept, need_weights=False)
    assert torch.equal(only[0], both[0]) and only[1] is None
    rest = sbc.sbc_gated_grad(dh, x, gate, up, kept, need_input=False, grad_dtype=torch.float32)
    assert rest[0] is None and torch.equal(rest[1], both[1]) and torch.equal(rest[2], both[2])


def test_gated_gradient_against_differences():
    """The gradient of a random weighting of the outputs along random directions, against differences of the 64-bit block."""
    x, gate, up, dh = problem(70, 64, 96, torch.float16)
    h, kept = sbc.sbc_gated(x, gate, up, "gelu", keep=True)
    grads = sbc.sbc_gated_grad(dh, x, gate, up, kept, grad_dtype=torch.float32)

    def total(a, b, c):
        return float((act64(a @ b.t(), "gelu")[0] * (a @ c.t()) * dh.double()).sum())

    args = [t.double() for t in (x, gate, up)]
    for i in range(3):
        way = torch.randn(args[i].shape, generator=gen(9 + i), device=DEV, dtype=torch.float64)
        eps = 1e-4
        there, back = ([a + s * eps * way if j == i else a for j, a in enumerate(args)] for s in (1, -1))
        slope = (total(*there) - total(*back)) / (2 * eps)
        got = float((grads[i].double() * way).sum())
        # the rounding of dg and du, and of dx, half a step of each term; they have independent signs
        noise = 2 * STEP[torch.float16] * float((grads[i].double() * way).norm()) * 8
        assert abs(got - slope) <= noise + 1e-5 * abs(slope) + 1e-4


def strided(t, lead, gap):
    room = torch.full((t.shape[0] * (t.shape[1] + gap) + lead,), 7.0, device=DEV, dtype=t.dtype)
    view = room[lead:].view(t.shape[0], t.shape[1] + gap)[:, :t.shape[1]]
    view.copy_(t)
    return room, view


@pytest.mark.parametrize("tokens", [4, 20, 90])
@pytest.mark.parametrize("sizes", [(64, 80), (65, 33)])
def test_gated_of_any_rows(tokens, sizes):
    """Rows at any place and distance give the same numbers; nothing is written between the rows of a result."""
    x, gate, up, dh = problem(tokens, *sizes, torch.bfloat16)
    for leads in ((0, 8, 16), (1, 2, 3), (8, 1, 0)):
        (_, xs), (_, gs), (_, us) = (strided(t, lead, gap) for t, lead, gap in zip((x, gate, up), leads, (8, 3, 1)))
        room, out = strided(torch.zeros_like(dh), 3, 5)
        check_forward(sbc.sbc_gated(xs, gs, us, out=out), x, gate, up, "silu")
        inside = torch.zeros_like(room, dtype=torch.bool)
        inside[3:].view(tokens, dh.shape[1] + 5)[:, :dh.shape[1]] = True
        assert bool((room[~inside] == 7).all())
        h, kept = sbc.sbc_gated(xs, gs, us, keep=True, out=out)
        check_forward(h, x, gate, up, "silu")
        check_backward(*sbc.sbc_gated_grad(strided(dh, 1, 2)[1], xs, gs, us, kept), dh, x, gate, up, "silu")


@pytest.mark.parametrize("tokens", [7, 200])
def test_gated_tokens_apart(tokens):
    """What is not finite stays in its token's row."""
    x, gate, up, dh = problem(tokens, 72, 136, torch.bfloat16)
    want = sbc.sbc_gated(x, gate, up)
    bad = x.clone()
    bad[2, 5], bad[4, 0] = float("nan"), float("inf")
    got = sbc.sbc_gated(bad, gate, up)
    keep = [i for i in range(tokens) if i not in (2, 4)]
    assert torch.equal(got[keep], want[keep]) and bool(torch.isnan(got[2]).all()) and not bool(torch.isfinite(got[4]).any())


def test_gated_without_tokens():
    x, gate, up, _ = problem(4, 24, 40, torch.bfloat16)
    none = x[:0]
    h, kept = sbc.sbc_gated(none, gate, up, keep=True)
    assert h.shape == (0, 40)
    dx, dgate, dup = sbc.sbc_gated_grad(none.new_zeros(0, 40), none, gate, up, kept)
    assert dx.shape == (0, 24) and not dgate.any() and not dup.any()


def test_gated_repeats_its_bits_in_a_graph_and_on_a_stream():
    x, gate, up, dh = problem(300, 650, 520, torch.float16)
    few = x[:3]

    def step(stream=None):
        h, kept = sbc.sbc_gated(x, gate, up, keep=True, stream=stream)
        return (sbc.sbc_gated(few, gate, up, stream=stream), h) + sbc.sbc_gated_grad(dh, x, gate, up, kept, stream=stream)

    want = step()
    assert all(torch.equal(a, b) for a, b in zip(step(), want))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = step(stream)
    torch.cuda.current_stream().wait_stream(stream)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for t in got:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_gated_wide_and_long():
    """The kernel's many tiles of both kinds, tails in all axes: against 32-bit products of the same rounded numbers."""
    for tokens, inner, hidden in ((4100, 264, 2056), (9216, 512, 4608), (300, 4104, 264)):
        x, gate, up, dh = problem(tokens, inner, hidden, torch.bfloat16)
        h, kept = sbc.sbc_gated(x, gate, up, keep=True)
        check_forward(h, x, gate, up, "silu")
        check_backward(*sbc.sbc_gated_grad(dh, x, gate, up, kept), dh, x, gate, up, "silu")


def test_gated_refusals():
    x, gate, up, dh = problem(40, 24, 40, torch.bfloat16)
    h, kept = sbc.sbc_gated(x, gate, up, keep=True)
    for call, error in ((lambda: sbc.sbc_gated(x.float(), gate.float(), up.float()), TypeError), (lambda: sbc.sbc_gated(x, gate.half(), up), TypeError),
                        (lambda: sbc.sbc_gated(x, gate, up[:8]), ValueError), (lambda: sbc.sbc_gated(x[:, :8], gate, up), ValueError),
                        (lambda: sbc.sbc_gated(x, gate, up, "tanh"), ValueError), (lambda: sbc.sbc_gated(x, gate[:0], up[:0]), ValueError),
                        (lambda: sbc.sbc_gated(x, gate.t().contiguous().t(), up), ValueError), (lambda: sbc.sbc_gated(x, gate, up, out=h[:8]), ValueError),
                        (lambda: sbc.sbc_gated(x, gate, up, status=torch.zeros(1, device=DEV)), TypeError),
                        (lambda: sbc.sbc_gated_grad(dh[:8], x, gate, up, kept), ValueError), (lambda: sbc.sbc_gated_grad(dh, x, gate, up, kept[:8]), ValueError),
                        (lambda: sbc.sbc_gated_grad(dh, x, gate, up, kept.half()), TypeError),
                        (lambda: sbc.sbc_gated_grad(dh, x, gate, up, kept, grad_dtype=torch.float16), TypeError)):
        with pytest.raises(error):
            call()
