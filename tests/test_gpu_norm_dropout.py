"""Layer norm and dropout on the GPU against plain computations in 64 bits.

Tolerances (u = 2^-24).  A sum over a row of n values goes through at most S = n / 1024 + 64 roundings (up to 32
values in turn in a thread, then a tree; long rows: eight values a thread for each 8192).  So the mean is off by at most
S u mean|x|, a normalised value h by (that / sigma)(1 + |h|) + |h| (S + 12) u, and what is made of them as written below.
A sum over rows goes through at most rows / 148 + 45 roundings (rows of a group in turn, the groups of a block, sixteen
rows of blocks).  A result's rounding is half a step of its type.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_1805_08768_b200 import binding as sbc

DEV = torch.device("cuda:0")
U = 2.0 ** -24
STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def values(rows, cols, dtype, seed):
    g = gen(seed)
    return (torch.randn(rows, cols, generator=g, device=DEV) * 2 + torch.randn(rows, 1, generator=g, device=DEV)).to(dtype)


def norm_parts(x, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    sigma = (x.sub(mean).square().mean(1, keepdim=True) + eps).sqrt()
    h = (x - mean) / sigma
    s = x.shape[1] / 1024 + 64
    dh = s * U * x.abs().mean(1, keepdim=True) / sigma * (1 + h.abs()) + h.abs() * (s + 12) * U
    return h, sigma, dh


def check_forward(y, x, w, b, eps):
    h, _, dh = norm_parts(x, eps)
    w = torch.ones(x.shape[1], device=DEV, dtype=torch.float64) if w is None else w.double()
    b = torch.zeros(x.shape[1], device=DEV, dtype=torch.float64) if b is None else b.double()
    want = h * w + b
    allowed = dh * w.abs() + 2 * U * ((h * w).abs() + b.abs()) + STEP[y.dtype] * want.abs() + TINY[y.dtype]
    assert bool(((y.double() - want).abs() <= allowed).all())


def check_backward(dx, dw, db, dy, x, w, eps):
    rows, cols = x.shape
    h, sigma, dh = norm_parts(x, eps)
    d = dy.double()
    t = d if w is None else d * w.double()
    s = cols / 1024 + 64
    mean, dot = t.mean(1, keepdim=True), (t * h).mean(1, keepdim=True)
    if dx is not None:
        want = (t - mean - h * dot) / sigma
        d_dot = s * U * (t * h).abs().mean(1, keepdim=True) + (t.abs() * dh).mean(1, keepdim=True)
        inside = 5 * U * (t.abs() + mean.abs() + (h * dot).abs()) + s * U * t.abs().mean(1, keepdim=True) + dh * dot.abs() + h.abs() * d_dot + dh * d_dot
        rel = (s + 8) * U + s * U * x.double().abs().mean(1, keepdim=True) / sigma
        allowed = inside / sigma + rel * (t.abs() + mean.abs() + (h * dot).abs()) / sigma + STEP[dx.dtype] * want.abs() + TINY[dx.dtype]
        assert bool(((dx.double() - want).abs() <= allowed).all())
    depth = (rows / 148 + 45) * U
    for got, terms, off in ((dw, d * h, d.abs() * dh), (db, d, 0 * d)):
        want = terms.sum(0)
        allowed = depth * terms.abs().sum(0) + off.sum(0) + STEP[got.dtype] * want.abs() + TINY[got.dtype]
        assert bool(((got.double() - want).abs() <= allowed).all())


SHAPES = [(1, 1), (1, 8), (35, 650), (7, 9), (257, 33), (100, 2601), (8191, 130), (3, 4096), (600, 4096), (5, 8184), (5, 8185), (9, 16376), (9, 16377), (4, 40001), (2, 131072)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_layer_norm(shape, dtype):
    rows, cols = shape
    x, dy = values(rows, cols, dtype, 1), values(rows, cols, dtype, 2)
    for kind in {torch.float32, dtype}:
        w, b = (torch.randn(cols, generator=gen(s), device=DEV).to(kind) for s in (3, 4))
        y, stats = sbc.sbc_layer_norm(x, w, b, 1e-5)
        check_forward(y, x, w, b, 1e-5)
        dx, dw, db = sbc.sbc_layer_norm_grad(dy, x, stats, w)
        assert dx.dtype == dtype and dw.dtype == db.dtype == kind
        check_backward(dx, dw, db, dy, x, w, 1e-5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [8, 37, 651, 9000])
def test_layer_norm_without_weights_and_parts(cols, dtype):
    x, dy = values(50, cols, dtype, 1), values(50, cols, dtype, 2)
    y, stats = sbc.sbc_layer_norm(x, eps=1e-3)
    check_forward(y, x, None, None, 1e-3)
    b = torch.randn(cols, generator=gen(3), device=DEV)
    check_forward(sbc.sbc_layer_norm(x, None, b, 1e-3)[0], x, None, b, 1e-3)
    dx, dw, db = sbc.sbc_layer_norm_grad(dy, x, stats)
    check_backward(dx, dw, db, dy, x, None, 1e-3)
    only = sbc.sbc_layer_norm_grad(dy, x, stats, need_weights=False)
    assert torch.equal(only[0], dx) and only[1] is None and only[2] is None
    sums = sbc.sbc_layer_norm_grad(dy, x, stats, need_input=False)
    assert sums[0] is None and torch.equal(sums[1], dw) and torch.equal(sums[2], db)
    assert sbc.sbc_layer_norm_grad(dy, x, stats, weight_dtype=dtype)[1].dtype == dtype


def strided(t, lead, gap):
    """The same values in rows that begin `lead` elements behind a buffer's start, `gap` elements apart."""
    room = torch.full((t.shape[0] * (t.shape[1] + gap) + lead,), 77.0, device=DEV, dtype=t.dtype)
    view = room[lead:].view(t.shape[0], t.shape[1] + gap)[:, :t.shape[1]]
    view.copy_(t)
    return room, view


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [16, 75, 1300, 9001])
def test_layer_norm_of_any_rows(cols, dtype):
    """Rows at any place and distance; results go to rows at others, and nothing is written between them."""
    rows = 37
    x, dy = values(rows, cols, dtype, 1), values(rows, cols, dtype, 2)
    w, b = torch.randn(cols, generator=gen(3), device=DEV), torch.randn(cols, generator=gen(4), device=DEV)
    for (lead, gap), (lead2, gap2) in (((1, 5), (0, 0)), ((0, 3), (3, 3)), ((2, 1), (2, 1)), ((8, 8), (7, 4))):
        _, xs = strided(x, lead, gap)
        _, dys = strided(dy, lead2, gap2)
        room, out = strided(torch.zeros_like(x), lead2, gap2)
        y, stats = sbc.sbc_layer_norm(xs, w, b, out=out)
        check_forward(y, x, w, b, 1e-5)
        inside = torch.zeros_like(room, dtype=torch.bool)
        inside[lead2:].view(rows, cols + gap2)[:, :cols] = True
        assert bool((room[~inside] == 77).all())
        dx, dw, db = sbc.sbc_layer_norm_grad(dys, xs, stats, w, out=out)
        check_backward(dx, dw, db, dy, x, w, 1e-5)
        assert bool((room[~inside] == 77).all())


@pytest.mark.parametrize("cols", [64, 650, 20000])
def test_layer_norm_in_place(cols):
    x, dy = values(40, cols, torch.bfloat16, 1), values(40, cols, torch.bfloat16, 2)
    y, stats = sbc.sbc_layer_norm(x)
    dx, dw, db = sbc.sbc_layer_norm_grad(dy, x, stats)
    a = x.clone()
    assert torch.equal(sbc.sbc_layer_norm(a, out=a)[0], y) and torch.equal(a, y)
    for over in ("dy", "x"):
        t = {"dy": dy.clone(), "x": x.clone()}
        got = sbc.sbc_layer_norm_grad(t["dy"], t["x"], stats, out=t[over])
        assert torch.equal(got[0], dx) and torch.equal(got[1], dw) and torch.equal(got[2], db)


def test_layer_norm_rows_apart():
    """What is not finite stays in its row; a constant row is the bias; sums of large and small rows keep both."""
    x = values(9, 130, torch.float32, 1)
    y, _ = sbc.sbc_layer_norm(x)
    bad = x.clone()
    bad[3, 17], bad[5, 0] = float("nan"), float("inf")
    got, _ = sbc.sbc_layer_norm(bad)
    keep = [0, 1, 2, 4, 6, 7, 8]
    assert torch.equal(got[keep], y[keep]) and bool(torch.isnan(got[[3, 5]]).all())
    flat = torch.full((4, 1000), 3.7, device=DEV)
    b = torch.randn(1000, generator=gen(2), device=DEV)
    assert bool(((sbc.sbc_layer_norm(flat, None, b)[0] - b).abs() <= (1000 / 1024 + 64) * U * 3.7 / 1e-5 ** 0.5 + 1e-6).all())
    far = torch.randn(6, 4096, generator=gen(3), device=DEV) + 10000.0   # the mean is far above the deviations
    check_forward(sbc.sbc_layer_norm(far)[0], far, None, None, 1e-5)


def test_layer_norm_without_rows():
    x = torch.zeros(0, 24, device=DEV, dtype=torch.bfloat16)
    w = torch.randn(24, device=DEV)
    y, stats = sbc.sbc_layer_norm(x, w)
    dx, dw, db = sbc.sbc_layer_norm_grad(x, x, stats, w)
    assert y.shape == dx.shape == (0, 24) and not dw.any() and not db.any()


def test_layer_norm_repeats_its_bits():
    x, dy = values(3000, 650, torch.float32, 1), values(3000, 650, torch.float32, 2)
    _, stats = sbc.sbc_layer_norm(x)
    first = sbc.sbc_layer_norm_grad(dy, x, stats)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, sbc.sbc_layer_norm_grad(dy, x, stats)))


def test_layer_norm_beyond_31_bits():
    """More than 2^31 elements: the last rows are what they are alone."""
    rows, cols = 70000, 32768
    x = torch.empty(rows, cols, device=DEV, dtype=torch.bfloat16).normal_(generator=gen(1))
    y, stats = sbc.sbc_layer_norm(x)
    assert torch.equal(y[-5:], sbc.sbc_layer_norm(x[-5:])[0])
    dx, _, _ = sbc.sbc_layer_norm_grad(x, x, stats, need_weights=False, out=y)
    assert torch.equal(dx[-5:], sbc.sbc_layer_norm_grad(x[-5:], x[-5:], stats[-5:].contiguous(), need_weights=False)[0])


def test_layer_norm_refusals():
    x = values(4, 16, torch.bfloat16, 1)
    w = torch.ones(16, device=DEV)
    _, stats = sbc.sbc_layer_norm(x, w)
    for call, error in ((lambda: sbc.sbc_layer_norm(x.t()), ValueError), (lambda: sbc.sbc_layer_norm(x.double()), TypeError),
                        (lambda: sbc.sbc_layer_norm(x, w[:8]), ValueError), (lambda: sbc.sbc_layer_norm(x, w.half()), TypeError),
                        (lambda: sbc.sbc_layer_norm(x, w, w.bfloat16()), TypeError), (lambda: sbc.sbc_layer_norm(x, eps=-1.0), sbc.SbcError),
                        (lambda: sbc.sbc_layer_norm(x, out=x[:2]), ValueError), (lambda: sbc.sbc_layer_norm(x, out=x.float()), TypeError),
                        (lambda: sbc.sbc_layer_norm(x.expand(3, 4, 16)), TypeError), (lambda: sbc.sbc_layer_norm_grad(x[:3], x, stats, w), ValueError),
                        (lambda: sbc.sbc_layer_norm_grad(x.float(), x, stats, w), TypeError), (lambda: sbc.sbc_layer_norm_grad(x, x, stats[:2], w), ValueError),
                        (lambda: sbc.sbc_layer_norm_grad(x, x, stats, w, weight_dtype=torch.float16), TypeError),
                        (lambda: sbc.sbc_layer_norm(x[:, :0]), sbc.SbcError)):
        with pytest.raises(error):
            call()


# ---- dropout ------------------------------------------------------------------------

def philox(counter, key):
    """Philox-4x32-10 of uint32 words [..., 4] and [..., 2], in Python's numbers."""
    c, k = [int(v) for v in counter], [int(v) for v in key]
    for _ in range(10):
        p, q = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(q >> 32) ^ c[1] ^ k[0], q & 0xFFFFFFFF, (p >> 32) ^ c[3] ^ k[1], p & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(n, key, step, at, dropped):
    """Which of n elements are kept."""
    out = np.zeros((n + 7) // 8 * 8, dtype=bool)
    for b in range((n + 7) // 8):
        c = b + at
        words = philox((c & 0xFFFFFFFF, c >> 32, step & 0xFFFFFFFF, step >> 32), (key & 0xFFFFFFFF, key >> 32))
        for j in range(8):
            out[8 * b + j] = (words[j // 2] >> (16 * (j % 2)) & 0xFFFF) >= dropped
    return torch.from_numpy(out[:n]).to(DEV)


def test_philox_answers():
    """The published generator's known answers hold for the plain form that the kernel is compared with."""
    assert philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert philox((ones,) * 4, (ones,) * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert philox((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def rng_of(key, step):
    return torch.tensor([key, step], dtype=torch.int64, device=DEV)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1, 1), (1, 8), (3, 7), (35, 65), (16, 64), (2, 1003)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999, 1.0])
def test_dropout(shape, dtype, p):
    x, r = values(*shape, dtype, 1), values(*shape, dtype, 2)
    dropped = round(65536 * p)
    key, step, at = 0x1234567890ABCDEF, 0x500000007, (1 << 33) + 5
    keep = kept(x.numel(), key, step, at, dropped).view(shape)
    scale = 65536 / (65536 - dropped) if dropped < 65536 else 0.0
    for res in (None, r):
        y = sbc.sbc_dropout(x, p, rng_of(key, step), at, residual=res)
        base = torch.zeros_like(x) if res is None else res
        assert torch.equal(y[~keep], base[~keep])
        want = base.double() + x.double() * scale
        # the scale is off by u of itself, the sum and the type round once each
        allowed = U * (x.double() * scale).abs() + (U + STEP[dtype]) * want.abs() + TINY[dtype]
        assert bool(((y.double() - want).abs() <= allowed)[keep].all())


@pytest.mark.parametrize("dtype", TYPES)
def test_dropout_of_any_rows(dtype):
    """The numbers go by an element's place in the matrix, whatever the strides; results may be x or the residual."""
    rows, cols = 29, 51
    x, r = values(rows, cols, dtype, 1), values(rows, cols, dtype, 2)
    rng = rng_of(7, 9)
    want = sbc.sbc_dropout(x, 0.3, rng, 11, residual=r)
    plain = sbc.sbc_dropout(x, 0.3, rng, 11)
    for lead, gap in ((1, 0), (0, 5), (3, 2)):
        _, xs = strided(x, lead, gap)
        _, rs = strided(r, lead, 0)
        room, out = strided(torch.zeros_like(x), 2, 3)
        assert torch.equal(sbc.sbc_dropout(xs, 0.3, rng, 11, residual=rs, out=out), want)
        inside = torch.zeros_like(room, dtype=torch.bool)
        inside[2:].view(rows, cols + 3)[:, :cols] = True
        assert bool((room[~inside] == 77).all())
        a = xs.clone()
        assert torch.equal(sbc.sbc_dropout(a, 0.3, rng, 11, out=a), plain)
        assert torch.equal(sbc.sbc_dropout(xs, 0.3, rng, 11, residual=rs, out=rs), want)
    a = x.clone()
    assert torch.equal(sbc.sbc_dropout(a, 0.3, rng, 11, residual=r, out=a), want)


def test_dropout_numbers_are_a_step_s_own():
    """A matrix in parts draws what the whole draws; another step or key draws anew; the share that is kept is p's."""
    x = torch.ones(1000, 64, device=DEV)
    rng = rng_of(123, 0)
    whole = sbc.sbc_dropout(x, 0.25, rng)
    assert torch.equal(torch.cat([sbc.sbc_dropout(x[:400], 0.25, rng, 0), sbc.sbc_dropout(x[400:], 0.25, rng, 400 * 8)]), whole)
    share = float((whole > 0).float().mean())
    assert abs(share - 0.75) < 6 * (0.75 * 0.25 / x.numel()) ** 0.5
    for other in (rng_of(123, 1), rng_of(124, 0)):
        both = ((sbc.sbc_dropout(x, 0.25, other) > 0) & (whole > 0)).float().mean()
        assert abs(float(both) - 0.75 ** 2) < 6 * (0.5625 * 0.4375 / x.numel()) ** 0.5


def test_dropped_infinities_do_not_count():
    x = torch.full((64, 64), float("inf"), device=DEV)
    x[::2] = float("nan")
    r = values(64, 64, torch.float32, 1)
    rng = rng_of(5, 6)
    keep = kept(x.numel(), 5, 6, 0, 32768).view(64, 64)
    y = sbc.sbc_dropout(x, 0.5, rng, residual=r)
    assert torch.equal(y[~keep], r[~keep]) and not bool(torch.isfinite(y[keep]).any())


def test_dropout_captured_draws_anew():
    x = values(64, 640, torch.bfloat16, 1)
    rng = rng_of(99, 0)
    out = torch.empty_like(x)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        sbc.sbc_dropout(x, 0.5, rng, out=out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            rng[1:].add_(1)
            sbc.sbc_dropout(x, 0.5, rng, out=out)
    rng[1] = 0
    seen = []
    for step in (1, 2, 3):
        graph.replay()
        torch.cuda.synchronize()
        assert int(rng[1]) == step
        seen.append(out.clone())
        assert torch.equal(out, sbc.sbc_dropout(x, 0.5, rng_of(99, step)))
    assert not torch.equal(seen[0], seen[1])


def test_dropout_beyond_31_bits():
    rows, cols = 66000, 32768
    x = torch.ones(rows, cols, device=DEV, dtype=torch.bfloat16)
    rng = rng_of(3, 4)
    y = sbc.sbc_dropout(x, 0.5, rng, out=x)
    tail = torch.ones(3, cols, device=DEV, dtype=torch.bfloat16)
    assert torch.equal(y[-3:], sbc.sbc_dropout(tail, 0.5, rng, (rows - 3) * cols // 8))


def test_dropout_on_another_stream():
    x = values(512, 640, torch.float32, 1)
    rng = rng_of(1, 2)
    want = sbc.sbc_dropout(x, 0.5, rng)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = sbc.sbc_dropout(x, 0.5, rng, stream=stream)
    y, stats = sbc.sbc_layer_norm(x, stream=stream)
    dx, dw, db = sbc.sbc_layer_norm_grad(x, x, stats, stream=stream)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(got, want)
    y0, stats0 = sbc.sbc_layer_norm(x)
    assert torch.equal(y, y0) and all(torch.equal(a, b) for a, b in zip((dx, dw, db), sbc.sbc_layer_norm_grad(x, x, stats0)))


def test_dropout_refusals():
    x = values(4, 16, torch.bfloat16, 1)
    rng = rng_of(1, 2)
    for call, error in ((lambda: sbc.sbc_dropout(x, 1.5, rng), ValueError), (lambda: sbc.sbc_dropout(x, float("nan"), rng), ValueError),
                        (lambda: sbc.sbc_dropout(x, 0.5, rng[:1]), ValueError), (lambda: sbc.sbc_dropout(x, 0.5, rng.int()), TypeError),
                        (lambda: sbc.sbc_dropout(x, 0.5, rng.cpu()), TypeError), (lambda: sbc.sbc_dropout(x, 0.5, rng, -1), ValueError),
                        (lambda: sbc.sbc_dropout(x, 0.5, rng, residual=x.float()), TypeError), (lambda: sbc.sbc_dropout(x, 0.5, rng, residual=x[:2]), ValueError),
                        (lambda: sbc.sbc_dropout(x.t(), 0.5, rng), ValueError), (lambda: sbc.sbc_dropout(x, 0.5, rng, out=x[:, :8]), ValueError)):
        with pytest.raises(error):
            call()
