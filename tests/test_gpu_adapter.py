"""Low-rank adapters on the GPU against plain computations in 64 bits.

Tolerances.  Operands go into the products as bfloat16 terms that they are the exact sum of; where a result is 16 bits wide two
terms are taken, which leaves less than 2^-15 of a factor.  A running sum of n products takes at most n / 16 + 64 additions (of
blocks and warps, too); each loses at most 2^-22 of a number no larger than the sum of the magnitudes where the tensor cores add
to it, and 2^-24 where sums start from zero (adapters or tokens in 32 bits): there the products of one step of 32 still lose
2^-20 of that step's magnitudes, counted for each.  A result is rounded once, half a step of its type.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_1805_08768_b200 import binding as sbc

DEV = torch.device("cuda:0")
STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25}
KINDS = [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16),
         (torch.float16, torch.float32)]


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def problem(tokens, inner, outer, rank, count, kind, seed=1, ids=None):
    dtype, weights = kind
    g = gen(seed)
    x = torch.randn(tokens, inner, generator=g, device=DEV).to(dtype)
    base = torch.randn(tokens, outer, generator=g, device=DEV).to(dtype)
    dy = (torch.randn(tokens, outer, generator=g, device=DEV) / outer ** 0.5).to(dtype)
    down = (torch.randn(count, rank, inner, generator=g, device=DEV) / inner ** 0.5).to(weights)
    up = (torch.randn(count, rank, outer, generator=g, device=DEV) / rank ** 0.5).to(weights)
    if ids is None:
        ids = torch.randint(-1, count, (tokens,), generator=g, device=DEV, dtype=torch.int32)
    return x, base, dy, down, up, ids


def lost(length):
    return (length / 16 + 64) * 2.0 ** -22


def near(got, want, allowed):
    allowed = allowed + STEP[got.dtype] * want.abs() + TINY[got.dtype]
    assert bool(((got.double() - want).abs() <= allowed).all())


def expected(x, base, dy, dx_base, down, up, ids, scale):
    """For every result: (want, what it may be off by before its rounding)"""
    cut = 2.0 ** -15
    count, rank, inner = down.shape
    outer = up.shape[2]
    y, ey = base.double().clone(), torch.zeros(base.shape, dtype=torch.float64, device=DEV)
    dx, ex = dx_base.double().clone(), torch.zeros(dx_base.shape, dtype=torch.float64, device=DEV)
    dd, ed = (torch.zeros(down.shape, dtype=torch.float64, device=DEV) for _ in range(2))
    du, eu = (torch.zeros(up.shape, dtype=torch.float64, device=DEV) for _ in range(2))
    wide = x.dtype == torch.float32
    for i in range(count):
        k = torch.nonzero(ids == i)[:, 0]
        if not len(k):
            continue
        a, b, d, p = x[k].double(), dy[k].double(), down[i].double(), up[i].double()

        def into(v, f):
            return v @ f.t(), lost(inner if f is d else outer) * (v.abs() @ f.abs().t())

        def out(m, em, f, by):
            c = 0 if wide else 2 * cut
            return by * (m @ f), abs(by) * (em @ f.abs() + (lost(rank) + c) * ((m.abs() + em) @ f.abs()))

        m, em = into(a, d)
        w, ew = out(m, em, p, scale)
        y[k] += w
        ey[k] += ew
        n, en = into(b, p)
        n, en = scale * n, abs(scale) * en + 2.0 ** -23 * (scale * n).abs()
        w, ew = out(n, en, d, 1.0)
        dx[k] += w
        ex[k] += ew
        c = 0 if down.dtype == torch.float32 else 2 * cut
        dd[i] = n.t() @ a
        ed[i] = en.t() @ a.abs() + (lost(len(k)) + c) * ((n.abs() + en).t() @ a.abs())
        du[i] = scale * (m.t() @ b)
        eu[i] = abs(scale) * (em.t() @ b.abs() + (lost(len(k)) + c) * ((m.abs() + em).t() @ b.abs()))
    ey += 2.0 ** -23 * (y.abs() + base.double().abs())
    ex += 2.0 ** -23 * (dx.abs() + dx_base.double().abs())
    return (y, ey), (dx, ex), (dd, ed), (du, eu)


def check_all(x, base, dy, down, up, ids, scale=2.0, plan=None):
    dx_base = torch.randn(x.shape, generator=gen(77), device=DEV).to(x.dtype)
    y_of, dx_of, dd_of, du_of = expected(x, base, dy, dx_base, down, up, ids, scale)
    near(sbc.sbc_adapter(x, down, up, ids, scale, base, plan), *y_of)
    y, kept = sbc.sbc_adapter(x, down, up, ids, scale, base, plan, keep=True)
    near(y, *y_of)
    dx, dd, du = sbc.sbc_adapter_grad(dy, x, down, up, kept, scale, dx_base)
    assert dx.dtype == x.dtype and dd.dtype == down.dtype and du.dtype == up.dtype
    near(dx, *dx_of)
    near(dd, *dd_of)
    near(du, *du_of)
    none = (ids < 0) | (ids >= down.shape[0])
    assert torch.equal(y[none], base[none]) and torch.equal(dx[none], dx_base[none])
    return y, dx, dd, du


SHAPES = [(1, 1, 1, 1, 1), (1, 16, 24, 3, 2), (5, 650, 300, 8, 8), (64, 128, 128, 16, 64), (65, 33, 65, 17, 3), (130, 2600, 130, 4, 1), (200, 96, 1000, 64, 2),
          (333, 777, 129, 33, 5), (500, 256, 512, 100, 3), (100, 64, 264, 128, 2), (1000, 40, 70, 12, 300), (700, 1032, 520, 48, 7)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", SHAPES)
def test_adapter(shape, kind):
    check_all(*problem(*shape, kind))


@pytest.mark.parametrize("kind", [KINDS[1], KINDS[2]])
def test_adapter_long(kind):
    check_all(*problem(3000, 4096, 1024, 64, 3, kind))
    tokens = 4096
    ids = torch.arange(tokens, device=DEV, dtype=torch.int32) // 700 - 1      # requests one behind the other
    check_all(*problem(tokens, 264, 2056, 16, 5, kind, ids=ids))


@pytest.mark.parametrize("case", ["none", "one", "last", "alternating", "beyond"])
@pytest.mark.parametrize("tokens", [40, 300])
def test_adapter_ids(case, tokens):
    """Nobody has an adapter; all the same one; the last; two in turns; numbers that are no adapter's."""
    ids = {"none": torch.full((tokens,), -1), "one": torch.zeros(tokens), "last": torch.full((tokens,), 6), "alternating": torch.arange(tokens) % 2 * 5,
           "beyond": torch.arange(tokens) % 9}[case].to(DEV, torch.int32)
    args = problem(tokens, 72, 136, 8, 7, KINDS[1], ids=ids)
    x, base, dy, down, up, _ = args
    y, dx, dd, du = check_all(*args)
    present = set(ids.tolist())
    for i in range(7):
        if i not in present:
            assert not dd[i].any() and not du[i].any()
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    sbc.sbc_adapter(x, down, up, ids, 2.0, base, status=status)
    plan = sbc.sbc_adapter_plan(ids, 7, status=status)
    assert int(status) == (sbc.STATUS_RANGE if case == "beyond" else 0)
    check_all(*args, plan=plan)


@pytest.mark.parametrize("tokens,count", [(1, 1), (31, 3), (64, 1), (65, 2), (2000, 5), (2000, 1500), (40000, 33), (5000, 32768)])
def test_plan(tokens, count):
    """The plan's own words: every token once, an adapter's tokens one behind the other in the order they came, tiles of 64."""
    ids = torch.randint(-1, count + 1, (tokens,), generator=gen(1), device=DEV, dtype=torch.int32)
    plan = sbc.sbc_adapter_plan(ids, count)
    words = plan.room.view(torch.int32).cpu()
    most = tokens // 64 + min(count + 1, tokens)
    tiles = words[:4 * (1 + most)].view(-1, 4)
    offsets = words[4 * (1 + most):][:count + 2]
    order = words[4 * (1 + most) + count + 2:][:tokens].long()
    bins = torch.where((ids >= 0) & (ids < count), ids, torch.full_like(ids, count)).cpu().long()
    assert torch.equal(order, torch.sort(bins, stable=True)[1])
    numbers = torch.bincount(bins, minlength=count + 1)
    assert torch.equal(offsets.long(), torch.cat((torch.zeros(1, dtype=torch.long), numbers.cumsum(0))))
    want = [(b, int(offsets[b]) + i, min(64, int(n) - i)) for b, n in enumerate(numbers.tolist()) if n for i in range(0, n, 64)]
    assert int(tiles[0, 0]) == len(want) <= most
    assert [tuple(t[:3]) for t in tiles[1:1 + len(want)].tolist()] == want


def strided(t, lead, gap):
    room = torch.full((t.shape[0] * (t.shape[1] + gap) + lead,), 7.0, device=DEV, dtype=t.dtype)
    view = room[lead:].view(t.shape[0], t.shape[1] + gap)[:, :t.shape[1]]
    view.copy_(t)
    return room, view


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tokens,sizes", [(9, (64, 72)), (200, (64, 72)), (9, (65, 71)), (200, (65, 71))])
def test_adapter_of_any_rows(tokens, sizes, kind):
    """Rows at any place and distance; results over the base and between other data; nothing else is written."""
    x, base, dy, down, up, ids = problem(tokens, *sizes, 8, 3, kind)
    y_of, dx_of, dd_of, du_of = expected(x, base, dy, x, down, up, ids, 2.0)
    for lead, gap in ((0, 0), (1, 2), (2, 1), (3, 0), (8, 8)):
        (_, xs), (_, dys) = strided(x, lead, gap), strided(dy, lead, gap)
        room, out = strided(base, lead, gap)
        inside = torch.zeros_like(room, dtype=torch.bool)
        inside[lead:].view(tokens, base.shape[1] + gap)[:, :base.shape[1]] = True
        near(sbc.sbc_adapter(xs, down, up, ids, 2.0, out, out=out), *y_of)
        assert bool((room[~inside] == 7).all())
        out.copy_(base)
        y, kept = sbc.sbc_adapter(xs, down, up, ids, 2.0, out, keep=True, out=out)
        near(y, *y_of)
        assert bool((room[~inside] == 7).all())
        room, out = strided(x, lead, gap)
        dx, dd, du = sbc.sbc_adapter_grad(dys, xs, down, up, kept, 2.0, out, out=out)
        near(dx, *dx_of)
        near(dd, *dd_of)
        near(du, *du_of)
        inside = torch.zeros_like(room, dtype=torch.bool)
        inside[lead:].view(tokens, x.shape[1] + gap)[:, :x.shape[1]] = True
        assert bool((room[~inside] == 7).all())


@pytest.mark.parametrize("tokens", [10, 100])
def test_adapter_without_base_and_parts(tokens):
    x, base, dy, down, up, ids = problem(tokens, 72, 80, 8, 3, KINDS[2])
    zero, zero_x = torch.zeros_like(base), torch.zeros_like(x)
    want, kept = sbc.sbc_adapter(x, down, up, ids, 0.5, zero, keep=True)
    got, _ = sbc.sbc_adapter(x, down, up, ids, 0.5, keep=True)
    assert torch.equal(got, want)
    assert torch.equal(sbc.sbc_adapter(x, down, up, ids, 0.5), sbc.sbc_adapter(x, down, up, ids, 0.5, zero))
    all_of = sbc.sbc_adapter_grad(dy, x, down, up, kept, 0.5)
    assert torch.equal(all_of[0], sbc.sbc_adapter_grad(dy, x, down, up, kept, 0.5, zero_x)[0])
    one = sbc.sbc_adapter_grad(dy, x, down, up, kept, 0.5, need_adapters=False)
    two = sbc.sbc_adapter_grad(dy, x, down, up, kept, 0.5, need_input=False)
    assert torch.equal(one[0], all_of[0]) and one[1] is None and two[0] is None
    assert torch.equal(two[1], all_of[1]) and torch.equal(two[2], all_of[2])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tokens", [12, 150])
def test_adapter_tokens_apart(tokens, kind):
    """What is not finite in a token's rows stays in its own results and its own adapter's gradients."""
    ids = torch.arange(tokens, device=DEV, dtype=torch.int32) % 4
    x, base, dy, down, up, _ = problem(tokens, 72, 136, 8, 4, kind, ids=ids)

    def run(x, dy):
        y, kept = sbc.sbc_adapter(x, down, up, ids, 2.0, base, keep=True)
        return (sbc.sbc_adapter(x, down, up, ids, 2.0, base), y) + sbc.sbc_adapter_grad(dy, x, down, up, kept, 2.0)

    want = run(x, dy)
    bad_x, bad_dy = x.clone(), dy.clone()
    bad_x[5, 3], bad_dy[9, 7] = float("nan"), float("inf")        # adapter 1 both
    got = run(bad_x, bad_dy)
    keep = [i for i in range(tokens) if i not in (5, 9)]
    for a, b in zip(got[:3], want[:3]):
        assert torch.equal(a[keep], b[keep])
    assert bool(torch.isnan(got[0][5]).all()) and bool(torch.isnan(got[1][5]).all()) and torch.equal(got[1][9], want[1][9])
    for a, b in zip(got[3:], want[3:]):
        assert torch.equal(a[[0, 2, 3]], b[[0, 2, 3]]) and not bool(torch.isfinite(a[1]).all())


def test_adapter_large_numbers_in_32_bits():
    """Values up to the type's largest are cut into terms without becoming infinite."""
    x = torch.full((70, 32), 3.4028e38, device=DEV)
    x[:, 1:] = 0
    down = torch.full((1, 1, 32), 1.1754944e-38, device=DEV)
    up = torch.ones(1, 1, 48, device=DEV)
    ids = torch.zeros(70, dtype=torch.int32, device=DEV)
    y = sbc.sbc_adapter(x, down, up, ids)
    want = float(x[0, 0].double() * down[0, 0, 0].double())
    assert bool(((y.double() - want).abs() <= 2.0 ** -20 * want).all())


def test_adapter_without_tokens():
    x, base, dy, down, up, ids = problem(4, 24, 40, 8, 3, KINDS[1])
    y, kept = sbc.sbc_adapter(x[:0], down, up, ids[:0], 1.0, base[:0], keep=True)
    assert y.shape == (0, 40) and sbc.sbc_adapter(x[:0], down, up, ids[:0]).shape == (0, 40)
    dx, dd, du = sbc.sbc_adapter_grad(dy[:0], x[:0], down, up, kept)
    assert dx.shape == (0, 24) and not dd.any() and not du.any()


def test_adapter_gradient_against_differences():
    x, base, dy, down, up, ids = problem(90, 48, 56, 6, 3, KINDS[0])
    y, kept = sbc.sbc_adapter(x, down, up, ids, 1.5, base, keep=True)
    grads = sbc.sbc_adapter_grad(dy, x, down, up, kept, 1.5)

    def total(a, d, u):
        s = 0.0
        for i in range(3):
            k = torch.nonzero(ids == i)[:, 0]
            s += float(((1.5 * (a[k] @ d[i].t()) @ u[i]) * dy[k].double()).sum())
        return s

    args = [t.double() for t in (x, down, up)]
    for i in range(3):
        way = torch.randn(args[i].shape, generator=gen(9 + i), device=DEV, dtype=torch.float64)
        there, back = ([a + s * 1e-3 * way if j == i else a for j, a in enumerate(args)] for s in (1, -1))
        slope = (total(*there) - total(*back)) / 2e-3      # (linear in each: exact but for rounding)
        got = float((grads[i].double() * way).sum())
        assert abs(got - slope) <= 1e-5 * float((grads[i].double() * way).abs().sum())


@pytest.mark.parametrize("kind", [KINDS[0], KINDS[1]])
def test_adapter_repeats_its_bits_in_a_graph_and_on_a_stream(kind):
    x, base, dy, down, up, ids = problem(777, 136, 264, 16, 6, kind)

    def step(stream=None):
        y, kept = sbc.sbc_adapter(x, down, up, ids, 2.0, base, keep=True, stream=stream)
        few = sbc.sbc_adapter(x[:40], down, up, ids[:40], 2.0, base[:40], stream=stream)
        return (y, few) + sbc.sbc_adapter_grad(dy, x, down, up, kept, 2.0, x, stream=stream)

    want = step()
    for _ in range(3):
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
    perm = torch.randperm(777, generator=gen(5), device=DEV)
    x.copy_(x[perm])           # other tokens and adapters in the same places
    ids.copy_(ids[perm])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, step()))


def test_adapter_refusals():
    x, base, dy, down, up, ids = problem(80, 24, 40, 8, 3, KINDS[1])
    y, kept = sbc.sbc_adapter(x, down, up, ids, 1.0, base, keep=True)
    plan = sbc.sbc_adapter_plan(ids[:40], 3)
    for call, error in ((lambda: sbc.sbc_adapter(x, down.half(), up, ids), TypeError), (lambda: sbc.sbc_adapter(x, down.float(), up, ids), TypeError),
                        (lambda: sbc.sbc_adapter(x, down[0], up[0], ids), TypeError), (lambda: sbc.sbc_adapter(x, down[:, :4], up, ids), TypeError),
                        (lambda: sbc.sbc_adapter(x, down, up[:2], ids), ValueError), (lambda: sbc.sbc_adapter(x[:, :8], down, up, ids), ValueError),
                        (lambda: sbc.sbc_adapter(x, down, up, ids[:40]), ValueError), (lambda: sbc.sbc_adapter(x, down, up, ids.long()), TypeError),
                        (lambda: sbc.sbc_adapter(x, down, up, None), ValueError), (lambda: sbc.sbc_adapter(x, down, up, None, plan=plan), ValueError),
                        (lambda: sbc.sbc_adapter(x, down, up, ids, base=base[:4]), ValueError), (lambda: sbc.sbc_adapter(x, down, up, ids, base=base.float()), TypeError),
                        (lambda: sbc.sbc_adapter(x, down.new_zeros(3, 129, 24), up.new_zeros(3, 129, 40), ids), ValueError),
                        (lambda: sbc.sbc_adapter_plan(ids, 0), ValueError), (lambda: sbc.sbc_adapter_plan(ids.cpu(), 3), TypeError),
                        (lambda: sbc.sbc_adapter_grad(dy[:, :8], x, down, up, kept), ValueError),
                        (lambda: sbc.sbc_adapter_grad(dy, x, down[:2].contiguous(), up[:2].contiguous(), kept), ValueError),
                        (lambda: sbc.sbc_adapter_grad(dy, x, down, up, sbc.AdapterKept(kept.mid[:1], kept.plan)), TypeError)):
        with pytest.raises((error, ValueError) if error is TypeError else error):
            call()
