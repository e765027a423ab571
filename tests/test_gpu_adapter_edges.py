"""Adapters of operands that are not finite: a batch with a plan and single tokens give what the definition gives.

Tolerances of what stays finite are those of test_gpu_adapter."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_1805_08768_b200 import binding as sbc
from test_gpu_adapter import DEV, KINDS, expected, gen, near, problem

INF, NAN = float("inf"), float("nan")


def alike(got, want, allowed):
    """NaNs and infinities of either sign in the same places, the others near."""
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.isposinf(), want.isposinf()) and torch.equal(got.isneginf(), want.isneginf())
    fine = want.isfinite()
    near(got[fine], want[fine], allowed[fine])


def spoilt(t, seed, parts, share=0.02, dtype=None):
    """A few values of t replaced; in place."""
    g = gen(seed)
    hit = torch.rand(t.shape, generator=g, device=DEV) < share
    which = torch.randint(0, len(parts), t.shape, generator=g, device=DEV)
    t.copy_(torch.where(hit, torch.tensor(parts, device=DEV, dtype=t.dtype)[which], t))


def check(x, base, dy, down, up, ids, scale=2.0):
    dx_base = torch.randn(x.shape, generator=gen(77), device=DEV).to(x.dtype)
    y_of, dx_of, dd_of, du_of = expected(x, base, dy, dx_base, down, up, ids, scale)
    y, kept = sbc.sbc_adapter(x, down, up, ids, scale, base, keep=True)
    alike(y, *y_of)
    alike(sbc.sbc_adapter(x, down, up, ids, scale, base), *y_of)
    for t in range(0, x.shape[0], 64):     # single tokens
        part = slice(t, t + 64)
        alike(sbc.sbc_adapter(x[part], down, up, ids[part], scale, base[part]), y_of[0][part], y_of[1][part])
    same = base.clone()
    assert torch.equal(sbc.sbc_adapter(x, down, up, ids, scale, same, out=same).nan_to_num(7.0), y.nan_to_num(7.0))
    dx, dd, du = sbc.sbc_adapter_grad(dy, x, down, up, kept, scale, dx_base)
    alike(dx, *dx_of)
    alike(dd, *dd_of)
    alike(du, *du_of)


SHAPES = [(130, 40, 72, 8, 3), (200, 37, 51, 5, 2), (300, 264, 520, 40, 4), (700, 1032, 520, 70, 2)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", SHAPES)
def test_infinite_inputs(shape, kind):
    """An infinity times a factor of few digits (whose lower terms are zeros) is an infinity; times a zero it is none."""
    x, base, dy, down, up, ids = problem(*shape, kind)
    tokens, inner, outer, rank, count = shape
    for t, s in ((down, 5), (up, 6)):      # few digits: halves and quarters; zeros in one adapter
        t.copy_((t * 4).round() / 4 + 0.25)
        spoilt(t[0], s, [0.0])
    x[3::7, 5] = INF
    x[4::9, inner - 1] = -INF
    dy[2::8, 1] = -INF
    dy[1::11, outer - 1] = INF
    check(x, base, dy, down, up, ids)


@pytest.mark.parametrize("kind", KINDS)
def test_infinite_factors_bases_and_nans(kind):
    x, base, dy, down, up, ids = problem(200, 72, 136, 8, 5, kind)
    down[0, 1, 3], down[1, 2, 71], up[0, 3, 5], up[2, 0, 135] = INF, -INF, -INF, NAN
    x[:, 3] = x[:, 3].round()              # zeros among what meets an infinite factor
    spoilt(base, 9, [INF, -INF, NAN])
    x[11, 0], dy[12, 3] = NAN, NAN
    check(x, base, dy, down, up, ids)


@pytest.mark.parametrize("kind", KINDS)
def test_nothing_is_finite(kind):
    """A step that has come apart altogether still ends, and says so everywhere."""
    x, base, dy, down, up, ids = problem(1000, 264, 520, 16, 3, kind)
    ids.clamp_(min=0)
    for value in (INF, NAN):
        x.fill_(value)
        dy.fill_(value)
        check(x, base, dy, down, up, ids)


def test_whole_operands_beside_small_terms():
    """A float32 factor so small that its first bfloat16 term is a zero still makes an infinity of one, and numbers of the type's
    end stay numbers."""
    x, base, dy, down, up, ids = problem(100, 24, 40, 4, 2, KINDS[0])
    down[:, 0, 2] = 1e-41
    x[5, 2], x[6, 3] = INF, 3e38
    ids[5] = ids[6] = 1
    down[1, :, 3] = 0.5
    up[1] = 2.0 ** -4
    check(x, base, dy, down, up, ids)


@pytest.mark.parametrize("kind", [KINDS[2], KINDS[4]])
def test_terms_at_their_largest(kind):
    """Two factors whose lower terms are as large as they can be, and a base that takes their product's larger part away: two terms
    of each and all of their products leave less than 2 x 2^-15 of it (both seconds' product alone is nearly 2^-14)."""
    tokens, inner, outer = 70, 24, 48
    v = 1 + 2.0 ** -7 - 2.0 ** -23
    x = torch.zeros(tokens, inner, device=DEV, dtype=kind[0])
    x[:, 3] = 1
    base = torch.full((tokens, outer), -1.0, device=DEV, dtype=kind[0])
    down, up = torch.zeros(1, 1, inner, device=DEV), torch.full((1, 1, outer), v, device=DEV)
    down[0, 0, 3] = v
    ids = torch.zeros(tokens, dtype=torch.int32, device=DEV)
    y_of = expected(x, base, base, torch.zeros_like(x), down, up, ids, 1.0)[0]
    near(sbc.sbc_adapter(x, down, up, ids, 1.0, base), *y_of)
    # the same on the way back: dy up^T is v, its product with down v^2
    dy = torch.zeros_like(base)
    dy[:, 5] = 1
    dx_base = torch.full_like(x, -1.0)
    _, kept = sbc.sbc_adapter(x, down, up, ids, 1.0, base, keep=True)
    dx_of = expected(x, base, dy, dx_base, down, up, ids, 1.0)[1]
    near(sbc.sbc_adapter_grad(dy, x, down, up, kept, 1.0, dx_base)[0], *dx_of)
