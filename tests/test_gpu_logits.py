"""Top logits and the distillation loss on the GPU against plain computations in 64 bits.

Selected values and indices are compared for equality.  Tolerances, derived beforehand (u = 2^-24):
  - a sum of cols exponentials relative to its largest: an exponential is off by 2^-22 plus u times
    its argument (terms with large arguments are small), a thread adds cols / 256 of them or fewer
    (rows in segments: fewer), partial sums meet in about 20 more steps: eps = (cols / 256 + 64) u
  - a logarithm's argument adds the rounding of numbers of the size L = max |logit| / temperature + log cols:
    delta = eps + 4 u L
  - loss: each outcome's term moves by at most p delta + (p + q) eps, and sum p = sum q = 1; cross
    entropy by 2 delta
  - gradient: every share (q, the teacher's, the label's) is off by its own size times 4 delta, the
    result is rounded once to the logits' type
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_1805_08768_b200 import binding as sbc

DEV = torch.device("cuda:0")
U = 2.0 ** -24
ROUND = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
INF = math.inf


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def logits(rows, cols, dtype, seed, scale=3.0, masked=0.0):
    g = gen(seed)
    z = torch.randn(rows, cols, generator=g, device=DEV) * scale
    if masked:
        z = z.masked_fill(torch.rand(rows, cols, generator=g, device=DEV) < masked, -INF)
    return z.to(dtype)


# ---- the largest logits ------------------------------------------------------------

def check_top(z, k, tau):
    values, indices, rest = sbc.sbc_top_logits(z, k, tau)
    # one NaN for all: torch sorts those with a sign bit elsewhere
    want, order = torch.sort(torch.where(torch.isnan(z), math.nan, z.double()), dim=1, descending=True, stable=True)
    assert values.dtype == torch.float32 and indices.dtype == torch.int32
    assert torch.equal(indices.long(), order[:, :k])
    assert bool(((values.double() == want[:, :k]) | (torch.isnan(values) & torch.isnan(want[:, :k]))).all())
    out = torch.logsumexp(want[:, k:] / tau, 1) if k < z.shape[1] else torch.full((z.shape[0],), -INF, device=DEV).double()
    finite = torch.isfinite(out)
    assert torch.equal(finite, torch.isfinite(rest)) and bool((rest[~finite].double().isnan() == out[~finite].isnan()).all())
    clean = torch.where(torch.isfinite(want), want, torch.zeros_like(want))
    size = clean.abs().amax(1) / tau + math.log(z.shape[1])
    allowed = (z.shape[1] / 256 + 64) * U + 4 * U * size
    assert bool(((rest.double() - out).abs() <= allowed)[finite].all()), float(((rest.double() - out).abs() - allowed)[finite].max())


TOPS = [(1, 1, 1), (3, 2, 1), (2, 2, 2), (5, 7, 3), (4, 8, 8), (3, 9, 4), (2, 63, 63), (2, 65, 17), (3, 255, 100), (3, 256, 256), (2, 257, 256),
        (2, 300, 256), (3, 1000, 1), (2, 1023, 200), (3, 2049, 256), (1, 4099, 64), (40, 5000, 30), (1, 10000, 32), (700, 10000, 64),
        (2, 50001, 128), (1, 131072, 256), (1, 262147, 5), (300, 20011, 128),
        (160, 131072, 256), (150, 110003, 1), (149, 102401, 40)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols,k", TOPS)
def test_top_logits(rows, cols, k, dtype):
    check_top(logits(rows, cols, dtype, rows + cols), k, 1.0 if cols % 2 else 2.5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols", [(3, 300), (2, 1000), (300, 10000), (3, 20000), (3, 40000), (1, 131072), (150, 110003)])
@pytest.mark.parametrize("k", [127, 129, 131, 201, 255])
def test_top_logits_of_odd_counts(rows, cols, k, dtype):
    """Lists of any length in front of the row that a block holds: one, two, four and eight blocks a row, and streamed."""
    check_top(logits(rows, cols, dtype, rows + k), k, 1.5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,k", [(3, 40, 7), (2, 700, 64), (1, 10000, 64), (320, 10000, 200), (2, 40000, 256), (148, 104003, 100)])
@pytest.mark.parametrize("kind", ["equal", "zeros", "few_values", "masked", "nearly_all_masked", "empty", "steps", "huge", "nan"])
def test_top_logits_ties_and_masks(kind, rows, cols, k, dtype):
    g = gen(7)
    if kind == "equal":
        z = torch.full((rows, cols), -1.25, device=DEV)
    elif kind == "zeros":
        z = torch.zeros(rows, cols, device=DEV)
        z[:, ::3] = -0.0
    elif kind == "few_values":
        z = torch.randint(-2, 3, (rows, cols), generator=g, device=DEV).float()
    elif kind == "masked":
        z = logits(rows, cols, torch.float32, 3, masked=0.5)
    elif kind == "nearly_all_masked":       # fewer values than are sent
        z = torch.full((rows, cols), -INF, device=DEV)
        z[:, cols // 3] = 2.0
        z[:, cols - 1] = -3.0
    elif kind == "empty":
        z = torch.full((rows, cols), -INF, device=DEV)
        z[0, 1] = 0.5
    elif kind == "steps":                   # ascending and descending runs: one thread's groups hold all the large ones
        z = torch.linspace(-4, 4, cols, device=DEV).repeat(rows, 1)
        z[0] = z[0].flip(0)
    elif kind == "huge":
        z = logits(rows, cols, torch.float32, 3) * 1e30
        z[:, 3] = 3e38
    else:
        z = logits(rows, cols, torch.float32, 3)
        z[0, cols // 2], z[0, 5] = math.nan, -math.nan
        z[-1, 2] = INF
    z = z.to(dtype)
    check_top(z, k, 1.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols,k", [(8, 40, 7), (8, 700, 64), (8, 3000, 33), (7, 40000, 200), (8, 450000, 5), (150, 110003, 100)])
def test_top_logits_with_infinities(rows, cols, k, dtype):
    """More infinities than are sent leave an infinite rest, a NaN that is left makes it a NaN."""
    z = logits(rows, cols, dtype, 3)
    places = torch.randperm(cols, generator=gen(8), device=DEV)
    z[0, places[:k + 1]] = INF
    z[1, places[:k]] = INF                       # all of them are sent
    z[2, places[:min(2 * k + 500, cols)]] = INF
    z[3] = INF
    z[4, places[:k]], z[4, places[k]] = math.nan, INF
    z[5, places[:k + 1]], z[5, places[k + 1]] = math.nan, INF
    z[6, places[:3]], z[6, places[3:k + 2]], z[6, places[k + 2:]] = math.nan, INF, -INF
    check_top(z, k, 2.0)
    rest = sbc.sbc_top_logits(z, k, 2.0)[2]
    want = torch.full((7,), INF, device=DEV)
    want[5] = math.nan
    assert bool(((rest[:7] == want) | (torch.isnan(rest[:7]) & torch.isnan(want)))[[0, 2, 3, 4, 5, 6]].all())
    assert bool(torch.isfinite(rest[1]))


def test_top_logits_strides_and_empty():
    room = logits(1, 200_000, torch.bfloat16, 9).view(-1)
    for offset, stride in ((1, 5003), (3, 5010), (0, 5001), (7, 6000)):
        check_top(torch.as_strided(room, (30, 5001), (stride, 1), offset), 40, 2.0)
    values, indices, rest = sbc.sbc_top_logits(torch.empty(0, 10, device=DEV), 3)
    assert values.shape == (0, 3) and indices.shape == (0, 3) and rest.shape == (0,)


# ---- distillation ------------------------------------------------------------------

def plain(z, values, indices, rest, tau, alpha, labels, grad_loss):
    """(loss, gradient by autograd, sizes that rounding errors go by), all float64."""
    z = z.double().clone()
    rows, cols = z.shape
    none = (z == -INF).all(1)
    z[none] = 0
    z.requires_grad_(True)
    used = indices >= 0
    index = indices.long().clamp(min=0)
    teacher = torch.where(used, values.double() / tau, torch.full_like(values, -INF).double())
    rest = torch.full((rows,), -INF, device=DEV).double() if rest is None else rest.double()
    teacher = torch.cat((teacher, rest[:, None]), 1)
    untaught = (teacher == -INF).all(1)
    p = torch.softmax(torch.where(untaught[:, None], torch.zeros_like(teacher), teacher), 1)
    sent = torch.zeros(rows, cols + 1, dtype=torch.bool, device=DEV).scatter_(1, torch.where(used, index, cols), True)[:, :cols]
    log_q = torch.log_softmax(z / tau, 1)
    others = torch.logsumexp(log_q.masked_fill(sent, -INF), 1) if not bool(sent.all()) else None
    outside = torch.full((rows,), -INF, device=DEV).double() if others is None else others
    pairs = torch.cat((log_q.gather(1, index), outside[:, None]), 1)
    kl = torch.where(p > 0, p * (torch.log(p) - torch.where(p > 0, pairs, torch.zeros_like(pairs))), torch.zeros_like(p)).sum(1)
    live = (~none & ~untaught).double()
    loss = alpha * tau * tau * torch.where(live > 0, kl, torch.zeros_like(kl))
    log_q1 = torch.log_softmax(z, 1)
    hot = torch.zeros_like(z)
    has = torch.zeros(rows, device=DEV).double()
    if labels is not None:
        has = ((labels >= 0) & ~none).double()
        word = labels.clamp(min=0)[:, None]
        hot = hot.scatter(1, word, 1.0) * has[:, None]
        loss = loss - (1 - alpha) * torch.where(has > 0, log_q1.gather(1, word)[:, 0], torch.zeros_like(has))
    g = torch.ones(rows, device=DEV).double() if grad_loss is None else grad_loss.double()
    (loss * g).sum().backward()
    with torch.no_grad():
        q = log_q.exp()
        target = torch.where(sent, torch.zeros_like(q), (log_q - outside[:, None]).exp() * p[:, -1:])
        target = torch.nan_to_num(target).scatter_add(1, index, torch.where(used, p[:, :-1], torch.zeros_like(p[:, :-1])))
        size = g.abs()[:, None] * (alpha * tau * (q + target) * live[:, None] + (1 - alpha) * has[:, None] * (log_q1.exp() + hot))
        grad = torch.where(none[:, None], torch.zeros_like(z), z.grad)
    return loss.detach(), grad, size


def check_distill(z, values, indices, rest, tau=1.0, alpha=1.0, labels=None, grad_loss=None):
    about = dict(rest=rest, temperature=tau, alpha=alpha, labels=labels)
    want, want_grad, size = plain(z, values, indices, rest, tau, alpha, labels, grad_loss)
    finite = torch.where(torch.isfinite(z.double()), z.double(), torch.zeros_like(z).double()).abs().amax()
    eps = (z.shape[1] / 256 + 64) * U
    big = float(finite) + float(values[torch.isfinite(values)].abs().max() if bool(torch.isfinite(values).any()) else 0)
    delta = eps + 4 * U * (big / min(tau, 1.0) + math.log(z.shape[1]) + 1)
    loss, stats = sbc.sbc_distill_loss(z, values, indices, **about)
    allowed = alpha * tau * tau * (2 * delta + 4 * eps) + (1 - alpha) * 2 * delta
    allowed = allowed + 8 * U * want.abs()
    assert bool(((loss.double() - want).abs() <= allowed).all()), float((loss.double() - want).abs().max())
    grad = sbc.sbc_distill_grad(z, values, indices, stats, grad_loss, **about)
    allowed = 4 * delta * size + ROUND[z.dtype] * want_grad.abs() + (1e-37 if z.dtype != torch.float16 else 2.0 ** -25)
    off = (grad.double() - want_grad).abs() - allowed
    assert bool((off <= 0).all()), float(off.max())
    # one call for both gives the same, also in the logits' place
    loss2, grad2 = sbc.sbc_distill_loss_grad(z, values, indices, grad_loss, **about)
    assert torch.equal(loss, loss2) and torch.equal(grad, grad2)
    place = z.clone()
    loss3, grad3 = sbc.sbc_distill_loss_grad(place, values, indices, grad_loss, out=place, **about)
    assert grad3.data_ptr() == place.data_ptr() and torch.equal(place, grad) and torch.equal(loss3, loss)
    place = z.clone()
    sbc.sbc_distill_grad(place, values, indices, stats, grad_loss, out=place, **about)
    assert torch.equal(place, grad)
    return loss, grad


def message(z, k, tau, seed, spread=1.0):
    teacher = z.float() + spread * torch.randn(z.shape, generator=gen(seed), device=DEV)
    return sbc.sbc_top_logits(teacher, k, tau)


DISTILLS = [(1, 1, 1), (2, 2, 1), (3, 7, 7), (3, 8, 2), (4, 9, 3), (2, 17, 16), (3, 64, 5), (2, 130, 256 // 4), (35, 1000, 32), (1, 10000, 32),
            (330, 10000, 64), (2, 50001, 128), (1, 131072, 200), (310, 20011, 17), (1, 4097, 256)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols,k", DISTILLS)
def test_distill(rows, cols, k, dtype):
    z = logits(rows, cols, dtype, cols)
    tau = [1.0, 2.0, 4.0, 0.7][(rows + cols) % 4]
    grad_loss = torch.rand(rows, generator=gen(2), device=DEV) - 0.2
    values, indices, rest = message(z, k, tau, 5)
    check_distill(z, values, indices, rest, tau, grad_loss=grad_loss)
    labels = torch.randint(-1, cols, (rows,), generator=gen(3), device=DEV)
    labels[0] = int(indices[0, 0])
    check_distill(z, values, indices, rest, tau, alpha=0.6, labels=labels, grad_loss=grad_loss)
    check_distill(z, values, indices, None, 1.0, alpha=0.25, labels=labels)
    check_distill(z, values, indices, None, tau, alpha=0.0, labels=labels)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,k", [(6, 50, 8), (4, 3000, 64), (1, 9000, 32), (400, 3001, 16)])
def test_distill_masks_and_empty_rows(rows, cols, k, dtype):
    z = logits(rows, cols, dtype, 11, masked=0.4)
    z[rows // 2] = -INF
    teacher = (z.float() + torch.randn(rows, cols, generator=gen(4), device=DEV))
    values, indices, rest = sbc.sbc_top_logits(teacher, k, 2.0)
    labels = indices[:, 0].long()
    labels[values[:, 0] == -INF] = -1
    for alpha, use in ((1.0, None), (0.5, labels)):
        for tau in (1.0, 2.0):
            loss, grad = check_distill(z, values, indices, rest, tau, alpha, use)
            assert float(loss[rows // 2]) == 0 and not bool(grad[rows // 2].any())
    # a teacher that says nothing: no divergence; labels still count
    quiet = values.clone()
    quiet[0] = -INF
    silence = rest.clone()
    silence[0] = -INF
    loss, grad = check_distill(z, quiet, indices, silence, 2.0)
    assert float(loss[0]) == 0 and not bool(grad[0].any())
    check_distill(z, quiet, indices, silence, 2.0, 0.5, labels)
    # slots that are not used
    some = indices.clone()
    some[:, 1::3] = -1
    check_distill(z, values, some, rest, 2.0)
    some[:] = -1
    check_distill(z, values, some, rest, 2.0, 0.5, labels)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_masks_of_the_types_lowest_value(dtype, tau):
    """Words ruled out by the lowest value instead of -inf; a row of nothing else is uniform."""
    low = torch.finfo(dtype).min
    z = logits(5, 900, dtype, 11)
    z[torch.rand(5, 900, generator=gen(1), device=DEV) < 0.5] = low
    z[2] = low
    check_top(z, 40, tau)
    values, indices, rest = sbc.sbc_top_logits(z, 40, tau)
    values = torch.where(values > low, values + torch.randn(5, 40, generator=gen(2), device=DEV), values)
    loss, grad = sbc.sbc_distill_loss_grad(z, values, indices, rest=rest, temperature=tau)
    # the uniform row: all distances are zero, so no size of a logit enters
    delta = (900 / 256 + 64 + 4 * 10) * U
    want, want_grad, _ = plain(z[2:3], values[2:3], indices[2:3], rest[2:3], tau, 1.0, None, None)
    assert abs(float(loss[2]) - float(want)) <= tau * tau * 6 * delta
    assert float((grad[2].double() - want_grad).abs().max()) <= 4 * delta + ROUND[dtype] * float(want_grad.abs().max())
    keep = torch.tensor([0, 1, 3, 4], device=DEV)
    alike = torch.where(z > low, z, -INF)[keep].contiguous()
    check_distill(alike, values[keep].contiguous(), indices[keep].contiguous(), rest[keep].contiguous(), tau)
    other, other_grad = sbc.sbc_distill_loss_grad(alike, values[keep].contiguous(), indices[keep].contiguous(), rest=rest[keep].contiguous(),
                                                  temperature=tau)
    assert torch.equal(loss[keep], other) and torch.equal(grad[keep], other_grad)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tau", [1.0, 2.0])
@pytest.mark.parametrize("rows,cols,k", [(6, 50, 8), (4, 3000, 64), (2, 40000, 32)])
def test_divergence_without_weight(rows, cols, k, tau, dtype):
    """alpha = 0 leaves the cross entropy alone, also where the student rules out what the teacher sent (an infinite
    divergence); a NaN among the logits still makes the row's loss NaN."""
    z = logits(rows, cols, dtype, 11)
    values, indices, rest = message(z, k, tau, 5)
    z.scatter_(1, indices[:, 1::2].long(), -INF)
    labels = z.argmax(1)
    labels[0] = -1
    about = dict(rest=rest, temperature=tau, alpha=0.0, labels=labels)
    x = z.double().requires_grad_(True)
    log_q = torch.log_softmax(x, 1)
    want = -log_q.gather(1, labels.clamp(min=0)[:, None])[:, 0] * (labels >= 0)
    (want_grad,) = torch.autograd.grad(want.sum(), x)
    size = (log_q.detach().exp() + torch.zeros_like(z).double().scatter(1, labels.clamp(min=0)[:, None], 1.0)) * (labels >= 0)[:, None]
    finite = torch.where(torch.isfinite(z), z.double().abs(), torch.zeros_like(z).double())
    delta = (cols / 256 + 64) * U + 4 * U * (float(finite.max()) + math.log(cols) + 1)
    loss, stats = sbc.sbc_distill_loss(z, values, indices, **about)
    assert bool(((loss.double() - want.detach()).abs() <= 2 * delta + 8 * U * want.detach().abs()).all()) and float(loss[0]) == 0
    for grad in (sbc.sbc_distill_grad(z, values, indices, stats, **about), sbc.sbc_distill_loss_grad(z, values, indices, **about)[1]):
        assert bool(((grad.double() - want_grad).abs() <= 4 * delta * size + ROUND[dtype] * want_grad.abs() + 1e-37).all())
    assert torch.equal(sbc.sbc_distill_loss_grad(z, values, indices, **about)[0], loss)
    z[rows - 1, int(indices[rows - 1, 0])] = math.nan
    again = sbc.sbc_distill_loss(z, values, indices, **about)[0]
    assert bool(torch.isnan(again[-1])) and torch.equal(again[:-1], loss[:-1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0])
@pytest.mark.parametrize("rows,cols,k", [(5, 900, 40), (2, 40000, 16)])
def test_one_side_of_the_types_lowest_value(rows, cols, k, tau, dtype):
    """A student whose words are all ruled out by the lowest value is uniform, whatever the teacher says; a teacher of
    lowest values is uniform over its words, whatever the student says.  All distances on that side are zero, so only
    the other side's logits enter the tolerance."""
    low = torch.finfo(dtype).min
    usual = logits(rows, cols, dtype, 11)
    values, indices, rest = message(usual, k, tau, 4)
    size = float(usual.double().abs().max()) + float(values.abs().max())
    delta = (cols / 256 + 64) * U + 4 * U * (size / min(tau, 1.0) + math.log(cols) + 1)
    lowest = torch.full_like(usual, low)
    quiet = torch.full_like(values, low)
    cases = [(lowest, values, rest), (lowest, values, None)]
    if tau >= 1.0:      # (beyond it the lowest value divided by the temperature is -inf: such a teacher says nothing)
        cases += [(usual, quiet, None), (lowest, quiet, None)]
    for z, v, r in cases:
        want, want_grad, parts = plain(z, v, indices, r, tau, 1.0, None, None)
        loss, grad = sbc.sbc_distill_loss_grad(z, v, indices, rest=r, temperature=tau)
        assert bool(((loss.double() - want).abs() <= tau * tau * 6 * delta + 8 * U * want.abs()).all()), (loss, want)
        tiny = 1e-37 if dtype != torch.float16 else 2.0 ** -25
        assert bool(((grad.double() - want_grad).abs() <= 4 * delta * parts + ROUND[dtype] * want_grad.abs() + tiny).all())
        again, stats = sbc.sbc_distill_loss(z, v, indices, r, tau)
        assert torch.equal(again, loss) and torch.equal(sbc.sbc_distill_grad(z, v, indices, stats, rest=r, temperature=tau), grad)


def test_distill_everything_sent_and_nothing_left():
    z = logits(5, 100, torch.float32, 3)
    values, indices, rest = message(z, 100, 1.0, 2)
    assert bool((rest == -INF).all())
    check_distill(z, values, indices, rest, 1.0)
    check_distill(z, values, indices, None, 2.0)


@pytest.mark.parametrize("cols,k", [(500, 10), (2000, 1000), (3000, 1024)])
def test_distill_many_words_in_any_order(cols, k):
    z = logits(7, cols, torch.float32, 3)
    indices = torch.stack([torch.randperm(cols, generator=gen(i), device=DEV)[:k] for i in range(7)]).to(torch.int32)
    values = z.gather(1, indices.long()) + torch.randn(7, k, generator=gen(8), device=DEV)
    check_distill(z, values, indices, torch.full((7,), 1.5, device=DEV), 1.5)


@pytest.mark.parametrize("shift", [-3000.0, 800.0])
def test_distill_large_logits(shift):
    z = logits(4, 600, torch.float32, 3) * 20 + shift
    values, indices, rest = message(z, 12, 1.0, 2, spread=30.0)
    check_distill(z, values, indices, rest, 1.0)
    check_distill(z, values, indices, rest, 3.0, 0.5, indices[:, 1].long().contiguous())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset,extra,out_offset", [(0, 0, 0), (1, 1, 1), (3, 5, 2), (8, 8, 4)])
def test_distill_strides(dtype, offset, extra, out_offset):
    rows, cols, k = 21, 1003, 16
    room = logits(1, offset + rows * (cols + extra) + 8, dtype, 2).view(-1)
    z = torch.as_strided(room, (rows, cols), (cols + extra, 1), offset)
    values, indices, rest = message(z.contiguous(), k, 1.0, 5)
    loss, grad = check_distill(z.contiguous(), values, indices, rest)
    wide = torch.full((rows, cols + 9), 7.0, device=DEV, dtype=dtype)
    out = wide[:, out_offset:out_offset + cols]
    loss2, _ = sbc.sbc_distill_loss_grad(z, values, indices, rest=rest, out=out)
    delta = ((cols / 256 + 64) + 4 * 30) * U          # rows are cut into vectors elsewhere: sums in another order
    assert bool(((loss2 - loss).abs() <= 4 * delta).all())
    assert bool(((out.double() - grad.double()).abs() <= 8 * delta + 2 * ROUND[dtype] * grad.double().abs()).all())
    assert bool((wide[:, :out_offset] == 7).all()) and bool((wide[:, out_offset + cols:] == 7).all())


def test_gradient_is_the_slope_of_the_loss():
    """Central differences along random directions of entries +-1.  With steps of 1/16 the cubic term of each
    of the log-sums is at most h^2 / 6 * 8 / tau^3 times its weight tau^2; the losses are off by 1e-5 at most."""
    rows, cols, k, tau, alpha, h = 6, 800, 20, 2.0, 0.5, 1 / 16
    z = logits(rows, cols, torch.float32, 3)
    values, indices, rest = message(z, k, tau, 2)
    labels = torch.randint(0, cols, (rows,), generator=gen(4), device=DEV)
    about = dict(rest=rest, temperature=tau, alpha=alpha, labels=labels)
    _, grad = sbc.sbc_distill_loss_grad(z, values, indices, **about)
    for seed in range(5):
        v = torch.sign(torch.randn(rows, cols, generator=gen(50 + seed), device=DEV))
        up, _ = sbc.sbc_distill_loss(z + h * v, values, indices, **about)
        down, _ = sbc.sbc_distill_loss(z - h * v, values, indices, **about)
        slope = (up.double() - down.double()) / (2 * h)
        allowed = h * h / 6 * 8 * (2 * alpha / tau + (1 - alpha)) + 1e-5 / h
        assert bool(((grad.double() * v).sum(1) - slope).abs().max() <= allowed)


def test_nan_and_infinity_stay_in_their_rows():
    z = logits(6, 700, torch.float32, 3)
    values, indices, rest = message(z, 16, 1.0, 2)
    bad = z.clone()
    bad[1, 400], bad[3, int(indices[3, 0])] = math.nan, INF
    loss, grad = sbc.sbc_distill_loss_grad(bad, values, indices, rest=rest)
    clean, clean_grad = sbc.sbc_distill_loss_grad(z, values, indices, rest=rest)
    rows = torch.tensor([False, True, False, True, False, False], device=DEV)
    assert torch.equal(torch.isnan(loss), rows) and torch.equal(torch.isnan(grad).any(1), rows)
    assert torch.equal(loss[~rows], clean[~rows]) and torch.equal(grad[~rows], clean_grad[~rows])


def test_words_beyond_the_vocabulary_are_reported():
    z = logits(3, 100, torch.float32, 3)
    values, indices, rest = message(z, 8, 1.0, 2)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    good, _ = sbc.sbc_distill_loss(z, values, indices, rest, status=status)
    assert int(status.item()) == 0
    wrong, ignored = indices.clone(), indices.clone()
    wrong[1, 3], ignored[1, 3] = 100, -1
    loss, _ = sbc.sbc_distill_loss(z, values, wrong, rest, status=status)
    assert int(status.item()) == sbc.STATUS_RANGE
    assert torch.equal(loss, sbc.sbc_distill_loss(z, values, ignored, rest)[0])
    status.zero_()
    labels = torch.tensor([5, 100, 7], device=DEV)
    loss, grad = sbc.sbc_distill_loss_grad(z, values, indices, rest=rest, alpha=0.5, labels=labels, status=status)
    assert int(status.item()) == sbc.STATUS_RANGE
    labels[1] = -1
    again, grad2 = sbc.sbc_distill_loss_grad(z, values, indices, rest=rest, alpha=0.5, labels=labels)
    assert torch.equal(loss, again) and torch.equal(grad, grad2)


def test_no_rows():
    z = torch.empty(0, 50, device=DEV)
    values, indices = torch.empty(0, 4, device=DEV), torch.empty(0, 4, dtype=torch.int32, device=DEV)
    loss, stats = sbc.sbc_distill_loss(z, values, indices)
    assert loss.shape == (0,) and stats.shape[0] == 0
    loss, grad = sbc.sbc_distill_loss_grad(z, values, indices)
    assert loss.shape == (0,) and grad.shape == (0, 50)


def test_refusals():
    z = logits(3, 100, torch.float32, 3)
    values, indices, rest = message(z, 8, 1.0, 2)
    for k in (0, 101, 257):
        with pytest.raises(ValueError):
            sbc.sbc_top_logits(z, k)
    for tau in (0.0, -1.0, math.nan):
        with pytest.raises(sbc.SbcError):
            sbc.sbc_top_logits(z, 3, tau)
        with pytest.raises(sbc.SbcError):
            sbc.sbc_distill_loss(z, values, indices, rest, temperature=tau)
    for alpha in (-0.1, 1.1, math.nan):
        with pytest.raises(sbc.SbcError):
            sbc.sbc_distill_loss(z, values, indices, rest, alpha=alpha)
    with pytest.raises(TypeError):
        sbc.sbc_distill_loss(z.double(), values, indices)
    with pytest.raises(TypeError):
        sbc.sbc_distill_loss(z, values, indices.long())
    with pytest.raises(TypeError):
        sbc.sbc_distill_loss(z, values, indices, labels=torch.zeros(3, device=DEV, dtype=torch.int32))
    with pytest.raises(ValueError):
        sbc.sbc_distill_loss(z, values[:2], indices[:2])
    with pytest.raises(ValueError):
        sbc.sbc_distill_loss(z, values, indices, rest[:2])
    with pytest.raises(ValueError):
        sbc.sbc_distill_loss_grad(z, values, indices, out=z.bfloat16())
    with pytest.raises(ValueError):
        sbc.sbc_distill_loss(z.t(), values, indices)


def test_work_on_another_stream():
    z = logits(40, 3000, torch.bfloat16, 3)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    values, indices, rest = sbc.sbc_top_logits(z, 16, 2.0, stream=side)
    loss, grad = sbc.sbc_distill_loss_grad(z, values, indices, rest=rest, temperature=2.0, stream=side)
    side.synchronize()
    again, grad2 = sbc.sbc_distill_loss_grad(z, values, indices, rest=rest, temperature=2.0)
    assert torch.equal(loss, again) and torch.equal(grad, grad2)


def test_logits_of_more_than_2_31_elements():
    """The last rows of a long matrix come out as those of a matrix of their own."""
    rows, cols, k = 33000, 66000, 20
    z = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    for lo in range(0, rows, 3300):
        z[lo:lo + 3300] = 3 * torch.randn(3300, cols, generator=gen(lo), device=DEV)
    assert z.numel() > 2 ** 31
    values, indices, rest = sbc.sbc_top_logits(z, k, 2.0)
    few = z[-200:].contiguous()
    part = sbc.sbc_top_logits(few, k, 2.0)
    assert torch.equal(values[-200:], part[0]) and torch.equal(indices[-200:], part[1])
    check_top(few[-3:], k, 2.0)
    values += torch.randn(values.shape, generator=gen(1), device=DEV)
    loss, stats = sbc.sbc_distill_loss(z, values, indices, rest, 2.0)
    grad = sbc.sbc_distill_grad(z, values, indices, stats, rest=rest, temperature=2.0)
    one, one_grad = sbc.sbc_distill_loss_grad(few, values[-200:].contiguous(), indices[-200:].contiguous(), rest=rest[-200:].contiguous(), temperature=2.0)
    want, want_grad, size = plain(few[-4:], values[-4:], indices[-4:], rest[-4:], 2.0, 1.0, None, None)
    delta = (cols / 256 + 64 + 4 * 40) * U
    assert bool(((loss[-4:] - want).abs() <= 4 * 10 * delta).all()) and bool(((loss[-200:] - one).abs() <= 4 * 10 * delta).all())
    allowed = 4 * delta * size + ROUND[z.dtype] * want_grad.abs() + 1e-37
    assert bool(((grad[-4:].double() - want_grad).abs() <= allowed).all())


def test_calls_in_a_graph():
    z = logits(64, 5000, torch.bfloat16, 3)
    run = lambda: sbc.sbc_distill_loss_grad(z, *sbc.sbc_top_logits(z, 16, 2.0)[:2], temperature=2.0)   # noqa: E731
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, grad = run()
    z.copy_(logits(64, 5000, torch.bfloat16, 9))
    graph.replay()
    again, grad2 = run()
    assert torch.equal(loss, again) and torch.equal(grad, grad2)
