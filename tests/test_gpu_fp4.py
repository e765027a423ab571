"""4-bit floating point on the GPU against plain computations in 64 bits.

Quantised values are compared for equality: every rounding decision of the format is that of exact
arithmetic.  A product's tolerance follows from its sums: the products of two grid values and two
block scales are exact in 32 bits, each of the ceil(cols / 64) accumulations into the 32-bit sum
(and the adds inside the unit, counted as four more) may lose two bits more than a rounded addition
of numbers no larger than sum |a b|, and the result is rounded once to the output's type.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_1805_08768_b200 import binding as sbc

DEV = torch.device("cuda:0")
BLOCK = {"e8m0": 32, "e4m3": 16}
GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def nearest(y, table):
    """Entry of an ascending table nearest to y >= 0, the even index on a tie, the last one beyond it."""
    hi = torch.searchsorted(table, y.contiguous()).clamp(max=len(table) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = table[hi] - y, y - table[lo]
    take_hi = (up < down) | ((up == down) & (hi % 2 == 0)) | (y >= table[-1])
    return torch.where(take_hi, table[hi], table[lo])


def plain_round(x, fmt):
    """x as its 4-bit form along the rows stands for it, float64; blocks with a non-finite value are NaN."""
    x = x.double()
    rows, cols = x.shape
    size = BLOCK[fmt]
    x = torch.cat((x, x.new_zeros(rows, -cols % size)), 1).reshape(rows, -1, size)
    bad = ~torch.isfinite(x).all(2)
    clean = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
    amax = clean.abs().amax(2)
    log2 = torch.frexp(amax)[1] - 1
    if fmt == "e8m0":
        e = torch.where(amax > 0, log2 - 2, torch.full_like(log2, -127)).clamp(-127, 127)
        scale = torch.ldexp(torch.ones_like(amax), e)
    else:
        top = clean.abs().max()
        g = max(-126, math.frexp(float(top))[1] - 1 - 10) if float(top) > 0 else 0
        table = torch.arange(0, 127, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn).double()
        scale = nearest(amax / 6 / 2.0 ** g, table) * 2.0 ** g
    y = clean.abs() / torch.where(scale > 0, scale, torch.full_like(scale, math.inf))[:, :, None]
    out = torch.sign(clean) * nearest(y, GRID) * scale[:, :, None]
    out[bad] = math.nan
    return out.reshape(rows, -1)[:, :cols]


def same(got, want):
    """Equal, the wanted value taken to the result's type (beyond its largest number: infinity)."""
    want = want.to(got.dtype).double()
    return bool(((got.double() == want) | (torch.isnan(got) & torch.isnan(want))).all())


def values(rows, cols, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, device=DEV) * torch.exp(2 * torch.randn(1, cols, generator=g, device=DEV))
    return x.to(dtype)


SHAPES = [(1, 1), (1, 650), (3, 16), (5, 17), (2, 33), (127, 31), (128, 128), (129, 129), (35, 650), (300, 1300), (257, 4096),
          (1000, 2), (8, 10000)]


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", SHAPES)
def test_quantise_both_ways(shape, dtype, fmt):
    x = values(*shape, dtype, 1 + shape[0])
    q, q_t = sbc.sbc_fp4_quantise_both(x, fmt)
    assert same(sbc.sbc_fp4_dequantise(q), plain_round(x, fmt))
    assert same(sbc.sbc_fp4_dequantise(q_t), plain_round(x.t(), fmt))
    # one orientation at a time writes the same bytes
    one, other = sbc.sbc_fp4_quantise(x, fmt), sbc.sbc_fp4_quantise(x, fmt, transposed=True)
    for a, b in ((one, q), (other, q_t)):
        assert torch.equal(a.values, b.values) and torch.equal(a.scales, b.scales) and torch.equal(a.tensor_scale, b.tensor_scale)


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
@pytest.mark.parametrize("offset,extra", [(0, 8), (1, 0), (3, 5), (4, 4), (2, 2)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantise_strides_and_offsets(dtype, offset, extra, fmt):
    rows, cols = 67, 333
    room = values(1, offset + rows * (cols + extra) + 64, dtype, 5).view(-1)
    x = torch.as_strided(room, (rows, cols), (cols + extra, 1), offset)
    q, q_t = sbc.sbc_fp4_quantise_both(x, fmt)
    assert same(sbc.sbc_fp4_dequantise(q), plain_round(x, fmt))
    assert same(sbc.sbc_fp4_dequantise(q_t), plain_round(x.t(), fmt))
    # a strided output keeps what stands between its rows
    wide = torch.full((rows, cols + 7), 7.0, device=DEV)
    sbc.sbc_fp4_dequantise(q, out=wide[:, 3:3 + cols])
    assert same(wide[:, 3:3 + cols], plain_round(x, fmt))
    assert bool((wide[:, :3] == 7).all()) and bool((wide[:, 3 + cols:] == 7).all())


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
def test_every_midpoint_and_its_neighbours(fmt):
    """Blocks whose largest value fixes the scale, the others on and next to the grid's midpoints."""
    rows = []
    mids = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float32)
    for scale in [1.0, 1.125, 1.25, 1.375, 1.5, 1.625, 1.75, 1.875]:
        at = mids * scale                                     # exact
        row = torch.cat((at, torch.nextafter(at, torch.tensor(math.inf))))
        low = torch.nextafter(at, torch.tensor(-math.inf))
        rows.append(torch.cat((row, torch.tensor([6 * scale, -6 * scale]))))
        rows.append(torch.cat((-low, low, torch.tensor([6 * scale, 0.0]))))
    x = torch.stack(rows).to(DEV).repeat(1, 2)
    x = torch.cat((x, x * 2.0 ** -20, x * 2.0 ** 40 if fmt == "e8m0" else x * 4))
    assert same(sbc.sbc_fp4_dequantise(sbc.sbc_fp4_quantise(x, fmt)), plain_round(x, fmt))


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
def test_zeros_extremes_and_non_finite_blocks(fmt):
    x = torch.zeros(12, 96, device=DEV)
    x[1] = 1e-45
    x[2, 5] = 3e38
    x[3, 40:] = torch.linspace(-1e-40, 1e-40, 56, device=DEV)
    x[4, 3], x[4, 50] = math.inf, 1.0
    x[5, 70], x[5, 1] = math.nan, -2.0
    x[6] = -math.inf
    x[7] = 1.17549435e-38
    x[8, ::2], x[8, 1::2] = -0.0, 1e-3
    x[9] = torch.logspace(-44, 38, 96, device=DEV)
    x[10] = -3.4028234e38
    if fmt == "e4m3":      # keep g where the small rows still matter, too
        assert same(sbc.sbc_fp4_dequantise(sbc.sbc_fp4_quantise(x[:2].contiguous(), fmt)), plain_round(x[:2], fmt))
    assert same(sbc.sbc_fp4_dequantise(sbc.sbc_fp4_quantise(x, fmt)), plain_round(x, fmt))
    assert same(sbc.sbc_fp4_dequantise(sbc.sbc_fp4_quantise(x, fmt, transposed=True)), plain_round(x.t(), fmt))
    z = torch.zeros(3, 40, device=DEV)
    assert not bool(sbc.sbc_fp4_dequantise(sbc.sbc_fp4_quantise(z, fmt)).any())


def plain_product(a, b):
    a, b = sbc.sbc_fp4_dequantise(a).double(), sbc.sbc_fp4_dequantise(b).double()
    return a @ b.t(), a.abs() @ b.abs().t()


def check_product(got, a, b):
    want, size = plain_product(a, b)
    allowed = (math.ceil(a.cols / 64) + 4) * 2.0 ** -22 * size + ROUND[got.dtype] * want.abs() + 1e-30
    assert bool(((got.double() - want).abs() <= allowed).all()), float(((got.double() - want).abs() - allowed).max())


PRODUCTS = [(1, 650, 10000), (1, 64, 128), (16, 256, 128), (1, 1, 1), (3, 5, 7), (17, 65, 129), (2, 8192, 256), (35, 650, 1000),
            (128, 512, 128), (129, 513, 130), (255, 300, 257), (256, 256, 256), (257, 1000, 300), (700, 1300, 2600), (16, 4096, 4096),
            (513, 96, 33), (64, 2048, 1000), (5000, 300, 1024), (4097, 128, 9000), (129, 70, 5)]


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
@pytest.mark.parametrize("shape", PRODUCTS)
def test_product(shape, fmt):
    tokens, inner, outer = shape
    a = sbc.sbc_fp4_quantise(values(tokens, inner, torch.bfloat16, 3), fmt)
    b = sbc.sbc_fp4_quantise(values(outer, inner, torch.float32, 4), fmt)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for dtype in (torch.float32, torch.bfloat16):
        check_product(sbc.sbc_fp4_product(a, b, dtype, status=status), a, b)
    again = sbc.sbc_fp4_product(a, b, torch.float32)
    assert torch.equal(again, sbc.sbc_fp4_product(a, b, torch.float32))        # same sums every time
    assert int(status.item()) == 0


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
def test_product_with_exact_small_integers(fmt):
    """Grid values with scale one everywhere: sums are whole numbers of quarters and must be exact."""
    g = torch.Generator(device=DEV).manual_seed(11)
    table = torch.cat((GRID, -GRID)).float()
    x = table[torch.randint(0, 16, (40, 320), generator=g, device=DEV)]
    w = table[torch.randint(0, 16, (200, 320), generator=g, device=DEV)]
    x[:, ::16], w[:, ::16] = 6.0, 6.0
    a, b = sbc.sbc_fp4_quantise(x, fmt), sbc.sbc_fp4_quantise(w, fmt)
    assert torch.equal(sbc.sbc_fp4_dequantise(a), x)
    assert torch.equal(sbc.sbc_fp4_product(a, b, torch.float32).double(), x.double() @ w.double().t())


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
@pytest.mark.parametrize("tokens", [21, 201, 513])
@pytest.mark.parametrize("outer,stride,at", [(131, 140, 5), (130, 140, 5), (130, 140, 4), (130, 141, 4), (131, 142, 2)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_product_writes_only_its_output(fmt, tokens, outer, stride, at, dtype):
    """Odd and even row lengths, strides and offsets: where words of two results are stored, and where not."""
    a = sbc.sbc_fp4_quantise(values(tokens, 200, torch.bfloat16, 3) / 16, fmt)
    b = sbc.sbc_fp4_quantise(values(outer, 200, torch.float32, 4) / 16, fmt)
    room = torch.full((tokens + 2, stride), 7.0, device=DEV, dtype=dtype)
    out = room[1:tokens + 1, at:at + outer]
    sbc.sbc_fp4_product(a, b, out=out)
    check_product(out, a, b)
    inside = torch.zeros_like(room, dtype=torch.bool)
    inside[1:tokens + 1, at:at + outer] = True
    assert bool((room[~inside] == 7).all())


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
@pytest.mark.parametrize("tokens", [1, 40, 300])
def test_nan_blocks_reach_only_their_rows(fmt, tokens):
    x, w = values(tokens, 700, torch.float32, 3), values(140, 700, torch.float32, 4)
    x[tokens // 2, 100], w[77, 650] = math.nan, math.inf
    a, b = sbc.sbc_fp4_quantise(x, fmt), sbc.sbc_fp4_quantise(w, fmt)
    got = sbc.sbc_fp4_product(a, b, torch.float32)
    want = torch.zeros_like(got, dtype=torch.bool)
    want[tokens // 2], want[:, 77] = True, True
    assert torch.equal(torch.isnan(got), want)


def test_sizes_agree_with_the_library():
    for rows in (1, 127, 128, 129, 5000):
        for cols in (1, 31, 32, 33, 64, 65, 128, 129, 4097):
            for fmt, code in sbc.FP4_FORMATS.items():
                values, scales = sbc._fp4_sizes(rows, cols, fmt)
                assert values == rows * sbc.lib().sbc_fp4_row_bytes(cols)
                assert scales == sbc.lib().sbc_fp4_scale_bytes(rows, cols, code)
                assert sbc.lib().sbc_fp4_workspace_bytes(rows, cols, code) == sbc.FP4_WORKSPACE_BYTES
                q = sbc.Fp4Tensor.empty(rows, cols, fmt, DEV)
                assert q.values.shape == (rows, values // rows) and q.scales.numel() == scales and q.nbytes == values + scales + 4
                assert q.values.data_ptr() == q.desc.values and q.scales.data_ptr() == q.desc.scales
                assert q.tensor_scale.data_ptr() == q.desc.tensor_scale and q.tensor_scale.shape == (1,)


@pytest.mark.parametrize("shape", [(40, 800), (41, 799), (32768, 1), (300, 400)])
def test_the_tensor_scale_looks_at_every_element(shape):
    """On both sides of the size from which a kernel of its own finds the largest magnitude."""
    rows, cols = shape
    for r, c in ((0, 0), (rows - 1, cols - 1), (rows // 2, cols // 3)):
        x = torch.full(shape, 1.0, device=DEV)
        x[r, c] = -1000.0
        q = sbc.sbc_fp4_quantise(x, "e4m3")
        assert float(q.tensor_scale) == 0.5          # 2^(9 - 10)
        assert same(sbc.sbc_fp4_dequantise(q), plain_round(x, "e4m3"))


def test_refusals():
    x = values(4, 64, torch.float32, 1)
    with pytest.raises(TypeError):
        sbc.sbc_fp4_quantise(x.double())
    with pytest.raises(TypeError):
        sbc.sbc_fp4_quantise(x.cpu())
    with pytest.raises(TypeError):
        sbc.sbc_fp4_quantise(x[0])
    with pytest.raises(ValueError):
        sbc.sbc_fp4_quantise(x.t())
    with pytest.raises(ValueError):
        sbc.sbc_fp4_quantise(x, "e5m2")
    with pytest.raises(ValueError):
        sbc.sbc_fp4_quantise(x[:0])
    a, b = sbc.sbc_fp4_quantise(x, "e8m0"), sbc.sbc_fp4_quantise(x, "e4m3")
    with pytest.raises(ValueError):
        sbc.sbc_fp4_product(a, b)
    with pytest.raises(ValueError):
        sbc.sbc_fp4_product(a, sbc.sbc_fp4_quantise(values(4, 65, torch.float32, 1), "e8m0"))
    with pytest.raises(ValueError):
        sbc.sbc_fp4_product(a, a, out=torch.empty(3, 4, device=DEV))
    with pytest.raises(ValueError):
        sbc.Fp4Tensor(a.values[:3], a.scales, a.tensor_scale, 4, 64, "e8m0")
    with pytest.raises(TypeError):
        sbc.sbc_fp4_product(a, a, status=torch.zeros(1, device=DEV))
    with pytest.raises(ValueError):
        sbc.Fp4Tensor(a.values, a.scales[:-512], a.tensor_scale, 4, 64, "e8m0")


def test_work_on_another_stream():
    side = torch.cuda.Stream()
    x, w = values(33, 650, torch.bfloat16, 3), values(300, 650, torch.float32, 4)
    torch.cuda.synchronize()
    a, b = sbc.sbc_fp4_quantise(x, stream=side), sbc.sbc_fp4_quantise(w, stream=side)
    got = sbc.sbc_fp4_product(a, b, torch.float32, stream=side)
    side.synchronize()
    check_product(got, a, b)


def test_matrices_of_more_than_2_31_elements():
    """The last rows and columns of a long matrix come out as those of a matrix of their own."""
    rows, cols = 66000, 32800
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    for lo in range(0, rows, 6600):
        x[lo:lo + 6600] = torch.randn(6600, cols, generator=torch.Generator(device=DEV).manual_seed(lo), device=DEV)
    assert x.numel() > 2 ** 31
    q, q_t = sbc.sbc_fp4_quantise_both(x, "e8m0")
    out = sbc.sbc_fp4_dequantise(q, torch.bfloat16)
    assert same(out[-300:], plain_round(x[-300:], "e8m0")) and same(out[:10], plain_round(x[:10], "e8m0"))
    out_t = sbc.sbc_fp4_dequantise(q_t, torch.bfloat16)
    last = x[:, -40:].t().contiguous()
    assert same(out_t[-40:], plain_round(last, "e8m0"))
    del out, out_t, q_t
    x[rows - 1, cols - 1] = 4096.0        # the tensor's largest is its last element
    e = sbc.sbc_fp4_quantise(x, "e4m3")
    assert float(e.tensor_scale) == 4.0
    # a product whose result has more than 2^31 elements
    del x, e
    a = sbc.sbc_fp4_quantise(values(66000, 64, torch.bfloat16, 1) / 16, "e8m0")
    b = sbc.sbc_fp4_quantise(values(32800, 64, torch.bfloat16, 2) / 16, "e8m0")
    y = sbc.sbc_fp4_product(a, b, torch.bfloat16)
    tail = sbc.Fp4Tensor(a.values[65920:].contiguous(), a.scales[65920 // 128 * 512:].contiguous(), a.tensor_scale, 80, 64, "e8m0")
    check_product(y[65920:].contiguous(), tail, b)


def test_calls_in_a_graph():
    """A recorded sequence of calls runs again on new inputs."""
    x, w = values(200, 650, torch.bfloat16, 3), values(300, 650, torch.float32, 4)
    w4 = sbc.sbc_fp4_quantise(w, "e4m3")
    sbc.sbc_fp4_product(sbc.sbc_fp4_quantise(x, "e4m3"), w4, torch.float32)      # kernels loaded before the recording
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = sbc.sbc_fp4_product(sbc.sbc_fp4_quantise(x, "e4m3"), w4, torch.float32)
    for seed in (7, 8):
        x.copy_(values(200, 650, torch.bfloat16, seed))
        graph.replay()
        assert torch.equal(y, sbc.sbc_fp4_product(sbc.sbc_fp4_quantise(x, "e4m3"), w4, torch.float32))


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_row_of_the_largest_length(dtype, fmt):
    """2^31 - 1 columns, the largest a header's matrix has, expanded to rows at every kind of offset: its
    last blocks come out as those of a short row."""
    cols, tail = 2 ** 31 - 1, 32 * 20 - 1
    x = torch.ones(1, cols, dtype=dtype, device=DEV)
    x[0, -tail:] = values(1, tail, dtype, 6)[0].clamp(-64, 64)
    x[0, -1] = 448.0
    q = sbc.sbc_fp4_quantise(x, fmt)
    short = plain_round(x[:, -tail - 64:], fmt)       # holds the tensor's largest, so its tensor scale
    one, want = short[:, :64].to(dtype), short[:, 64:]
    del x
    room = torch.empty(cols + 16, dtype=dtype, device=DEV)
    for offset in (0, 1, 16 // dtype.itemsize - 1):
        room.fill_(7.0)
        out = room[offset:offset + cols].view(1, cols)
        sbc.sbc_fp4_dequantise(q, out=out)
        assert same(out[:, -tail:], want)
        assert torch.equal(out[:, :64], one) and bool((out[:, :-tail:2 ** 20 + 1] == one[0, 0]).all())
        assert bool((room[:offset] == 7).all()) and bool((room[offset + cols:] == 7).all())


SMALLEST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,inner,outer", [(1, 650, 300), (16, 8192, 300), (128, 300, 131), (129, 70, 130), (300, 4096, 300)])
@pytest.mark.parametrize("size_a,size_b", [(1e-20, 1e-20), (1e-21, 3e-18), (1e-30, 1e-10), (1e-36, 1.0), (1e-30, 1e25), (1e25, 1e-35), (1e18, 1e17),
                                           (1e30, 1e5)])
def test_product_of_tensor_scales_beyond_32_bits(size_a, size_b, tokens, inner, outer, dtype):
    """Tensor scales whose product alone is below the smallest or above the largest number; the result counts.
    Tolerance as above, and half of the smallest number for results that are not normal ones."""
    a = sbc.sbc_fp4_quantise(torch.randn(tokens, inner, generator=torch.Generator(device=DEV).manual_seed(5), device=DEV) * size_a, "e4m3")
    b = sbc.sbc_fp4_quantise(torch.randn(outer, inner, generator=torch.Generator(device=DEV).manual_seed(6), device=DEV) * size_b, "e4m3")
    want, size = plain_product(a, b)
    got = sbc.sbc_fp4_product(a, b, dtype)
    allowed = (math.ceil(inner / 64) + 4) * 2.0 ** -22 * size + ROUND[dtype] * want.abs() + SMALLEST[dtype] / 2
    assert bool(((got.double() - want).abs() <= allowed).all())
    assert bool(torch.isfinite(got).all()) and bool((got != 0).any())


@pytest.mark.parametrize("tokens", [3, 40, 300])
def test_huge_tensor_scales_and_rows_of_zeros(tokens):
    """One value near the type's largest on each side fixes the tensor scales; rows of zeros stay zeros, and so do
    products of rows that the scale rounds to zero."""
    x, w = torch.zeros(tokens, 200, device=DEV), torch.zeros(150, 200, device=DEV)
    x[1, 7], w[70, 9] = 2e38, -3e38                  # in different places: their product with everything is 0
    x[2, 100], w[3, 100] = 1.0, 1.0                  # far below the smallest block scale
    a, b = sbc.sbc_fp4_quantise(x, "e4m3"), sbc.sbc_fp4_quantise(w, "e4m3")
    assert float(a.tensor_scale) * float(b.tensor_scale) > 2.0 ** 200
    for dtype in (torch.float32, torch.bfloat16):
        assert not bool(sbc.sbc_fp4_product(a, b, dtype).any())
    x[1, 9] = 2e38                                   # now one result is beyond the largest number, the others are not
    got = sbc.sbc_fp4_product(sbc.sbc_fp4_quantise(x, "e4m3"), b, torch.float32)
    assert float(got[1, 70]) == -math.inf
    got[1, 70] = 0
    assert not bool(got.any())


@pytest.mark.parametrize("rows,cols,gap", [(16, 64, 64), (17, 64, 64), (512, 64, 64), (40, 650, 14), (32768, 1, 7)])
def test_the_tensor_scale_of_rows_with_gaps(rows, cols, gap):
    """Slices on both sides of the rule by which a kernel of its own finds the largest magnitude.  A slice may not take
    20 times what its copy takes (a block that walks all rows by itself takes hundreds of times as long)."""
    x = torch.full((rows, cols + gap), 5000.0, device=DEV)[:, :cols]
    x.fill_(1.0)
    x[rows - 1, cols - 1] = -1000.0
    q = sbc.sbc_fp4_quantise(x, "e4m3")
    assert float(q.tensor_scale) == 0.5
    assert same(sbc.sbc_fp4_dequantise(q), plain_round(x, "e4m3"))

    def least(t):
        times = []
        for _ in range(7):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            for _ in range(4):
                sbc.sbc_fp4_quantise(t, "e4m3")
            end.record()
            end.synchronize()
            times.append(start.elapsed_time(end))
        return min(times)

    assert least(x) <= 20 * least(x.contiguous())
