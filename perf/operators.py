"""What the operators of distilled training are measured on.

A client of a distributed training round gets the weights in 4 bits, multiplies with them as they
are, learns from the few largest logits that a teacher sends for each position, and hands its own
weight update to the sparse binary encoder.  The operators are

  top      the k largest logits of every row, and the logarithm of the mass of all the others
  distill  the divergence of a student's softmax from such a row (and a label's cross entropy),
           forward, backward, and both in one call
  quantise values to 4-bit floating point with a scale per block, along the rows or both ways
  product  out = A B^T of two tensors held in 4 bits; with the quantisation of the activations,
           and as a training step (output, gradient of the input, gradient of the weights)

``run`` makes the plain computation in 32 bits, or, where ``own`` is set, the package's calls.

The 4-bit layout (both sides are handed the same bytes): element i of a row is nibble i % 2 (low
one first) of byte i // 2, rows are a multiple of 16 bytes apart; nibble = sign * 8 + index into
0, 0.5, 1, 1.5, 2, 3, 4, 6.  The scale of row r, block b is byte (r % 32) * 16 + (r % 128 // 32) * 4
+ b % 4 of tile (r // 128, b // 4), 512 bytes each.  Format "e8m0" has a power of two for 32 elements,
format "e4m3" an 8-bit float for 16 elements and a power of two for the whole tensor.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = {"e8m0": 32, "e4m3": 16}


def listed():
    return [
        # one answer of a teacher: a single position over the word model's vocabulary; latency
        dict(name="top_one_row", kind="top", rows=1, cols=10000, k=32, dtype="f32", tau=1.0, masked=False),
        # a batch of 64 sentences of 35 words, some words ruled out, positions without any word left
        dict(name="top_word_batch", kind="top", rows=2240, cols=10000, k=64, dtype="bf16", tau=2.0, masked=True),
        # the largest vocabulary, a message with many logits
        dict(name="top_wide", kind="top", rows=2048, cols=131072, k=128, dtype="bf16", tau=1.0, masked=False),
        # one sentence of one client: loss and gradient in one call, labels mixed in; latency
        dict(name="distill_sentence", kind="distill", rows=35, cols=10000, k=32, dtype="f32", tau=2.0, alpha=0.5,
             calls=1, masked=False),
        # a client's batch over the word model's vocabulary, ruled-out words and empty positions
        dict(name="distill_word_batch", kind="distill", rows=4480, cols=10000, k=64, dtype="bf16", tau=2.0, alpha=1.0,
             calls=1, masked=True),
        # forward and backward as two calls (autograd's order); an odd vocabulary, so rows start at odd places
        dict(name="distill_wide_two_calls", kind="distill", rows=4095, cols=50001, k=128, dtype="bf16", tau=1.0,
             alpha=0.7, calls=2, masked=False),
        # the word model's embedding as the server sends it: to 4 bits, and expanded by the client
        dict(name="quantise_embedding", kind="quantise", rows=10000, cols=650, dtype="f32", format="e4m3", both=False),
        # the activations of a long batch, along the rows for the forward product, along the columns for the backward one
        dict(name="quantise_activations", kind="quantise", rows=16384, cols=4096, dtype="bf16", format="e8m0", both=True),
        # one token's logits of the word model: 650 hidden units (no multiple of a block), 10000 words; latency
        dict(name="product_one_token", kind="product", tokens=1, inner=650, outer=10000, format="e4m3", dtype="bf16",
             step=False),
        # sixteen tokens through a large layer: the weights' bytes count
        dict(name="product_few_tokens", kind="product", tokens=16, inner=8192, outer=8192, format="e8m0", dtype="bf16",
             step=False),
        # a training step of the word model's gates: output, input gradient, weight gradient
        dict(name="product_gates_step", kind="product", tokens=2240, inner=1300, outer=2600, format="e8m0", dtype="bf16",
             step=True),
        # a large layer over a long batch: arithmetic counts
        dict(name="product_large", kind="product", tokens=8192, inner=8192, outer=8192, format="e4m3", dtype="bf16",
             step=False),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["top", "distill", "quantise", "product"])
    if kind in ("top", "distill"):
        cols = _spread(rng, 64, 131072)
        rows = _spread(rng, 1, min(8192, (1 << 27) // cols))
        case = dict(kind=kind, rows=rows, cols=cols, k=min(cols, _spread(rng, 1, 256)), dtype=rng.choice(["f32", "bf16"]),
                    tau=rng.choice([1.0, 2.0, 4.0]), masked=rng.random() < 0.4)
        if kind == "distill":
            case.update(alpha=rng.choice([1.0, 0.9, 0.5]), calls=rng.choice([1, 2]))
        return case
    if kind == "quantise":
        cols = _spread(rng, 1, 16384)
        return dict(kind=kind, rows=_spread(rng, 1, min(65536, (1 << 26) // cols)), cols=cols, dtype=rng.choice(["f32", "bf16"]),
                    format=rng.choice(["e8m0", "e4m3"]), both=rng.random() < 0.5)
    step = rng.random() < 0.35
    inner, outer = _spread(rng, 16, 8192), _spread(rng, 16, 16384)
    most = int(1.0e12 / (2.0 * inner * outer * (3 if step else 1)))
    return dict(kind=kind, tokens=_spread(rng, 1, max(1, min(8192, most))), inner=inner, outer=outer,
                format=rng.choice(["e8m0", "e4m3"]), dtype=rng.choice(["f32", "bf16"]), step=step)


# ---- inputs -----------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)


def _logits(case, g):
    """Logits over a vocabulary whose words differ in frequency (rank to the -1), float32."""
    rows, cols = case["rows"], case["cols"]
    rank = torch.randperm(cols, generator=g, device="cuda").float()
    z = torch.randn(rows, cols, generator=g, device="cuda").mul_(2.0).sub_(torch.log1p(rank))
    if case["masked"]:
        gone = torch.rand(rows, cols, generator=g, device="cuda") < 0.3
        gone |= (torch.rand(rows, 1, generator=g, device="cuda") < 0.02)
        z.masked_fill_(gone, -math.inf)
    return z


def _activations(rows, cols, g):
    """Values whose columns differ in size, a few of them by a lot."""
    size = torch.exp(0.5 * torch.randn(cols, generator=g, device="cuda"))
    size = torch.where(torch.rand(cols, generator=g, device="cuda") < 0.01, size * 20, size)
    return torch.randn(rows, cols, generator=g, device="cuda") * size


def prepare(case, seed):
    g = _generator(seed)
    dtype = DTYPES[case["dtype"]]
    state = dict(case=dict(case))
    if case["kind"] == "top":
        state["logits"] = _logits(case, g).to(dtype)
    elif case["kind"] == "distill":
        z = _logits(case, g)
        teacher = z + 1.5 * torch.randn(z.shape, generator=g, device="cuda")
        state["logits"] = z.to(dtype)
        del z
        values, indices = teacher.topk(case["k"], dim=1)
        state["values"], state["indices"] = values, indices.to(torch.int32)
        state["rest"] = torch.logsumexp(teacher.scatter_(1, indices, -math.inf).div_(case["tau"]), 1)
        del teacher
        label = indices[:, 0].masked_fill(torch.rand(case["rows"], generator=g, device="cuda") < 0.1, -1)
        label = label.masked_fill(values[:, 0] == -math.inf, -1)
        state["labels"] = label if case["alpha"] < 1 else None
        used = (torch.rand(case["rows"], generator=g, device="cuda") < 0.95).float()
        state["grad_loss"] = used / case["rows"]
    elif case["kind"] == "quantise":
        state["x"] = _activations(case["rows"], case["cols"], g).to(dtype)
    else:
        tokens, inner, outer = case["tokens"], case["inner"], case["outer"]
        state["x"] = _activations(tokens, inner, g).to(dtype)
        w = torch.randn(outer, inner, generator=g, device="cuda") / inner ** 0.5
        if case["step"]:   # a step quantises its weights anew, they change every time
            state["w"] = w
            state["dy"] = (torch.randn(tokens, outer, generator=g, device="cuda") / tokens
                           * torch.exp(torch.randn(tokens, 1, generator=g, device="cuda"))).to(dtype)
        else:              # the weights as they came from the server: in 4 bits
            state["w4"] = _pack(w, case["format"])
    return state


# ---- the plain form -----------------------------------------------------------------

def _power(e):
    """2**e as float32 for whole e in [-149, 127], by its bits."""
    e = e.to(torch.int32)
    bits = torch.where(e >= -126, (e + 127) << 23, torch.ones_like(e) << (e + 149).clamp(0, 22))
    return bits.view(torch.float32)


def _exponent(x):
    """floor(log2(x)) of positive float32."""
    return torch.frexp(x)[1] - 1


def _blocks(x, fmt):
    """(x padded and cut into blocks, float32; the blocks' scales; the tensor's scale) for rows of x."""
    size = BLOCK[fmt]
    x = torch.nn.functional.pad(x.float(), (0, -x.shape[1] % size)).view(x.shape[0], -1, size)
    amax = x.abs().amax(2)
    if fmt == "e8m0":
        e = torch.where(amax > 0, _exponent(amax) - 2, -127).clamp(-127, 127)
        return x, _power(e), torch.ones((), device=x.device)
    top = amax.amax()
    tensor = _power(torch.where(top > 0, _exponent(top) - 10, 0).clamp(-126, 127))
    return x, (amax / (tensor * 6.0)).to(torch.float8_e4m3fn).float(), tensor


def _codes(y):
    """Index of the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 to y >= 0; a tie goes to the even index."""
    return ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0))


def _grid():
    return torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda")


def _nibbles(x, scale, tensor):
    s = (scale * tensor)[:, :, None]
    y = torch.where(s > 0, x.abs() / s, 0.0)
    return _codes(y) + 8 * torch.signbit(x).to(torch.uint8)


def _round(x, fmt):
    """x (rows, cols) as its 4-bit form along the rows stands for it, float32."""
    b, scale, tensor = _blocks(x, fmt)
    v = _grid()[_nibbles(b, scale, tensor).int()] * (scale * tensor)[:, :, None]
    return v.view(x.shape[0], -1)[:, :x.shape[1]]


def _pack(w, fmt):
    """w in the 4-bit layout that the head of this file describes: (values, scales, tensor scale)."""
    rows, cols = w.shape
    b, scale, tensor = _blocks(w, fmt)
    n = _nibbles(b, scale, tensor).view(rows, -1)
    n = torch.nn.functional.pad(n, (0, -n.shape[1] % 32))
    values = (n[:, 0::2] | (n[:, 1::2] << 4)).contiguous()
    code = torch.frexp(scale)[1].add(126).to(torch.uint8) if fmt == "e8m0" else scale.to(torch.float8_e4m3fn).view(torch.uint8)
    code = torch.nn.functional.pad(code, (0, -code.shape[1] % 4, 0, -rows % 128))
    code = code.view(code.shape[0] // 128, 4, 32, code.shape[1] // 4, 4).permute(0, 3, 2, 1, 4)
    return values, code.reshape(-1).contiguous(), tensor.reshape(1)


def _unpack(packed, rows, cols, fmt):
    values, code, tensor = packed
    n = torch.stack((values & 15, values >> 4), 2).view(rows, -1)[:, :cols]
    blocks = -(-cols // BLOCK[fmt])
    code = code.view(-(-rows // 128), -(-blocks // 4), 32, 4, 4).permute(0, 3, 2, 1, 4)
    code = code.reshape(-(-rows // 128) * 128, -1)[:rows, :blocks]
    scale = _power(code.int() - 127) if fmt == "e8m0" else code.contiguous().view(torch.float8_e4m3fn).float()
    scale = (scale * tensor).repeat_interleave(BLOCK[fmt], 1)[:, :cols]
    return _grid()[n.int()] * scale


def _plain_top(s, c):
    z = s["logits"].float()
    ordered, index = torch.sort(z, dim=1, descending=True, stable=True)
    values, rest = ordered[:, :c["k"]], ordered[:, c["k"]:] / c["tau"]
    if rest.shape[1] == 0:
        return values, index[:, :c["k"]].to(torch.int32), torch.full_like(values[:, 0], -math.inf)
    high = rest[:, 0]
    total = torch.exp(rest - torch.where(high > -math.inf, high, 0.0)[:, None]).sum(1)
    return values.contiguous(), index[:, :c["k"]].to(torch.int32), high + torch.log(total)


def _plain_distill(s, c):
    z, index, tau, alpha = s["logits"].float(), s["indices"].long(), c["tau"], c["alpha"]
    t, rest = s["values"] / tau, s["rest"]
    # the teacher: its sent words, and one more outcome for all the others
    both = torch.cat((t, rest[:, None]), 1)
    high = both.amax(1)
    taught = high > -math.inf
    p = torch.exp(both - torch.where(taught, high, 0.0)[:, None])
    total = p.sum(1)
    p = p / torch.where(taught, total, 1.0)[:, None]
    # the student, likewise
    top = z.amax(1)
    seen = top > -math.inf
    top = torch.where(seen, top, 0.0)[:, None]
    e = torch.exp((z - top) / tau)
    at = torch.gather(z, 1, index)
    mass = torch.exp((at - top) / tau)
    others = e.clone().scatter_(1, index, 0.0).sum(1)
    whole = torch.where(seen, others + mass.sum(1), 1.0)
    # the divergence: sum over the outcomes of p d - p + q with d = log p - log q, where every term is
    # positive; p (exp(-d) - 1 + d) keeps a small d's digits
    shift = (high - top[:, 0] / tau) + (torch.log(total) - torch.log(whole))
    d = torch.cat((t - at / tau, ((rest - top[:, 0] / tau) - torch.log(others))[:, None]), 1) - shift[:, None]
    q_of = torch.cat((mass, others[:, None]), 1) / whole[:, None]
    term = torch.where(d.abs() < 0.5, p * (torch.expm1(-d) + d), p * d - p + q_of)
    live = (taught & seen).float()
    gap = torch.where(p > 0, term, q_of).sum(1)
    loss = alpha * tau * tau * torch.where(live > 0, gap, 0.0)
    share = others / whole
    less = torch.where(share > 0, 1.0 - p[:, -1] / share, 0.0)
    q = e / whole[:, None]
    grad = q * less[:, None]
    grad.scatter_(1, index, torch.gather(q, 1, index) - p[:, :-1])
    grad *= (alpha * tau * live)[:, None]
    if s["labels"] is not None:
        label = s["labels"]
        has = ((label >= 0) & seen).float()
        word = label.clamp(min=0)[:, None]
        e1 = torch.exp(z - top)
        sum1 = torch.where(seen, e1.sum(1), 1.0)
        cross = torch.log(sum1) - (torch.gather(z, 1, word) - top)[:, 0]
        loss = loss + (1 - alpha) * torch.where(has > 0, cross, 0.0)
        q1 = e1 / sum1[:, None]
        q1.scatter_add_(1, word, torch.full_like(cross, -1.0)[:, None])
        grad += q1 * ((1 - alpha) * has)[:, None]
    return loss, (grad * s["grad_loss"][:, None]).to(s["logits"].dtype)


def _plain(s):
    c = s["case"]
    if c["kind"] == "top":
        return _plain_top(s, c)
    if c["kind"] == "distill":
        return _plain_distill(s, c)
    if c["kind"] == "quantise":
        x = s["x"]
        out = (_round(x, c["format"]).to(x.dtype),)
        return out + (_round(x.t(), c["format"]).to(x.dtype),) if c["both"] else out
    x, fmt = s["x"], c["format"]
    if not c["step"]:
        return (_round(x, fmt) @ _unpack(s["w4"], c["outer"], c["inner"], fmt).t()).to(x.dtype)
    w, dy = s["w"], s["dy"]
    y = (_round(x, fmt) @ _round(w, fmt).t()).to(x.dtype)
    dx = (_round(dy, fmt) @ _round(w.t(), fmt).t()).to(x.dtype)
    dw = _round(dy.t(), fmt) @ _round(x.t(), fmt).t()
    return y, dx, dw


# ---- the package's calls ---------------------------------------------------------------

def _own(s):
    from paper_1805_08768_b200 import binding as sbc

    c = s["case"]
    if c["kind"] == "top":
        return sbc.sbc_top_logits(s["logits"], c["k"], c["tau"])
    if c["kind"] == "distill":
        about = dict(rest=s["rest"], temperature=c["tau"], alpha=c["alpha"], labels=s["labels"])
        if c["calls"] == 1:
            return sbc.sbc_distill_loss_grad(s["logits"], s["values"], s["indices"], s["grad_loss"], **about)
        loss, stats = sbc.sbc_distill_loss(s["logits"], s["values"], s["indices"], **about)
        return loss, sbc.sbc_distill_grad(s["logits"], s["values"], s["indices"], stats, s["grad_loss"], **about)
    if c["kind"] == "quantise":
        x = s["x"]
        if not c["both"]:
            return (sbc.sbc_fp4_dequantise(sbc.sbc_fp4_quantise(x, c["format"]), x.dtype),)
        q, q_t = sbc.sbc_fp4_quantise_both(x, c["format"])
        return sbc.sbc_fp4_dequantise(q, x.dtype), sbc.sbc_fp4_dequantise(q_t, x.dtype)
    x, fmt = s["x"], c["format"]
    if not c["step"]:
        w4 = sbc.Fp4Tensor(*s["w4"], rows=c["outer"], cols=c["inner"], format=fmt)
        return sbc.sbc_fp4_product(sbc.sbc_fp4_quantise(x, fmt), w4, x.dtype)
    x4, x4_t = sbc.sbc_fp4_quantise_both(x, fmt)
    w4, w4_t = sbc.sbc_fp4_quantise_both(s["w"], fmt)
    y = sbc.sbc_fp4_product(x4, w4, x.dtype)
    dy4, dy4_t = sbc.sbc_fp4_quantise_both(s["dy"], fmt)
    return y, sbc.sbc_fp4_product(dy4, w4_t, x.dtype), sbc.sbc_fp4_product(dy4_t, x4_t, torch.float32)


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ------------------------------------------------------

def _fp4_bytes(rows, cols, fmt):
    return rows * cols * 0.5 + rows * -(-cols // BLOCK[fmt])


def work(case):
    c = case
    width = {"f32": 4, "bf16": 2}[c["dtype"]]
    if c["kind"] == "top":
        n = c["rows"] * c["cols"]
        return {"bytes": n * width + c["rows"] * (c["k"] * 8 + 4), "flops": 3 * n}
    if c["kind"] == "distill":
        n = c["rows"] * c["cols"]
        return {"bytes": n * width * (2 if c["calls"] == 1 else 3) + c["rows"] * (c["k"] * 8 + 24), "flops": 8 * n}
    if c["kind"] == "quantise":
        n, ways = c["rows"] * c["cols"], 2 if c["both"] else 1
        small = _fp4_bytes(c["rows"], c["cols"], c["format"]) + (_fp4_bytes(c["cols"], c["rows"], c["format"]) if c["both"] else 0)
        return {"bytes": n * width * (1 + ways) + 2 * small, "flops": 6 * n * ways}
    t, i, o, fmt = c["tokens"], c["inner"], c["outer"], c["format"]
    if not c["step"]:
        return {"bytes": t * i * width + _fp4_bytes(o, i, fmt) + t * o * width, "flops": 2 * t * i * o}
    return {"bytes": 2 * t * (i + o) * width + 2 * o * i * 4, "flops": 6 * t * i * o}


# ---- the definitions in 64 bits -----------------------------------------------------------

def _exact_round(x, fmt):
    """The value nearest to each element among (4-bit value) * (block scale) * (tensor scale), float64."""
    size = BLOCK[fmt]
    x = x.double()
    rows, cols = x.shape
    x = torch.cat((x, x.new_zeros(rows, -cols % size)), 1).reshape(rows, -1, size)
    high = x.abs().max(2).values

    def floor_log2(v):
        return ((v.view(torch.int64) >> 52) & 2047) - 1023

    if fmt == "e8m0":
        scale = torch.ldexp(torch.ones_like(high), (floor_log2(high) - 2).clamp(-127, 127))
    else:
        most = high.max()
        tensor = torch.ldexp(torch.ones_like(most), (floor_log2(most) - 10).clamp(-126, 127) if float(most) > 0 else torch.zeros_like(most).long())
        table = torch.arange(0, 127, dtype=torch.uint8, device=x.device).view(torch.float8_e4m3fn).double()
        scale = _exact_nearest(high / 6 / tensor, table) * tensor
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    y = _exact_nearest(x.abs() / torch.where(scale > 0, scale, math.inf)[:, :, None], table)
    return (torch.sign(x) * y * scale[:, :, None]).reshape(rows, -1)[:, :cols]


def _exact_nearest(y, table):
    """The table's entry nearest to y, the one of even index on a tie, the last one beyond it."""
    above = torch.searchsorted(table, y.contiguous()).clamp(max=len(table) - 1)
    below = (above - 1).clamp(min=0)
    up, down = table[above] - y, y - table[below]
    return torch.where((up < down) | ((up == down) & (above % 2 == 0)) | (y >= table[-1]), table[above], table[below])


def _exact_distill(s, c, part):
    tau, alpha = c["tau"], c["alpha"]
    z, index = s["logits"][part].double(), s["indices"][part].long()
    teacher = torch.cat((s["values"][part].double() / tau, s["rest"][part].double()[:, None]), 1)
    empty = torch.isinf(teacher).all(1) | torch.isinf(z).all(1)
    none = torch.isinf(z).all(1)
    z = torch.where(none[:, None], torch.zeros_like(z), z)
    log_p = torch.log_softmax(torch.where(empty[:, None], torch.zeros_like(teacher), teacher), 1)
    log_q = torch.log_softmax(z / tau, 1)
    sent = torch.zeros_like(z, dtype=torch.bool).scatter_(1, index, True)
    others = torch.logsumexp(torch.where(sent, torch.full_like(z, -math.inf), log_q), 1)
    pairs = torch.cat((log_q.gather(1, index), others[:, None]), 1)
    p = log_p.exp()
    kl = torch.where(p > 0, p * (log_p - pairs), torch.zeros_like(p)).sum(1)
    q = log_q.exp()
    target = torch.where(sent, torch.zeros_like(q), torch.exp(log_q + (log_p[:, -1:] - others[:, None])))
    target = torch.where(torch.isnan(target), torch.zeros_like(target), target)
    target.scatter_(1, index, p[:, :-1])
    live = (~empty).double()
    loss = alpha * tau ** 2 * kl * live
    grad = alpha * tau * (q - target) * live[:, None]
    if s["labels"] is not None:
        label = s["labels"][part]
        has = ((label >= 0) & ~none).double()
        log_q1 = torch.log_softmax(z, 1)
        word = label.clamp(min=0)[:, None]
        loss = loss - (1 - alpha) * torch.where(has > 0, log_q1.gather(1, word)[:, 0], torch.zeros_like(has))
        hot = torch.zeros_like(z).scatter_(1, word, 1.0)
        grad = grad + (1 - alpha) * (log_q1.exp() - hot) * has[:, None]
    return loss, grad * s["grad_loss"][part].double()[:, None]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "top":
        values, rests = [], []
        for lo in range(0, c["rows"], 256):
            z = s["logits"][lo:lo + 256].double().sort(1, descending=True).values
            values.append(z[:, :c["k"]])
            rests.append(torch.logsumexp(z[:, c["k"]:] / c["tau"], 1) if c["k"] < c["cols"]
                         else torch.full_like(z[:, 0], -math.inf))
        return torch.cat(values), None, torch.cat(rests)
    if c["kind"] == "distill":
        parts = [_exact_distill(s, c, slice(lo, lo + 256)) for lo in range(0, c["rows"], 256)]
        return tuple(torch.cat(x) for x in zip(*parts))
    if c["kind"] == "quantise":
        out = (_exact_round(s["x"], c["format"]),)
        return out + (_exact_round(s["x"].t(), c["format"]),) if c["both"] else out
    x, fmt = s["x"], c["format"]
    if not c["step"]:
        g = _generator(seed)
        _activations(c["tokens"], c["inner"], g)
        w = torch.randn(c["outer"], c["inner"], generator=g, device="cuda") / c["inner"] ** 0.5
        return _exact_round(x, fmt) @ _exact_round(w, fmt).t()
    w, dy = s["w"], s["dy"]
    return (_exact_round(x, fmt) @ _exact_round(w, fmt).t(),
            _exact_round(dy, fmt) @ _exact_round(w.t(), fmt).t(),
            _exact_round(dy.t(), fmt) @ _exact_round(x.t(), fmt).t())
