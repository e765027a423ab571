"""What the operators of a client's own layers are measured on.

Between two rounds a client trains the block of a language model that it was sent: a normalisation, a
gated feed-forward block, a projection that all clients share with a low-rank adapter of each client
beside it, and dropout on the way back into the residual.  The operators are

  norm     layer norm, forward, and backward with the sums over rows that its weight and bias get
  dropout  values kept with probability 1 - p by a counter-based generator and added to a residual;
           the backward pass draws the same numbers again, no mask is kept
  gated    h = act(x G^T) * (x U^T), forward for one token or many, and backward (x, G, U)
  adapter  y = base + s (x D_i^T) P_i, i the adapter of the token's client or request, forward for
           single tokens of many requests or for long ones, and backward (x, D, P)

``run`` makes the plain computation in 32 bits, or, where ``own`` is set, the package's calls.

The generator is Philox-4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as
1, 2, 3", 2011): key = seed, counter = (number of the group of eight elements + at, step), 64 bits
each, low word first.  Its four words are eight halves, low ones first, for the group's eight elements
in row-major order.  An element is dropped if its half is below d = round(65536 p), and scaled by
65536 / (65536 - d) if not.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


def listed():
    return [
        # one sentence of 35 words in the word model's 650 hidden units, there and back; latency
        dict(name="norm_sentence", kind="norm", rows=35, cols=650, dtype="f32", weights="f32", step=True),
        # a batch's normalisation where no gradient is asked for; an odd width, so rows start at odd places
        dict(name="norm_odd_forward", kind="norm", rows=8191, cols=2601, dtype="f16", weights="f16", step=False),
        # a long batch of a wide model, there and back, the weights in 32 bits
        dict(name="norm_long_step", kind="norm", rows=16384, cols=4096, dtype="bf16", weights="f32", step=True),
        # one sentence's hidden units, there and back; latency
        dict(name="dropout_sentence", kind="dropout", rows=35, cols=650, dtype="f32", p=0.5),
        # a long batch of a wide model on its way into the residual, and its gradient
        dict(name="dropout_long", kind="dropout", rows=16384, cols=4096, dtype="bf16", p=0.1),
        # one token through the word model's block: latency, 650 is no multiple of 16 bytes' worth
        dict(name="gated_one_token", kind="gated", tokens=1, inner=650, hidden=2600, dtype="bf16", act="silu", step=False),
        # sixteen sequences' next tokens through a large block: the weights' bytes count
        dict(name="gated_few_tokens", kind="gated", tokens=16, inner=4096, hidden=16384, dtype="bf16", act="silu", step=False),
        # a training step of the word model's block on 64 sentences of 35 words
        dict(name="gated_word_step", kind="gated", tokens=2240, inner=650, hidden=2600, dtype="f16", act="gelu", step=True),
        # a training step of a large block on a long batch: arithmetic counts
        dict(name="gated_large_step", kind="gated", tokens=8192, inner=4096, hidden=8192, dtype="bf16", act="silu", step=True),
        # the next token of 32 requests, each with one of 64 adapters: latency
        dict(name="adapter_single_tokens", kind="adapter", tokens=32, inner=4096, outer=4096, rank=16, adapters=64, requests=32,
             dtype="bf16", weights="bf16", step=False),
        # a step of eight clients' adapters beside the word model's gates, the adapters in 32 bits as their updates are
        dict(name="adapter_clients_step", kind="adapter", tokens=2240, inner=650, outer=2600, rank=8, adapters=8, requests=8,
             dtype="bf16", weights="f32", step=True),
        # prompts and long sequences of twelve requests, a step of their adapters beside a large projection
        dict(name="adapter_long_step", kind="adapter", tokens=8191, inner=4096, outer=8192, rank=64, adapters=8, requests=12,
             dtype="bf16", weights="bf16", step=True),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["norm", "dropout", "gated", "adapter"])
    if kind in ("norm", "dropout"):
        cols = _spread(rng, 8, 16384)
        case = dict(kind=kind, rows=_spread(rng, 1, min(65536, (1 << 26) // cols)), cols=cols, dtype=rng.choice(["f32", "bf16", "f16"]))
        if kind == "norm":
            case.update(weights=rng.choice(["f32", case["dtype"]]), step=rng.random() < 0.7)
        else:
            case.update(p=rng.choice([0.05, 0.1, 0.3, 0.5]))
        return case
    step, inner = rng.random() < 0.5, _spread(rng, 16, 8192)
    if kind == "gated":
        hidden = _spread(rng, 16, 16384)
        most = int(1.5e12 / (4.0 * inner * hidden * (3 if step else 1)))
        return dict(kind=kind, tokens=_spread(rng, 1, max(1, min(8192, most))), inner=inner, hidden=hidden, dtype=rng.choice(["bf16", "f16"]),
                    act=rng.choice(["silu", "gelu"]), step=step)
    outer, rank, adapters = _spread(rng, 16, 8192), _spread(rng, 1, 64), _spread(rng, 1, 64)
    most = int(5.0e11 / (2.0 * (inner + outer) * rank * adapters * (3 if step else 1)))
    tokens = _spread(rng, 1, max(1, min(8192, most)))
    dtype = rng.choice(["f32", "bf16", "f16"])
    return dict(kind=kind, tokens=tokens, inner=inner, outer=outer, rank=rank, adapters=adapters, requests=min(tokens, _spread(rng, 1, 64)),
                dtype=dtype, weights=rng.choice(["f32", dtype]), step=step)


# ---- inputs -----------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 6151 + 29)


def _activations(rows, cols, g):
    """Values whose columns differ in size and place, a few of them by a lot."""
    size = torch.exp(0.5 * torch.randn(cols, generator=g, device="cuda"))
    size = torch.where(torch.rand(cols, generator=g, device="cuda") < 0.01, size * 10, size)
    return torch.randn(rows, cols, generator=g, device="cuda") * size + 0.3 * torch.randn(cols, generator=g, device="cuda")


def _gradients(rows, cols, g):
    """Gradients whose rows differ in size (loss scaling keeps 16-bit ones, and the sums over them, in range)."""
    return torch.randn(rows, cols, generator=g, device="cuda") * torch.exp(0.7 * torch.randn(rows, 1, generator=g, device="cuda")) * 0.25


def _adapter_of_tokens(case, g):
    """Every token's adapter, -1 where a request has none: requests of unequal lengths, one behind the other."""
    tokens, requests = case["tokens"], case["requests"]
    cuts = torch.randperm(max(tokens - 1, 1), generator=g, device="cuda")[:requests - 1] + 1   # where a new request begins
    request = torch.zeros(tokens + 1, dtype=torch.int64, device="cuda").index_fill_(0, cuts, 1)[:tokens].cumsum(0)
    which = torch.randint(0, case["adapters"], (requests,), generator=g, device="cuda")
    which = which.masked_fill(torch.rand(requests, generator=g, device="cuda") < 0.05, -1)
    return which[request].to(torch.int32)


def prepare(case, seed):
    g = _generator(seed)
    c, dtype = case, DTYPES[case["dtype"]]
    state = dict(case=dict(case))
    if c["kind"] == "norm":
        state["x"] = _activations(c["rows"], c["cols"], g).to(dtype)
        state["weight"] = (1 + 0.2 * torch.randn(c["cols"], generator=g, device="cuda")).to(DTYPES[c["weights"]])
        state["bias"] = (0.1 * torch.randn(c["cols"], generator=g, device="cuda")).to(DTYPES[c["weights"]])
        if c["step"]:
            state["dy"] = _gradients(c["rows"], c["cols"], g).to(dtype)
    elif c["kind"] == "dropout":
        state["x"] = _activations(c["rows"], c["cols"], g).to(dtype)
        state["residual"] = _activations(c["rows"], c["cols"], g).to(dtype)
        state["dy"] = _gradients(c["rows"], c["cols"], g).to(dtype)
        # the generator's key, and how many steps were made with it
        state["rng"] = torch.tensor([(int(seed) * 0x9E3779B97F4A7C15 + 12345) % (1 << 63), int(seed) % 1000003 + 7], device="cuda")
        state["at"] = 1 << 20   # what earlier layers took of the step's numbers
    elif c["kind"] == "gated":
        state["x"] = _activations(c["tokens"], c["inner"], g).to(dtype)
        for name in ("gate", "up"):
            state[name] = (torch.randn(c["hidden"], c["inner"], generator=g, device="cuda") / c["inner"] ** 0.5).to(dtype)
        if c["step"]:
            state["dh"] = _gradients(c["tokens"], c["hidden"], g).to(dtype)
    else:
        state["x"] = _activations(c["tokens"], c["inner"], g).to(dtype)
        # what the shared projection gave for these tokens
        state["base"] = torch.randn(c["tokens"], c["outer"], generator=g, device="cuda").to(dtype)
        state["ids"] = _adapter_of_tokens(c, g)
        weights = DTYPES[c["weights"]]
        state["down"] = (torch.randn(c["adapters"], c["rank"], c["inner"], generator=g, device="cuda") / c["inner"] ** 0.5).to(weights)
        state["up"] = (0.3 * torch.randn(c["adapters"], c["rank"], c["outer"], generator=g, device="cuda") / c["rank"] ** 0.5).to(weights)
        state["scale"] = 2.0
        if c["step"]:
            state["dy"] = (_gradients(c["tokens"], c["outer"], g) * (4 / c["outer"] ** 0.5)).to(dtype)
            # the input's gradient through the shared projection
            state["dx_base"] = _gradients(c["tokens"], c["inner"], g).to(dtype)
    return state


# ---- the plain form -----------------------------------------------------------------

def _plain_norm(s, c):
    x, w, b = s["x"].float(), s["weight"].float(), s["bias"].float()
    centred = x - x.mean(1, keepdim=True)
    rstd = torch.rsqrt((centred * centred).mean(1, keepdim=True) + EPS)
    hat = centred * rstd
    y = (hat * w + b).to(s["x"].dtype)
    if not c["step"]:
        return y
    dy = s["dy"].float()
    t = dy * w
    dx = rstd * (t - t.mean(1, keepdim=True) - hat * (t * hat).mean(1, keepdim=True))
    return y, dx.to(s["x"].dtype), (dy * hat).sum(0).to(s["weight"].dtype), dy.sum(0).to(s["bias"].dtype)


LOW = 0xFFFFFFFF


def _plain_halves(rng, at, n):
    """The generator's halves for n elements, int64."""
    block = torch.arange(-(-n // 8), device="cuda") + at
    key, step = rng[0], rng[1]
    a, b = block & LOW, (block >> 32) & LOW
    c, d = (step & LOW).expand_as(a), ((step >> 32) & LOW).expand_as(a)
    k0, k1 = key & LOW, (key >> 32) & LOW
    for _ in range(10):
        # (64 bits wrap around; the words above and below the middle are right all the same)
        first, second = a * 0xD2511F53, c * 0xCD9E8D57
        a, b, c, d = ((second >> 32) & LOW) ^ b ^ k0, second & LOW, ((first >> 32) & LOW) ^ d ^ k1, first & LOW
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    words = torch.stack((a, b, c, d), 1)
    return torch.stack((words & 0xFFFF, words >> 16), 2).reshape(-1)[:n]


def _plain_dropout(s, c):
    x = s["x"]
    dropped = round(65536 * c["p"])
    keep = _plain_halves(s["rng"], s["at"], x.numel()).view_as(x) >= dropped
    scale = torch.where(keep, 65536.0 / (65536 - dropped), 0.0)
    return (s["residual"].float() + x.float() * scale).to(x.dtype), (s["dy"].float() * scale).to(x.dtype)


def _act(g, act):
    """(act(g), its derivative)"""
    if act == "silu":
        e = torch.sigmoid(g)
        return g * e, e * (1 + g * (1 - e))
    p = 0.5 * torch.erfc(g * -math.sqrt(0.5))
    return g * p, p + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))


def _plain_gated(s, c):
    dtype = s["x"].dtype
    x, gate, up = s["x"].float(), s["gate"].float(), s["up"].float()
    u = x @ up.t()
    value, slope = _act(x @ gate.t(), c["act"])
    h = (value * u).to(dtype)
    if not c["step"]:
        return h
    dh = s["dh"].float()
    dg, du = dh * u * slope, dh * value
    return h, (dg @ gate + du @ up).to(dtype), (dg.t() @ x).to(dtype), (du.t() @ x).to(dtype)


def _plain_adapter(s, c):
    dtype, scale = s["x"].dtype, s["scale"]
    n, rank, inner = s["down"].shape
    x, down, up = s["x"].float(), s["down"].float().view(n * rank, inner), s["up"].float().view(n * rank, -1)
    # all adapters side by side; a token's own columns are left, the others are zeros
    mine = (s["ids"][:, None] == torch.arange(n, device="cuda")).repeat_interleave(rank, 1).float()
    mid = (x @ down.t()) * mine
    y = (s["base"].float() + scale * (mid @ up)).to(dtype)
    if not c["step"]:
        return y
    dy = s["dy"].float()
    dmid = scale * (dy @ up.t()) * mine
    dx = (s["dx_base"].float() + dmid @ down).to(dtype)
    return y, dx, (dmid.t() @ x).view_as(s["down"]).to(s["down"].dtype), (scale * (mid.t() @ dy)).view_as(s["up"]).to(s["up"].dtype)


PLAIN = {"norm": _plain_norm, "dropout": _plain_dropout, "gated": _plain_gated, "adapter": _plain_adapter}


# ---- the package's calls ---------------------------------------------------------------

def _own(s):
    from paper_1805_08768_b200 import binding as sbc

    c = s["case"]
    if c["kind"] == "norm":
        y, stats = sbc.sbc_layer_norm(s["x"], s["weight"], s["bias"], EPS)
        if not c["step"]:
            return y
        return (y,) + tuple(sbc.sbc_layer_norm_grad(s["dy"], s["x"], stats, s["weight"]))
    if c["kind"] == "dropout":
        return (sbc.sbc_dropout(s["x"], c["p"], s["rng"], s["at"], residual=s["residual"]),
                sbc.sbc_dropout(s["dy"], c["p"], s["rng"], s["at"]))
    if c["kind"] == "gated":
        if not c["step"]:
            return sbc.sbc_gated(s["x"], s["gate"], s["up"], c["act"])
        h, kept = sbc.sbc_gated(s["x"], s["gate"], s["up"], c["act"], keep=True)
        return (h,) + tuple(sbc.sbc_gated_grad(s["dh"], s["x"], s["gate"], s["up"], kept))
    if not c["step"]:
        return sbc.sbc_adapter(s["x"], s["down"], s["up"], s["ids"], s["scale"], s["base"])
    y, kept = sbc.sbc_adapter(s["x"], s["down"], s["up"], s["ids"], s["scale"], s["base"], keep=True)
    return (y,) + tuple(sbc.sbc_adapter_grad(s["dy"], s["x"], s["down"], s["up"], kept, s["scale"], s["dx_base"]))


def run(state):
    return _own(state) if own else PLAIN[state["case"]["kind"]](state, state["case"])


# ---- what a pass cannot do without ------------------------------------------------------

def work(case):
    c = case
    width = {"f32": 4, "bf16": 2, "f16": 2}
    w = width[c["dtype"]]
    if c["kind"] in ("norm", "dropout"):
        n = c["rows"] * c["cols"]
        if c["kind"] == "dropout":
            return {"bytes": 5 * n * w, "flops": 6 * n}
        return {"bytes": n * w * (4 if c["step"] else 2) + c["cols"] * width[c["weights"]] * (4 if c["step"] else 2), "flops": n * (18 if c["step"] else 7)}
    t, i = c["tokens"], c["inner"]
    if c["kind"] == "gated":
        h = c["hidden"]
        if c["step"]:
            return {"bytes": w * (2 * t * i + 2 * t * h + 4 * h * i), "flops": 12 * t * i * h}
        return {"bytes": w * (t * i + t * h + 2 * h * i), "flops": 4 * t * i * h}
    o, r = c["outer"], c["rank"]
    adapters = min(c["adapters"], c["requests"]) * r * (i + o) * width[c["weights"]]
    if c["step"]:   # the gradients of adapters that no token has are zeros, and written too
        return {"bytes": w * t * (3 * i + 3 * o) + 4 * t + adapters + c["adapters"] * r * (i + o) * width[c["weights"]], "flops": 6 * t * r * (i + o)}
    return {"bytes": w * t * (i + 2 * o) + 4 * t + adapters, "flops": 2 * t * r * (i + o)}


# ---- the definitions in 64 bits -----------------------------------------------------------

def _exact_norm(s, c):
    x = s["x"].double()
    w, b = s["weight"].double(), s["bias"].double()
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    sigma = torch.sqrt(var + EPS)
    y = (x - mean) / sigma * w + b
    if not c["step"]:
        return y
    dy = s["dy"].double()
    cols = x.shape[1]
    # d y_k / d x_j = w_k ((k == j) - 1 / n - hat_j hat_k / n) / sigma
    z = (x - mean) / sigma
    dot = torch.einsum("rk,k,rk->r", dy, w, z)[:, None]
    dx = (dy * w - (dy @ w)[:, None] / cols - z * dot / cols) / sigma
    return y, dx, torch.einsum("rk,rk->k", dy, z), torch.einsum("rk->k", dy)


def _exact_halves(key, step, at, n):
    """The halves again, with products of 32-bit words put together from 16-bit pieces."""
    def split(a, m):
        low, high = m & 0xFFFF, m >> 16
        p, q = (a & 0xFFFF) * low, (a >> 16) * high
        middle = (a >> 16) * low + (a & 0xFFFF) * high + (p >> 16)
        return (q + (middle >> 16)) % (1 << 32), ((middle % 65536) << 16) + p % 65536

    number = torch.arange((n + 7) // 8, device="cuda") + at
    x = [number % (1 << 32), number >> 32, torch.full_like(number, step % (1 << 32)), torch.full_like(number, step >> 32)]
    for r in range(10):
        h0, l0 = split(x[0], 0xD2511F53)
        h1, l1 = split(x[2], 0xCD9E8D57)
        k = [(key % (1 << 32) + r * 0x9E3779B9) % (1 << 32), ((key >> 32) + r * 0xBB67AE85) % (1 << 32)]
        x = [h1 ^ x[1] ^ k[0], l1, h0 ^ x[3] ^ k[1], l0]
    halves = torch.empty(len(number), 8, dtype=torch.int64, device="cuda")
    for j in range(4):
        halves[:, 2 * j], halves[:, 2 * j + 1] = x[j] % 65536, x[j] // 65536
    return halves.view(-1)[:n]


def _exact_dropout(s, c):
    x = s["x"].double()
    key, step = (int(v) for v in s["rng"].tolist())
    below = int(c["p"] * 65536 + 0.5)
    halves = _exact_halves(key, step, s["at"], x.numel()).view_as(x)
    factor = torch.where(halves < below, 0.0, 1 / (1 - below / 65536)).double()
    return s["residual"].double() + factor * x, factor * s["dy"].double()


def _exact_gated(s, c):
    x, gate, up = s["x"].double(), s["gate"].double(), s["up"].double()
    g, u = torch.nn.functional.linear(x, gate), torch.nn.functional.linear(x, up)
    if c["act"] == "silu":
        share = 1 / (1 + torch.exp(-g))
        slope = share + g * share * (1 - share)
    else:
        share = 0.5 * (1 + torch.erf(g / math.sqrt(2)))
        slope = share + g * torch.exp(-g ** 2 / 2) / math.sqrt(2 * math.pi)
    h = g * share * u
    if not c["step"]:
        return h
    dh = s["dh"].double()
    dup = dh * (g * share)
    dgate = dh * u * slope
    del g, share, slope, u
    return h, torch.mm(dgate, gate) + torch.mm(dup, up), torch.mm(dgate.T, x), torch.mm(dup.T, x)


def _exact_adapter(s, c):
    x, y, scale = s["x"].double(), s["base"].double(), s["scale"]
    step = c["step"]
    if step:
        dy, dx = s["dy"].double(), s["dx_base"].double()
        grads = torch.zeros_like(s["down"], dtype=torch.float64), torch.zeros_like(s["up"], dtype=torch.float64)
    for i in range(c["adapters"]):
        rows = torch.nonzero(s["ids"] == i)[:, 0]
        d, p = s["down"][i].double(), s["up"][i].double()
        y[rows] += scale * (x[rows] @ d.T @ p)
        if step:
            dx[rows] += scale * (dy[rows] @ p.T @ d)
            grads[0][i] = scale * ((dy[rows] @ p.T).T @ x[rows])
            grads[1][i] = scale * ((x[rows] @ d.T).T @ dy[rows])
    return (y, dx) + grads if step else y


EXACT = {"norm": _exact_norm, "dropout": _exact_dropout, "gated": _exact_gated, "adapter": _exact_adapter}


def exact(case, seed):
    return EXACT[case["kind"]](prepare(case, seed), case)
