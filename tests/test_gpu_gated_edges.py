"""The gated block where its sizes and its activations end."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_1805_08768_b200 import binding as sbc

from test_gpu_gated import DEV, STEP, act64


def test_gated_widest_inputs():
    """One token as wide as a call takes: positions go up to a step of the kernel's loop below 2^31.  All but some thousand of x's
    values are zeros, the others and the weights small whole numbers, so both sums are exact in any order; so are
    their product (below 2^24) and its one rounding."""
    inner = (1 << 31) - 513
    gen = torch.Generator(device=DEV).manual_seed(3)
    at = torch.cat([torch.arange(0, 700, device=DEV), torch.randint(700, inner - 2100, (1000,), generator=gen, device=DEV),
                    torch.arange(inner - 2100, inner, device=DEV)]).unique()
    rows = []
    for _ in range(3):
        row = torch.zeros(1, inner, dtype=torch.bfloat16, device=DEV)
        row[0, at] = torch.randint(-2, 3, (at.numel(),), generator=gen, device=DEV).bfloat16()
        rows.append(row)
    x, gate, up = rows
    # where x is zero, weights that are not count for nothing
    for w in (gate, up):
        w[0, at[at.numel() // 2] + 1] = 5.0
    values = [r[0, at].double() for r in rows]
    g, u = float((values[0] * values[1]).sum()), float((values[0] * values[2]).sum())
    if g < 0:
        gate.neg_()
        g = -g
    assert 0 < g < 4096 and 0 < abs(u) < 4096
    want = torch.tensor(g * u, dtype=torch.float64, device=DEV).bfloat16()
    assert torch.equal(sbc.sbc_gated(x, gate, up, "relu")[0, 0], want)


@pytest.mark.parametrize("tokens", [1, 20, 100])
@pytest.mark.parametrize("act", ["silu", "gelu_tanh", "sigmoid"])
def test_gated_small_activations(act, tokens):
    """Activations near the type's smallest numbers, times factors near its largest: they keep their digits.  Off by (8 + 2 |z|)
    2^-23 of itself (z: the sigmoid's argument) or, where the share is below 2^-126, a step of 2^-149; times g, that is."""
    g = -torch.cat([torch.arange(60, 104, 0.5, device=DEV), torch.arange(80, 92, 0.0625, device=DEV)]).bfloat16()
    if act == "gelu_tanh":
        g = -torch.arange(7, 12, 0.0625, device=DEV).bfloat16()
    hidden = g.numel()
    x = torch.zeros(tokens, 16, dtype=torch.bfloat16, device=DEV)
    x[:, 2], x[:, 3] = 1, 1
    gate, up = (torch.zeros(hidden, 16, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    gate[:, 2], up[:, 3] = g, 2.0 ** 110
    g64 = g.double()
    value, slope = act64(g64, act)
    if act == "gelu_tanh":     # (1 + tanh(t) cancels: by the exponential)
        c = 2 * (2 / torch.pi) ** 0.5
        z, dz = c * (g64 + 0.044715 * g64 ** 3), c * (1 + 3 * 0.044715 * g64 ** 2)
        share = 1 / (1 + torch.exp(-z))
        value, slope = g64 * share, share * (1 + g64 * dz * (1 - share))
    else:
        z = g64
        share = torch.sigmoid(z)
    off = (8 + 2 * z.abs()) * 2.0 ** -23
    factor = 1.0 if act == "sigmoid" else g64.abs()
    allowed = (off * value.abs() + 2.0 ** -149 * factor) * 2.0 ** 110 + STEP[torch.bfloat16] * (value * 2.0 ** 110).abs()
    h = sbc.sbc_gated(x, gate, up, act)
    assert bool(((h.double() - value * 2.0 ** 110).abs() <= allowed).all()) and float(value.abs().min()) < 2.0 ** -126
    h, kept = sbc.sbc_gated(x, gate, up, act, keep=True)
    assert bool(((h.double() - value * 2.0 ** 110).abs() <= allowed).all())
    # what is kept for the backward pass: u act'(g) and act(g); the slope's two parts differ by what z and dz are off, too
    got = kept[:, :hidden].double()
    if act == "gelu_tanh":
        steep = 1 + (g64 * dz).abs()
    else:
        steep = 1 + g64.abs()
    slack = (off + 2.0 ** -20) * share * steep + 2.0 ** -149 * steep
    assert bool(((got[..., 0] * 2.0 ** -110 - slope).abs() <= slack).all())
    assert bool(((got[..., 1] - value).abs() <= off * value.abs() + 2.0 ** -149 * (1 + factor)).all())


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu", "sigmoid"])
def test_gated_slopes_of_infinities(act):
    """At plus infinity a slope is its limit."""
    x = torch.zeros(40, 16, dtype=torch.bfloat16, device=DEV)
    x[:, 0] = 1
    gate, up = (torch.zeros(24, 16, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    gate[:, 0], up[:, 0] = float("inf"), 1
    x[:, 1:] = 0
    gate[:, 1:] = 0
    h, kept = sbc.sbc_gated(x, gate, up, act, keep=True)
    limit = 0.0 if act == "sigmoid" else 1.0
    assert bool((kept[:, :24, 0] == limit).all())
