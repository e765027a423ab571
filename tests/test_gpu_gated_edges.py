"""The gated block where its sizes end; what is computed is exact, so results are compared for equality."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_1805_08768_b200 import binding as sbc

DEV = torch.device("cuda:0")


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
