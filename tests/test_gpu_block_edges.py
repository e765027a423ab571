"""The operators of a client's own layers behind autograd, where a caller asks for less, or for more, than a whole step."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_1805_08768_b200 import binding as sbc
from paper_1805_08768_b200 import block, distill

DEV = torch.device("cuda:0")


def randn(*shape, seed, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


@pytest.mark.parametrize("tokens", [30, 100])
def test_fixed_adapters_beside_a_trained_projection(tokens):
    """Only the shared projection learns: its gradient is what it gets without the adapters, for few tokens and for many."""
    x = randn(tokens, 64, seed=1, dtype=torch.bfloat16)
    w = randn(96, 64, seed=2).requires_grad_(True)
    down, up = randn(3, 5, 64, seed=3), randn(3, 5, 96, seed=4)
    ids = (torch.arange(tokens, device=DEV) % 4 - 1).to(torch.int32)
    dy = randn(tokens, 96, seed=6, dtype=torch.bfloat16)
    for plan in (None, sbc.sbc_adapter_plan(ids, 3)):
        y = block.adapter(x, down, up, ids, 1.5, distill.fp4_linear(x, w), plan)
        (got,) = torch.autograd.grad(y, w, dy)
        (want,) = torch.autograd.grad(distill.fp4_linear(x, w), w, dy)
        assert torch.equal(got, want)
