"""Layer norm at the sizes where rows are shorter than what a thread loads; tolerances as in test_gpu_norm_dropout."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_1805_08768_b200 import binding as sbc
from test_gpu_norm_dropout import DEV, TYPES, check_backward, check_forward, strided, values


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 2, 3, 4, 5, 6, 7])
def test_layer_norm_of_rows_shorter_than_a_granule(cols, dtype):
    """Many rows begin within one granule of eight: each has its own values and no other's, whatever the rows' distance."""
    w, b = torch.randn(cols, device=DEV), torch.randn(cols, device=DEV)
    for rows in (2, 3, 4, 61, 4096):
        x, dy = values(rows, cols, dtype, 1), values(rows, cols, dtype, 2)
        for lead, gap in ((0, 0), (0, 1), (3, 0), (1, 2)):
            room, xs = strided(x, lead, gap)
            out_room, out = strided(torch.zeros_like(x), lead, gap)
            y, stats = sbc.sbc_layer_norm(xs, w, b, out=out)
            check_forward(y, x, w, b, 1e-5)
            inside = torch.zeros_like(out_room, dtype=torch.bool)
            inside[lead:].view(rows, cols + gap)[:, :cols] = True
            assert bool((out_room[~inside] == 77).all())
            dx, dw, db = sbc.sbc_layer_norm_grad(dy, xs, stats, w)
            check_backward(dx, dw, db, dy, x, w, 1e-5)


@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm_rows_do_not_see_their_neighbours(dtype):
    """What lies beside a row, NaNs and infinities of other rows among it, does not count."""
    for cols in (2, 7, 9, 33):
        x = values(40, cols, dtype, 1)
        want, _ = sbc.sbc_layer_norm(x)
        for bad in (float("nan"), float("inf")):
            spoilt = x.clone()
            spoilt[1::2] = bad
            assert torch.equal(sbc.sbc_layer_norm(spoilt)[0][::2], want[::2])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [8193, 9000, 16384, 20001])
def test_layer_norm_gradients_of_many_long_rows(cols, dtype):
    """Rows longer than a group holds, several for every block (two an SM), so that its sums over rows go on from row to row."""
    rows = 2 * torch.cuda.get_device_properties(DEV).multi_processor_count * 3 + 5
    x, dy = values(rows, cols, dtype, 1), values(rows, cols, dtype, 2)
    w, b = torch.randn(cols, device=DEV), torch.randn(cols, device=DEV)
    y, stats = sbc.sbc_layer_norm(x, w, b)
    check_forward(y, x, w, b, 1e-5)
    dx, dw, db = sbc.sbc_layer_norm_grad(dy, x, stats, w)
    check_backward(dx, dw, db, dy, x, w, 1e-5)
    _, dw2, db2 = sbc.sbc_layer_norm_grad(dy, x, stats, w, need_input=False)
    assert torch.equal(dw, dw2) and torch.equal(db, db2)
