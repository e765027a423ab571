"""Refusals of the operators of a client's own layers that the host makes: no kernel is launched, no GPU is needed.

Every call below has addresses that nothing lies behind; each must be refused before anything is enqueued."""
import ctypes as C

import pytest

from paper_1805_08768_b200 import binding as sbc
from paper_1805_08768_b200 import build

OK, BAD, SMALL = sbc.SBC_OK, sbc.SBC_EINVAL, sbc.SBC_ECAPACITY
P = 1 << 20   # a 16-byte aligned address


@pytest.fixture(scope="module")
def lib():
    build.build()
    return sbc.lib()


def changed(good, **by):
    """The good arguments with one or more of them changed, by name."""
    args = dict(good)
    args.update(by)
    return list(args.values())


NORM = dict(x=P, dtype=1, rows=4, cols=8, x_stride=8, weight=P, bias=P, weight_dtype=1, eps=1e-5, y=P, y_stride=8, stats=P, stream=None)


@pytest.mark.parametrize("by", [dict(x=None), dict(y=None), dict(dtype=3), dict(rows=-1), dict(cols=0), dict(cols=1 << 31), dict(x_stride=7),
                                dict(y_stride=7), dict(weight_dtype=2), dict(weight=P + 1), dict(eps=-1.0), dict(eps=float("nan")),
                                dict(eps=float("inf")), dict(x=P + 1), dict(stats=P + 4)])
def test_layer_norm_refuses(lib, by):
    assert lib.sbc_layer_norm(*changed(NORM, **by)) == BAD


def test_layer_norm_of_no_rows(lib):
    assert lib.sbc_layer_norm(*changed(NORM, rows=0, x=None, y=None)) == OK
    assert lib.sbc_layer_norm_workspace_bytes(-1, 8) == 0 and lib.sbc_layer_norm_workspace_bytes(4, 0) == 0
    assert lib.sbc_layer_norm_workspace_bytes(0, 8) > 0


NORM_GRAD = dict(dy=P, dy_stride=8, x=P, x_stride=8, dtype=1, rows=4, cols=8, stats=P, weight=P, weight_dtype=1, dx=P, dx_stride=8, dweight=P,
                 dbias=P, workspace=P, workspace_bytes=1 << 20, stream=None)


@pytest.mark.parametrize("by", [dict(dy=None), dict(x=None), dict(stats=None), dict(dy_stride=3), dict(dx_stride=3), dict(weight_dtype=2),
                                dict(dx=None, dweight=None, dbias=None), dict(workspace=None), dict(workspace=P + 8), dict(dweight=P + 1)])
def test_layer_norm_grad_refuses(lib, by):
    assert lib.sbc_layer_norm_grad(*changed(NORM_GRAD, **by)) == BAD


def test_layer_norm_grad_wants_its_workspace(lib):
    need = lib.sbc_layer_norm_workspace_bytes(4, 8)
    assert lib.sbc_layer_norm_grad(*changed(NORM_GRAD, workspace_bytes=need - 1)) == SMALL
    assert lib.sbc_layer_norm_grad(*changed(NORM_GRAD, rows=0, dweight=None, dbias=None)) == OK


DROP = dict(x=P, dtype=0, rows=4, cols=8, x_stride=8, residual=None, residual_stride=0, p=0.5, rng=P, at=0, out=P, out_stride=8, stream=None)


@pytest.mark.parametrize("by", [dict(x=None), dict(out=None), dict(dtype=-1), dict(p=-0.1), dict(p=1.1), dict(p=float("nan")), dict(rng=None),
                                dict(rng=P + 4), dict(at=-1), dict(at=(1 << 62) + 1), dict(residual=P, residual_stride=7), dict(cols=0),
                                dict(x_stride=3), dict(out_stride=3), dict(x=P + 2)])
def test_dropout_refuses(lib, by):
    assert lib.sbc_dropout(*changed(DROP, **by)) == BAD


def test_dropout_of_no_rows(lib):
    assert lib.sbc_dropout(*changed(DROP, rows=0, x=None, out=None)) == OK


def gated_weights(**by):
    d = sbc.GatedDesc(P, P, 24, 24, 16, 24, 1, 0)
    for name, value in by.items():
        setattr(d, name, value)
    return C.byref(d)


GATED = dict(w=None, x=P, tokens=100, x_stride=24, h=P, h_stride=16, kept=None, workspace=None, workspace_bytes=0, status=None, stream=None)
BAD_WEIGHTS = [dict(dtype=0), dict(dtype=3), dict(act=5), dict(act=-1), dict(hidden=0), dict(inner=0), dict(hidden=(1 << 31) - 1),
               dict(gate=None), dict(up=None), dict(gate_stride=23), dict(up=P + 1)]


@pytest.mark.parametrize("by", BAD_WEIGHTS)
def test_gated_refuses_weights(lib, by):
    assert lib.sbc_gated(*changed(GATED, w=gated_weights(**by))) == BAD
    assert lib.sbc_gated_workspace_bytes(gated_weights(**by), 100, P, 24, 0, 0) == 0


@pytest.mark.parametrize("by", [dict(w=None), dict(x=None), dict(h=None), dict(tokens=-1), dict(x_stride=23), dict(h_stride=15), dict(kept=P + 8),
                                dict(status=P + 2)])
def test_gated_refuses(lib, by):
    assert lib.sbc_gated(*changed(dict(GATED, w=gated_weights()), **by)) == BAD


def test_gated_workspace(lib):
    """Aligned rows need none; odd ones are copied, each matrix that has them, except for few tokens."""
    w = gated_weights()
    assert lib.sbc_gated_workspace_bytes(w, 100, P, 24, 0, 0) == 0
    assert lib.sbc_gated_workspace_bytes(w, 100, P + 2, 24, 0, 0) >= 100 * 24 * 2
    assert lib.sbc_gated_workspace_bytes(w, 5, P + 2, 25, 0, 0) == 0
    assert lib.sbc_gated_workspace_bytes(w, 5, P + 2, 25, 1, 0) >= 5 * 24 * 2
    assert lib.sbc_gated_workspace_bytes(w, 5, P, 24, 0, 1) >= 2 * 5 * 16 * 2
    assert lib.sbc_gated_kept_bytes(5, 15) == 5 * 16 * 8 and lib.sbc_gated_kept_bytes(5, 0) == 0
    odd = gated_weights(inner=23, gate_stride=23, up_stride=23)
    need = lib.sbc_gated_workspace_bytes(odd, 100, P, 24, 0, 0)
    assert need >= 2 * 16 * 24 * 2
    assert lib.sbc_gated(*changed(GATED, w=odd)) == BAD
    assert lib.sbc_gated(*changed(GATED, w=odd, workspace=P, workspace_bytes=need - 1)) == SMALL
    assert lib.sbc_gated(*changed(GATED, w=gated_weights(), tokens=0, x=None, h=None)) == OK


GATED_GRAD = dict(w=None, x=P, tokens=100, x_stride=24, dh=P, dh_stride=16, kept=P, dx=P, dx_stride=24, dgate=P, dup=P, grad_dtype=1, grad_stride=24,
                  workspace=P, workspace_bytes=1 << 30, status=None, stream=None)


@pytest.mark.parametrize("by", [dict(w=None), dict(x=None), dict(dh=None), dict(kept=None), dict(kept=P + 8), dict(dgate=None), dict(dup=None),
                                dict(dx=None, dgate=None, dup=None), dict(grad_dtype=2), dict(grad_stride=23), dict(dx_stride=23), dict(dh_stride=15),
                                dict(workspace=None), dict(tokens=-1)])
def test_gated_grad_refuses(lib, by):
    assert lib.sbc_gated_grad(*changed(dict(GATED_GRAD, w=gated_weights()), **by)) == BAD


def test_gated_grad_wants_its_workspace(lib):
    need = lib.sbc_gated_workspace_bytes(gated_weights(), 100, P, 24, 0, 1)
    assert lib.sbc_gated_grad(*changed(GATED_GRAD, w=gated_weights(), workspace_bytes=need - 1)) == SMALL
    assert lib.sbc_gated_grad(*changed(GATED_GRAD, w=gated_weights(), tokens=0, dgate=None, dup=None)) == OK


def adapters(**by):
    d = sbc.AdaptersDesc(P, P, 3, 4, 24, 16, 0, 0)
    for name, value in by.items():
        setattr(d, name, value)
    return C.byref(d)


ADAPTER = dict(w=None, x=P, dtype=1, tokens=10, x_stride=24, ids=P, plan=None, scale=1.0, base=None, base_stride=0, out=P, out_stride=16, mid=None,
               status=None, stream=None)


@pytest.mark.parametrize("by", [dict(down=None), dict(up=None), dict(count=0), dict(count=sbc.ADAPTER_COUNT + 1), dict(rank=0), dict(rank=sbc.ADAPTER_RANK + 1),
                                dict(inner=0), dict(outer=(1 << 30) + 1), dict(dtype=2), dict(reserved=1), dict(down=P + 2)])
def test_adapter_refuses_adapters(lib, by):
    assert lib.sbc_adapter(*changed(ADAPTER, w=adapters(**by))) == BAD


@pytest.mark.parametrize("by", [dict(w=None), dict(x=None), dict(out=None), dict(ids=None), dict(ids=P + 2), dict(tokens=-1), dict(tokens=sbc.ADAPTER_FEW + 1),
                                dict(mid=P), dict(plan=P), dict(plan=P + 8, mid=P), dict(plan=P, mid=P + 8), dict(x_stride=23), dict(out_stride=15),
                                dict(base=P, base_stride=15), dict(dtype=3), dict(status=P + 1)])
def test_adapter_refuses(lib, by):
    assert lib.sbc_adapter(*changed(dict(ADAPTER, w=adapters()), **by)) == BAD


def test_adapter_plan_refuses(lib):
    need = lib.sbc_adapter_plan_bytes(10, 3)
    assert need > 0 and lib.sbc_adapter_plan_bytes(-1, 3) == 0 and lib.sbc_adapter_plan_bytes(10, 0) == 0 and lib.sbc_adapter_plan_bytes((1 << 24) + 1, 3) == 0
    assert lib.sbc_adapter_mid_bytes(10, 17) == 10 * 32 * 6 and lib.sbc_adapter_mid_bytes(10, 0) == 0
    for ids, tokens, count, plan, size in ((None, 10, 3, P, need), (P + 1, 10, 3, P, need), (P, -1, 3, P, need), (P, 10, 0, P, need), (P, 10, 3, None, need),
                                           (P, 10, 3, P + 8, need)):
        assert lib.sbc_adapter_plan(ids, tokens, count, plan, size, None, None) == BAD
    assert lib.sbc_adapter_plan(P, 10, 3, P, need - 1, None, None) == SMALL
    assert lib.sbc_adapter(*changed(ADAPTER, w=adapters(), tokens=0, x=None, out=None, ids=None)) == OK


ADAPTER_GRAD = dict(w=None, dy=P, dy_stride=16, x=P, x_stride=24, dtype=1, tokens=10, plan=P, mid=P, scale=1.0, base=None, base_stride=0, dx=P,
                    dx_stride=24, ddown=P, dup=P, dmid=P, stream=None)


@pytest.mark.parametrize("by", [dict(w=None), dict(dy=None), dict(x=None), dict(plan=None), dict(mid=None), dict(dmid=None), dict(dx=None, ddown=None, dup=None),
                                dict(dy_stride=15), dict(dx_stride=23), dict(base=P, base_stride=23), dict(ddown=P + 2), dict(dup=P + 1), dict(plan=P + 4)])
def test_adapter_grad_refuses(lib, by):
    assert lib.sbc_adapter_grad(*changed(dict(ADAPTER_GRAD, w=adapters()), **by)) == BAD


def test_block_functions_check_before_the_library():
    """Arguments that are not on a GPU are refused by the binding itself."""
    import torch

    x = torch.zeros(4, 8)
    for call in (lambda: sbc.sbc_layer_norm(x), lambda: sbc.sbc_dropout(x, 0.5, torch.zeros(2, dtype=torch.int64)), lambda: sbc.sbc_gated(x, x, x),
                 lambda: sbc.sbc_adapter(x, x[None], x[None], None), lambda: sbc.sbc_adapter_plan(torch.zeros(3, dtype=torch.int32), 2)):
        with pytest.raises(TypeError):
            call()
