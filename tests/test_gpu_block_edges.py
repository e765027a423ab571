"""The operators of a client's own layers behind autograd, where a caller asks for less, or for more, than a whole step."""
import pytest
import torch
from torch.utils.checkpoint import checkpoint

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_1805_08768_b200 import binding as sbc
from paper_1805_08768_b200 import block, distill
from paper_1805_08768_b200.dsgd import DelayedSGD

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


def test_updates_are_of_the_call_that_asks():
    """Clients in any order, weights and delays of any call: nothing is answered from an earlier one.  (95 positions: a client's
    part of the batch begins at odd places.)"""
    toy = block.ToyAdapters(3, DEV, positions=95)
    other = [w + 0.05 * randn(*w.shape, seed=s) for s, w in enumerate(toy.weights)]

    def ask(client, weights, delay):
        toy.numbers.rng[1] = 5
        return toy.local_update(client, weights, delay)

    before = [w.clone() for w in toy.weights]
    first = ask(1, toy.weights, 2)                     # not the first client first
    assert all(torch.equal(a, b) for a, b in zip(before, toy.weights))
    assert all(bool(torch.isfinite(u).all()) and float(u.abs().max()) > 0 for u in first)
    assert all(torch.equal(a, b) for a, b in zip(first, ask(1, toy.weights, 2)))
    for another in (ask(1, other, 2), ask(1, toy.weights, 1), ask(2, toy.weights, 2)):
        assert not torch.equal(first[1], another[1])
    assert all(torch.equal(a, b) for a, b in zip(first, ask(1, toy.weights, 2)))
    with pytest.raises(IndexError):
        toy.local_update(3, toy.weights, 1)


def test_clients_together_and_alone():
    """Without dropout a client's update in the batch is the one that it gets alone, up to roundings that fall to the other side
    (as in test_gpu_block: within 2^-6 of the whole)."""
    toy = block.ToyAdapters(3, DEV)
    toy.block.p = 0.0
    weights = [w + 0.05 * randn(*w.shape, seed=s) for s, w in enumerate(toy.weights)]
    together = toy.local_updates(weights, 1)
    for c in range(3):
        for a, b in zip(together[c], toy.local_update(c, weights, 1)):
            assert a.shape == b.shape and float((a - b).double().norm()) <= 2.0 ** -6 * float(b.double().norm())


def test_federated_run_of_all_clients_in_one_batch():
    toy = block.ToyAdapters(3, DEV)
    run = DelayedSGD(toy.weights, 3, 0.05, 2, local_updates=toy.local_updates)
    before = [w.clone() for w in run.weights]
    for _ in range(3):
        run.round()
    run.check()
    assert len(run.last_updates) == 3 and not torch.equal(run.last_updates[0][1], run.last_updates[1][1])
    assert all(not torch.equal(a, b) and bool(torch.isfinite(b).all()) for a, b in zip(before, run.weights))
    with pytest.raises(ValueError):
        DelayedSGD(toy.weights, 3, 0.05, 2)
    with pytest.raises(ValueError):
        DelayedSGD(toy.weights, 3, 0.05, 2, toy.local_update, local_updates=toy.local_updates)
    short = DelayedSGD(toy.weights, 2, 0.05, 2, local_updates=toy.local_updates)
    with pytest.raises(ValueError):
        short.round()


@pytest.mark.parametrize("reentrant", [False, True])
def test_block_that_is_computed_again(reentrant):
    """A block under activation checkpointing gives the output and the gradients that it gives without, its dropout's numbers
    taken before; without them it is refused."""
    b = block.AdaptedBlock(96, 160, DEV, p=0.5, seed=3)
    ids = (torch.arange(70, device=DEV) % 4).to(torch.int32)
    plan = sbc.sbc_adapter_plan(ids, 4)
    dy = randn(70, 96, seed=6, dtype=torch.bfloat16)
    numbers = block.DropoutNumbers(5, DEV)

    def grads(run):
        leaves = [t.requires_grad_(True) for t in (randn(70, 96, seed=1, dtype=torch.bfloat16), randn(4, 6, 160, seed=3), randn(4, 6, 96, seed=4))]
        y = run(*leaves)
        y.backward(dy)
        return [y.detach()] + [t.grad for t in leaves]

    at = numbers.take(70 * 96)
    want = grads(lambda x, d, u: b.train(x, d, u, plan, numbers, at))
    got = grads(lambda x, d, u: checkpoint(lambda *t: b.train(*t, plan, numbers, at), x, d, u, use_reentrant=reentrant))
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    with pytest.raises(RuntimeError, match="taken in a backward pass"):
        grads(lambda x, d, u: checkpoint(lambda *t: b.train(*t, plan, numbers), x, d, u, use_reentrant=reentrant))


@pytest.mark.parametrize("tokens", [20, 90])
def test_ids_that_are_no_adapters_are_told(tokens):
    """With and without gradients, for few tokens and for many: the caller sees it, and the token is one without an adapter."""
    x, base = randn(tokens, 40, seed=1), randn(tokens, 56, seed=2)
    down, up = randn(3, 5, 40, seed=3), randn(3, 5, 56, seed=4).requires_grad_(True)
    ids = (torch.arange(tokens, device=DEV) % 3).to(torch.int32)
    wrong = ids.clone()
    wrong[tokens // 2] = 3
    told = torch.zeros(1, dtype=torch.int32, device=DEV)
    for grad in (True, False):
        with torch.set_grad_enabled(grad):
            right = block.adapter(x, down, up, ids, 1.5, base, status=told)
            assert int(told) == 0
            y = block.adapter(x, down, up, wrong, 1.5, base, status=told)
        assert int(told) == sbc.STATUS_RANGE
        told.zero_()
        others = torch.arange(tokens, device=DEV) != tokens // 2
        assert torch.equal(y[~others], base[~others]) and torch.equal(y[others], right[others])
    b = block.AdaptedBlock(96, 160, DEV, seed=3)
    b.serve(randn(tokens, 96, seed=1, dtype=torch.bfloat16), randn(3, 6, 160, seed=3), randn(3, 6, 96, seed=4), wrong, told)
    assert int(told) == sbc.STATUS_RANGE
