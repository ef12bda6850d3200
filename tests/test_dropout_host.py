"""The key of dropout's modules on the host, with a stand-in for the kernel:
gradients under activation checkpointing, and that masks do not repeat."""

import pytest
import torch
from torch.utils.checkpoint import checkpoint

from paper_2609_02846_amd import dropout as module
from paper_2609_02846_amd.dropout import Dropout


@pytest.fixture(autouse=True)
def stand_in(monkeypatch):
    """Dropout by a host generator of the same key."""
    def forward(x, p, seed, tensor_id=0, residual=None):
        g = torch.Generator().manual_seed((int(seed) * 1000003 + int(tensor_id)) % 2 ** 63)
        y = torch.where(torch.rand(x.shape, generator=g) >= p, x / (1 - p), torch.zeros(()))
        return y if residual is None else residual + y
    monkeypatch.setattr(module, "dropout_forward", forward)


def gradients(m, x, w, reentrant=None):
    """Of x and w through two calls of a branch: checkpointed ones unless
    ``reentrant`` is None."""
    torch.manual_seed(7)
    x, w = x.clone().requires_grad_(), w.clone().requires_grad_()
    branch = lambda t: m(t * w, residual=t).square()  # noqa: E731
    call = branch if reentrant is None else lambda t: checkpoint(branch, t, use_reentrant=reentrant)  # noqa: E731
    call(call(x)).sum().backward()
    return x.grad, w.grad


@pytest.mark.parametrize("reentrant", [True, False])
def test_gradients_under_checkpointing(reentrant):
    """A recomputed call draws the mask of the call that it repeats."""
    x, w = torch.randn(30, 40), torch.randn(40)
    want = gradients(Dropout(0.3), x, w)
    for got, exp in zip(gradients(Dropout(0.3), x, w, reentrant), want):
        assert torch.equal(got, exp)


@pytest.mark.parametrize("reentrant", [True, False])
def test_a_counted_key_is_refused_in_a_recomputed_call(reentrant):
    """With a seed of its own the module counts its calls and cannot tell which
    one is repeated: an error, not another mask's gradients."""
    x, w = torch.randn(30, 40), torch.randn(40)
    gradients(Dropout(0.3, seed=5), x, w)
    with pytest.raises(RuntimeError, match="seed"):
        gradients(Dropout(0.3, seed=5), x, w, reentrant)


def test_modules_and_runs():
    """By default modules draw unrelated masks, and torch's generator state
    brings a run's masks back."""
    x = torch.ones(1000)
    torch.manual_seed(3)
    a, b = Dropout(0.5), Dropout(0.5)
    first = [a(x), b(x), a(x)]
    state = torch.get_rng_state()
    later = [a(x), b(x)]
    all_ = first + later
    assert all(not torch.equal(p, q) for i, p in enumerate(all_) for q in all_[:i])
    torch.set_rng_state(state)
    assert all(torch.equal(p, q) for p, q in zip([Dropout(0.5)(x), Dropout(0.5)(x)], later))


def test_seeded_calls():
    """Call c draws with key seed + c; evaluation draws nothing."""
    x = torch.ones(100)
    m = Dropout(0.5, seed=9, layer_id=2)
    calls = [m(x), m.eval()(x), m.train()(x)]
    assert torch.equal(calls[0], module.dropout_forward(x, 0.5, 9, 2)) and calls[1] is x
    assert torch.equal(calls[2], module.dropout_forward(x, 0.5, 10, 2))


def test_a_resumed_run_goes_on_with_the_count():
    """The count of a seeded module is part of the state dict; a state without
    one, or with one that the module has no use for, loads too."""
    x = torch.ones(100)
    m = torch.nn.Sequential(Dropout(0.5, seed=9), torch.nn.Identity())
    m(x), m(x)
    state = m.state_dict()
    want = m(x)
    resumed = torch.nn.Sequential(Dropout(0.5, seed=9), torch.nn.Identity())
    resumed.load_state_dict(state)
    assert torch.equal(resumed(x), want)
    assert all(isinstance(v, torch.Tensor) for v in state.values())
    m.load_state_dict({})                             # from before there was a count
    torch.nn.Sequential(Dropout(0.5), torch.nn.Identity()).load_state_dict(state)
    assert not torch.nn.Sequential(Dropout(0.5)).state_dict()
    with pytest.raises(RuntimeError, match="other"):
        m.load_state_dict({"0.other": torch.ones(1)})
