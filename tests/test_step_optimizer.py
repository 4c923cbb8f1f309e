"""Which optimizer calls a TrainStep takes, and that a refused one changes nothing.  The kernels are replaced by a record of the calls:
no GPU is needed."""
import types

import pytest


@pytest.fixture
def made(monkeypatch):
    import torch
    from paper_2201_02791_amd import step as module
    kb, calls = module.kb, []

    def adamw(plan, lr, beta1, beta2, eps, t, stream=None):
        if beta1 >= 1.0:
            raise kb.KgeError(-1, "beta1")
        calls.append(("adamw", t))

    def other(kind, p, g, m, v, lr, beta1, beta2, eps, t, **_):
        if beta1 >= 1.0:
            raise kb.KgeError(-1, "beta1")
        assert kind == kb.OPT_SGD or (m is not None and v is not None)
        calls.append(("sgd" if kind == kb.OPT_SGD else "adam", t))
    monkeypatch.setattr(kb, "adamw_step", adamw)
    monkeypatch.setattr(kb, "optimizer_step", other)

    def make(bf16_block=False):
        ts = object.__new__(module.TrainStep)
        ts.torch, ts.cg, ts.dH0, ts.layers, ts.grads, ts.block = torch, None, None, [], [], None
        ts.M, ts.dM = torch.ones(3, 8), torch.ones(3, 8)
        if bf16_block:
            f = lambda *s: torch.ones(s)  # noqa: E731
            ts.block = types.SimpleNamespace(W=f(8, 8), W_rows=f(8, 8).bfloat16(), b=f(8), gamma=f(8), beta=f(8), dW=f(8, 8), db=f(8),
                                             dgamma=f(8), dbeta=f(8))
        del calls[:]
        return ts
    return kb, make, calls


def test_a_bf16_block_after_a_refused_first_call(made):
    kb, make, calls = made
    ts = make(bf16_block=True)
    for kind in (kb.OPT_ADAM, kb.OPT_SGD):
        with pytest.raises(ValueError):
            ts.optimizer_step(kind)
    with pytest.raises(ValueError):
        ts.optimizer_step()                       # its default
    ts.optimizer_step(kb.OPT_ADAMW)
    with pytest.raises(ValueError):
        ts.optimizer_step()
    ts.optimizer_step(kb.OPT_ADAMW)
    assert calls == [("adamw", 1), ("adamw", 2)]


@pytest.mark.parametrize("first,second", [("OPT_ADAM", "OPT_ADAMW"), ("OPT_ADAMW", "OPT_ADAM"), ("OPT_SGD", "OPT_ADAM"), ("OPT_SGD", "OPT_ADAMW")])
@pytest.mark.parametrize("lazy", [False, True])
def test_state_of_another_kind(made, first, second, lazy):
    kb, make, calls = made
    ts = make()
    first, second = getattr(kb, first), getattr(kb, second)
    if not lazy:
        ts.init_optimizer(first)
    ts.optimizer_step(first)
    with pytest.raises(ValueError, match="another kind"):
        ts.optimizer_step(second)
    ts.optimizer_step(first)
    assert [t for _, t in calls] == [1, 2]
    ts.init_optimizer(second)
    ts.optimizer_step(second)
    assert calls[-1][1] == 1


@pytest.mark.parametrize("kind", ["OPT_SGD", "OPT_ADAM", "OPT_ADAMW"])
def test_a_call_that_the_library_refuses_is_no_step(made, kind):
    kb, make, calls = made
    ts, kind = make(), getattr(kb, kind)
    ts.optimizer_step(kind)
    with pytest.raises(kb.KgeError):
        ts.optimizer_step(kind, beta1=1.0)
    ts.optimizer_step(kind)
    assert [t for _, t in calls] == [1, 2]


def test_plain_gradient_descent_beside_any_state(made):
    kb, make, calls = made
    for kind in (kb.OPT_ADAM, kb.OPT_ADAMW):
        ts = make()
        ts.init_optimizer(kind)
        ts.optimizer_step(kb.OPT_SGD)
        ts.optimizer_step(kind)
        assert calls[0] == ("sgd", 1) and calls[1][1] == 2


def test_no_such_kind(made):
    kb, make, calls = made
    ts = make()
    for call in (ts.optimizer_step, ts.init_optimizer):
        with pytest.raises(ValueError):
            call(7)
    ts.optimizer_step(kb.OPT_ADAMW)
    assert calls == [("adamw", 1)]
