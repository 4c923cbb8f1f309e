"""Updates of a training step whose gradients have a largest norm, and after a step on drawn negatives: the number of a step, the rows of the
entity table that it takes, the memory that a captured step keeps."""
import math
import sys

import numpy as np
import pytest

from gpu_util import SEED, rel_err
from test_gpu_dense import kb    # noqa: F401  (the fixture)
from test_gpu_hard_negatives import make

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def states(ts):
    """Every tensor of the optimizer's state, by name"""
    out = {}
    for name, s in ts.opt_state.items():
        for k, t in (s.items() if isinstance(s, dict) else zip("mv", s)):
            if t is not None:
                out[name, k] = t
    return out


def same(a, b):
    import torch
    for (k, p, _, _), (_, q, _, _) in zip(a._opt_pairs(), b._opt_pairs()):
        assert torch.equal(p, q), k
    for (k, x), y in zip(states(a).items(), states(b).values()):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), k


def copy_gradients(a, b):
    for (_, _, g, _), (_, _, h, _) in zip(a._opt_pairs(), b._opt_pairs()):
        h.copy_(g)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("cone", [True, False])
def test_a_step_that_is_left_out_has_no_number(kb, cone, bits):  # noqa: F811
    """Gradients that are not finite leave parameters, moments and the number of the step as they are: what follows is what would have
    followed without that step, the first one's bias corrections among it"""
    say(cone, bits)
    spec, part, pos, step = make(kb, cone)
    a, b = step(), step()
    for ts in (a, b):
        ts.init_optimizer(kb.OPT_ADAMW, bits)
    for number, (before, after) in enumerate([(1, 0), (0, 2), (3, 0)]):
        a.run(spec.neg_mode, SEED, number)
        kept = a.dM[0, 0].item()
        for _ in range(before):
            a.dM[0, 0] = math.inf if number else math.nan
            a.optimizer_step(kb.OPT_ADAMW, lr=0.05, max_norm=1.0)
        a.dM[0, 0] = kept
        b.run(spec.neg_mode, SEED, number)                      # for its sub-graph's rows
        copy_gradients(a, b)
        for ts in (a, b):
            ts.optimizer_step(kb.OPT_ADAMW, lr=0.05, max_norm=1.0)
        for _ in range(after):
            a.dM[0, 0] = -math.inf
            a.optimizer_step(kb.OPT_ADAMW, lr=0.05, max_norm=1.0)
        same(a, b)
        assert a.opt_t == b.opt_t == number + 1


def test_steps_with_and_without_a_largest_norm_are_numbered_together(kb):  # noqa: F811
    """A norm that nothing reaches scales nothing: steps with it, left-out ones among them, and steps without it are the steps without it"""
    import torch
    spec, part, pos, step = make(kb)
    a, b = step(), step()
    for ts in (a, b):
        ts.init_optimizer(kb.OPT_ADAMW)
        ts.run(spec.neg_mode, SEED, 0)
    copy_gradients(a, b)
    kept = a.dM[0, 0].item()
    steps = 0
    for how in ("plain", "norm", "bad", "plain", "bad", "norm", "sgd", "plain", "bad", "sgd", "norm"):
        say(how)
        if how == "bad":
            a.dM[0, 0] = math.nan
            a.optimizer_step(kb.OPT_ADAMW, lr=0.05, max_norm=1e30)
            a.dM[0, 0] = kept
            continue
        steps += 1
        kind = kb.OPT_SGD if how == "sgd" else kb.OPT_ADAMW
        a.optimizer_step(kind, lr=0.05, **(dict(max_norm=1e30) if how == "norm" else {}))
        b.optimizer_step(kind, lr=0.05)
        for (k, p, _, _), (_, q, _, _) in zip(a._opt_pairs(), b._opt_pairs()):
            # of a step, lr at most while the gradients stay: the two corrections come from the host's pow there and from products here, off by a
            # rounding each, and so may be what follows (two products, a root and a reciprocal of two roundings each, the product with lr): 16
            # are allowed.  The update's own rounding may fall to the other side: two halves of a step of a number that was up to 0.6 larger
            assert bool(((p - q).abs() <= steps * U * (16 * 0.05 + 2 * (q.abs() + 0.6))).all()), k
    assert a.opt_t == b.opt_t == steps
    a.opt_t = b.opt_t = 40                                       # as a program that goes on from saved moments sets it
    for ts in (a, b):
        ts.optimizer_step(kb.OPT_ADAMW, lr=0.05, max_norm=1e30)
    assert a.opt_t == b.opt_t == 41
    torch.cuda.synchronize()


def test_the_norm_counts_steps_that_are_made(kb):  # noqa: F811
    import torch
    g = [torch.randn(300, 7, device="cuda"), torch.randn(5000, device="cuda")]
    number = torch.full((1,), 2 ** 40, dtype=torch.int64, device="cuda")
    want = [float(x) for x in kb.grad_norm(g, 0.5)]
    for bad in (None, math.inf, None, math.nan, -math.inf, None):
        if bad is not None:
            g[0][2, 3], kept = bad, g[0][2, 3].item()
        norm, factor = kb.grad_norm(g, 0.5, t_dev=number)
        if bad is not None:
            assert math.isnan(float(factor))
            g[0][2, 3] = kept
        else:
            assert [float(norm), float(factor)] == want
    assert int(number) == 2 ** 40 + 3
    ones = [torch.ones(1, device="cuda") for _ in range(100)]    # more tensors than a launch has
    kb.grad_norm(ones, 0.5, t_dev=number)
    assert int(number) == 2 ** 40 + 4
    for other in (torch.zeros(1, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.int64)):
        with pytest.raises(kb.KgeError):
            kb.grad_norm(ones, 0.5, t_dev=other)


def test_a_refused_step_has_no_number_and_leaves_the_gradients(kb):  # noqa: F811
    import torch
    spec, part, pos, step = make(kb)
    for kind in (kb.OPT_ADAM, kb.OPT_ADAMW):
        ts = step()
        ts.init_optimizer(kind)
        ts.run(spec.neg_mode, SEED, 0)
        was = [(p.clone(), g.clone()) for _, p, g, _ in ts._opt_pairs()]
        for how in (dict(beta1=1.0), dict(beta2=-0.5), dict(max_norm=-1.0), dict(max_norm=math.nan)):
            with pytest.raises(kb.KgeError):
                ts.optimizer_step(kind, **dict(dict(max_norm=1e-3), **how))
            assert ts.opt_t == 0
            assert all(torch.equal(x, p) and torch.equal(y, g) for (x, y), (_, p, g, _) in zip(was, ts._opt_pairs()))
        ts.optimizer_step(kind, max_norm=1e-3)
        assert ts.opt_t == 1


def test_replays_of_a_captured_step_are_steps(kb):  # noqa: F811
    """A step captured after an eager one counts on the device: each replay has a number of its own, but for those that are left out"""
    import torch
    spec, part, pos, step = make(kb)
    a, b = step(), step()
    for ts in (a, b):
        ts.init_optimizer(kb.OPT_ADAMW)
        ts.run(spec.neg_mode, SEED, 0)
    copy_gradients(a, b)
    for ts in (a, b):
        ts.optimizer_step(kb.OPT_ADAMW, lr=0.05, max_norm=0.01)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.optimizer_step(kb.OPT_ADAMW, lr=0.05, max_norm=0.01)
    kept = a.dM[0, 0].item()
    for number in (2, 3, 4):
        graph.replay()
        a.dM[0, 0] = math.inf
        graph.replay()                                           # left out
        a.dM[0, 0] = kept
        b.optimizer_step(kb.OPT_ADAMW, lr=0.05, max_norm=0.01)
        same(a, b)
        assert a.opt_t == b.opt_t == number
    for ts in (a, b):
        ts.optimizer_step(kb.OPT_ADAMW, lr=0.05)
    same(a, b)


def test_replays_of_a_step_captured_before_any_have_its_number(kb):  # noqa: F811
    import torch
    spec, part, pos, step = make(kb)
    a, b = step(), step()
    for ts in (a, b):
        ts.init_optimizer(kb.OPT_ADAMW)
        ts.run(spec.neg_mode, SEED, 0)
        ts.opt_t = 5
    copy_gradients(a, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.optimizer_step(kb.OPT_ADAMW, lr=0.05, max_norm=0.01)
    assert a.opt_t == 6
    kept = a.dM[0, 0].item()
    for _ in range(3):
        a.dM[0, 0] = math.nan
        graph.replay()                                           # left out
        a.dM[0, 0] = kept
        graph.replay()
        torch.cuda.synchronize()
        b.opt_t = 5
        b.optimizer_step(kb.OPT_ADAMW, lr=0.05, max_norm=0.01)
        same(a, b)
        assert b.opt_t == 6 and a.opt_t == 6
    for how in (dict(max_norm=0.01), dict(), dict(max_norm=0.01)):
        for ts in (a, b):
            ts.optimizer_step(kb.OPT_ADAMW, lr=0.05, **how)
        if how:
            graph.replay()                                       # its number is its own
            b.opt_t, kept_t = 5, b.opt_t
            b.optimizer_step(kb.OPT_ADAMW, lr=0.05, max_norm=0.01)
            assert b.opt_t == 6
            b.opt_t = kept_t
        assert a.opt_t == b.opt_t
    for (k, p, _, _), (_, q, _, _) in zip(a._opt_pairs(), b._opt_pairs()):
        # the step without max_norm takes its corrections from the device for one, from the host for the other: a rounding of each
        assert bool(((p - q).abs() <= 7 * U * (16 * 0.05 + 2 * (q.abs() + 0.6))).all()), k


def warm(ts, bits):
    """Moments of many steps before: every row has some"""
    import torch
    for (_, k), t in states(ts).items():
        if k.endswith("scale"):
            t.fill_(2.0 ** -9)
        elif t.element_size() == 1:
            t.view(torch.uint8).fill_(0x38)                      # 1 in e4m3, 0.5 in e5m2
        else:
            t.fill_(2e-3)


@pytest.mark.parametrize("cone", [True, False])
@pytest.mark.parametrize("name,bits", [("OPT_ADAM", 32), ("OPT_ADAMW", 32), ("OPT_ADAMW", 8)])
@pytest.mark.parametrize("most", [None, 0.05])
def test_rows_that_only_candidates_reach_are_left(kb, name, bits, cone, most):  # noqa: F811
    """An update after a step on drawn negatives takes the rows that a step on those negatives takes, moments included"""
    import torch
    say(name, bits, cone, most)
    kind = getattr(kb, name)
    spec, part, pos, step = make(kb, cone, n_entities=6000, n_pos=40, n_neg=2)
    a, b = step(), step()
    a.set_candidates(60)
    for ts in (a, b):
        ts.init_optimizer(kind, bits)
        warm(ts, bits)
    a.run_hard(spec.neg_mode, SEED, 0, torch.rand(len(pos), 2, device="cuda"))
    b.set_dropout_state(SEED, 0)
    b.neg_ent.copy_(a.neg_ent)
    b.neg_side.copy_(a.neg_side)
    b.compute_graph()
    b.forward()
    b.score_loss()
    b.backward()
    copy_gradients(a, b)                                         # atomics leave other last bits
    torch.cuda.synchronize()
    if cone:
        every = kb.ComputeGraph(part, len(a.layers))
        kb.compute_graph(part, every, a.pos, a.cand_ent)
        read, drawn = (cg.input_rows()[0] != 0 for cg in (every, b.cg))
        assert (read & ~drawn).sum() > 100 and not (drawn & ~read).any()
        assert not bool((a.dH0[torch.from_numpy(~drawn).cuda()] != 0).any())
    was = {k: t.clone() for k, t in states(a).items()}
    table = a.H0.clone()
    for ts in (a, b):
        ts.optimizer_step(kind, lr=0.05, max_norm=most)
    same(a, b)
    if cone:
        left = torch.from_numpy(~drawn).cuda()
        assert torch.equal(a.H0[left], table[left]) and not torch.equal(a.H0, table)
        for k in "mv":
            assert torch.equal(states(a)["H0", k].view(torch.uint8)[left], was["H0", k].view(torch.uint8)[left])


def test_a_captured_step_keeps_its_workspace(kb):  # noqa: F811
    """Draws of other settings want a larger workspace: the one that a graph was captured with is not given away"""
    import torch
    spec, part, pos, step = make(kb, n_pos=8, n_neg=3)
    ts = step()
    ts.set_candidates(40000)
    u = torch.rand(len(pos), 3, device="cuda")
    ts.run_hard(spec.neg_mode, SEED, 0, u, top_k=10)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ts.run_hard(spec.neg_mode, SEED, 0, u, top_k=10)
    small = ts.cand_workspace.numel()
    ts.run_hard(spec.neg_mode, SEED, 0, u, top_p=0.9)
    assert ts.cand_workspace.numel() > small
    others = [torch.full((small,), 7, dtype=torch.uint8, device="cuda") for _ in range(64)]
    torch.cuda.synchronize()
    for i in range(3):
        u.copy_(torch.rand(len(pos), 3, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = ts.choice.clone(), ts.neg_ent.clone()
        assert all(bool((t == 7).all()) for t in others)
        ts.run_hard(spec.neg_mode, SEED, 0, u, top_k=10)
        torch.cuda.synchronize()
        assert torch.equal(got[0], ts.choice) and torch.equal(got[1], ts.neg_ent)


@pytest.mark.parametrize("dropout", [0.0, 0.3])
@pytest.mark.parametrize("msg", [0, 1])
@pytest.mark.parametrize("order", ["ORDER_PROJECT_FIRST", "ORDER_RELATION_WEIGHTS"])
def test_gradients_by_the_drawn_negatives_sub_graph_only_candidates_left_out(kb, order, msg, dropout):  # noqa: F811
    """The backward pass over the drawn negatives' sub-graph is that over the candidates', which the forward pass took"""
    import torch
    from paper_2201_02791_amd import synth
    from paper_2201_02791_amd.step import TrainStep
    say(order, msg, dropout)
    spec, part, pos, _ = make(kb, n_entities=6000, n_pos=40, n_neg=2)
    ts = TrainStep(part, synth.make_params(spec, part.n_vert), spec.acts, msg, cone=True, order=getattr(kb, order), dropout=dropout)
    ts.set_batch(pos, 2)
    ts.set_candidates(60)
    ts.run_hard(spec.neg_mode, SEED, 0, torch.rand(len(pos), 2, device="cuda"))
    drawn = ts.cg.input_rows()[1]
    got = [g.clone() for _, _, g, _ in ts._opt_pairs()]
    kb.compute_graph(part, ts.cg, ts.pos, ts.cand_ent)
    assert ts.cg.input_rows()[1] > drawn + 100
    ts.backward()
    torch.cuda.synchronize()
    for x, (k, _, y, _) in zip(got, ts._opt_pairs()):
        # the same terms in another order; messages in bf16 may be rounded to the other side, by 2^-8 of one of them
        assert rel_err(x.cpu().numpy(), y.cpu().numpy()) <= (2.0 ** -7 if msg else 1e-5), k
        assert k == "M" or float(y.abs().max()) > 0


@pytest.mark.parametrize("number", [True, False])
def test_steps_on_another_stream_count_there(kb, number):  # noqa: F811
    """The number of a step is written and read in the order of the stream that the step runs on, also while that one lags behind"""
    import torch
    spec, part, pos, step = make(kb)
    a, b = step(), step()
    for ts in (a, b):
        ts.init_optimizer(kb.OPT_ADAMW)
        ts.run(spec.neg_mode, SEED, 0)
    copy_gradients(a, b)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    stream = side.cuda_stream if number else side
    for how in (dict(), dict(max_norm=0.01), dict(), dict(max_norm=0.01), dict(kind=kb.OPT_SGD), dict(max_norm=0.01)):
        with torch.cuda.stream(side):
            torch.cuda._sleep(2_000_000)
        a.optimizer_step(**dict(dict(kind=kb.OPT_ADAMW, lr=0.05, stream=stream), **how))
        b.optimizer_step(**dict(dict(kind=kb.OPT_ADAMW, lr=0.05), **how))
    assert a.opt_t == b.opt_t == 6
    same(a, b)


def test_numbers_below_one_are_refused(kb):  # noqa: F811
    import torch
    spec, part, pos, step = make(kb)
    for kind in (kb.OPT_ADAM, kb.OPT_ADAMW):
        ts = step()
        ts.init_optimizer(kind)
        ts.run(spec.neg_mode, SEED, 0)
        was = [(p.clone(), g.clone()) for _, p, g, _ in ts._opt_pairs()]
        for how in (dict(max_norm=1e-3), dict()):
            ts.opt_t = -1
            with pytest.raises(kb.KgeError, match="starts at 1"):
                ts.optimizer_step(kind, **how)
            assert ts.opt_t == -1
            assert all(torch.equal(x, p) and torch.equal(y, g) for (x, y), (_, p, g, _) in zip(was, ts._opt_pairs()))
