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
