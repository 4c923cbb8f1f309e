"""The answering operators and clipping as a program uses them: training steps on negatives that the model takes for true, updates with the
gradients' norm limited, answers from a trained model's table."""
import math
import sys

import numpy as np
import pytest

import answer_ref as ref
from gpu_util import SEED, rel_err
from paper_2201_02791_amd import synth
from test_gpu_dense import kb    # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu
U = ref.U


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def make(kb, cone=True, n_entities=600, n_pos=512, n_neg=3, mode=1, msg=0):  # noqa: F811
    from paper_2201_02791_amd.step import TrainStep
    spec = synth.scaled(synth.WORKLOADS[0], name="hard", seed=23, n_entities=n_entities, n_relations=6, n_triples=4000,
                        d=32, n_bases=3, n_pos=n_pos, n_neg=n_neg, neg_mode=mode)
    head, rel, tail = synth.make_triples(spec)
    part = kb.build_partition(head, rel, tail, spec.n_entities, spec.n_relations, 1, 0, 2, spec.neg_domain)
    params = synth.make_params(spec, part.n_vert)
    params["M"] = np.asarray(params["M"]) * 30                   # scores that lie apart
    pos = synth.make_batch(spec, part.n_core)

    def step():
        ts = TrainStep(part, params, spec.acts, msg, cone=cone, order=kb.ORDER_RELATION_WEIGHTS)
        ts.set_batch(pos, n_neg)
        return ts
    return spec, part, pos, step


@pytest.mark.parametrize("cone", [True, False])
@pytest.mark.parametrize("n_cand,how", [(40, dict()), (17, dict(temperature=0.5, top_k=5)), (64, dict(top_p=0.8, min_p=0.01))])
def test_a_step_on_drawn_negatives(kb, orc, cone, n_cand, how):  # noqa: F811
    import torch
    say(cone, n_cand, how)
    spec, part, pos, step = make(kb, cone)
    a, b = step(), step()
    a.set_candidates(n_cand)
    for number in (0, 1):
        u = torch.rand(len(pos), 3, device="cuda")
        a.run_hard(spec.neg_mode, SEED, number, u, **how)
        torch.cuda.synchronize()
        # the candidates are what the uniform sampler draws, and their scores those of the scoring call
        ent, side = (torch.empty_like(x) for x in (a.cand_ent, a.cand_side))
        kb.sample_negatives(part, a.pos, n_cand, spec.neg_mode, SEED, number, ent, side)
        assert torch.equal(ent, a.cand_ent) and torch.equal(side, a.cand_side)
        H, M = a.H_out.double().cpu().numpy(), a.M.double().cpu().numpy()
        h, r, t = (part.export("core_" + k)[pos] for k in "hrt")
        e, s = ent.cpu().numpy(), side.cpu().numpy() != 0
        hh, tt = np.where(s, e, h[:, None]), np.where(s, t[:, None], e)
        want = (H[hh] * M[r][:, None] * H[tt]).sum(2)
        size = np.abs(H[hh] * M[r][:, None] * H[tt]).sum(2)
        got = a.cand_scores[:, 1:].double().cpu().numpy()
        own = e == np.where(s, h[:, None], t[:, None])
        assert np.isneginf(got[own]).all() and (np.abs(got - want)[~own] <= 2 * (32 + 8) * U * size[~own]).all()
        # the draws, and what they pick
        cols, _ = ref.sample(got, u.double().cpu().numpy(), **how)
        assert np.array_equal(a.choice.cpu().numpy(), cols)
        pick = np.where(cols < 0, np.arange(3)[None, :] % n_cand, cols)
        assert np.array_equal(a.neg_ent.cpu().numpy(), np.take_along_axis(e, pick, 1))
        assert np.array_equal(a.neg_side.cpu().numpy() != 0, np.take_along_axis(s, pick, 1))
        # the step on them: that of a plain step which is given these negatives
        b.set_dropout_state(SEED, number)
        b.neg_ent.copy_(a.neg_ent)
        b.neg_side.copy_(a.neg_side)
        b.compute_graph()
        b.forward()
        b.score_loss()
        b.backward()
        torch.cuda.synchronize()
        np.testing.assert_allclose(float(a.loss), float(b.loss), rtol=1e-5)
        rows = np.unique(np.concatenate([h, t, a.neg_ent.cpu().numpy().ravel()]))
        assert rel_err(a.H_out.cpu().numpy()[rows], b.H_out.cpu().numpy()[rows]) <= 1e-6
        for x, y in [(a.dH_out, b.dH_out), (a.dM, b.dM), (a.dH0, b.dH0)] + [(p[k], q[k]) for p, q in zip(a.grads, b.grads) for k in p]:
            assert rel_err(x.cpu().numpy(), y.cpu().numpy()) <= 1e-5
        # harder than uniform negatives: what was drawn scores above the candidates' mean
        drawn = np.take_along_axis(np.where(own, want, got), pick, 1)
        assert drawn.mean() > np.where(own, 0.0, got).sum() / (~own).sum()


def test_candidates_of_another_batch_are_refused(kb):  # noqa: F811
    import torch
    spec, part, pos, step = make(kb)
    ts = step()
    u = torch.rand(len(pos), 3, device="cuda")
    with pytest.raises(ValueError):
        ts.run_hard(spec.neg_mode, SEED, 0, u)
    with pytest.raises(ValueError):
        ts.set_candidates(0)
    ts.set_candidates(20)
    with pytest.raises(ValueError):
        ts.run_hard(spec.neg_mode, SEED, 0, u[:, :2])
    for other, n_neg in ((pos[:300], 3), (np.concatenate([pos, pos]), 3), (pos, 2), (pos, 0)):
        ts.set_batch(other, n_neg)
        with pytest.raises(ValueError):
            ts.run_hard(spec.neg_mode, SEED, 0, torch.rand(len(other), max(n_neg, 1), device="cuda"))
    ts.set_batch(pos[:300], 2)
    ts.set_candidates(5)
    ts.run_hard(spec.neg_mode, SEED, 0, u[:300, :2].contiguous())


def test_positives_that_have_no_other_candidate(kb):  # noqa: F811
    """Every candidate hidden: the row is empty, and the candidates themselves are taken, as a uniform step would"""
    import torch
    spec, part, pos, step = make(kb, mode=0)
    ts = step()
    t = torch.from_numpy(part.export("core_t")[pos].astype(np.int32)).cuda()
    ent, side = t[:, None].repeat(1, 4).contiguous(), torch.zeros((len(pos), 4), dtype=torch.uint8, device="cuda")
    ent[5, 2] = (ent[5, 2] + 1) % part.n_vert
    scores = torch.zeros((len(pos), 9), device="cuda")
    kb.hide_positives(part, ts.pos, ent, side, scores[:, 3:7])
    want = torch.zeros_like(scores)
    want[:, 3:7] = -math.inf
    want[5, 5] = 0
    assert torch.equal(scores, want)
    choice, _ = kb.sample_scores(scores[:, 3:7], torch.rand(len(pos), 3, device="cuda"))
    assert bool((choice[5] == 2).all()) and bool((torch.cat([choice[:5], choice[6:]]) == -1).all())
    ne, ns = torch.empty((len(pos), 3), dtype=torch.int32, device="cuda"), torch.empty((len(pos), 3), dtype=torch.uint8, device="cuda")
    kb.pick_negatives(ent, side, choice, ne, ns)
    assert torch.equal(ne[6], ent[6, :3]) and torch.equal(ne[5], ent[5, 2].expand(3))
    # heads replaced; indices outside the partition hide nothing
    h = torch.from_numpy(part.export("core_h")[pos].astype(np.int32)).cuda()
    scores = torch.zeros((len(pos), 1), device="cuda")
    bad = ts.pos.clone()
    bad[0], bad[1] = -1, part.n_core
    kb.hide_positives(part, bad, h[:, None].contiguous(), torch.ones((len(pos), 1), dtype=torch.uint8, device="cuda"), scores)
    assert bool((scores[:2] == 0).all()) and bool(torch.isneginf(scores[2:]).all())


@pytest.mark.parametrize("cone", [True, False])
@pytest.mark.parametrize("name", ["OPT_SGD", "OPT_ADAM", "OPT_ADAMW"])
def test_updates_with_a_largest_norm(kb, name, cone):  # noqa: F811
    """A step with max_norm is the step on gradients scaled beforehand"""
    import torch
    kind = getattr(kb, name)
    spec, part, pos, step = make(kb, cone)
    a, b = step(), step()
    for ts in (a, b):
        ts.init_optimizer(kind)
    for number in range(3):
        for ts in (a, b):
            ts.run(spec.neg_mode, SEED, number)
        for (_, _, g, _), (_, _, o, _) in zip(a._opt_pairs(), b._opt_pairs()):
            o.copy_(g)                                           # atomics leave other last bits
        torch.cuda.synchronize()
        total = ref.norm([g.double().cpu().numpy() for _, _, g, _ in a._opt_pairs()])
        most = total * (0.3 if number < 2 else 2.0)
        f = np.float32(ref.factor(total, float(np.float32(most))))
        for _, _, g, _ in b._opt_pairs():
            g.mul_(float(f))
        a.optimizer_step(kind, lr=0.05, max_norm=most)
        b.optimizer_step(kind, lr=0.05)
        assert abs(float(a.grad_norm) - total) <= 2 * U * total
        for (k, p, g, _), (_, q, h, _) in zip(a._opt_pairs(), b._opt_pairs()):
            # the factor's last bit moves a gradient by a rounding, and a step of lr by a few
            assert rel_err(p.cpu().numpy(), q.cpu().numpy()) <= 1e-5, k
            if kind != kb.OPT_ADAMW:
                assert rel_err(g.cpu().numpy(), h.cpu().numpy()) <= 4 * U
    if kind == kb.OPT_ADAMW:                                     # a step whose gradients are not finite is left out
        was = [p.clone() for _, p, _, _ in a._opt_pairs()]
        a.dM[0, 0] = math.inf
        a.optimizer_step(kind, max_norm=1.0)
        assert math.isinf(float(a.grad_norm)) and all(torch.equal(x, p) for x, (_, p, _, _) in zip(was, a._opt_pairs()))


def test_what_a_step_allocates_is_its_streams(kb):  # noqa: F811
    """Memory of another stream's would be given to that one's tensors while this one may still use it"""
    import torch
    spec, part, pos, step = make(kb)
    ts = step()
    ts.init_optimizer(kb.OPT_ADAMW)
    ts.set_candidates(20)
    u, side = torch.rand(len(pos), 3, device="cuda"), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ts.run_hard(spec.neg_mode, SEED, 0, u, stream=side)
    ts.optimizer_step(kb.OPT_ADAMW, max_norm=1.0, stream=side)
    torch.cuda.synchronize()
    segments = torch.cuda.memory_snapshot()
    for t in (ts.cand_workspace, ts.grad_workspace, ts.grad_norm, ts.grad_factor):
        at, = [s for s in segments if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]]
        assert at["stream"] == side.cuda_stream


def test_a_block_and_bf16_take_a_largest_norm_too(kb):  # noqa: F811
    import torch
    from test_gpu_feature_block import small
    spec, _, part, params, ts = small(kb, 32, 32, True)
    ts.init_optimizer(kb.OPT_ADAMW, 8)
    ts.run(spec.neg_mode, SEED, 0)
    torch.cuda.synchronize()
    total = ref.norm([g.double().cpu().numpy() for _, _, g, _ in ts._opt_pairs()])
    ts.optimizer_step(kb.OPT_ADAMW, max_norm=0.1)
    assert abs(float(ts.grad_norm) - total) <= 2 * U * total and len(ts.grad_plan.tensors) == len(ts._opt_pairs())


def test_a_captured_step_on_drawn_negatives(kb):  # noqa: F811
    """Candidates, their scores, draws, the step on them, the norm of its gradients and the update, captured and replayed"""
    import torch
    spec, part, pos, step = make(kb)
    ts = step()
    ts.set_candidates(30)
    ts.init_optimizer(kb.OPT_ADAMW)
    u = torch.rand(len(pos), 3, device="cuda")
    start = [p.clone() for _, p, _, _ in ts._opt_pairs()]

    def one():
        ts.run_hard(spec.neg_mode, SEED, 5, u, top_k=10)
        ts.optimizer_step(kb.OPT_ADAMW, lr=0.0, max_norm=0.01)   # the parameters stay, so that every replay has the same scores

    one()
    torch.cuda.synchronize()
    ts.opt_t = 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one()
    for i in range(3):
        u.copy_(torch.rand(len(pos), 3, device="cuda"))
        for x in (ts.choice, ts.neg_ent, ts.neg_side, ts.dH_out):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (ts.choice, ts.neg_ent, ts.neg_side, ts.dH_out)]
        norm = float(ts.grad_norm)
        ts.run_hard(spec.neg_mode, SEED, 5, u, top_k=10)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, (ts.choice, ts.neg_ent, ts.neg_side, ts.dH_out)))
        total = ref.norm([g.double().cpu().numpy() for _, _, g, _ in ts._opt_pairs()])
        assert abs(norm - total) <= 1e-5 * total                 # the gradients' atomics
    assert all(torch.equal(x, p) for x, (_, p, _, _) in zip(start, ts._opt_pairs()))


@pytest.mark.parametrize("full", [True, False])
def test_answers(kb, full):  # noqa: F811
    import torch
    from paper_2201_02791_amd.answer import Answers
    spec, part, pos, step = make(kb)
    ts = step()
    ts.run(spec.neg_mode, SEED, 0)
    H, M = ts.H_out, ts.M
    answers = Answers(H, M, full_rows=full)
    rows = kb.table4_decode(answers.table).double().cpu().numpy()
    n = 9
    ent = torch.arange(n, dtype=torch.int32, device="cuda") * 7
    rel = torch.arange(n, dtype=torch.int32, device="cuda") % 6
    S = answers.scores(ent, rel)
    x = (H.double().cpu().numpy() if full else rows)[ent.cpu().numpy()] * M.double().cpu().numpy()[rel.cpu().numpy()]
    assert (np.abs(S.double().cpu().numpy() - x @ rows.T) <= ref.scores_bound(x, rows, True)).all()
    u = torch.rand(n, 4, dtype=torch.float64, device="cuda")
    q = torch.arange(n, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for known in (None, (q, ent.long())):
        want = S.double().cpu().numpy()
        if known is not None:
            want[np.arange(n), ent.cpu().numpy()] = -math.inf
        for how in (dict(temperature=0.0), dict(temperature=0.5, top_k=20, top_p=0.9)):
            for stream in (None, side, side.cuda_stream):
                got, share = answers.ask(ent, rel, u, known=known, stream=stream, **how)
                torch.cuda.synchronize()
                cols, p = ref.sample(want, u.cpu().numpy(), **how)
                assert np.array_equal(got.cpu().numpy(), cols) and (np.abs(share.double().cpu().numpy() - p) <= U * p).all()
