"""The feature block and AdamW as a training step uses them: block, encoder, score, their gradients and the update, against
the same loop in 64 bits."""
import sys

import numpy as np
import pytest

import block_ref as ref
from gpu_util import SEED, rel_err
from paper_2201_02791_amd import synth
from test_gpu_dense import host, kb    # noqa: F401  (kb: the fixture)

pytestmark = pytest.mark.gpu
LR, B1, B2, EPS, WD = 0.01, 0.9, 0.999, 1e-8, 0.01
NORM_EPS = 1e-5


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def small(kb, f, d, cone=True, msg=0, act=ref.SILU, block=True):  # noqa: F811
    from paper_2201_02791_amd.step import TrainStep
    spec = synth.scaled(synth.WORKLOADS[0], name="block", seed=17, n_entities=600, n_relations=6, n_triples=5000,
                        d=d, n_bases=3, n_pos=512, n_neg=2, neg_mode=1)
    head, rel, tail = synth.make_triples(spec)
    part = kb.build_partition(head, rel, tail, spec.n_entities, spec.n_relations, 1, 0, 2, spec.neg_domain)
    params = synth.make_params(spec, part.n_vert)
    rng = np.random.default_rng(5)
    if block:
        n = lambda s, *shape: rng.normal(0, s, shape).astype(np.float32)  # noqa: E731
        params["block"] = dict(X=n(1.0, part.n_vert, f), W=n(f ** -0.5, f, d), b=n(0.1, d), gamma=1.0 + n(0.1, d), beta=n(0.1, d))
    ts = TrainStep(part, params, spec.acts, msg, cone=cone, order=kb.ORDER_RELATION_WEIGHTS,
                   block=dict(act=act, residual=f == d, eps=NORM_EPS) if block else None)
    ts.set_batch(synth.make_batch(spec, part.n_core), spec.n_neg)
    return spec, (head, rel, tail), part, params, ts


@pytest.mark.parametrize("f,d,cone", [(32, 32, True), (20, 32, False)], ids=["residual_subgraph", "narrow_features"])
def test_training_loop_with_a_block_matches_64_bits(kb, orc, f, d, cone):  # noqa: F811
    import torch
    say("feature block loop", f, d, cone)
    spec, triples, part, params, ts = small(kb, f, d, cone)
    op = orc.build_partition(*triples, spec.n_entities, spec.n_relations, 1, 0, 2, spec.neg_domain)
    pos = synth.make_batch(spec, part.n_core)
    blk = params["block"]
    P = dict(M=np.asarray(params["M"], np.float64), **{k: blk[k].astype(np.float64) for k in ("W", "b", "gamma", "beta")})
    for l in range(2):
        for k in ("V", "a", "W0"):
            P["%s%d" % (k, l)] = np.asarray(params[k][l], np.float64).copy()
    st = {k: (np.zeros_like(x), np.zeros_like(x)) for k, x in P.items()}
    X, eps = blk["X"].astype(np.float64), float(np.float32(NORM_EPS))
    ts.init_optimizer(kb.OPT_ADAMW, 32, WD)
    for step in range(4):
        ts.run(spec.neg_mode, SEED, step)
        torch.cuda.synchronize()
        Z, pre = ref.dense_forward(X, P["W"], P["b"], ref.SILU, X if f == d else None)
        H0, mean, rstd = ref.norm_forward(Z, P["gamma"], P["beta"], eps)
        layers = [dict(V=P["V%d" % l], a=P["a%d" % l], W0=P["W0%d" % l], act=spec.acts[l]) for l in range(2)]
        res = orc.train_step(op, layers, H0, P["M"], pos, spec.n_neg, spec.neg_mode, SEED, step)
        dZ, dgamma, dbeta = ref.norm_backward(Z, P["gamma"], mean, rstd, res["dH0"])
        _, dW, db = ref.dense_backward(X, P["W"], pre, dZ, ref.SILU)
        grads = dict(M=res["dM"], W=dW, b=db, gamma=dgamma, beta=dbeta)
        for l in range(2):
            for k in ("V", "a", "W0"):
                grads["%s%d" % (k, l)] = res["grads"][l]["d" + k]
        # the tolerances of the suite's other training loop: fp32 steps of a model with a ReLU, Adam's quotients after it
        np.testing.assert_allclose(float(ts.loss.cpu()[0]), res["loss"], rtol=1e-4)
        tol = 1e-4 if step == 0 else 1e-3
        assert rel_err(host(ts.H0), H0) <= tol
        for name, _, g, _ in ts._opt_pairs():
            assert rel_err(host(g), grads[name]) <= (1e-3 if step == 0 else 1e-2), (step, name)
        ts.optimizer_step(kb.OPT_ADAMW, LR, B1, B2, EPS)
        for k in P:
            wd = WD if P[k].ndim > 1 else 0.0
            P[k], m, v = ref.adamw(P[k], *st[k], grads[k], step + 1, LR, B1, B2, EPS, wd)
            st[k] = (m, v)
    torch.cuda.synchronize()
    for name, p, _, _ in ts._opt_pairs():
        assert rel_err(host(p), P[name]) <= 1e-2, name


@pytest.mark.parametrize("bits", [32, 8])
def test_bf16_block_keeps_its_copy_of_the_weight(kb, bits):  # noqa: F811
    import torch
    say("bf16 feature block", bits)
    spec, _, part, _, ts = small(kb, 128, 64, msg=kb.MSG_BF16)
    ts.init_optimizer(kb.OPT_ADAMW, bits)
    first = ts.block.W.clone()
    for step in range(3):
        ts.run(spec.neg_mode, SEED, step)
        ts.optimizer_step(kb.OPT_ADAMW, LR)
        torch.cuda.synchronize()
        assert all(bool(torch.isfinite(p).all()) for _, p, _, _ in ts._opt_pairs())
    assert bool((ts.block.W_rows == ts.block.W.to(torch.bfloat16)).all()) and bool((ts.block.W != first).any())
    assert ts.opt_state["W"]["m"].dtype == (torch.float32 if bits == 32 else torch.float8_e4m3fn)
    assert ts.opt_state["b"]["m"].dtype == torch.float32, "small tensors keep 32 bits"
    z, pre = ref.dense_forward(host(ts.block.X), host(ts.block.W_rows), host(ts.block.b), ref.SILU)
    ts.forward()
    torch.cuda.synchronize()
    bound = ref.dense_forward_bound(host(ts.block.X), host(ts.block.W_rows), host(ts.block.b), ref.SILU, None, "bf16")
    assert (np.abs(host(ts.block.Z) - z) <= bound[0]).all() and (np.abs(host(ts.block.pre) - pre) <= bound[1]).all()
    with pytest.raises(ValueError):
        ts.optimizer_step(kb.OPT_ADAM)


@pytest.mark.parametrize("cone", [True, False], ids=["mask", "nonzero_rows"])
def test_adamw_of_a_table_moves_the_rows_that_adam_moves(kb, cone):  # noqa: F811
    """Without weight decay AdamW is Adam: the same step as the per-tensor calls, on the same rows of the entity table."""
    import torch
    both = [small(kb, 0, 32, cone, block=False) for _ in range(2)]
    spec, ts, tw = both[0][0], both[0][4], both[1][4]
    tw.init_optimizer(kb.OPT_ADAMW, 32, 0.0)
    for x in (ts, tw):
        x.run(spec.neg_mode, SEED, 0)
    for (name, _, g, _), (_, _, h, _) in zip(ts._opt_pairs(), tw._opt_pairs()):
        h.copy_(g)                       # atomics in dM and the layers' gradients: the low bits of two runs differ
    before = ts.H0.clone()
    ts.optimizer_step(kb.OPT_ADAM, LR)
    tw.optimizer_step(kb.OPT_ADAMW, LR)
    torch.cuda.synchronize()
    moved = (tw.H0 != before).any(1)
    assert bool((moved == (ts.H0 != before).any(1)).all()) and bool(moved.any())
    for (name, p, _, _), (_, q, _, _) in zip(ts._opt_pairs(), tw._opt_pairs()):
        # the quotient's and the parameter's own roundings, in another order
        assert float((p - q).abs().max()) <= 2.0 ** -22 * (float(p.abs().max()) + 4 * LR), name


def test_step_with_a_block_replays_from_a_hip_graph(kb):  # noqa: F811
    import torch
    spec, _, part, _, ts = small(kb, 32, 32)
    ts.run(spec.neg_mode, SEED, 1)
    torch.cuda.synchronize()
    f = ts.block
    outs = [ts.H0, f.Z, f.pre, f.mean, f.rstd]
    sums = [f.dZ, f.dW, f.db, f.dgamma, f.dbeta]       # behind dH0, whose low bits come from atomics
    want = [x.clone() for x in outs + sums]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ts.run(spec.neg_mode, SEED, 1)
    for rep in range(3):
        for x in outs + sums + [f.workspace]:
            x.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, w in zip(outs, want):
            assert bool((x == w).all()), rep
        for x, w in zip(sums, want[len(outs):]):
            assert rel_err(host(x), host(w)) <= 1e-5, rep
