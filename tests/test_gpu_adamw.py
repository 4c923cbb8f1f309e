"""AdamW over a list of tensors against its definition: parameters within the rounding of fp32, moments of 8 bits bit for bit."""
import sys

import numpy as np
import pytest

import block_ref as ref
from test_gpu_dense import host, kb    # noqa: F401  (kb: the fixture)

pytestmark = pytest.mark.gpu
HYPER = dict(lr=0.01, beta1=0.9, beta2=0.999, eps=1e-8)
U = ref.U


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def gpu(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def make(shape, seed, rows="all", part=0.4):
    """(param, grad, which rows the step takes) of a tensor; gradients of all magnitudes, zeros among them"""
    rng = np.random.default_rng(seed)
    p = rng.normal(0, 1, shape).astype(np.float32)
    g = (rng.normal(0, 1, shape) * 10.0 ** rng.integers(-5, 1, shape)).astype(np.float32)
    g.reshape(-1)[::11] = 0.0
    on = np.ones(shape[0] if len(shape) == 2 else 1, bool)
    if rows != "all":
        on = rng.random(shape[0]) < part
        if rows == "nonzero":
            g[~on] = 0.0
            g[on, -1] = 1e-3
    return p, g, on


def as_rows(x):
    return x if x.ndim == 2 else x.reshape(1, -1)


def param_bound(p, m, v, g, t, wd):
    """fp32's rounding of p and of the step: the moments' roundings against the sum of their terms' magnitudes, and ten more"""
    lr, b1, b2, eps = (float(np.float32(HYPER[k])) for k in ("lr", "beta1", "beta2", "eps"))
    p, m, v, g = (np.abs(np.asarray(x, np.float64)) for x in (p, m, v, g))
    den = np.sqrt((b2 * v + (1 - b2) * g * g) / (1 - b2 ** t)) + eps
    step = (b1 * m + (1 - b1) * g) / (1 - b1 ** t) / den
    return 2 * U * (p + lr * (wd * p + step)) + 14 * U * lr * (wd * p + step)


def tensor(kb, p, g, bits, rows, on, wd, copy, shift=0):  # noqa: F811
    """The dict of one tensor; shift: its arrays start that many elements into their allocations"""
    import torch

    def place(t):
        if not shift:
            return t
        flat = torch.zeros(t.numel() + shift, dtype=torch.uint8, device="cuda").view(t.dtype) if t.element_size() == 1 else torch.zeros(
            t.numel() + shift, dtype=t.dtype, device="cuda")
        flat = flat[shift:].view(t.shape)
        flat.view(torch.uint8 if t.element_size() == 1 else t.dtype).copy_(t.view(torch.uint8) if t.element_size() == 1 else t)
        return flat
    q = gpu(p)
    st = kb.adamw_state(q, bits)
    out = dict(param=place(q), grad=place(gpu(g)), weight_decay=wd, rows=rows,
               row_mask=gpu((on * 3).astype(np.uint8)) if rows == "mask" else None,
               copy=place(torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")) if copy else None)
    return dict(out, m=place(st["m"]), v=place(st["v"]), m_scale=st["m_scale"], v_scale=st["v_scale"])


SHAPES = [(1, 1), (1, 255), (1, 256), (3, 4), (40, 5), (33, 30), (70, 64), (21, 100), (17, 256), (9, 259), (4, 1028), (1, 65001), (3000, 36)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("rows", ["all", "mask", "nonzero"])
def test_steps_of_a_list(kb, bits, rows):  # noqa: F811
    import torch
    say("adamw", bits, rows)
    for shift in (0, 1):
        cases = [make(s, i + 1, rows) for i, s in enumerate(SHAPES)]
        list_ = [tensor(kb, p, g, bits, rows, on, 0.0 if i % 2 else 0.1, i % 3 == 0, shift) for i, (p, g, on) in enumerate(cases)]
        plan = kb.AdamWTensors(list_)
        for t in (1, 2, 3):
            before = [{k: w[k].clone() for k in ("param", "m", "v", "m_scale", "v_scale", "copy") if w.get(k) is not None} for w in list_]
            kb.adamw_step(plan, t=t, **HYPER)
            torch.cuda.synchronize()
            for (p, g, on), w, b, shape in zip(cases, list_, before, SHAPES):
                say("tensor", shape, "t", t, "shift", shift)
                wd = float(np.float32(w["weight_decay"]))
                m, v = host(b["m"].float()), host(b["v"].float())
                if bits == 8:
                    spread = lambda s: np.repeat(host(s), ref.BLOCK, 1)[:, :shape[1]]  # noqa: E731
                    m, v = m * spread(b["m_scale"]), v * spread(b["v_scale"])
                m, v = m.astype(np.float32), v.astype(np.float32)
                want, m64, v64 = ref.adamw(host(b["param"]), m, v, g, t, wd=wd, **HYPER)
                got = host(w["param"])
                off = np.abs(got - want)[on]
                assert (off <= param_bound(host(b["param"]), m, v, g, t, wd)[on]).all()
                m32, v32 = ref.moments(m, v, g, HYPER["beta1"], HYPER["beta2"])
                if bits == 32:
                    np.testing.assert_array_equal(w["m"].cpu().numpy()[on], m32[on])
                    np.testing.assert_array_equal(w["v"].cpu().numpy()[on], v32[on])
                else:
                    for name, x, form in (("m", m32, ref.E4M3), ("v", v32, ref.E5M2)):
                        q, s = ref.encode(x, form, t)
                        np.testing.assert_array_equal(host(w[name + "_scale"])[on], s[on].astype(np.float64))
                        np.testing.assert_array_equal(host(w[name].float())[on], q[on])
                if w["copy"] is not None:
                    assert bool((w["copy"] == w["param"].to(torch.bfloat16))[gpu(on)].all())
                for name, old in b.items():       # rows that the step did not take: as they were, bit for bit
                    new = w[name][gpu(~on)] if w[name].element_size() > 1 else w[name].view(torch.uint8)[gpu(~on)]
                    old = old[gpu(~on)] if old.element_size() > 1 else old.view(torch.uint8)[gpu(~on)]
                    assert bool((new == old).all()), name


def test_more_tensors_than_a_launch_takes(kb):  # noqa: F811
    import torch
    cases = [make((1, 50 + i), i) for i in range(75)]
    both = [[tensor(kb, p, g, 8 if i % 2 else 32, "all", on, 0.01, False) for i, (p, g, on) in enumerate(cases)] for _ in range(2)]
    kb.adamw_step(both[0], t=1, **HYPER)
    for w in both[1]:
        kb.adamw_step([w], t=1, **HYPER)
    for a, b in zip(*both):
        assert bool((a["param"] == b["param"]).all()) and bool((a["m"].float() == b["m"].float()).all())
        assert not bool((a["param"] == gpu(cases[0][0][:1, :1])).all())
    kb.adamw_step([], t=1, **HYPER)
    empty = torch.empty((0, 8), device="cuda")
    kb.adamw_step([dict(param=empty, grad=empty.clone(), m=empty.clone(), v=empty.clone()), both[0][0]], t=2, **HYPER)


def test_averages_of_8_bits_follow_those_of_32(kb):  # noqa: F811
    """A gradient that stays for 3000 steps and then is gone for 3000: v must rise to g^2 and fall again, in steps of a thousandth where the
    format's numbers are up to a quarter (D) apart.  A step moves v by D v with probability 0.001 / D: its mean is v, its variance 0.001 D v^2.
    Where the average forgets (0.002 a step) that adds up to D / 2 <= 1/8 of v^2; where nothing pulls v back, its logarithm's variance
    over 3000 steps is at most 3 D <= 3/4.  The mean over 2048 elements is then within 0.1, four of its deviations, of one."""
    import torch
    rng = np.random.default_rng(2)
    g = np.exp(rng.normal(0, 1, (8, 256))).astype(np.float32)
    w8, w32 = (tensor(kb, np.zeros_like(g), g, bits, "all", None, 0.0, False) for bits in (8, 32))
    plan = kb.AdamWTensors([w8, w32])
    grads = [w["grad"] for w in (w8, w32)]
    for phase, scale in (("rise", 1.0), ("fall", 0.0)):
        for x in grads:
            x.mul_(scale)
        for t in range(1, 3001):
            kb.adamw_step(plan, lr=0.0, beta1=0.9, beta2=0.999, eps=1e-8, t=t + (3000 if phase == "fall" else 0))
        v8, v32 = host(w8["v"].float()) * host(w8["v_scale"]), host(w32["v"])
        say(phase, "v8 / v32: mean", (v8 / v32).mean(), "spread", (v8 / v32).std())
        assert 0.9 < (v8 / v32).mean() < 1.1, phase
        if phase == "rise":
            assert (v8 / v32).std() <= np.sqrt(1 / 8) * 1.1
        else:
            assert np.log(v8 / v32).std() <= np.sqrt(3 / 4) * 1.1
    assert bool((w8["param"] == 0).all()), "a learning rate of zero moves nothing"


def test_numbers_that_are_not_finite_and_blocks_of_zeros(kb):  # noqa: F811
    import torch
    p, g, on = make((4, 512), 1)
    g[1, 300], g[2, 5] = np.inf, np.nan
    g[3, :256] = 0.0
    w = tensor(kb, p, g, 8, "all", on, 0.0, False)
    kb.adamw_step([w], t=1, **HYPER)
    torch.cuda.synchronize()
    s = host(w["m_scale"])
    assert np.isnan(s[1, 1]) and np.isnan(s[2, 0]) and s[3, 0] == 0.0 and np.isfinite(s[[0, 1, 2, 3], [0, 0, 1, 1]]).all()
    assert not bool(w["m"].view(torch.uint8)[3, :256].any()) and not bool(w["v"].view(torch.uint8)[3, :256].any())
    new = host(w["param"])
    fine = np.ones((4, 512), bool)
    fine[1, 300] = fine[2, 5] = False
    assert np.isfinite(new[fine]).all() and not np.isfinite(new[2, 5])
    assert np.array_equal(new[3, :256], p[3, :256].astype(np.float64))


@pytest.mark.parametrize("bits", [32, 8])
def test_another_stream_a_step_number_on_the_device_and_a_graph(kb, bits):  # noqa: F811
    import torch
    shapes = [(200, 72), (1, 3001), (50, 300)]
    cases = [make(s, 5 + i, "mask" if i == 0 else "all") for i, s in enumerate(shapes)]
    fresh = lambda: [tensor(kb, p, g, bits, "mask" if i == 0 else "all", on, 0.1, i == 1) for i, (p, g, on) in enumerate(cases)]  # noqa: E731
    a, b = fresh(), fresh()
    for t in range(1, 5):
        kb.adamw_step(a, t=t, **HYPER)
    step = torch.ones(1, dtype=torch.int64, device="cuda")
    plan = kb.AdamWTensors(b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    kb.adamw_step(plan, t_dev=step, stream=side, **HYPER)       # t = 1
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kb.adamw_step(plan, t_dev=step, **HYPER)
    for t in range(2, 5):
        step.fill_(t)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
    for x, y in zip(a, b):
        for k in ("m", "v"):
            assert bool((x[k].view(torch.uint8) == y[k].view(torch.uint8)).all()), k
        # the corrections 1 / (1 - beta^t) come from the host's pow there and from products here: a rounding of each apart
        assert float((x["param"] - y["param"]).abs().max()) <= 8 * U * (float(x["param"].abs().max()) + 4 * HYPER["lr"])
