"""The norm of all gradients and their scaling, and AdamW with a factor from device memory, against their definitions in 64 bits."""
import math
import sys

import numpy as np
import pytest

import answer_ref as ref
from test_gpu_dense import kb    # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu
U = ref.U
HALF = {"f32": ref.U, "bf16": ref.H}


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def make(shapes, kind, seed, spread=3):
    """[(tensor, numbers in 64 bits, mask or None)]"""
    import torch
    rng = np.random.default_rng(seed)
    out = []
    for i, shape in enumerate(shapes):
        x = (rng.normal(0, 1, shape) * 10.0 ** rng.integers(-spread, spread + 1)).astype(np.float32)
        t = torch.from_numpy(x).cuda().to(torch.bfloat16 if kind == "bf16" else torch.float32)
        out.append((t, t.double().cpu().numpy(), None))
    return out


def check(kb, grads, most, scale=True, kind="f32"):  # noqa: F811
    import torch
    plan = kb.GradTensors([dict(grad=t, row_mask=None if m is None else torch.from_numpy(m).cuda()) for t, _, m in grads])
    counted = [x if m is None else x[m != 0] for _, x, m in grads]
    total = ref.norm(counted)
    norm, factor = (kb.clip_grads if scale else kb.grad_norm)(plan, most)
    f = ref.factor(total, most)
    assert abs(float(norm) - total) <= 2 * U * total             # a rounding to fp32; the sum in 64 bits is far below it
    assert abs(float(factor) - f) <= 2 * U * f
    f = float(factor)
    for t, x, m in grads:
        want = x * f if scale else x
        if m is not None:
            want = np.where((m != 0)[:, None], want, x)
        far = np.abs(t.double().cpu().numpy() - want)
        assert (far <= (HALF[kind] + (U if kind == "bf16" else 0.0)) * np.abs(want) + 2.0 ** -149 if kind == "f32" else
                far <= (ref.H + U) * np.abs(want) + 2.0 ** -133).all()
    return float(norm), f


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("shapes", [[(1,)], [(3,)], [(63,), (64,), (65,)], [(255, 3), (1, 257)], [(1000, 32), (10, 32), (4, 1024), (20, 4), (32, 32)],
                                    [(7, 5)] * 60, [(4097,)] * 3, [(0,), (5,), (0, 4)], [(300000,), (3,), (70001, 13)]])
def test_norm_and_scaling(kb, shapes, kind):  # noqa: F811
    for most in (0.1, 1e30, 0.0):
        for scale in (False, True):
            say(shapes[:4], len(shapes), kind, most, scale)
            check(kb, make(shapes, kind, len(shapes)), most, scale, kind)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d", [(1, 7), (5, 1), (1000, 3), (999, 17), (513, 64), (100, 200), (77, 256), (50, 257), (33, 1031), (20011, 40)])
def test_rows_that_do_not_count(kb, rows, d, kind):  # noqa: F811
    """Rows with a mask of zero are neither read - they hold infinities here - nor written"""
    import torch
    rng = np.random.default_rng(rows)
    say(rows, d, kind)
    grads = make([(rows, d), (31,)], kind, d)
    m = (rng.random(rows) < 0.6).astype(np.uint8) * 255
    t, x, _ = grads[0]
    t[torch.from_numpy(m == 0).cuda()] = math.inf
    x = t.double().cpu().numpy()
    plan = kb.GradTensors([dict(grad=t, row_mask=torch.from_numpy(m).cuda()), grads[1][0]])
    total = ref.norm([x[m != 0], grads[1][1]])
    norm, factor = kb.clip_grads(plan, 0.25 * total)
    assert abs(float(norm) - total) <= 2 * U * total and abs(float(factor) - 0.25) <= 4 * U
    got = t.double().cpu().numpy()
    assert np.isinf(got[m == 0]).all()
    got, x = got[m != 0], x[m != 0]
    assert (np.abs(got - x * float(factor)) <= (HALF[kind] + U) * np.abs(x) * 0.25 + 2.0 ** -133).all()


def test_shifted_and_mixed_types(kb):  # noqa: F811
    """Tensors that start at any element, of both types in one list"""
    import torch
    for shift in (1, 2, 3):
        base, half = torch.randn(5000, device="cuda"), torch.randn(5000, device="cuda").bfloat16()
        g = [base[shift:shift + 1201], half[shift:shift + 777].view(7, 111)]
        want = [t.double().cpu().numpy() for t in g]
        rest = (base[shift + 1201:].clone(), half[shift + 777:].clone(), base[:shift].clone())
        total = ref.norm(want)
        norm, factor = kb.clip_grads(kb.GradTensors(g), 0.5 * total)
        assert abs(float(norm) - total) <= 2 * U * total
        for t, x, h in zip(g, want, (U, ref.H + U)):
            assert (np.abs(t.double().cpu().numpy() - x * float(factor)) <= h * np.abs(x)).all()
        assert torch.equal(rest[0], base[shift + 1201:]) and torch.equal(rest[1], half[shift + 777:]) and torch.equal(rest[2], base[:shift])


def test_large_and_small_numbers(kb):  # noqa: F811
    """Squares that leave fp32's range on either side"""
    for size in (1e30, 1e-30, 1e-42):
        x = np.full((300, 40), size, np.float32)
        import torch
        t = torch.from_numpy(x.copy()).cuda()
        total = ref.norm([x])
        norm, factor = kb.clip_grads([t], total / 4)
        assert abs(float(norm) - total) <= 2 * U * total + 2.0 ** -150 and abs(float(factor) - 0.25) <= 1e-6 + 2.0 ** -149 / total
    t = torch.full((1000,), 3e38, device="cuda")                 # the norm is beyond fp32, the factor is not
    norm, factor = kb.clip_grads([t], 1.0)
    f = 1.0 / (float(np.float32(3e38)) * math.sqrt(1000))        # 1.05e-40, a subnormal number: off by half of fp32's smallest step, 2^-150
    assert math.isinf(float(norm)) and abs(float(factor) - f) <= 2.0 ** -150 + 2 * U * f
    assert abs(float(t.double().norm()) - 1) <= 2.0 ** -150 / f + 4 * U


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_gradients_that_are_not_finite(kb, bad):  # noqa: F811
    import torch
    t, o = torch.randn(70, 9, device="cuda"), torch.randn(1000, device="cuda")
    t[3, 4] = bad
    was = t.clone()
    norm, factor = kb.grad_norm([t, o], 1.0)
    assert not math.isfinite(float(norm)) and math.isnan(float(norm)) == math.isnan(bad) and math.isnan(float(factor))
    assert torch.equal(t.nan_to_num(7.0), was.nan_to_num(7.0))
    kb.clip_grads([t, o], 1.0)
    assert torch.isnan(t).all() and torch.isnan(o).all()


def test_a_factor_of_one_writes_nothing_and_no_limit(kb):  # noqa: F811
    import torch
    t = torch.randn(40000, device="cuda")
    was = t.clone()
    norm, factor = kb.clip_grads([t], 1e9)
    assert float(factor) == 1.0 and torch.equal(t, was)
    norm, factor = kb.grad_norm([t])
    assert float(factor) == 1.0 and abs(float(norm) - float(was.double().norm())) <= 2 * U * float(norm)
    z = torch.zeros(100, device="cuda")
    norm, factor = kb.clip_grads([z], 0.0)
    assert float(norm) == 0.0 and float(factor) == 1.0
    e = torch.empty(0, device="cuda")
    norm, factor = kb.clip_grads([e], 0.0)
    assert float(norm) == 0.0 and float(factor) == 1.0


def test_repeats_and_workspaces(kb):  # noqa: F811
    """The same bits again, from a workspace that held anything, on another stream, and in a list past one launch"""
    import torch
    grads = [torch.randn(1 + 977 * i, device="cuda") for i in range(110)]
    plan = kb.GradTensors(grads)
    first = [float(x) for x in kb.grad_norm(plan, 0.5)]
    assert abs(first[0] - ref.norm([g.double().cpu().numpy() for g in grads])) <= 2 * U * first[0]
    ws = torch.full((kb.grad_norm_workspace_bytes(110),), 255, dtype=torch.uint8, device="cuda")
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for stream in (None, other, None):
        n, f = kb.grad_norm(plan, 0.5, workspace=ws, stream=stream)
        torch.cuda.synchronize()
        assert [float(n), float(f)] == first
        ws.fill_(254)
    n, f = kb.clip_grads(plan, 0.5)
    assert [float(n), float(f)] == first
    after = ref.norm([g.double().cpu().numpy() for g in grads])
    assert abs(after - 0.5) <= 4 * U


def test_captured_and_replayed(kb):  # noqa: F811
    import torch
    g = [torch.randn(5000, 8, device="cuda"), torch.randn(300, device="cuda")]
    mask = torch.ones(5000, dtype=torch.uint8, device="cuda")
    plan = kb.GradTensors([dict(grad=g[0], row_mask=mask), g[1]])
    norm, factor = torch.empty((), device="cuda"), torch.empty((), device="cuda")
    ws = torch.empty(kb.grad_norm_workspace_bytes(2), dtype=torch.uint8, device="cuda")
    kb.clip_grads(plan, 1.0, norm, factor, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kb.clip_grads(plan, 1.0, norm, factor, ws)
    for i in range(4):
        for t in g:
            t.copy_(torch.randn_like(t) * (i + 1))
        mask.copy_((torch.rand(5000, device="cuda") < 0.5).to(torch.uint8))
        want = [t.double().cpu().numpy() for t in g]
        m = mask.cpu().numpy() != 0
        graph.replay()
        torch.cuda.synchronize()
        total = ref.norm([want[0][m], want[1]])
        assert abs(float(norm) - total) <= 2 * U * total
        got = g[0].double().cpu().numpy()
        assert np.array_equal(got[~m], want[0][~m]) and (np.abs(got - want[0] * float(factor))[m] <= U * np.abs(want[0][m])).all()


def test_more_than_2_to_31_elements(kb):  # noqa: F811
    import torch
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    n = (1 << 31) + 1000
    t = torch.full((n,), 0.5, device="cuda")
    t[-1] = 2.0
    total = math.sqrt(0.25 * (n - 1) + 4.0)
    norm, factor = kb.clip_grads([t], total / 2)
    assert abs(float(norm) - total) <= 2 * U * total and abs(float(factor) - 0.5) <= U
    f = float(factor)
    assert float(t[-1]) == np.float32(2.0 * f) and bool((t[:-1] == 0.5 * f).all())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("rows", ["all", "mask", "nonzero"])
def test_adamw_takes_the_factor(kb, bits, rows):  # noqa: F811
    """A step with a factor is the step with gradients multiplied by it beforehand, bit for bit; a NaN leaves everything"""
    import torch
    torch.manual_seed(3)
    shape = (300, 70)
    p = torch.randn(shape, device="cuda")
    g = torch.randn(shape, device="cuda") * (torch.rand(shape[0], 1, device="cuda") < 0.5)
    mask = (torch.rand(shape[0], device="cuda") < 0.5).to(torch.uint8)

    def tensors(g):
        t = dict(param=p.clone(), grad=g, rows=rows, row_mask=mask if rows == "mask" else None, weight_decay=0.1,
                 copy=torch.zeros(shape, dtype=torch.bfloat16, device="cuda"), **kb.adamw_state(p, bits))
        return [t]
    factor = torch.tensor([0.37], device="cuda")
    a, b = tensors(g), tensors(g * 0.37)
    for t in (1, 2, 3):
        kb.adamw_step(a, lr=0.1, t=t, factor=factor)
        kb.adamw_step(b, lr=0.1, t=t)
        for k in ("param", "m", "v", "m_scale", "v_scale", "copy"):
            if a[0][k] is not None:
                x, y = a[0][k], b[0][k]
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), (k, t)
    was = {k: a[0][k].clone() for k in ("param", "m", "v", "copy")}
    kb.adamw_step(a, lr=0.1, t=4, factor=torch.tensor(math.nan, device="cuda"))
    for k, x in was.items():
        assert torch.equal(a[0][k].view(torch.uint8), x.view(torch.uint8)), k


def test_a_step_whose_gradients_are_clipped(kb):  # noqa: F811
    """The two calls as a program makes them: the norm of the gradients of a list, then AdamW over it with the factor"""
    import torch
    torch.manual_seed(4)
    ps = [torch.randn(50, 20, device="cuda"), torch.randn(9, device="cuda")]
    gs = [torch.randn_like(p) * 5 for p in ps]
    mask = (torch.arange(50, device="cuda") % 3 != 0).to(torch.uint8)
    own = [dict(param=p.clone(), grad=g, **kb.adamw_state(p)) for p, g in zip(ps, gs)]
    own[0].update(rows="mask", row_mask=mask)
    norm, factor = kb.grad_norm([dict(grad=gs[0], row_mask=mask), gs[1]], 2.0)
    kb.adamw_step(own, lr=0.1, t=1, factor=factor)
    total = ref.norm([gs[0].double().cpu().numpy()[mask.cpu().numpy() != 0], gs[1].double().cpu().numpy()])
    f = 2.0 / total
    for i, (p, g) in enumerate(zip(ps, gs)):
        x, y = p.double(), g.double() * f
        m, v = 0.1 * y, 0.001 * y * y
        want = x - 0.1 * (m / 0.1) / ((v / 0.001).sqrt() + 1e-8)
        if i == 0:
            want = torch.where(mask[:, None] != 0, want, x)
        # of the first step, lr, every factor cancels but eps: a dozen roundings and those of fp32's 0.9 and 0.999
        assert (own[i]["param"].double() - want).abs().max().item() <= 20 * U * 5 + 0.1 * 1e-4
