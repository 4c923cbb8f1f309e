"""Dense layer (forward and backward pass) against its formula in 64 bits: types, odd and ragged sizes, strides, activations,
residuals, rows of nothing, infinities, other streams, graphs."""
import sys

import numpy as np
import pytest

import block_ref as ref

pytestmark = pytest.mark.gpu
ACTS = {"identity": ref.IDENTITY, "relu": ref.RELU, "silu": ref.SILU}


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


@pytest.fixture(scope="module")
def kb():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2201_02791_amd import binding
    binding.load()
    return binding


def tt(kind):
    import torch
    return torch.float32 if kind == "f32" else torch.bfloat16


def dev(x, kind="f32", wide=0, shift=0):
    """The matrix on the device in a type (rounded to it); wide > 0: as columns shift .. of a wider matrix of 7s."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(tt(kind)).cuda()
    if not wide or x.ndim != 2:
        return t
    buf = torch.full((x.shape[0], x.shape[1] + wide), 7.0, dtype=tt(kind), device="cuda")
    buf[:, shift:shift + x.shape[1]] = t
    return buf[:, shift:shift + x.shape[1]]


def host(t):
    return t.detach().cpu().double().numpy()


def inputs(n, di, do, seed, std=1.0):
    rng = np.random.default_rng(seed)
    return (rng.normal(0, std, (n, di)), rng.normal(0, 1.0 / np.sqrt(di), (di, do)), rng.normal(0, 0.3, do).astype(np.float32),
            rng.normal(0, std, (n, do)), rng.normal(0, 0.1, (n, do)), rng.normal(0, 0.1, (n, di)))


SIZES = [(1, 1, 1), (1, 1000, 517), (2, 7, 3), (3, 64, 32), (17, 256, 129), (128, 128, 128), (129, 33, 127), (255, 200, 200),
         (300, 203, 517), (1000, 32, 31), (600, 70, 50), (700, 30, 129), (1500, 140, 70), (2049, 130, 258), (5, 4100, 20)]


def within(got, want, bound, what):
    bad = np.abs(got - want) > bound
    assert not bad.any(), "%s: %d of %d are off, worst %g of its bound" % (
        what, bad.sum(), bad.size, float(np.max(np.abs(got - want) / np.maximum(bound, 1e-300))))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("n,di,do", SIZES)
def test_forward(kb, kind, act, n, di, do):
    say("dense forward", kind, act, n, di, do)
    X, W, b, R, _, _ = inputs(n, di, do, n + di + do)
    dX, dW, dR, db = dev(X, kind), dev(W, kind), dev(R, kind), dev(b)
    for res, bias in ((False, True), (True, True), (True, False)):
        layer = dict(W=dW, b=db if bias else None, act=ACTS[act])
        Y, pre = kb.dense_forward(layer, dX, R=dR if res else None, keep_pre=True)
        x, w, r = host(dX), host(dW), host(dR) if res else None
        y, z = ref.dense_forward(x, w, b.astype(np.float64) if bias else None, ACTS[act], r)
        by, bz = ref.dense_forward_bound(x, w, b.astype(np.float64) if bias else None, ACTS[act], r, kind)
        within(host(pre), z, bz, "pre")
        within(host(Y), y, by, "Y")
        again, none = kb.dense_forward(layer, dX, R=dR if res else None)
        assert none is None and bool((again == Y).all()), "the same call gives the same bits"


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("n,di,do", SIZES)
def test_backward(kb, kind, act, n, di, do):
    say("dense backward", kind, act, n, di, do)
    X, W, b, R, G, A = inputs(n, di, do, 3 * n + di + do)
    dX, dW, dG, dA = dev(X, kind), dev(W, kind), dev(G, kind), dev(A, kind)
    layer = dict(W=dW, b=dev(b), act=ACTS[act])
    pre = kb.dense_forward(layer, dX, keep_pre=True)[1]
    x, w, z, g = host(dX), host(dW), host(pre), host(dG)
    for add in (None, dA):
        got = kb.dense_backward(layer, dX, pre if act != "identity" else None, dG, add=add)
        a = None if add is None else host(add)
        want = ref.dense_backward(x, w, z, g, ACTS[act], a)
        bound = ref.dense_backward_bound(x, w, z, g, ACTS[act], a, kind)
        for k, name in enumerate(("dX", "dW", "db")):
            within(host(got[name]), want[k], bound[k], name)
        again = kb.dense_backward(layer, dX, pre, dG, add=add)
        assert all(bool((again[k] == got[k]).all()) for k in got), "the same call gives the same bits"
    part = kb.dense_backward(layer, dX, pre, dG, need_dX=False)
    assert part["dX"] is None and bool((part["dW"] == got["dW"]).all()) and bool((part["db"] == got["db"]).all())
    part = kb.dense_backward(layer, dX, pre, dG, need_dW=False)
    assert part["dW"] is None and part["db"] is None
    within(host(part["dX"]), host(kb.dense_backward(layer, dX, pre, dG)["dX"]), 0.0, "dX alone")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,di,do,act", [(4100, 60, 64, "silu"), (4096, 64, 100, "relu"), (4173, 33, 200, "identity"), (4101, 128, 31, "relu"),
                                         (4255, 100, 128, "silu"), (4127, 127, 257, "relu"), (4100, 250, 64, "silu"), (5000, 200, 128, "relu"),
                                         (4300, 256, 256, "silu"), (4129, 255, 515, "identity"), (33000, 96, 96, "silu"), (4100, 300, 40, "silu"),
                                         (16387, 128, 128, "silu"), (16400, 66, 200, "relu"), (17000, 120, 72, "identity"),
                                         (20001, 100, 257, "silu"), (200003, 256, 96, "silu"), (200000, 72, 136, "relu")])
def test_long_matrices_of_narrow_rows(kb, kind, n, di, do, act):
    """Every width class of the kernels that keep W in registers, both ways round, beside widths that they do not take."""
    say("dense rows", kind, n, di, do, act)
    X, W, b, R, G, A = inputs(n, di, do, n + 1)
    x, r, g, a = (dev(z, kind) for z in (X, R, G, A))
    layer = dict(W=dev(W, kind), b=dev(b), act=ACTS[act])
    Y, pre = kb.dense_forward(layer, x, R=r, keep_pre=True)
    args = host(x), host(layer["W"]), b.astype(np.float64), ACTS[act], host(r)
    for got, want, bound, what in zip((Y, pre), ref.dense_forward(*args), ref.dense_forward_bound(*args, kind), ("Y", "pre")):
        within(host(got), want, bound, what)
    if di == do:
        own = kb.dense_forward(layer, x, R=x, keep_pre=True)
        args = (*args[:4], host(x))
        within(host(own[0]), ref.dense_forward(*args)[0], ref.dense_forward_bound(*args, kind)[0], "R = X")
        assert bool((own[1] == pre).all()) and bool((kb.dense_forward(layer, x, R=x)[0] == own[0]).all())
    bare = kb.dense_forward(dict(layer, b=None), x)[0]
    within(host(bare), ref.dense_forward(args[0], args[1], None, ACTS[act])[0],
           ref.dense_forward_bound(args[0], args[1], None, ACTS[act], None, kind)[0], "Y alone")
    for add in (None, a):
        got = kb.dense_backward(layer, x, pre, g, add=add, need_dW=False)["dX"]
        args = host(x), host(layer["W"]), host(pre), host(g), ACTS[act], None if add is None else host(add)
        within(host(got), ref.dense_backward(*args)[0], ref.dense_backward_bound(*args, kind)[0], "dX")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_many_rows_in_chunks(kb, kind):
    """The weights' gradient over more rows than a chunk holds, the last chunk a short one."""
    n, di, do = 70001, 40, 24
    say("dense chunks", kind)
    X, W, b, _, G, _ = inputs(n, di, do, 5)
    dX, dG = dev(X, kind), dev(G, kind)
    layer = dict(W=dev(W, kind), b=dev(b), act=ref.SILU)
    Y, pre = kb.dense_forward(layer, dX, keep_pre=True)
    got = kb.dense_backward(layer, dX, pre, dG)
    args = host(dX), host(layer["W"]), host(pre), host(dG), ref.SILU, None
    for k, name in enumerate(("dX", "dW", "db")):
        within(host(got[name]), ref.dense_backward(*args)[k], ref.dense_backward_bound(*args, kind)[k], name)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,di,do,wide,shift", [(70, 37, 45, 3, 1), (260, 128, 64, 8, 8), (131, 96, 100, 1, 0)])
def test_strided_rows_keep_what_lies_between(kb, kind, n, di, do, wide, shift):
    import torch
    say("dense strides", kind, n, di, do, wide, shift)
    X, W, b, R, G, A = inputs(n, di, do, 9)
    flat = [dev(z, kind) for z in (X, R, G, A)]
    views = [dev(z, kind, wide, shift) for z in (X, R, G, A)]
    layer = dict(W=dev(W, kind), b=dev(b), act=ref.SILU)
    Y, pre = kb.dense_forward(layer, flat[0], R=flat[1], keep_pre=True)
    out = [torch.full((n + 2, w + wide), 5.0, dtype=tt(kind), device="cuda") for w in (do, do, di)]
    vY, vpre, vdX = (o[1:n + 1, shift:shift + w] for o, w in zip(out, (do, do, di)))
    kb.dense_forward(layer, views[0], R=views[1], Y=vY, pre=vpre)
    assert bool((vY == Y).all()) and bool((vpre == pre).all())
    want = kb.dense_backward(layer, flat[0], pre, flat[2], add=flat[3])
    got = kb.dense_backward(layer, views[0], vpre, views[2], add=views[3], dX=vdX)
    assert all(bool((got[k] == want[k]).all()) for k in want)
    for o, v in zip(out, (vY, vpre, vdX)):
        v.fill_(5.0)
        assert bool((o == 5.0).all()), "what lies around the rows stays as it was"


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_in_place_residual_and_added_gradient(kb, kind):
    n, d = 300, 72
    X, W, b, R, G, A = inputs(n, d, d, 4)
    layer = dict(W=dev(W, kind), b=dev(b), act=ref.RELU)
    x, r, g, a = (dev(z, kind) for z in (X, R, G, A))
    Y, pre = kb.dense_forward(layer, x, R=r, keep_pre=True)
    kb.dense_forward(layer, x, R=r, Y=r)
    assert bool((r == Y).all())
    own, _ = kb.dense_forward(layer, x, R=x)
    y, _ = ref.dense_forward(host(x), host(layer["W"]), b.astype(np.float64), ref.RELU, host(x))
    within(host(own), y, ref.dense_forward_bound(host(x), host(layer["W"]), b.astype(np.float64), ref.RELU, host(x), kind)[0], "R = X")
    want = kb.dense_backward(layer, x, pre, g, add=a)["dX"]
    kb.dense_backward(layer, x, pre, g, add=a, dX=a)
    assert bool((a == want).all())


def test_no_rows(kb):
    import torch
    layer = dict(W=torch.ones((5, 6), device="cuda"), b=None, act=ref.RELU)
    X, none = torch.empty((0, 5), device="cuda"), torch.empty((0, 6), device="cuda")
    Y, pre = kb.dense_forward(layer, X, keep_pre=True)
    assert tuple(Y.shape) == (0, 6) and tuple(pre.shape) == (0, 6)
    g = kb.dense_backward(layer, X, none, none)
    assert tuple(g["dX"].shape) == (0, 5) and not bool(g["dW"].any()) and not bool(g["db"].any())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n", [150, 4200, 16500])
def test_numbers_that_are_not_finite(kb, kind, n):
    """Infinities, NaN and numbers near the type's largest reach the results that fp32 products of them have, and no others."""
    import torch
    di, do = (72, 33) if n > 10000 else (40, 33)
    X, W, b, _, G, _ = inputs(n, di, do, 8)
    W[3] = np.abs(W[3]) + 0.1
    X[5, 3], X[7, 3], X[9, 2], X[11, 3] = np.inf, -np.inf, np.nan, 3.3e38 / 64
    X[13, 3], X[13, 4] = np.inf, np.inf                      # of either sign where W[4] is negative
    layer = dict(W=dev(W, kind), b=dev(b), act=ref.IDENTITY)
    x = dev(X, kind)
    Y, _ = kb.dense_forward(layer, x)
    with np.errstate(all="ignore"):
        want = host(x) @ host(layer["W"]) + b
    got = host(Y)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    inf = np.isinf(want)
    assert inf.any() and np.array_equal(got[inf], want[inf]) and np.array_equal(np.isinf(got), inf)
    fine = np.isfinite(want)
    assert np.abs(got[fine] / want[fine] - 1).max() < 1.0    # and the huge ones are no infinities
    G[3, 5], G[4, 6] = np.inf, np.nan
    g = kb.dense_backward(layer, dev(np.ones((n, di)), kind), None, dev(G, kind))
    with np.errstate(all="ignore"):
        dX, dW, db = ref.dense_backward(np.ones((n, di)), host(layer["W"]), None, host(dev(G, kind)), ref.IDENTITY)
    for a, w in ((g["dX"], dX), (g["dW"], dW), (g["db"], db)):
        a = host(a)
        assert np.array_equal(np.isnan(a), np.isnan(w)) and np.array_equal(a[np.isinf(w)], w[np.isinf(w)])
        assert np.array_equal(np.isinf(a), np.isinf(w))
    relu = dict(layer, act=ref.RELU)
    y, pre = kb.dense_forward(relu, x, keep_pre=True)
    assert np.array_equal(np.isnan(host(y)), np.isnan(want)), "ReLU keeps a NaN"
    assert not bool(torch.isnan(kb.dense_backward(relu, dev(np.ones((n, di)), kind), pre, dev(np.ones((n, do)), kind))["dW"]).any())


def test_gradients_against_differences(kb):
    """L = <C, Y> moved by +-h along a random direction of each input.  Central differences are off by h^2 / 6 of the third
    derivative (|silu'''| < 0.4, and L is linear else) and by fp32's rounding of Y (about 2^-22 of sum |C Y|) over 2 h."""
    import torch
    n, di, do, h = 200, 24, 40, 2.0 ** -6
    X, W, b, R, C, _ = inputs(n, di, do, 12)
    rng = np.random.default_rng(3)
    x, w, bb = dev(X), dev(W), dev(b)
    layer = dict(W=w, b=bb, act=ref.SILU)
    c = dev(C)
    _, pre = kb.dense_forward(layer, x, keep_pre=True)
    g = kb.dense_backward(layer, x, pre, c)
    L = lambda X_, W_, b_: float((kb.dense_forward(dict(W=W_, b=b_, act=ref.SILU), X_)[0].double() * c.double()).sum())
    size = float((kb.dense_forward(layer, x)[0].double() * c.double()).abs().sum())
    for name, at, grad in (("X", 0, g["dX"]), ("W", 1, g["dW"]), ("b", 2, g["db"])):
        base = [x, w, bb]
        step = dev(rng.normal(0, 1, tuple(base[at].shape)))
        up, down = list(base), list(base)
        up[at], down[at] = base[at] + h * step, base[at] - h * step
        got = (L(*up) - L(*down)) / (2 * h)
        want = float((grad.double() * step.double()).sum())
        moved = host(step) @ host(w) if at == 0 else host(x) @ host(step) if at == 1 else np.broadcast_to(host(step), (n, do))
        bound = h * h / 6 * 0.4 * float(np.abs(host(c) * moved ** 3).sum()) + 2.0 ** -22 * size / h + 2.0 ** -20 * float((grad.abs() * step.abs()).sum())
        assert abs(got - want) <= bound, (name, got, want, bound)
        assert bound < 0.2 * float((grad.double() ** 2).sum().sqrt() * (step.double() ** 2).sum().sqrt()), "the bound says something"


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,di,do", [(700, 96, 80), (17000, 128, 96), (3000, 256, 200), (200000, 136, 72)])
def test_another_stream_and_a_graph(kb, kind, n, di, do):
    import torch
    X, W, b, R, G, _ = inputs(n, di, do, 2)
    layer = dict(W=dev(W, kind), b=dev(b), act=ref.SILU)
    x, r, c = dev(X, kind), dev(R, kind), dev(G, kind)
    Y, pre = kb.dense_forward(layer, x, R=r, keep_pre=True)
    g = kb.dense_backward(layer, x, pre, c)
    want = [Y, pre, g["dX"], g["dW"], g["db"]]
    out = [torch.zeros_like(t) for t in want]
    ws = torch.empty(kb.dense_workspace_bytes(layer, n), dtype=torch.uint8, device="cuda")

    def call(stream=None):
        kb.dense_forward(layer, x, R=r, Y=out[0], pre=out[1], stream=stream)
        kb.dense_backward(layer, x, out[1], c, dX=out[2], dW=out[3], db=out[4], workspace=ws, stream=stream)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    side.synchronize()
    assert all(bool((a == b_).all()) for a, b_ in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for rep in range(3):
        for o in out + [ws]:
            o.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(bool((a == b_).all()) for a, b_ in zip(out, want)), rep


# one size for each kernel: few results; tiles of 64 x 128 (fp32); tiles of 128 x 128; rows past W in registers (fp32, bf16)
KERNELS = [(150, 40, 33), (12000, 200, 200), (50000, 136, 136), (17000, 128, 128), (200000, 136, 72)]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,di,do", KERNELS)
def test_relu_hides_what_is_not_finite(kb, kind, n, di, do):
    """Where pre is not above zero, dY counts for nothing, whatever it is: bit for bit what zeros there give."""
    import torch
    say("relu hides", kind, n, di, do)
    X, W, b, Z, G, _ = inputs(n, di, do, 21)
    Z[2], Z[5, ::2], Z[6, ::3] = np.nan, 0.0, -np.inf
    layer = dict(W=dev(W, kind), b=dev(b), act=ref.RELU)
    x, pre, clean = dev(X, kind), dev(Z, kind), dev(G, kind)
    hidden = ~(pre > 0)
    clean[hidden] = 0.0
    for what in (float("inf"), float("nan"), -3.3e38):
        dirty = clean.clone()
        dirty[hidden] = what
        want, got = (kb.dense_backward(layer, x, pre, g) for g in (clean, dirty))
        for k in want:
            assert bool((got[k] == want[k]).all()), (k, what)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,di,do", KERNELS[1:])
def test_numbers_that_are_not_finite_in_long_matrices(kb, kind, n, di, do):
    say("dense not finite", kind, n, di, do)
    X, W, b, _, G, _ = inputs(n, di, do, 22)
    W[3] = np.abs(W[3]) + 0.1
    at = n - 40                                              # in the last tiles and in the first
    for r in (0, at):
        X[r + 5, 3], X[r + 7, 3], X[r + 9, 2], X[r + 11, 3] = np.inf, -np.inf, np.nan, 3.3e38 / 64
        X[r + 13, 3], X[r + 13, 4] = np.inf, np.inf
        G[r + 3, 5], G[r + 4, 6] = np.inf, np.nan
    layer = dict(W=dev(W, kind), b=dev(b), act=ref.IDENTITY)
    x, g = dev(X, kind), dev(G, kind)
    ones = dev(np.ones((n, di)), kind)
    back = kb.dense_backward(layer, ones, None, g)
    with np.errstate(all="ignore"):
        want = host(x) @ host(layer["W"]) + b
        dX, dW, db = ref.dense_backward(host(ones), host(layer["W"]), None, host(g), ref.IDENTITY)
    for a, w in ((kb.dense_forward(layer, x)[0], want), (back["dX"], dX), (back["dW"], dW), (back["db"], db)):
        a = host(a)
        assert np.isinf(w).any() and np.isnan(w).any()
        assert np.array_equal(np.isnan(a), np.isnan(w)) and np.array_equal(np.isinf(a), np.isinf(w))
        assert np.array_equal(a[np.isinf(w)], w[np.isinf(w)])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,di,do", [(70, 37, 45), (4000, 203, 150), (12000, 200, 200), (17000, 128, 128), (200000, 136, 72)])
def test_nothing_between_the_rows_counts(kb, kind, n, di, do):
    """Rows apart by columns of NaN: bit for bit what the same rows without them give."""
    import torch
    say("dense gaps of NaN", kind, n, di, do)
    X, W, b, Z, G, _ = inputs(n, di, do, 23)
    apart = lambda t, wide: torch.cat([t, torch.full((n, wide), float("nan"), dtype=t.dtype, device="cuda")], 1)[:, :t.shape[1]]
    layer = dict(W=dev(W, kind), b=dev(b), act=ref.SILU)
    x, z, g = dev(X, kind), dev(Z, kind), dev(G, kind)
    want = kb.dense_backward(layer, x, z, g, add=x)
    Y, pre = kb.dense_forward(layer, x, R=g, keep_pre=True)
    for wide in (1, 8):
        xs, zs, gs = (apart(t, wide) for t in (x, z, g))
        got = kb.dense_backward(layer, xs, zs, gs, add=xs)
        for k in want:
            assert bool((got[k] == want[k]).all()), (k, wide)
        Ys, pres = kb.dense_forward(layer, xs, R=gs, keep_pre=True)
        assert bool((Ys == Y).all()) and bool((pres == pre).all()), wide


def test_results_on_a_callers_stream_are_of_its_memory(kb):
    """Memory that work on the current stream still writes is no place for another stream's results."""
    import torch
    X, W, b, _, G, _ = inputs(4096, 64, 512, 24)
    layer = dict(W=dev(W), b=dev(b), act=ref.IDENTITY)
    x, g, a = dev(X), dev(G), torch.zeros((4096, 4096), device="cuda")
    want = kb.dense_forward(layer, x)[0].clone()
    grads = {k: v.clone() for k, v in kb.dense_backward(layer, x, None, g).items()}
    norm = dict(gamma=None, beta=None, eps=1e-5)
    normed = kb.layer_norm_forward(norm, want)[0].clone()
    side, out = torch.cuda.Stream(), torch.empty_like(a)
    for stream in (side, side.cuda_stream):
        torch.cuda.synchronize()
        for _ in range(40):
            torch.mm(a, a, out=out)                          # tens of milliseconds that the fills below wait for
        late = [torch.empty_like(t) for t in [want, normed] + list(grads.values()) for _ in range(3)]
        for t in late:
            t.fill_(7.0)
        del late, t
        Y = kb.dense_forward(layer, x, stream=stream)[0]
        got = kb.dense_backward(layer, x, None, g, stream=stream)
        N = kb.layer_norm_forward(norm, want, stream=stream)[0]
        torch.cuda.synchronize()
        assert bool((Y == want).all()) and bool((N == normed).all())
        assert all(bool((got[k] == grads[k]).all()) for k in grads)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,di,do", [(29082, 203, 517), (3000, 700, 129), (2600, 9, 3), (70000, 66, 65), (140000, 20, 21), (300, 1030, 1100)])
def test_weights_gradients_of_few_and_many_chunks(kb, kind, n, di, do):
    say("dense chunks", kind, n, di, do)
    X, _, _, Z, G, _ = inputs(n, di, do, 25)
    x, z, g = dev(X, kind), dev(Z, kind), dev(G, kind)
    layer = dict(W=dev(np.zeros((di, do)), kind), b=None, act=ref.RELU)
    got = kb.dense_backward(layer, x, z, g, need_dX=False)
    args = (host(x), host(layer["W"]), host(z), host(g), ref.RELU)
    want, bound = ref.dense_backward(*args), ref.dense_backward_bound(*args, None, kind)
    within(host(got["dW"]), want[1], bound[1], "dW")
    within(host(got["db"]), want[2], bound[2], "db")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,di,do,act", [(30000, 129, 160, "silu"), (14541, 160, 129, "relu"), (9000, 388, 416, "identity"), (12001, 260, 257, "silu")])
def test_last_columns_of_a_wide_result(kb, kind, n, di, do, act):
    """Results one to 32 columns wider than whole tiles."""
    say("dense narrow", kind, n, di, do, act)
    X, W, b, R, G, A = inputs(n, di, do, 26)
    x, r, g, a = (dev(z, kind) for z in (X, R, G, A))
    layer = dict(W=dev(W, kind), b=dev(b), act=ACTS[act])
    Y, pre = kb.dense_forward(layer, x, R=r, keep_pre=True)
    got = kb.dense_backward(layer, x, pre, g, add=a)
    b64 = b.astype(np.float64)
    forward = (host(x), host(layer["W"]), b64, ACTS[act], host(r))
    for t, w, e, name in zip((Y, pre), ref.dense_forward(*forward), ref.dense_forward_bound(*forward, kind), ("Y", "pre")):
        within(host(t), w, e, name)
    back = (host(x), host(layer["W"]), host(pre), host(g), ACTS[act], host(a))
    for k, w, e in zip(("dX", "dW", "db"), ref.dense_backward(*back), ref.dense_backward_bound(*back, kind)):
        within(host(got[k]), w, e, k)


@pytest.mark.parametrize("kind,n,di,do", [("f32", 17003, 128, 768), ("f32", 16500, 80, 384), ("f32", 17000, 640, 72), ("bf16", 200001, 72, 264),
                                          ("bf16", 200016, 264, 72)])
def test_several_groups_of_columns_of_a_long_matrix(kb, kind, n, di, do):
    say("dense groups", kind, n, di, do)
    X, W, b, R, G, _ = inputs(n, di, do, 27)
    x, r, g = dev(X, kind), dev(R, kind), dev(G, kind)
    layer = dict(W=dev(W, kind), b=dev(b), act=ref.RELU)
    Y, pre = kb.dense_forward(layer, x, R=r, keep_pre=True)
    dX = kb.dense_backward(layer, x, pre, g, need_dW=False)["dX"]
    w, b64 = host(layer["W"]), b.astype(np.float64)
    for part in (slice(0, 300), slice(n // 2, n // 2 + 1000), slice(n - 4000, n)):      # every group and wavefront, first and last tiles
        forward = (host(x[part]), w, b64, ref.RELU, host(r[part]))
        for t, want, e, name in zip((Y, pre), ref.dense_forward(*forward), ref.dense_forward_bound(*forward, kind), ("Y", "pre")):
            within(host(t[part]), want, e, name)
        back = (host(x[part]), w, host(pre[part]), host(g[part]), ref.RELU)
        within(host(dX[part]), ref.dense_backward(*back)[0], ref.dense_backward_bound(*back, None, kind)[0], "dX")
    again = kb.dense_forward(layer, x, R=r)[0]
    assert bool((again == Y).all())
