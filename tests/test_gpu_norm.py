"""Layer norm (forward and backward pass) against its formula in 64 bits."""
import sys

import numpy as np
import pytest

import block_ref as ref
from test_gpu_dense import dev, host, kb, tt, within    # noqa: F401  (kb: the fixture)

pytestmark = pytest.mark.gpu
EPS = 1e-5
# every group of lanes, both sides of its limits, and rows that are no multiple of four
SIZES = [(1, 1), (3, 2), (50, 17), (33, 64), (16, 65), (9, 128), (200, 131), (1000, 256), (7, 257), (65, 512), (5, 1000), (6, 1025),
         (11, 2048), (3, 2049), (4, 4097), (2, 8192), (3, 8193), (2, 16384), (2100, 40)]


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def inputs(n, d, seed):
    rng = np.random.default_rng(seed)
    X = rng.normal(0, 1, (n, d)) * rng.uniform(0.2, 3.0, (n, 1)) + rng.normal(0, 2, (n, 1))
    return X, rng.normal(1, 0.2, d).astype(np.float32), rng.normal(0, 0.2, d).astype(np.float32), rng.normal(0, 0.1, (n, d))


@pytest.mark.parametrize("kx,ky", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("n,d", SIZES)
def test_forward_and_backward(kb, kx, ky, n, d):  # noqa: F811
    say("layer norm", kx, ky, n, d)
    X, gamma, beta, G = inputs(n, d, n + d)
    x, g = dev(X, kx), dev(G, ky)
    norm = dict(gamma=dev(gamma), beta=dev(beta), eps=EPS)
    Y, mean, rstd = kb.layer_norm_forward(norm, x, out_dtype=tt(ky))
    eps = float(np.float32(EPS))
    g64, b64 = gamma.astype(np.float64), beta.astype(np.float64)
    for got, want, bound, what in zip((Y, mean, rstd), ref.norm_forward(host(x), g64, b64, eps),
                                      ref.norm_forward_bound(host(x), g64, b64, eps, ky), ("Y", "mean", "rstd")):
        within(host(got), want, bound, what)
    got = kb.layer_norm_backward(norm, x, mean, rstd, g)
    args = host(x), g64, host(mean), host(rstd), host(g)
    for k, name in enumerate(("dX", "dgamma", "dbeta")):
        within(host(got[name]), ref.norm_backward(*args)[k], ref.norm_backward_bound(*args, kx)[k], name)
    again = kb.layer_norm_backward(norm, x, mean, rstd, g)
    assert all(bool((again[k] == got[k]).all()) for k in got), "the same call gives the same bits"
    part = kb.layer_norm_backward(norm, x, mean, rstd, g, need_dX=False)
    assert part["dX"] is None and bool((part["dgamma"] == got["dgamma"]).all()) and bool((part["dbeta"] == got["dbeta"]).all())
    bare = dict(gamma=None, beta=None, eps=EPS)
    one, zero = np.ones(d), np.zeros(d)
    within(host(kb.layer_norm_forward(bare, x, out_dtype=tt(ky))[0]), ref.norm_forward(host(x), one, zero, eps)[0],
           ref.norm_forward_bound(host(x), one, zero, eps, ky)[0], "Y without weights")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,wide,shift", [(70, 37, 3, 1), (300, 128, 8, 4), (131, 200, 1, 0), (9, 4096, 5, 5)])
def test_strided_rows_keep_what_lies_between(kb, kind, n, d, wide, shift):  # noqa: F811
    import torch
    say("layer norm strides", kind, n, d, wide, shift)
    X, gamma, beta, G = inputs(n, d, 4)
    norm = dict(gamma=dev(gamma), beta=dev(beta), eps=EPS)
    mean, rstd = kb.layer_norm_forward(norm, dev(X, kind))[1:]
    out = [torch.full((n + 2, d + wide), 5.0, dtype=tt(kind), device="cuda") for _ in range(2)]
    vY, vdX = (o[1:n + 1, shift:shift + d] for o in out)
    got_m = kb.layer_norm_forward(norm, dev(X, kind, wide, shift), Y=vY)
    x64, g64, b64, e = host(dev(X, kind)), gamma.astype(np.float64), beta.astype(np.float64), float(np.float32(EPS))
    for got, want, bound in zip((vY, *got_m[1:]), ref.norm_forward(x64, g64, b64, e), ref.norm_forward_bound(x64, g64, b64, e, kind)):
        within(host(got), want, bound, "forward")
    got = kb.layer_norm_backward(norm, dev(X, kind, wide, shift), mean, rstd, dev(G, kind, wide, shift), dX=vdX)
    args = x64, g64, host(mean), host(rstd), host(dev(G, kind))
    for k, name in enumerate(("dX", "dgamma", "dbeta")):
        within(host(got[name]), ref.norm_backward(*args)[k], ref.norm_backward_bound(*args, kind)[k], name)
    for o, v in zip(out, (vY, vdX)):
        v.fill_(5.0)
        assert bool((o == 5.0).all()), "what lies around the rows stays as it was"


def test_rows_of_one_value_and_rows_far_from_zero(kb):  # noqa: F811
    """A row without spread becomes beta; a mean a thousand times the spread costs the digits that the input itself lacks."""
    import torch
    n, d = 64, 96
    X, gamma, beta, G = inputs(n, d, 1)
    X = X * 1e-1 + 1000.0
    X[:8] = 3.0
    x = dev(X)
    norm = dict(gamma=dev(gamma), beta=dev(beta), eps=EPS)
    Y, mean, rstd = kb.layer_norm_forward(norm, x)
    want = ref.norm_forward(host(x), gamma.astype(np.float64), beta.astype(np.float64), float(np.float32(EPS)))
    bound = ref.norm_forward_bound(host(x), gamma.astype(np.float64), beta.astype(np.float64), float(np.float32(EPS)), "f32")
    within(host(Y), want[0], bound[0], "Y")
    assert bool((Y[:8] == norm["beta"]).all()) and bool(torch.isfinite(rstd).all())


def test_a_row_that_is_not_finite_stays_alone(kb):  # noqa: F811
    import torch
    n, d = 40, 72
    X, gamma, beta, G = inputs(n, d, 2)
    clean = kb.layer_norm_forward(dict(gamma=dev(gamma), beta=dev(beta), eps=EPS), dev(X))[0]
    X[3, 5], X[17, 0] = np.nan, np.inf
    Y = kb.layer_norm_forward(dict(gamma=dev(gamma), beta=dev(beta), eps=EPS), dev(X))[0]
    bad = torch.isnan(Y).any(1)
    assert bad.nonzero().flatten().tolist() == [3, 17]
    assert bool((Y[~bad] == clean[~bad]).all())


def test_no_rows(kb):  # noqa: F811
    import torch
    norm = dict(gamma=torch.ones(12, device="cuda"), beta=None, eps=EPS)
    X, one = torch.empty((0, 12), device="cuda"), torch.empty(0, device="cuda")
    assert tuple(kb.layer_norm_forward(norm, X)[0].shape) == (0, 12)
    g = kb.layer_norm_backward(norm, X, one, one, X)
    assert not bool(g["dgamma"].any()) and not bool(g["dbeta"].any())


def test_gradients_against_differences(kb):  # noqa: F811
    """L = <C, Y> moved by +-h along a direction: off by O(h^2) of L's third derivative along it, here below 40 h^2 of the
    gradient's size (rows of 48, spread 1, a direction of size 1 an element), and by fp32's rounding over 2 h."""
    n, d, h = 60, 48, 2.0 ** -9
    rng = np.random.default_rng(6)
    X, gamma, beta, C = rng.normal(0, 1, (n, d)), rng.normal(1, 0.2, d), rng.normal(0, 0.2, d), rng.normal(0, 1, (n, d))
    x, c = dev(X), dev(C)
    base = [x, dev(gamma), dev(beta)]
    L = lambda a: float((kb.layer_norm_forward(dict(gamma=a[1], beta=a[2], eps=EPS), a[0])[0].double() * c.double()).sum())  # noqa: E731
    norm = dict(gamma=base[1], beta=base[2], eps=EPS)
    Y, mean, rstd = kb.layer_norm_forward(norm, x)
    g = kb.layer_norm_backward(norm, x, mean, rstd, c)
    size = float((Y.double() * c.double()).abs().sum())
    for at, grad in enumerate((g["dX"], g["dgamma"], g["dbeta"])):
        step = dev(rng.normal(0, 1, tuple(base[at].shape)))
        up, down = list(base), list(base)
        up[at], down[at] = base[at] + h * step, base[at] - h * step
        got, want = (L(up) - L(down)) / (2 * h), float((grad.double() * step.double()).sum())
        scale = float((grad.double() * step.double()).abs().sum())
        assert abs(got - want) <= 40 * h * h * scale + 2.0 ** -22 * size / h, (at, got, want)


def test_another_stream_and_a_graph(kb):  # noqa: F811
    import torch
    n, d = 3000, 136
    X, gamma, beta, G = inputs(n, d, 3)
    norm = dict(gamma=dev(gamma), beta=dev(beta), eps=EPS)
    x, c = dev(X, "bf16"), dev(G)
    Y, mean, rstd = kb.layer_norm_forward(norm, x, out_dtype=torch.float32)
    g = kb.layer_norm_backward(norm, x, mean, rstd, c)
    want = [Y, mean, rstd, g["dX"], g["dgamma"], g["dbeta"]]
    out = [torch.zeros_like(t) for t in want]
    ws = torch.empty(kb.layer_norm_workspace_bytes(d, n), dtype=torch.uint8, device="cuda")

    def call(stream=None):
        kb.layer_norm_forward(norm, x, Y=out[0], mean=out[1], rstd=out[2], stream=stream)
        kb.layer_norm_backward(norm, x, out[1], out[2], c, dX=out[3], dgamma=out[4], dbeta=out[5], workspace=ws, stream=stream)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    side.synchronize()
    assert all(bool((a == b).all()) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for rep in range(3):
        for o in out + [ws]:
            o.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(bool((a == b).all()) for a, b in zip(out, want)), rep
