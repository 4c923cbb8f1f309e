"""Calls of the vertex-feature block and of AdamW that the library refuses, none of which needs a GPU, and the 64-bit forms that
the GPU tests measure against, checked by differences."""
import ctypes as C
import os

import numpy as np
import pytest

import block_ref as ref


@pytest.fixture(scope="module")
def kb():
    from paper_2201_02791_amd import build, binding
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    binding.load()
    return binding


EINVAL, ENOMEM, ERANGE = -1, -2, -4
P = C.c_void_p(1 << 12)          # an aligned address that is never used: every call below is refused before that
N0 = C.c_void_p(0)
L = lambda x: C.c_int64(x)  # noqa: E731


def test_struct_layouts(kb):
    assert C.sizeof(kb._Dense) == 4 * 4 + 2 * 8 and C.sizeof(kb._Norm) == 4 * 4 + 2 * 8
    assert C.sizeof(kb._AdamWTensor) == 8 * 8 + 2 * 8 + 2 * 4 + 4 + 4 and C.sizeof(kb._AdamW) == 4 * 4 + 8 + 8


@pytest.mark.parametrize("change,status,word", [
    (dict(d_in=0), EINVAL, "widths"), (dict(d_out=65537), EINVAL, "widths"), (dict(act=3), EINVAL, "act"), (dict(dtype=2), EINVAL, "type"),
    (dict(n=-1), EINVAL, "negative"), (dict(n=1 << 31), ERANGE, "rows"), (dict(ldx=7), EINVAL, "stride"), (dict(ldy=3), EINVAL, "stride"),
    (dict(ldr=3), EINVAL, "stride"), (dict(W=None), EINVAL, "NULL"), (dict(X=N0), EINVAL, "NULL"), (dict(X=C.c_void_p(4098)), EINVAL, "aligned")])
def test_dense_forward(kb, change, status, word):
    a = dict(d_in=8, d_out=4, act=1, dtype=0, n=5, ldx=8, ldy=4, ldr=4, W=1 << 12, X=P)
    a.update(change)
    d = kb._Dense(a["d_in"], a["d_out"], a["act"], a["dtype"], a["W"], None)
    rc = kb.load().kge_dense_forward(C.byref(d), L(a["n"]), a["X"], L(a["ldx"]), P, L(a["ldr"]), P, L(a["ldy"]), N0, L(0), N0)
    assert rc == status and word.encode() in kb.load().kge_last_error()
    if set(change) & {"d_in", "d_out", "act", "dtype", "n"}:
        assert kb.load().kge_dense_workspace_bytes(C.byref(d), L(a["n"])) == 0


def test_dense_backward(kb):
    lib = kb.load()
    d = kb._Dense(8, 4, 1, 0, 1 << 12, None)
    call = lambda X=P, pre=P, dY=P, add=N0, dX=P, dW=P, ws=P, size=1 << 20, d=d: lib.kge_dense_backward(  # noqa: E731
        C.byref(d), L(5), X, L(8), pre, L(4), dY, L(4), add, L(8), dX, L(8), dW, P, ws, C.c_size_t(size), N0)
    for got, status in ((call(X=N0), EINVAL), (call(pre=N0), EINVAL), (call(dY=N0), EINVAL), (call(add=P, dX=N0), EINVAL),
                        (call(ws=N0), EINVAL), (call(ws=C.c_void_p(4096 + 64)), EINVAL), (call(size=16), ENOMEM),
                        (call(d=kb._Dense(8, 4, 1, 0, None, None)), EINVAL)):
        assert got == status
    wide = kb._Dense(65536, 65536, 0, 0, 1 << 12, None)
    assert lib.kge_dense_backward(C.byref(wide), L(5), P, L(65536), N0, L(0), P, L(65536), N0, L(0), N0, L(0), P, P, P, C.c_size_t(1 << 62), N0) == ERANGE
    assert lib.kge_dense_backward(None, L(5), P, L(8), P, L(4), P, L(4), N0, L(8), P, L(8), P, P, P, C.c_size_t(1 << 20), N0) == EINVAL


def test_dense_outputs_that_are_inputs(kb):
    lib, d = kb.load(), kb._Dense(8, 8, 1, 0, 1 << 12, None)
    X, R, Y, Z = (C.c_void_p((k + 1) << 12) for k in range(4))
    forward = lambda X, R, Y, pre: lib.kge_dense_forward(C.byref(d), L(5), X, L(8), R, L(8), Y, L(8), pre, L(8), N0)  # noqa: E731
    for call in ((X, N0, X, N0), (X, X, X, Z), (X, R, Y, X), (X, R, Y, R), (X, R, Y, Y)):
        assert forward(*call) == EINVAL and b"may not be" in lib.kge_last_error()
    backward = lambda dX, ws: lib.kge_dense_backward(C.byref(d), L(5), X, L(8), Y, L(8), Z, L(8), R, L(8), dX, L(8), ws, ws, ws,  # noqa: E731
                                                     C.c_size_t(1 << 20), N0)
    for dX in (X, Y, Z):
        assert backward(dX, P) == EINVAL and b"may not be" in lib.kge_last_error()


def test_layer_norm(kb):
    lib = kb.load()
    fwd = lambda p, n=5, X=P, Y=P, ldx=8: lib.kge_layer_norm_forward(C.byref(p), L(n), X, L(ldx), Y, L(8), N0, N0, N0)  # noqa: E731
    ok = kb._Norm(8, 0, 0, 1e-5, None, None)
    for got, status in ((fwd(kb._Norm(0, 0, 0, 1e-5, None, None)), EINVAL), (fwd(kb._Norm(16385, 0, 0, 1e-5, None, None)), EINVAL),
                        (fwd(kb._Norm(8, 2, 0, 1e-5, None, None)), EINVAL), (fwd(kb._Norm(8, 0, 0, -1.0, None, None)), EINVAL),
                        (fwd(kb._Norm(8, 0, 0, float("nan"), None, None)), EINVAL), (fwd(ok, n=-1), EINVAL), (fwd(ok, n=1 << 31), ERANGE),
                        (fwd(ok, X=N0), EINVAL), (fwd(ok, Y=N0), EINVAL), (fwd(ok, ldx=7), EINVAL), (fwd(ok, X=C.c_void_p(4097)), EINVAL)):
        assert got == status
    bwd = lambda mean=P, ws=P, size=1 << 20, dg=P: lib.kge_layer_norm_backward(  # noqa: E731
        C.byref(ok), L(5), P, L(8), mean, P, P, L(8), P, L(8), dg, N0, ws, C.c_size_t(size), N0)
    assert bwd(mean=N0) == EINVAL and bwd(ws=N0) == EINVAL and bwd(size=8) == ENOMEM and bwd(ws=C.c_void_p(4104)) == EINVAL
    assert lib.kge_layer_norm_workspace_bytes(C.byref(kb._Norm(0, 0, 0, 0.0, None, None)), L(5)) == 0


@pytest.mark.parametrize("change,status", [
    (dict(n_rows=-1), EINVAL), (dict(d=-1), EINVAL), (dict(state_bits=16), EINVAL), (dict(rows=3), EINVAL), (dict(param=None), EINVAL),
    (dict(m=None), EINVAL), (dict(state_bits=8), EINVAL), (dict(m_scale=1 << 12), EINVAL), (dict(rows=1), EINVAL),
    (dict(row_mask=1 << 12), EINVAL), (dict(rows=2, d=70000), EINVAL), (dict(n_rows=1 << 40, d=1 << 30), ERANGE),
    (dict(n_rows=1, d=1 << 36), ERANGE), (dict(param=(1 << 12) + 2), EINVAL), (dict(copy=(1 << 12) + 1), EINVAL)])
def test_adamw(kb, change, status):
    a = dict(param=1 << 12, grad=1 << 12, m=1 << 12, v=1 << 12, n_rows=3, d=8, state_bits=32, rows=0, weight_decay=0.0)
    a.update(change)
    t = kb._AdamWTensor(**a)
    o = kb._AdamW(0.01, 0.9, 0.999, 1e-8, 1, None)
    assert kb.load().kge_adamw_step(C.byref(o), C.byref(t), C.c_int32(1), N0) == status


def test_adamw_hyper_parameters(kb):
    t = kb._AdamWTensor(n_rows=0, d=8, state_bits=32)
    call = lambda *o, n=1: kb.load().kge_adamw_step(C.byref(kb._AdamW(*o)), C.byref(t), C.c_int32(n), N0)  # noqa: E731
    assert call(0.01, 0.9, 0.999, 1e-8, 1, None) == 0                 # nothing to update: nothing runs
    assert call(0.01, 1.0, 0.999, 1e-8, 1, None) == EINVAL and call(0.01, 0.9, -0.1, 1e-8, 1, None) == EINVAL
    assert call(0.01, 0.9, 0.999, 1e-8, 0, None) == EINVAL and call(0.01, 0.9, 0.999, 1e-8, 1, None, n=-1) == EINVAL
    assert call(0.01, 0.9, 0.999, 1e-8, 1, (1 << 12) + 4) == EINVAL
    assert kb.load().kge_adamw_step(None, C.byref(t), C.c_int32(1), N0) == EINVAL


def test_binding_refuses_shapes_types_and_host_tensors(kb):
    import torch
    f = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)  # noqa: E731
    layer = dict(W=f(8, 4), b=f(4), act=kb.ACT_RELU)
    bad = [lambda: kb.dense_forward(layer, f(5, 7)), lambda: kb.dense_forward(layer, f(5, 8, dt=torch.bfloat16)),
           lambda: kb.dense_forward(layer, f(5, 8, dt=torch.float16)), lambda: kb.dense_forward(layer, f(8, 5).t()),
           lambda: kb.dense_forward(dict(layer, b=f(3)), f(5, 8)), lambda: kb.dense_forward(layer, f(5, 8), R=f(4, 4)),
           lambda: kb.dense_forward(layer, f(1, 8).expand(5, 8)), lambda: kb.dense_forward(dict(layer, W=f(4, 8).t()), f(5, 8)),
           lambda: kb.dense_backward(layer, f(5, 8), f(5, 4), f(5, 3)), lambda: kb.dense_backward(layer, f(5, 8), f(4, 4), f(5, 4)),
           lambda: kb.layer_norm_forward(dict(gamma=f(7)), f(5, 8)), lambda: kb.layer_norm_forward(dict(), f(8)),
           lambda: kb.layer_norm_backward(dict(), f(5, 8), None, f(5), f(5, 8)), lambda: kb.layer_norm_backward(dict(), f(5, 8), f(5), f(4), f(5, 8)),
           lambda: kb.dense_forward(layer, f(5, 8)), lambda: kb.layer_norm_forward(dict(), f(5, 8))]          # host memory
    t = dict(param=f(3, 8), grad=f(3, 8), m=f(3, 8), v=f(3, 8))
    bad += [lambda: kb.AdamWTensors([dict(t, grad=f(3, 7))]), lambda: kb.AdamWTensors([dict(t, m_scale=f(3, 1), v_scale=f(3, 1))]),
            lambda: kb.AdamWTensors([dict(t, rows="some")]), lambda: kb.AdamWTensors([dict(t, rows="mask", row_mask=f(3))]),
            lambda: kb.AdamWTensors([dict(t, copy=f(3, 8))]), lambda: kb.AdamWTensors([dict(t, param=f(8, 3).t())]),
            lambda: kb.adamw_step([t]), lambda: kb.adamw_state(f(3, 8), 4)]
    for i, call in enumerate(bad):
        with pytest.raises(kb.KgeError) as e:
            call()
        assert e.value.status == EINVAL, i


def test_the_plain_gradients_by_differences():
    rng = np.random.default_rng(1)
    n, di, do, h = 6, 5, 4, 1e-5
    X, W, b, G, gamma = rng.normal(size=(n, di)), rng.normal(size=(di, do)), rng.normal(size=do), rng.normal(size=(n, do)), rng.normal(size=do)

    def slope(f, x):
        out = np.zeros_like(x)
        for i in np.ndindex(x.shape):
            e = np.zeros_like(x)
            e[i] = h
            out[i] = (f(x + e) - f(x - e)) / (2 * h)
        return out
    for a in (ref.IDENTITY, ref.SILU):
        pre = ref.dense_forward(X, W, b, a)[1]
        dX, dW, db = ref.dense_backward(X, W, pre, G, a)
        L = lambda X_, W_, b_: (ref.dense_forward(X_, W_, b_, a)[0] * G).sum()  # noqa: E731
        for got, want in ((dX, slope(lambda x: L(x, W, b), X)), (dW, slope(lambda w: L(X, w, b), W)), (db, slope(lambda c: L(X, W, c), b))):
            np.testing.assert_allclose(got, want, atol=1e-7, rtol=1e-7)
    Z = rng.normal(size=(n, do))
    Y, mean, rstd = ref.norm_forward(Z, gamma, b, 1e-3)
    dX, dg, db = ref.norm_backward(Z, gamma, mean, rstd, G)
    L = lambda z, g, c: (ref.norm_forward(z, g, c, 1e-3)[0] * G).sum()  # noqa: E731
    for got, want in ((dX, slope(lambda z: L(z, gamma, b), Z)), (dg, slope(lambda g: L(Z, g, b), gamma)), (db, slope(lambda c: L(Z, gamma, c), b))):
        np.testing.assert_allclose(got, want, atol=1e-7, rtol=1e-6)


def test_the_plain_8_bit_moments():
    """Numbers come from the format, at most one of its distances off; the mean over steps is the number itself."""
    import torch
    rng = np.random.default_rng(4)
    x = (rng.normal(size=(3, 300)) * np.exp(rng.normal(0, 2, (3, 300)))).astype(np.float32)
    for form, dt, y in ((ref.E4M3, torch.float8_e4m3fn, x), (ref.E5M2, torch.float8_e5m2, x * x)):
        mean = np.zeros(x.shape)
        for t in range(1, 2001):
            q, s = ref.encode(y, form, t)
            if t < 4:
                assert np.array_equal(torch.from_numpy(q).to(dt).double().numpy(), q)
                spread = np.repeat(s, ref.BLOCK, 1)[:, :300]
                unit = np.ldexp(1.0, np.maximum(np.frexp(np.abs(y) / spread)[1] - 1, form["least"]) - form["digits"]) * spread
                assert (np.abs(q * spread - y) < unit).all() and (np.abs(q * spread - y) > 0.5 * unit).any()
            mean += q * spread / 2000
        big = np.abs(y) > 1e-3 * np.abs(y).max(1, keepdims=True)
        # 2000 offsets spread their mean by at most half a distance (an eighth of the number) over sqrt(2000); six of that
        assert (np.abs(mean - y) <= 6.0 / 8.0 / np.sqrt(2000.0) * np.abs(y))[big].all()
