"""The dense layer on bf16 rows of 129 to 256 terms in matrices long enough for the kernels that keep W in registers, both ways
round, with everything that is optional in their epilogue."""
import numpy as np
import pytest

import block_ref as ref
from test_gpu_dense import ACTS, host, kb, say, within    # noqa: F401  (kb: the fixture)

pytestmark = pytest.mark.gpu


def parts_of(n):
    """Rows of the first, middle and last rounds of tiles; a round is 256 tiles of 32 rows."""
    return [slice(0, 600), slice(n // 2, n // 2 + 1500), slice(n - 9000, n - 8000), slice(n - 700, n)]


def made(n, di, do, seed):
    """x, r, g, a of bf16 on the device, and the layer's W and b."""
    import torch
    gen = torch.Generator("cuda").manual_seed(seed)
    z = lambda std, *shape: torch.randn(shape, generator=gen, device="cuda") * std  # noqa: E731
    x, r, g, a, w = (t.bfloat16() for t in (z(1.0, n, di), z(1.0, n, do), z(0.1, n, do), z(0.1, n, di), z(di ** -0.5, di, do)))
    return x, r, g, a, w, z(0.3, do)


# whole tiles in the loop without branches, and an incomplete last one; the width of the group, less, and terms that are no multiple
# of eight (the loop with branches)
SIZES = [(200003, 256, 256), (200032, 256, 256), (210011, 200, 136), (200001, 136, 200), (200003, 129, 250), (200017, 240, 120)]


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("n,di,do", SIZES)
def test_wide_bf16_rows(kb, act, n, di, do):  # noqa: F811
    import torch
    say("wide bf16 rows", act, n, di, do)
    x, r, g, a, W, b = made(n, di, do, n + di)
    layer = dict(W=W, b=b, act=ACTS[act])
    w, b64 = host(W), host(b)

    def forward(res, bias, Y, pre):
        for p in parts_of(n):
            args = host(x[p]), w, b64 if bias else None, ACTS[act], None if res is None else host(res[p])
            for got, want, bound, what in zip((Y, pre), ref.dense_forward(*args), ref.dense_forward_bound(*args, "bf16"), ("Y", "pre")):
                if got is not None:
                    within(host(got[p]), want, bound, what)

    Y, pre = kb.dense_forward(layer, x, R=r, keep_pre=True)
    forward(r, True, Y, pre)
    bare = dict(layer, b=None)
    for res, keep, lay in ((None, True, layer), (r, False, layer), (None, False, bare)):
        got = kb.dense_forward(lay, x, R=res, keep_pre=keep)
        forward(res, lay is layer, *got)
        if keep:
            assert bool((got[1] == pre).all())
        elif res is not None:
            assert bool((got[0] == Y).all())
    dX = {}
    for name, add in (("alone", None), ("added", a)):
        dX[name] = got = kb.dense_backward(layer, x, pre, g, add=add, need_dW=False)["dX"]
        for p in parts_of(n):
            args = host(x[p])[:, :1], w, host(pre[p]), host(g[p]), ACTS[act], None if add is None else host(add[p])
            at = ref.dense_backward_bound(*args, "bf16")[0]
            within(host(got[p]), ref.dense_backward(*args)[0], at, "dX " + name)
    # every other row: within two half steps of bf16 of what torch's own products in fp32 give
    z = pre.float()
    s = torch.sigmoid(z)
    P = g.float() * (1.0 if act == "identity" else (z > 0) if act == "relu" else s * (1 + z * (1 - s)))
    size = P.abs() @ layer["W"].float().abs().t()
    assert bool(((dX["alone"].float() - P @ layer["W"].float().t()).abs() <= 2.0 ** -7 * size).all())
    z = x.float() @ layer["W"].float() + layer["b"]
    size = x.float().abs() @ layer["W"].float().abs() + layer["b"].abs()
    assert bool(((pre.float() - z).abs() <= 2.0 ** -7 * size).all())


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("n,d", [(200003, 256), (200032, 256), (200009, 128), (210011, 200), (200005, 72)])
def test_a_bf16_residual_that_is_x(kb, act, n, d):  # noqa: F811
    """R = X: the same bits as a copy of X as R, in every row, with and without pre."""
    import torch
    say("bf16 residual", act, n, d)
    x, _, _, _, W, b = made(n, d, d, n + d)
    x[5, 3], x[n - 3, 1] = float("inf"), float("nan")
    layer = dict(W=W, b=b, act=ACTS[act])
    Y, pre = kb.dense_forward(layer, x, R=x.clone(), keep_pre=True)
    own, own_pre = kb.dense_forward(layer, x, R=x, keep_pre=True)
    bits = lambda t: t.view(torch.int16)  # noqa: E731
    fine = ~Y.isnan()
    assert bool((bits(own)[fine] == bits(Y)[fine]).all()) and bool((own.isnan() == Y.isnan()).all()) and int((~fine).any(1).sum()) <= 2
    assert bool((bits(own_pre)[~pre.isnan()] == bits(pre)[~pre.isnan()]).all()) and bool((own_pre.isnan() == pre.isnan()).all())
    alone = kb.dense_forward(layer, x, R=x)[0]
    assert bool((bits(alone)[fine] == bits(Y)[fine]).all()) and bool((alone.isnan() == Y.isnan()).all())
    w, b64 = host(W), host(b)
    for p in parts_of(n):
        rows = host(x[p])
        rows = rows[np.isfinite(rows).all(1)]
        got = host(own[p])[np.isfinite(host(x[p])).all(1)]
        args = rows, w, b64, ACTS[act], rows
        within(got, ref.dense_forward(*args)[0], ref.dense_forward_bound(*args, "bf16")[0], "Y")
