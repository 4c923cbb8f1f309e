"""Where the dense layer's results may lie, at a size for each of its kernels: in place of the residual or of the added gradient, and as
columns of a wider matrix at any element."""
import pytest

import block_ref as ref
from test_gpu_dense import KERNELS, host, kb, say, tt, within    # noqa: F401  (kb: the fixture)

pytestmark = pytest.mark.gpu
SIZES = KERNELS + [(200003, 256, 256), (200000, 72, 264), (17000, 64, 300), (30000, 129, 160)]


def made(kind, n, di, do):
    import torch
    gen = torch.Generator("cuda").manual_seed(n + di)
    z = lambda *s: torch.randn(s, generator=gen, device="cuda").to(tt(kind))  # noqa: E731
    layer = dict(W=z(di, do) * di ** -0.5, b=torch.randn(do, generator=gen, device="cuda"), act=ref.SILU)
    x, r, g, a = z(n, di), z(n, do), z(n, do), z(n, di)
    Y, pre = kb_forward(layer, x, r)
    return layer, x, r, g, a, Y, pre


def kb_forward(layer, x, r):
    from paper_2201_02791_amd import binding
    return binding.dense_forward(layer, x, R=r, keep_pre=True)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,di,do", SIZES)
def test_in_place(kb, kind, n, di, do):  # noqa: F811
    say("dense in place", kind, n, di, do)
    layer, x, r, g, a, Y, pre = made(kind, n, di, do)
    kb.dense_forward(layer, x, R=r, Y=r)
    assert bool((r == Y).all())
    want = kb.dense_backward(layer, x, pre, g, add=a, need_dW=False)["dX"]
    kb.dense_backward(layer, x, pre, g, add=a, dX=a, need_dW=False)
    assert bool((a == want).all())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,di,do", SIZES)
@pytest.mark.parametrize("wide,shift", [(3, 1), (8, 4), (1, 0)])
def test_columns_of_a_wider_matrix(kb, kind, n, di, do, wide, shift):  # noqa: F811
    """Bit for bit what dense results are, but for long bf16 rows, where another kernel, with another order of its sums, takes results that
    are off their words: rows of the first, middle and last tiles are held to the formula in 64 bits, and so by twice those
    bounds to one another."""
    import torch
    say("dense wider results", kind, n, di, do, wide, shift)
    layer, x, r, g, a, Y, pre = made(kind, n, di, do)
    out = [torch.full((n + 2, w + wide), 5.0, dtype=tt(kind), device="cuda") for w in (do, do, di)]
    vY, vpre, vdX = (o[1:n + 1, shift:shift + w] for o, w in zip(out, (do, do, di)))
    kb.dense_forward(layer, x, R=r, Y=vY, pre=vpre)
    kb.dense_backward(layer, x, vpre, g, add=a, dX=vdX, need_dW=False)
    dX = kb.dense_backward(layer, x, vpre.contiguous(), g, add=a, need_dW=False)["dX"]
    w, b = host(layer["W"]), host(layer["b"])
    for p in (slice(0, 300), slice(n // 2, n // 2 + 500), slice(max(0, n - 700), n)):
        forward = host(x[p]), w, b, ref.SILU, host(r[p])
        for got, want, bound, what in zip((vY, vpre), ref.dense_forward(*forward), ref.dense_forward_bound(*forward, kind), ("Y", "pre")):
            within(host(got[p]), want, bound, what)
        back = host(x[p])[:, :1], w, host(vpre[p]), host(g[p]), ref.SILU, host(a[p])
        within(host(vdX[p]), ref.dense_backward(*back)[0], ref.dense_backward_bound(*back, kind)[0], "dX")
    if kind == "f32" or n < 200000:
        assert bool((vY == Y).all()) and bool((vpre == pre).all()) and bool((vdX == dX).all())
    else:                        # every row: two bf16 numbers next to one another, or, near zero, as far apart as twice what fp32
        # sums of 264 terms of 14 in all may be off: 2 x 2 (264 + 8) 2^-24 x 14 < 2^-10
        for one, two in ((vY, Y), (vpre, pre), (vdX, dX)):
            assert bool(((one.float() - two.float()).abs() <= 2.0 ** -7 * two.float().abs() + 2.0 ** -10).all())
    first = vY.clone()
    vY.copy_(r)
    kb.dense_forward(layer, x, R=vY, Y=vY)                   # in place, with its own row stride
    assert bool((vY == first).all())
    for o, v in zip(out, (vY, vpre, vdX)):
        v.fill_(5.0)
        assert bool((o == 5.0).all()), "what lies around the rows stays as it was"
