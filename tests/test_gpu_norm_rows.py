"""Layer norm's backward pass over more rows than its blocks hold at once: dgamma and dbeta from integers, whose sums fp32 holds
exactly, bit for bit; dX row by row."""
import numpy as np
import pytest

import block_ref as ref
from test_gpu_dense import dev, host, kb, say, within    # noqa: F401  (kb: the fixture)

pytestmark = pytest.mark.gpu
# beyond 1024 blocks (512 above 2048 elements) of 64, 32, 16, 8, 4 rows or one row: two rounds and a remainder, or three and four
SIZES = [(70001, 40), (200003, 7), (40001, 100), (20003, 256), (50001, 130), (10001, 512), (20011, 300), (5003, 1000), (13001, 1024), (4101, 2048),
         (1301, 2049), (2051, 4096), (1101, 8192), (1101, 8193), (600, 16384)]


@pytest.mark.parametrize("kx,ky", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("n,d", SIZES)
def test_many_rows(kb, kx, ky, n, d):  # noqa: F811
    say("layer norm rows", kx, ky, n, d)
    rng = np.random.default_rng(n + d)
    X, G = rng.integers(-3, 4, (n, d)).astype(np.float32), rng.integers(-3, 4, (n, d)).astype(np.float32)
    mean, rstd = rng.integers(-1, 2, n).astype(np.float32), (2.0 ** rng.integers(-1, 2, n)).astype(np.float32)
    gamma = rng.normal(1, 0.2, d).astype(np.float32)
    assert 2 * 24 * n < 2 ** 24        # xh is a multiple of 1/2 up to 8, a term of 1/2 up to 24
    norm = dict(gamma=dev(gamma), beta=None, eps=1e-5)
    x, g, m, r = dev(X, kx), dev(G, ky), dev(mean), dev(rstd)
    blocks = min(1024 if d <= 2048 else 512, -(-n // ((16 if d <= 64 else 8 if d <= 128 else 4 if d <= 2048 else 1) * (4 if d <= 256 else 2 if d <= 512 else 1))))
    assert kb.layer_norm_workspace_bytes(d, n) == -(-blocks * 2 * d * 4 // 256) * 256 and blocks in (512, 1024)
    got = kb.layer_norm_backward(norm, x, m, r, g)
    X, G, mean, rstd = (t.astype(np.float64) for t in (X, G, mean, rstd))
    xh = (X - mean[:, None]) * rstd[:, None]
    assert np.array_equal(host(got["dgamma"]), (G * xh).sum(0)) and np.array_equal(host(got["dbeta"]), G.sum(0))
    args = gamma.astype(np.float64), mean, rstd
    step = max(1, 4000000 // d)
    for p in [slice(k, min(k + step, n)) for k in range(0, n, step)]:
        part = X[p], args[0], mean[p], rstd[p], G[p]
        within(host(got["dX"][p]), ref.norm_backward(*part)[0], ref.norm_backward_bound(*part, kx)[0], "dX")
    sums = kb.layer_norm_backward(norm, x, m, r, g, need_dX=False)
    assert all(bool((sums[k] == got[k]).all()) for k in ("dgamma", "dbeta"))
    again = kb.layer_norm_backward(norm, x, m, r, g)
    assert all(bool((again[k] == got[k]).all()) for k in got), "the same call gives the same bits"


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(70001, 40), (5003, 1000), (1301, 2049), (1101, 8193)])
def test_many_rows_forward_and_back(kb, kind, n, d):  # noqa: F811
    """Real numbers; a term of dgamma and dbeta passes through the sums of its lane's rows, of the block's groups and of the blocks,
    fewer than a hundred additions in place of n."""
    say("layer norm real rows", kind, n, d)
    rng = np.random.default_rng(n)
    X = rng.normal(0, 1, (n, d)) * rng.uniform(0.2, 3.0, (n, 1)) + rng.normal(0, 2, (n, 1))
    gamma, beta = rng.normal(1, 0.2, d).astype(np.float32), rng.normal(0, 0.2, d).astype(np.float32)
    x, g = dev(X, kind), dev(rng.normal(0, 0.1, (n, d)), kind)
    norm = dict(gamma=dev(gamma), beta=dev(beta), eps=1e-5)
    Y, mean, rstd = kb.layer_norm_forward(norm, x)
    args = host(x), gamma.astype(np.float64), beta.astype(np.float64), float(np.float32(1e-5))
    for got, want, bound in zip((Y, mean, rstd), ref.norm_forward(*args), ref.norm_forward_bound(*args, kind)):
        within(host(got), want, bound, "forward")
    got = kb.layer_norm_backward(norm, x, mean, rstd, g)
    x, g, mean, rstd = host(x), host(g), host(mean)[:, None], host(rstd)[:, None]
    xh = (x - mean) * rstd
    ex = 2.0 * ref.U * (np.abs(x) + np.abs(mean)) * rstd + ref.U * np.abs(xh)
    depth = 8 + 16 + 32 + 32 + 8                            # rows of a lane, groups of a block, 1024 / 32 blocks, 32 lanes of the second launch; its own products
    wide = depth * ref.U * np.abs(g * xh).sum(0) + (np.abs(g) * ex).sum(0)
    within(host(got["dgamma"]), (g * xh).sum(0), wide, "dgamma")
    within(host(got["dbeta"]), g.sum(0), depth * ref.U * np.abs(g).sum(0), "dbeta")
    within(host(got["dX"]), ref.norm_backward(x, args[1], mean[:, 0], rstd[:, 0], g)[0],
           ref.norm_backward_bound(x, args[1], mean[:, 0], rstd[:, 0], g, kind)[0], "dX")
