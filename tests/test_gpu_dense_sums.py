"""The dense layer's sums over many rows: from integers, whose sums fp32 holds exactly, bit for bit; from real numbers within the
roundings that a chunk's rows and the chunks' number make, where one lost chunk shows."""
import numpy as np
import pytest

import block_ref as ref
from test_gpu_dense import dev, host, kb, say, tt, within    # noqa: F401  (kb: the fixture)

pytestmark = pytest.mark.gpu


def chunks_of(kind, n, di, do):
    """[(first row, end)] of the chunks that the weights' gradient is cut into."""
    bm, bn = ((128, 32) if do <= 32 else (128, 64) if do <= 64 else (32, 128) if di <= 32 else (256, 128) if kind == "bf16" and di > 128 and do > 64 else (128, 128))
    tiles, at_once = -(-di // bm) * -(-do // bn), 256 if bm == 256 else 512
    most = 8 * (at_once // 8 // tiles) if tiles <= at_once // 8 else at_once // tiles
    rows = -(-n // max(1, min(most, -(-n // 256))))
    rows = -(-rows // 64) * 64
    return [(r, min(r + rows, n)) for r in range(0, n, rows)]


# one to more than 256 chunks: each form of the second launch, the last chunk a short one; every tile of the weights' gradient
SIZES = [(200, 40, 24, 1), (2600, 9, 3, 11), (3000, 200, 200, 12), (20003, 200, 100, 79), (29082, 203, 517, 46), (50001, 130, 140, 112),
         (70000, 66, 65, 274), (40007, 300, 20, 157), (140000, 20, 21, 438), (140003, 24, 200, 244), (131073, 130, 60, 228)]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["identity", "relu"])
@pytest.mark.parametrize("n,di,do,chunks", SIZES)
def test_integers_bit_for_bit(kb, kind, act, n, di, do, chunks):  # noqa: F811
    """Terms of up to 9, fewer than 2^17 a sum: every partial sum is an integer below 2^24, whatever the order."""
    import torch
    say("dense integer sums", kind, act, n, di, do)
    assert 9 * n < 2 ** 24
    gen = torch.Generator("cuda").manual_seed(n + di)
    x, g, z = (torch.randint(-3, 4, s, generator=gen, device="cuda").to(tt(kind)) for s in ((n, di), (n, do), (n, do)))
    X, G, Z = host(x), host(g), host(z)
    parts = chunks_of(kind, n, di, do)
    assert len(parts) == chunks
    layer = dict(W=dev(np.zeros((di, do)), kind), b=None, act=ref.RELU if act == "relu" else ref.IDENTITY)
    P = G * (Z > 0) if act == "relu" else G
    got = kb.dense_backward(layer, x, z, g, need_dX=False)
    dW, db = host(got["dW"]), host(got["db"])
    assert np.array_equal(dW, X.T @ P) and np.array_equal(db, P.sum(0))
    for r, e in parts:
        assert (X[r:e].T @ P[r:e]).any() and P[r:e].any(), "without this chunk the sums are others"
    assert kb.dense_workspace_bytes(layer, n) == -(-len(parts) * (di + 1) * do * 4 // 256) * 256


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,di,do,chunks", SIZES)
def test_real_numbers_within_what_chunks_round(kb, kind, n, di, do, chunks):  # noqa: F811
    """A term passes through at most its chunk's rows and then the chunks' number of additions: the depth that sum_bound takes."""
    import torch
    say("dense real sums", kind, n, di, do)
    gen = torch.Generator("cuda").manual_seed(n + do)
    x, z, g = ((torch.randn(shape, generator=gen, device="cuda") * s).to(tt(kind)) for s, shape in ((1.0, (n, di)), (1.0, (n, do)), (0.1, (n, do))))
    layer = dict(W=dev(np.zeros((di, do)), kind), b=None, act=ref.SILU)
    got = kb.dense_backward(layer, x, z, g, need_dX=False)
    x, z, g = host(x), host(z), host(g)
    P = g * ref.act_grad(z, ref.SILU)
    off = np.abs(g) * 8.0 * ref.U * (1.0 + np.abs(z)) + 2.0 * ref.U * np.abs(P)       # act', as the elementwise bounds count it
    parts = chunks_of(kind, n, di, do)
    depth = parts[0][1] + len(parts)
    wide_w = ref.sum_bound(depth, np.abs(x).T @ np.abs(P)) + np.abs(x).T @ off
    wide_b = ref.sum_bound(depth, np.abs(P).sum(0)) + off.sum(0)
    within(host(got["dW"]), x.T @ P, wide_w, "dW")
    within(host(got["db"]), P.sum(0), wide_b, "db")
    for r, e in parts[:3] + parts[-1:]:
        if e - r >= 64:
            assert (np.abs(x[r:e].T @ P[r:e]) > 2.0 * wide_w).any() and (np.abs(P[r:e].sum(0)) > 2.0 * wide_b).any(), "a lost chunk shows"
