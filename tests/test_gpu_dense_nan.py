"""Calls whose inputs are all NaN: fp32 results that are not finite are formed again term by term, which must not cost a training run
that has diverged its speed."""
import numpy as np
import pytest

import block_ref as ref
from test_gpu_dense import kb, say, tt    # noqa: F401  (kb: the fixture)

pytestmark = pytest.mark.gpu


# few results; rows past W in registers; tiles of 64 x 128 (fp32) or 128 x 128
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,di,do", [(250, 512, 512), (17000, 128, 128), (12000, 512, 512), (100000, 256, 256)])
def test_all_nan_takes_little_longer(kb, kind, n, di, do):  # noqa: F811
    """At most eight times the time of finite numbers, the least of five; the whole sums took 20 to 250 times."""
    import torch
    say("dense all NaN", kind, n, di, do)
    full = lambda v, *s: torch.full(s, v, dtype=tt(kind), device="cuda")  # noqa: E731

    def least(call):
        t = []
        for _ in range(6):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            call()
            b.record()
            torch.cuda.synchronize()
            t.append(a.elapsed_time(b))
        return min(t[1:])
    took = []
    for v in (0.5, float("nan")):
        x, g, z, layer = full(v, n, di), full(v, n, do), full(0.5, n, do), dict(W=full(0.5, di, do), b=None, act=ref.SILU)
        calls = [lambda: kb.dense_forward(layer, x, keep_pre=True), lambda: kb.dense_backward(layer, x, z, g, need_dW=False),
                 lambda: kb.dense_backward(layer, x, z, g, need_dX=False)]
        if v != v:
            Y, pre = calls[0]()
            back = kb.dense_backward(layer, x, z, g)
            assert all(bool(t.isnan().all()) for t in (Y, pre, *back.values()))
        took.append([least(c) for c in calls])
    say("ms", took)
    assert (np.array(took[1]) <= 8.0 * np.array(took[0]) + 0.02).all(), took
