"""Draws at the borders between the ways in which rows are taken: by a wavefront, a small block, a large block, split; and beside them."""
import sys

import numpy as np
import pytest

import answer_ref as ref
from test_gpu_dense import kb    # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu
U = ref.U


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def rows_of(rows, cols, kind):
    """(scores on the device, rows that are looked at): plain ones, equal scores in plenty, few scores, one score everywhere, nothing, odd numbers"""
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows * 7 + cols)
    s = torch.randn((rows, cols), generator=g, device="cuda") * 2
    some = [0, 1, 2, 3, 4, 5, rows // 2, rows - 1]
    s[1] = torch.round(s[1] * 2) / 2
    s[2, torch.rand(cols, generator=g, device="cuda") < 0.97] = -np.inf
    s[3] = -1.25
    s[4] = -np.inf
    s[5, ::3] = float("nan")
    s[5, cols - 1] = 9.0
    return s.bfloat16() if kind == "bf16" else s, some


def check(kb, s, some, u, **how):  # noqa: F811
    import torch
    on = {k: torch.from_numpy(v).cuda() if isinstance(v, np.ndarray) else v for k, v in how.items()}
    choice, prob = kb.sample_scores(s, u, want_prob=True, **on)
    at = {k: v[some] if isinstance(v, np.ndarray) else v for k, v in how.items()}
    want, share = ref.sample(s[some].double().cpu().numpy(), u[some].cpu().numpy(), **at)
    got = choice[some].cpu().numpy()
    assert np.array_equal(got, want), (np.argwhere(got != want)[:5], got[got != want][:5], want[got != want][:5])
    assert (np.abs(prob[some].double().cpu().numpy() - share) <= U * share).all()
    empty = choice < 0                                           # of the others one has no score to draw
    assert bool((empty.all(1) == empty.any(1)).all()) and int(empty.any(1).sum()) == 1 and bool((choice < s.shape[1]).all())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(4095, 1025), (4096, 1025), (4096, 1279), (4096, 2047), (4096, 2048), (4096, 2049), (511, 4097), (512, 4095), (512, 4096), (512, 4097),
                                       (512, 16385), (512, 65535), (512, 65536), (511, 65536), (512, 65537), (128, 32769), (127, 32769), (128, 65536),
                                       (255, 65537), (256, 65537), (256, 262143), (256, 262144), (256, 262145)])
def test_rows_at_the_borders(kb, rows, cols, kind):  # noqa: F811
    import torch
    s, some = rows_of(rows, cols, kind)
    g = torch.Generator(device="cuda").manual_seed(1)
    u = torch.rand((rows, 5), generator=g, device="cuda", dtype=torch.float64)
    u[:, 0], u[:, 1] = 0.0, 1.0 - 2.0 ** -53                     # the first and the last column that is left
    rng = np.random.default_rng(cols)
    f = lambda lo, hi: rng.uniform(lo, hi, rows).astype(np.float32)  # noqa: E731
    k = rng.integers(0, 90, rows).astype(np.int32)
    for how in (dict(), dict(top_k=50), dict(top_k=cols // 3), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=700, top_p=0.8, min_p=0.001, temperature=1.3),
                dict(temperature=f(0.3, 2.0), top_k=k, top_p=f(0.3, 1.1), min_p=f(0.0, 0.1))):
        say(rows, cols, kind, {k: v if np.isscalar(v) else "by row" for k, v in how.items()})
        check(kb, s, some, u, **how)
