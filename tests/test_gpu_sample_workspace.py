"""Draws from long rows stay inside the workspace that they ask for."""
import sys

import pytest

from test_gpu_dense import kb    # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(1, 70000), (3, 1000001), (40, 300000), (130, 400000)])
def test_nothing_behind_the_workspace_is_written(kb, rows, cols):  # noqa: F811
    import torch
    s = torch.randn(rows, cols, device="cuda")
    s[0] = 1.5                                                   # equal scores: every list is full
    u = torch.rand(rows, 3, device="cuda")
    k = torch.randint(0, 500, (rows,), dtype=torch.int32, device="cuda")
    for how in (dict(), dict(min_p=0.1), dict(top_k=cols // 2), dict(top_k=40), dict(top_k=k), dict(top_p=0.9), dict(top_p=0.9, top_k=cols // 2), dict(top_p=0.7, top_k=k),
                dict(temperature=0.0)):
        print("[case]", rows, cols, {a: b if isinstance(b, (int, float)) else "by row" for a, b in how.items()}, file=sys.stderr, flush=True)
        want = kb.sample_scores(s, u, want_prob=True, **how)
        n = kb.sample_workspace_bytes(rows, cols, **how)
        memory = torch.full((n + (1 << 20),), 0xA5, dtype=torch.uint8, device="cuda")
        got = kb.sample_scores(s, u, want_prob=True, workspace=memory[:n], **how)
        assert bool((memory[n:] == 0xA5).all())
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
