"""AdamW over a tensor whose rows are more wavefronts than one launch may have."""
import numpy as np
import pytest

from test_gpu_adamw import HYPER, make, tensor
from test_gpu_dense import host, kb, say    # noqa: F401  (kb: the fixture)

pytestmark = pytest.mark.gpu


def test_masked_rows_of_two_launches(kb):  # noqa: F811
    """Rows of 257 elements are two wavefronts each: 2^25 of them and more are more than a launch takes.  The rows that the mask takes,
    at both ends and where the launches meet, must move as the same rows of a small tensor do, and their neighbours not at all; so
    must a tensor in front and one behind."""
    import torch
    torch.cuda.empty_cache()
    n, d = (1 << 25) + 1000, 257
    if torch.cuda.mem_get_info()[0] < 110 << 30:
        pytest.skip("needs 90 GB of device memory")
    say("adamw", n, d)
    meet = 1 << 25                       # the second launch begins a few rows before this one
    at = torch.tensor([0, 1, 77, (1 << 24) + 3] + list(range(meet - 9, meet + 3)) + [n - 2, n - 1], device="cuda")
    beside = torch.tensor([2, 76, (1 << 24) + 2, meet - 10, meet + 3, n - 3], device="cuda")
    p, g, _ = make((len(at), d), 3)
    small = tensor(kb, p, g, 8, "all", None, 0.1, False)
    big = dict(weight_decay=0.1, rows="mask", row_mask=torch.zeros(n, dtype=torch.uint8, device="cuda"))
    for k in ("param", "grad"):
        big[k] = torch.empty((n, d), device="cuda")
        big[k][at], big[k][beside] = small[k], 5.0
    for k, dt in (("m", torch.float8_e4m3fn), ("v", torch.float8_e5m2)):
        codes = torch.empty((n, d), dtype=torch.uint8, device="cuda")
        codes[at], codes[beside] = 0, 9
        big[k] = codes.view(dt)
        big[k + "_scale"] = torch.empty((n, 2), device="cuda")
        big[k + "_scale"][at], big[k + "_scale"][beside] = 0.0, 2.0
    big["row_mask"][at] = 1
    ends = [[tensor(kb, *make((33, 40), 8 + i)[:2], 32, "all", None, 0.0, False) for i in range(2)] for _ in range(2)]
    kb.adamw_step([ends[0][0], big, ends[0][1]], t=1, **HYPER)
    kb.adamw_step([small] + ends[1], t=1, **HYPER)
    torch.cuda.synchronize()
    assert bool((big["param"][at] == small["param"]).all()) and not np.array_equal(host(small["param"]), p)
    for k in ("m_scale", "v_scale"):
        assert bool((big[k][at] == small[k]).all()) and bool((big[k][beside] == 2.0).all())
    # which of two neighbouring codes is taken goes by the element's index: here another one
    for k, part in (("m", 0.125), ("v", 0.25)):
        a, b = (host(t.float()) for t in (big[k].view(torch.uint8)[at].view(big[k].dtype), small[k]))
        assert (np.abs(a - b) <= part * np.maximum(np.maximum(np.abs(a), np.abs(b)), 2.0 ** -6 if k == "m" else 2.0 ** -14)).all()
        assert bool((big[k].view(torch.uint8)[beside] == 9).all())
    assert bool((big["param"][beside] == 5.0).all())
    for x, y in zip(*ends):
        assert all(bool((x[k] == y[k]).all()) for k in ("param", "m", "v"))
    del big
    torch.cuda.empty_cache()
