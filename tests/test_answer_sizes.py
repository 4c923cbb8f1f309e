"""Settings and sizes of the answering operators that a 32-bit argument does not hold are never cut to what it does.  None of it needs a GPU."""
import os

import pytest


@pytest.fixture(scope="module")
def kb():
    from paper_2201_02791_amd import build, binding
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    binding.load()
    return binding


MOST = 2 ** 31 - 1


@pytest.mark.parametrize("k", [MOST, 2 ** 31, 2 ** 32, 2 ** 32 + 5, 10 ** 12, 2 ** 63, 2 ** 70])
def test_a_top_k_that_is_more_than_any_row_has(kb, k):
    """As many as there are, however large the number: the largest that the library takes, which no row reaches"""
    import torch
    assert kb._sampling(1.0, k, 1.0, 0.0, 0, 3)[0].top_k == MOST
    rows = torch.ones(3, dtype=torch.int32)
    assert kb._sampling(1.0, rows, 1.0, 0.0, k, 3)[0].top_k == MOST
    assert kb._sampling(torch.ones(3), k, 1.0, 0.0, 0, 3)[0].top_k == MOST
    assert kb.sample_workspace_bytes(3, 100000, top_k=k) == kb.sample_workspace_bytes(3, 100000, top_k=MOST)


@pytest.mark.parametrize("k", [-1, -2 ** 31, -2 ** 31 - 1, -2 ** 32, -2 ** 32 + 5, -2 ** 70])
def test_a_top_k_below_zero_is_refused(kb, k):
    import torch
    for how in (dict(top_k=k), dict(top_k=torch.ones(3, dtype=torch.int32), most_k=k), dict(top_k=k, temperature=torch.ones(3))):
        with pytest.raises(kb.KgeError, match="top_k"):
            kb.sample_workspace_bytes(3, 100000, **how)
        with pytest.raises(kb.KgeError, match="top_k|device"):
            kb.sample_scores(torch.zeros(3, 9), torch.zeros(3, 4), **how)


def test_settings_in_range_are_kept(kb):
    for k in (0, 1, 50, MOST - 1):
        assert kb._sampling(0.5, k, 0.9, 0.1, 0, 3)[0].top_k == k
    with pytest.raises(TypeError):
        kb._sampling(0.5, 2.5, 0.9, 0.1, 0, 3)


@pytest.mark.parametrize("wide", [2 ** 31, 2 ** 32, 2 ** 32 + 40])
def test_sizes_past_32_bits_are_refused(kb, wide):
    """Tensors without memory: what is checked is the argument, before any launch"""
    import torch
    at = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="meta")  # noqa: E731
    i32, u8 = torch.int32, torch.uint8
    with pytest.raises(kb.KgeError, match="4096"):
        kb.table4_encode(at(1, wide))
    with pytest.raises(kb.KgeError, match="draws"):
        kb.sample_scores(at(1, 9), at(1, wide))
    with pytest.raises(kb.KgeError, match="candidates"):
        kb.pick_negatives(at(1, wide, dtype=i32), at(1, wide, dtype=u8), at(1, 4, dtype=i32), at(1, 4, dtype=i32), at(1, 4, dtype=u8))
    with pytest.raises(kb.KgeError, match="negatives"):
        kb.pick_negatives(at(1, 9, dtype=i32), at(1, 9, dtype=u8), at(1, wide, dtype=i32), at(1, wide, dtype=i32), at(1, wide, dtype=u8))

    class Part:
        handle = None
    with pytest.raises(kb.KgeError, match="candidates"):
        kb.hide_positives(Part(), at(1, dtype=i32), at(1, wide, dtype=i32), at(1, wide, dtype=u8), at(1, wide))


def test_a_step_number_is_an_aligned_address(kb):
    t = (kb._GradTensor * 1)()
    for at in (None, 4100):
        assert kb.load().kge_grad_norm_step(t, 1, 1.0, 4096, 4096, at, 4096, 1 << 20, None) == -1 and b"t_dev" in kb.load().kge_last_error()
    assert kb.load().kge_grad_norm_step(t, 1, -1.0, 4096, 4096, 4096, 4096, 1 << 20, None) == -1 and b"max_norm" in kb.load().kge_last_error()


def test_settings_of_adamw_are_checked_alone(kb):
    kb.check_adamw(0.1, 0.0, 0.5, 1e-8)
    for how in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan"))):
        with pytest.raises(kb.KgeError, match="beta"):
            kb.check_adamw(**how)


@pytest.mark.parametrize("rows,cols", [(16, 2900000), (1, 1000000), (4096, 300000), (9000, 300000)])
def test_workspaces_of_long_rows(kb, rows, cols):
    """Lists of scores are claimed where top-p's search writes them, and there alone: sums of 16 bytes for 1024 columns and those by digit are
    what the others need"""
    at_once = min(rows, 4096)
    without = at_once * (6 * 2048 * 8 + 1024 + 16 * cols // 1024 + 40 * (cols // 4096 + 1)) + 4096
    for how in (dict(), dict(min_p=0.1), dict(top_k=cols // 2), dict(top_k=cols // 2, temperature=0.5, min_p=0.01)):
        assert kb.sample_workspace_bytes(rows, cols, **how) <= without, how
    for how in (dict(top_p=0.9), dict(top_p=0.9, top_k=cols // 2)):
        assert 2 * at_once * cols <= kb.sample_workspace_bytes(rows, cols, **how) <= without + 3 * at_once * (cols + 65536), how
    kb.check_adamw(t=2 ** 40)
    with pytest.raises(kb.KgeError, match="starts at 1"):
        kb.check_adamw(t=0)
