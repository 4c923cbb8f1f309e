"""Draws from rows of scores against their definition: columns equal, shares within the rounding of fp32.

Weights are rounded to whole multiples of 2^-40 of the largest, in the library and in the 64-bit form, and everything after that is exact in both;
an exponential that differs in its last bit can move a weight by one such unit, which a draw meets with a probability below 2^-30."""
import math
import sys

import numpy as np
import pytest

import answer_ref as ref
from test_gpu_dense import kb    # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu
U = ref.U


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def gpu(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def scores_of(rows, cols, seed, std=2.0, ties=False, out=0.0, kind="f32"):
    rng = np.random.default_rng(seed)
    s = rng.normal(0, std, (rows, cols))
    if ties:
        s = np.round(s)
    s = s.astype(np.float32)
    s[rng.random((rows, cols)) < out] = -np.inf
    if kind == "bf16":
        s = ref.bf16(s).astype(np.float32)
    return s, rng.random((rows, 7))


def check(kb, s, u, kind="f32", scores=None, **how):  # noqa: F811
    import torch
    t = gpu(s) if scores is None else scores
    if kind == "bf16" and scores is None:
        t = t.bfloat16()
    on = {k: gpu(v) if isinstance(v, np.ndarray) else v for k, v in how.items()}
    choice, prob = kb.sample_scores(t, gpu(u), want_prob=True, **on)
    cols, share = ref.sample(s.astype(np.float64), u, **how)
    got = choice.cpu().numpy()
    assert np.array_equal(got, cols), (np.argwhere(got != cols)[:5], got[got != cols][:5], cols[got != cols][:5])
    assert (np.abs(prob.double().cpu().numpy() - share) <= U * share).all()
    return choice


SETTINGS = [dict(), dict(temperature=0.3), dict(temperature=0.0), dict(top_k=1), dict(top_k=3), dict(top_k=50), dict(top_k=1000), dict(top_p=0.9),
            dict(top_p=0.05), dict(top_p=0.9999), dict(min_p=0.1), dict(min_p=1.0), dict(top_k=40, top_p=0.8, temperature=1.7),
            dict(top_k=64, top_p=0.95, min_p=0.02, temperature=0.6), dict(top_p=0.7, min_p=0.05)]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [1, 2, 3, 63, 64, 65, 200, 256, 257, 1000, 1024, 1025, 4099])
def test_settings_by_columns(kb, cols, kind):  # noqa: F811
    for i, how in enumerate(SETTINGS):
        for ties, out in ((False, 0.0), (True, 0.1), (False, 0.97)):
            say(cols, kind, how, ties, out)
            check(kb, *scores_of(6, cols, 31 * cols + i, 2.0, ties, out, kind), kind, **how)


@pytest.mark.parametrize("cols", [8191, 8193, 16384, 16385, 32768, 32771, 65537, 131072, 300001])
@pytest.mark.parametrize("rows", [1, 3])
def test_settings_by_long_rows(kb, cols, rows):  # noqa: F811
    for i, how in enumerate(SETTINGS + [dict(top_k=600), dict(top_k=5000, top_p=0.9), dict(top_k=cols - 1), dict(top_k=cols + 5, top_p=0.5)]):
        for ties, kind, out in ((False, "f32", 0.0), (True, "bf16", 0.02)):
            say(cols, rows, how, ties, kind)
            check(kb, *scores_of(rows, cols, cols + i, 2.0, ties, out, kind), kind, **how)


@pytest.mark.parametrize("rows,cols", [(300, 100), (1000, 7), (257, 1500), (300, 20000), (5000, 64), (70000, 5)])
def test_many_rows(kb, rows, cols):  # noqa: F811
    for how in (dict(), dict(top_k=20, top_p=0.9), dict(top_p=0.6, min_p=0.01)):
        say(rows, cols, how)
        check(kb, *scores_of(rows, cols, rows), **how)


@pytest.mark.parametrize("cols", [5, 300, 3000, 40000, 200000])
def test_spreads_of_scores(kb, cols):  # noqa: F811
    """Nearly equal scores, one far above the others, all equal, an offset that leaves few bits, sorted both ways"""
    base, u = scores_of(1, cols, cols)
    rows = [base[0] * 1e-6, base[0] * 1e-3 + 1000, base[0] * 100, np.zeros(cols), np.full(cols, -7.25), np.sort(base[0]), np.sort(base[0])[::-1],
            np.where(np.arange(cols) == cols // 2, 40.0, base[0]), np.linspace(-1e30, 1e30, cols), base[0] * 1e-38, np.where(base[0] > 0, 0.0, -0.0)]
    s = np.array(rows, np.float32)
    u = np.random.default_rng(1).random((len(s), 9))
    for how in SETTINGS:
        say(cols, how)
        check(kb, s, u, **how)


@pytest.mark.parametrize("cols", [4, 100, 2000, 70000])
def test_rows_without_weights_and_odd_numbers(kb, cols):  # noqa: F811
    low = -3.4028235e38
    s, _ = scores_of(9, cols, 3)
    s[0] = -np.inf                                               # nothing to draw
    s[1] = np.nan
    s[2] = low                                                   # the lowest number is a number: all alike
    s[3, 1:] = -np.inf                                           # one column
    s[4, ::2] = np.nan
    s[5, 2] = np.inf                                             # what is infinite takes all
    s[6, [1, 3]] = np.inf
    s[7] = np.where(np.arange(cols) % 3 == 0, s[7], low)
    s[8, 0] = -np.inf
    u = np.random.default_rng(1).random((9, 6))
    for how in SETTINGS:
        say(cols, how)
        c = check(kb, s, u, **how)
        assert bool((c[:2] == -1).all()) and bool((c[3] == 0).all())


@pytest.mark.parametrize("cols", [1, 50, 1500, 50000])
def test_numbers_out_of_range(kb, cols):  # noqa: F811
    """Random numbers at the ends and outside, settings of rows that the host does not see"""
    s, _ = scores_of(8, cols, 5)
    u = np.tile(np.array([0.0, 1.0 - 2.0 ** -53, 1.0, 1.5, -0.5, math.nan, math.inf, -math.inf, 0.5]), (8, 1))
    check(kb, s, u)
    check(kb, s, u, top_k=5, top_p=0.5)
    u = np.random.default_rng(2).random((8, 5))
    t = np.array([1.0, 0.0, -1.0, math.nan, math.inf, 1e-45, 3e38, 0.5], np.float32)
    check(kb, s, u, temperature=t)
    check(kb, s, u, top_k=np.array([0, -3, 1, 2, 2 ** 31 - 1, -2 ** 31, 7, 40], np.int32))
    check(kb, s, u, top_k=np.array([0, -3, 1, 2, 2 ** 31 - 1, -2 ** 31, 7, 40], np.int32), most_k=6)
    check(kb, s, u, top_p=np.array([0.0, -1.0, math.nan, 1.0, 2.0, math.inf, -math.inf, 0.5], np.float32))
    check(kb, s, u, min_p=np.array([0.0, -1.0, math.nan, 1.0, 2.0, math.inf, 1e-45, 0.5], np.float32))


@pytest.mark.parametrize("cols", [30, 900, 30000, 100000])
def test_settings_of_rows(kb, cols):  # noqa: F811
    rng = np.random.default_rng(cols)
    s, u = scores_of(20, cols, 8)
    f = lambda lo, hi: rng.uniform(lo, hi, 20).astype(np.float32)  # noqa: E731
    k = rng.integers(0, 80, 20).astype(np.int32)
    check(kb, s, u, temperature=f(0.2, 2.0), top_k=k, top_p=f(0.3, 1.1), min_p=f(0.0, 0.2))
    check(kb, s, u, temperature=f(0.2, 2.0), top_k=k, top_p=f(0.3, 1.1), min_p=f(0.0, 0.2), most_k=50)
    check(kb, s, u, temperature=f(0.2, 2.0), top_p=f(0.3, 1.0), top_k=30)
    check(kb, s, u, temperature=f(0.2, 2.0), top_p=f(0.8, 1.0))


def test_ties_on_the_border(kb):  # noqa: F811
    """Equal scores of which top-k or top-p leave the first few, by column"""
    for cols in (10, 700, 20000, 150000):
        s = np.ones((3, cols), np.float32)
        s[1, cols // 2:] = 2.0
        s[2, ::2] = 3.0
        u = np.random.default_rng(3).random((3, 50))
        for how in (dict(top_k=3), dict(top_k=cols // 2 + 1), dict(top_p=0.3), dict(top_p=0.95), dict(top_k=cols // 2 + 2, top_p=0.99), dict(top_k=cols - 1)):
            say(cols, how)
            check(kb, s, u, **how)


def test_places_strides_and_kinds_of_random_numbers(kb):  # noqa: F811
    import torch
    for cols in (60, 2000, 40000):
        s, u = scores_of(5, cols, 4)
        for kind in ("f32", "bf16"):
            for shift in (1, 2, 3):
                wide = torch.full((5, cols + 9), math.inf, device="cuda", dtype=torch.bfloat16 if kind == "bf16" else torch.float32)
                wide[:, shift:shift + cols] = gpu(s)
                x = wide[:, shift:shift + cols]
                check(kb, x.float().cpu().numpy(), u, kind, x, top_k=30, top_p=0.9)
                check(kb, x.float().cpu().numpy(), u, kind, x)
        u32 = u.astype(np.float32)
        choice, prob = kb.sample_scores(gpu(s), gpu(u32), top_p=0.9)
        assert prob is None and np.array_equal(choice.cpu().numpy(), ref.sample(s.astype(np.float64), u32.astype(np.float64), top_p=0.9)[0])


def test_one_row_seen_by_all(kb):  # noqa: F811
    """Rows that start one element apart would be refused; a single row of stride zero is one row"""
    import torch
    s, _ = scores_of(1, 500, 4)
    u = np.random.default_rng(9).random((1, 300))
    check(kb, s, u, top_k=40)
    with pytest.raises(kb.KgeError):
        kb.sample_scores(gpu(s).expand(4, 500), torch.rand(4, 3, device="cuda"))


def test_no_columns_no_rows_no_draws(kb):  # noqa: F811
    import torch
    e = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    choice, prob = kb.sample_scores(e(4, 0), torch.rand(4, 3, device="cuda"), want_prob=True)
    assert bool((choice == -1).all()) and bool((prob == 0).all())
    assert kb.sample_scores(e(0, 5), e(0, 3))[0].shape == (0, 3) and kb.sample_scores(e(5, 5), e(5, 0))[0].shape == (5, 0)


@pytest.mark.parametrize("rows,cols", [(3, 100), (4, 3000), (2, 50000), (3, 400000), (400, 300)])
def test_repeats_workspaces_and_streams(kb, rows, cols):  # noqa: F811
    """The same draws from a workspace that held anything, on another stream, at once with other calls of their own workspaces"""
    import torch
    s, u = scores_of(rows, cols, 6)
    s, u = gpu(s), gpu(u)
    for how in (dict(top_k=50, top_p=0.9), dict(top_p=0.9), dict(), dict(top_k=3000, min_p=0.001)):
        say(rows, cols, how)
        want, p = kb.sample_scores(s, u, want_prob=True, **how)
        n = kb.sample_workspace_bytes(rows, cols, **how)
        streams = [torch.cuda.Stream() for _ in range(3)]
        torch.cuda.synchronize()
        outs = []
        for i, st in enumerate(streams):
            ws = torch.full((n,), 255 - i, dtype=torch.uint8, device="cuda")
            torch.cuda.synchronize()
            outs.append((kb.sample_scores(s, u, want_prob=True, workspace=ws, stream=st, **how), ws))
        torch.cuda.synchronize()
        for (c, q), _ in outs:
            assert torch.equal(c, want) and torch.equal(q, p)


@pytest.mark.parametrize("rows,cols", [(5, 60), (3, 5000), (2, 90000)])
def test_captured_and_replayed(kb, rows, cols):  # noqa: F811
    import torch
    for how in (dict(top_k=30, top_p=0.9), dict(top_p=0.8), dict()):
        say(rows, cols, how)
        s, u = torch.randn(rows, cols, device="cuda"), torch.rand(rows, 4, dtype=torch.float64, device="cuda")
        choice, prob = torch.empty((rows, 4), dtype=torch.int32, device="cuda"), torch.empty((rows, 4), device="cuda")
        ws = torch.empty(kb.sample_workspace_bytes(rows, cols, **how), dtype=torch.uint8, device="cuda")
        kb.sample_scores(s, u, choice=choice, prob=prob, workspace=ws, **how)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kb.sample_scores(s, u, choice=choice, prob=prob, workspace=ws, **how)
        for i in range(4):
            s.copy_(torch.randn(rows, cols, device="cuda") * (i + 1))
            u.copy_(torch.rand(rows, 4, dtype=torch.float64, device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            want, share = ref.sample(s.double().cpu().numpy(), u.cpu().numpy(), **how)
            assert np.array_equal(choice.cpu().numpy(), want) and (np.abs(prob.double().cpu().numpy() - share) <= U * share).all()


def test_offsets_past_32_bits(kb):  # noqa: F811
    import torch
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB")
    wide = torch.empty((3, 2_200_000_000), dtype=torch.bfloat16, device="cuda")
    s, u = scores_of(3, 5000, 11, kind="bf16")
    x = wide[:, 7:5007]
    x.copy_(gpu(s))
    check(kb, s, u, "bf16", x, top_k=20, top_p=0.9)
    check(kb, s, u, "bf16", x, top_p=0.9)


def test_shares_of_many_draws(kb):  # noqa: F811
    """Evenly spread random numbers come out in the softmax's shares, to one draw a column"""
    import torch
    s = torch.randn(1, 300, device="cuda")
    n = 200000
    u = ((torch.arange(n, dtype=torch.float64, device="cuda") + 0.5) / n)[None]
    choice, _ = kb.sample_scores(s, u, temperature=0.8)
    share = torch.softmax(s.double() / float(np.float32(0.8)), 1)[0] * n
    assert float((torch.bincount(choice[0].long(), minlength=300) - share).abs().max()) <= 1.0 + 1e-4


def test_pick_negatives(kb):  # noqa: F811
    import torch
    rng = np.random.default_rng(0)
    ent, side = rng.integers(0, 1000, (700, 9)).astype(np.int32), rng.integers(0, 2, (700, 9)).astype(np.uint8)
    choice = rng.integers(0, 9, (700, 20)).astype(np.int32)
    choice[5], choice[6, 3], choice[7, 0] = -1, 9, 2 ** 31 - 1
    ne, ns = torch.empty((700, 20), dtype=torch.int32, device="cuda"), torch.empty((700, 20), dtype=torch.uint8, device="cuda")
    kb.pick_negatives(gpu(ent), gpu(side), gpu(choice), ne, ns)
    c = np.where((choice < 0) | (choice >= 9), np.arange(20)[None, :] % 9, choice)
    assert np.array_equal(ne.cpu().numpy(), np.take_along_axis(ent, c, 1)) and np.array_equal(ns.cpu().numpy(), np.take_along_axis(side, c, 1))


def test_long_rows_of_zeros_and_negative_scores(kb):  # noqa: F811
    """Zero is where the digits of a score's bits have a border: scores of exactly zero, of either sign, beside those just below and above"""
    cols = 200000
    rng = np.random.default_rng(5)
    below = -np.abs(rng.normal(0, 2, cols)).astype(np.float32)
    below[:50000] *= np.float32(1e-40)                           # subnormal, and next to zero
    rows = []
    for zeros in (0.0, -0.0):
        s = below.copy()
        s[rng.permutation(cols)[:60000]] = zeros
        rows.append(s)
    rows.append(np.where(rng.random(cols) < 0.3, 0.0, below).astype(np.float32))
    rows.append(np.where(rng.random(cols) < 0.1, -rows[2], rows[2]).astype(np.float32))
    rows.append(np.where(rng.random(cols) < 0.5, np.float32(-1e-45), np.float32(0)).astype(np.float32))
    s, u = np.array(rows), rng.random((5, 9))
    above = [int((r >= 0).sum()) for r in s]
    for k in (59990, 60000, 60010, above[2] + 1, above[3] - 1, above[4], above[4] + 5):
        for how in (dict(top_k=k), dict(top_k=k, top_p=0.9999), dict(top_k=k, temperature=3e38, top_p=0.5)):
            say(k, how)
            check(kb, s, u, **how)
    for p in (0.2, 0.299, 0.3, 0.31, 0.5, 0.9):
        for t in (3e38, 1.0, 1e-3):
            say(p, t)
            check(kb, s, u, top_p=p, temperature=t)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_rows_of_millions(kb, kind):  # noqa: F811
    """More columns than 2^22, where a weight's unit is 2^-39, in every way that long rows go; lists that have no room"""
    s, u = scores_of(1, 4200001, 77, kind=kind)
    s[0, 1000000:1040000] = 3.0
    for how in (dict(), dict(top_k=10), dict(top_k=100000), dict(top_p=0.95), dict(top_p=0.5, min_p=0.01), dict(top_k=3000000, top_p=0.8), dict(temperature=0.0)):
        say(kind, how)
        check(kb, s, u, kind, **how)


@pytest.mark.parametrize("cols", [3, 100, 700, 1500, 9000, 40000, 70000])
def test_signalling_nan(kb, cols):  # noqa: F811
    """A NaN of any bits is no score, wherever it stands: beside the largest, first and last"""
    import torch
    s, u = scores_of(5, cols, cols, 1.0)
    bits = s.view(np.uint32)
    for r, at in enumerate((0, cols - 1, cols // 2, 1)):
        bits[r, at] = (0x7f800001, 0xff800001, 0x7fa00000, 0xffbfffff)[r]
        s[r, (at + 1) % cols] = 6.0
    s[4] = -np.inf
    bits[4, 0] = 0x7f800001
    half = torch.from_numpy((bits >> 16 | (np.isnan(s) * 1)).astype(np.uint16).view(np.int16)).cuda().view(torch.bfloat16)
    for how in (dict(), dict(temperature=0.0), dict(top_k=2), dict(top_p=0.9), dict(min_p=0.3)):
        say(cols, how)
        t = torch.from_numpy(s.view(np.int32).copy()).cuda().view(torch.float32)
        clean = np.where(np.isnan(s), -np.inf, s)
        check(kb, clean, u, scores=t, **how)
        clean = np.where(np.isnan(s), -np.inf, (bits & np.uint32(0xffff0000)).view(np.float32))
        check(kb, clean, u, "bf16", scores=half, **how)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_few_draws_of_long_rows(kb, kind):  # noqa: F811
    """Enough rows for parts of 16384, and so few draws that each weighs its part again; rows of every kind in one call: a plain top-p, no top-p,
    one score, min-p above top-p's first digit and below it, ties of both cuts, infinities, nothing"""
    rows, cols = 9, 2_900_000
    s, u = scores_of(rows, cols, 77, 2.0, out=0.01, kind=kind)
    s[4] = np.round(s[4] * 2) / 2
    s[5] = np.round(s[5] * 2) / 2
    s[6, [17, 40_000, 2_899_999]] = np.inf
    s[7] = np.nan
    s[8, 1_000_000:] = -np.inf
    say(kind)
    check(kb, s, u, kind, temperature=np.array([0.9, 1, 0, 1.5, 0.8, 1, 1, 1, 3], np.float32), top_k=np.array([0, 0, 0, 0, 0, 200_000, 0, 5, 700_000], np.int32),
          top_p=np.array([0.9, 1, 0.5, 0.95, 0.7, 0.8, 0.6, 0.5, 0.3], np.float32), min_p=np.array([0, 0, 0, 0.4, 0.001, 0, 0.5, 0, 1e-4], np.float32))
    check(kb, s, u, kind, temperature=1.1, top_p=0.97, min_p=0.01)
    check(kb, s[:, :2_000_001], u, kind, temperature=2.0, top_p=0.4)


def test_more_long_rows_than_a_batch(kb):  # noqa: F811
    import torch
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    rows, cols = 4100, 262200
    s = torch.randn(rows, cols, device="cuda", dtype=torch.bfloat16)
    u = torch.rand(rows, 2, dtype=torch.float64, device="cuda")
    some = [0, 1, 4095, 4096, 4099]
    for how in (dict(top_p=0.9), dict(top_k=30000, top_p=0.9), dict(top_k=20), dict()):
        say(rows, cols, how)
        choice, prob = kb.sample_scores(s, u, want_prob=True, **how)
        want, share = ref.sample(s[some].double().cpu().numpy(), u[some].cpu().numpy(), **how)
        assert np.array_equal(choice[some].cpu().numpy(), want) and (np.abs(prob[some].double().cpu().numpy() - share) <= U * share).all()
        assert bool((choice >= 0).all()) and bool((choice < cols).all()) and bool((prob > 0).all())
