"""Tables of 4 bits and the scores of questions against them: codes, scales and rows bit for bit, scores within fp32's rounding of sums in 64 bits."""
import math
import sys

import numpy as np
import pytest

import answer_ref as ref
from test_gpu_dense import kb    # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def rows_of(n, d, seed, kind="f32"):
    rng = np.random.default_rng(seed)
    x = rng.normal(0, 1, (n, d)) * 10.0 ** rng.integers(-4, 4, (n, 1))
    x[rng.random((n, d)) < 0.05] = 0.0
    x = x.astype(np.float32)
    return ref.bf16(x).astype(np.float32) if kind == "bf16" else x


def gpu(x, kind="f32"):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t.bfloat16() if kind == "bf16" else t


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(1, 1), (3, 4), (17, 31), (16, 32), (5, 33), (40, 64), (33, 100), (20, 200), (9, 256), (7, 1000), (2, 4096), (70, 129)])
def test_codes_scales_and_rows(kb, n, d, kind):  # noqa: F811
    import torch
    say(n, d, kind)
    x = rows_of(n, d, n * 7 + d, kind)
    if n > 2:
        x[1] = 0.0                                               # a row of nothing, and a group of one small number
        x[2, :32] = 0.0
        x[2, min(5, d - 1)] = 1e-30
    codes, scales = ref.encode(gpu(x, kind).double().cpu().numpy())        # of the numbers that the call gets: 1e-30 is rounded for bf16
    t = kb.table4_encode(gpu(x, kind))
    assert np.array_equal(t.scales.double().cpu().numpy(), scales)
    assert np.array_equal(t.codes.cpu().numpy(), ref.pack(codes))
    want = ref.decode(codes, scales, d)
    assert np.array_equal(kb.table4_decode(t).double().cpu().numpy(), want)        # a number times a bf16 one: exact
    assert np.array_equal(kb.table4_decode(t, dtype=torch.bfloat16).double().cpu().numpy(), ref.bf16(want))
    ids = torch.tensor([n - 1, 0, 0, -1, n, 2 ** 31 - 1, n // 2], dtype=torch.int32, device="cuda")
    got = kb.table4_decode(t, rows=ids).double().cpu().numpy()
    assert np.array_equal(got[[0, 1, 2, 6]], want[[n - 1, 0, 0, n // 2]]) and np.isnan(got[3:6]).all()


def test_borders_between_two_numbers(kb):  # noqa: F811
    """Elements on the borders and next to them on both sides, at scales of all sorts"""
    borders = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], np.float32)
    rows = []
    for s in (1.0, 1.9921875, 2.0 ** -120, 3.0 * 2.0 ** 100, 1.0078125):
        b = borders * np.float32(s)
        rows.append(np.concatenate([[6.0 * s], b, np.nextafter(b, np.float32(0)), np.nextafter(b, np.float32(np.inf)), -b]).astype(np.float32))
    x = np.array(rows)
    codes, scales = ref.encode(x)
    t = kb.table4_encode(gpu(x))
    assert np.array_equal(t.scales.double().cpu().numpy(), scales) and np.array_equal(t.codes.cpu().numpy(), ref.pack(codes))


def test_scales_at_the_ends_of_the_range(kb):  # noqa: F811
    x = np.zeros((12, 32), np.float32)
    x[:, 3] = [3.4028235e38, 1e-45, 2.0 ** -126, 2.0 ** -125, 6 * 2.0 ** -126, np.nextafter(np.float32(6 * 2.0 ** -126), np.float32(1)), 3.0, 1e-40, 5.9999995,
               6.0000005, 6.046875, 6.05]
    x[:, 20] = -x[:, 3] / 3
    codes, scales = ref.encode(x)
    t = kb.table4_encode(gpu(x))
    assert np.array_equal(t.scales.double().cpu().numpy(), scales) and np.array_equal(t.codes.cpu().numpy(), ref.pack(codes))


def test_numbers_up_to_the_largest_stay_finite(kb):  # noqa: F811
    """Past bf16's largest number, 255 2^120, six of the next scale would be infinite"""
    import torch
    most, edge = np.finfo(np.float32).max, np.float32(255 * 2.0 ** 120)
    x = np.zeros((6, 40), np.float32)
    x[:, 3] = [most, -most, edge, np.nextafter(edge, most), np.nextafter(edge, np.float32(0)), most / 2]
    x[:, 35] = x[::-1, 3] / 5
    codes, scales = ref.encode(x)
    t = kb.table4_encode(gpu(x))
    assert np.array_equal(t.scales.double().cpu().numpy(), scales) and np.array_equal(t.codes.cpu().numpy(), ref.pack(codes))
    want = ref.decode(codes, scales, 40)
    got = kb.table4_decode(t).double().cpu().numpy()
    assert np.isfinite(got).all() and np.array_equal(got, want) and abs(got[0, 3]) == float(edge)
    assert np.array_equal(kb.table4_decode(t, dtype=torch.bfloat16).double().cpu().numpy(), ref.bf16(want))


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_groups_that_are_not_finite(kb, bad):  # noqa: F811
    x = rows_of(4, 70, 1)
    x[2, 40] = bad
    t = kb.table4_encode(gpu(x))
    got = kb.table4_decode(t).cpu().numpy()
    clean = x.copy()
    clean[2, 32:64] = 0
    codes, scales = ref.encode(clean)
    want = ref.decode(codes, scales, 70)
    assert np.isnan(got[2, 32:64]).all()
    want[2, 32:64] = got[2, 32:64] = 0
    assert np.array_equal(got.astype(np.float64), want)
    s = kb.table4_scores(t, gpu(x[:2])).cpu().numpy()
    assert np.isnan(s[:, 2]).all() and np.isfinite(np.delete(s, 2, 1)).all()


def test_strided_rows_and_places(kb):  # noqa: F811
    """X and out as columns of wider matrices, at any element; what lies between rows is not written; encoding into a table again"""
    import torch
    n, d = 37, 45
    wide = gpu(rows_of(n, 64, 5))
    for shift in (0, 1, 3):
        X = wide[:, shift:shift + d]
        codes, scales = ref.encode(X.cpu().numpy())
        t = kb.table4_encode(X)
        assert np.array_equal(t.codes.cpu().numpy(), ref.pack(codes))
        for dtype in (torch.float32, torch.bfloat16):
            out = torch.full((n, 60), 7.0, dtype=dtype, device="cuda")
            kb.table4_decode(t, out=out[:, shift:shift + d])
            want = ref.decode(codes, scales, d)
            assert np.array_equal(out[:, shift:shift + d].double().cpu().numpy(), want if dtype == torch.float32 else ref.bf16(want))
            assert bool((out[:, :shift] == 7).all()) and bool((out[:, shift + d:] == 7).all())
        kb.table4_encode(gpu(rows_of(n, d, 6)), table=t)
        assert not np.array_equal(t.codes.cpu().numpy(), ref.pack(codes))
        half = wide.bfloat16()[:, shift:shift + d]
        assert np.array_equal(kb.table4_encode(half).codes.cpu().numpy(), ref.pack(ref.encode(half.double().cpu().numpy())[0]))


def make(kb, n, d, q, kind, rel, seed):  # noqa: F811
    rng = np.random.default_rng(seed)
    E = rows_of(n, d, seed)
    codes, scales = ref.encode(E) if n * d <= 40000 else (None, None)
    t = kb.table4_encode(gpu(E))
    rows = ref.decode(codes, scales, d) if codes is not None else kb.table4_decode(t).double().cpu().numpy()
    X = rows_of(max(q, 5), d, seed + 1, kind)
    M = rng.normal(0, 1, (7, d)).astype(np.float32) if rel else None
    return t, rows, X, M, rng.integers(0, len(X), q).astype(np.int32), rng.integers(0, 7, q).astype(np.int32)


def check(kb, t, rows, X, M, fixed, r, kind):  # noqa: F811
    got = kb.table4_scores(t, gpu(X, kind), fixed=gpu(fixed), M=None if M is None else gpu(M), rel=None if M is None else gpu(r))
    x = X.astype(np.float64)[fixed]
    if M is not None:
        x = x * M.astype(np.float64)[r]
    far = np.abs(got.double().cpu().numpy() - ref.scores(x, rows))
    assert (far <= ref.scores_bound(x, rows, M is not None)).all()
    return got


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rel", [True, False])
@pytest.mark.parametrize("q", [1, 2, 4, 5, 16, 17, 32, 33, 64, 70])
def test_scores_by_questions(kb, q, rel, kind):  # noqa: F811
    for n, d in ((100, 40), (17, 200), (64, 256)):
        say(q, rel, kind, n, d)
        check(kb, *make(kb, n, d, q, kind, rel, q + d), kind)


@pytest.mark.parametrize("n", [1, 15, 16, 17, 63, 65, 1000])
@pytest.mark.parametrize("d", [1, 4, 31, 32, 33, 64, 95, 96, 97, 128, 130, 160, 225, 257, 512])
def test_scores_by_sizes(kb, n, d):  # noqa: F811
    for q, kind, rel in ((1, "f32", True), (3, "bf16", False), (20, "f32", True), (9, "bf16", False), (9, "bf16", True)):
        say(n, d, q, kind, rel)
        check(kb, *make(kb, n, d, q, kind, rel, n + d), kind)


@pytest.mark.parametrize("d", [800, 1024, 1700, 2048, 4000, 4096])
@pytest.mark.parametrize("q", [1, 5, 20, 65])
def test_scores_of_wide_rows(kb, d, q):  # noqa: F811
    for kind, rel in (("f32", True), ("bf16", False)):
        say(d, q, kind, rel)
        check(kb, *make(kb, 50, d, q, kind, rel, d + q), kind)


@pytest.mark.parametrize("n,d,q", [(14541, 200, 1), (14541, 200, 40), (70001, 72, 3), (300007, 32, 7), (40000, 256, 16)])
def test_scores_of_long_tables(kb, n, d, q):  # noqa: F811
    say(n, d, q)
    a = make(kb, n, d, q, "f32", True, n)
    got = check(kb, *a, "f32")
    again = check(kb, *a, "f32")
    import torch
    assert torch.equal(got, again)


def test_questions_without_ids_and_strides(kb):  # noqa: F811
    import torch
    t, rows, X, M, fixed, r = make(kb, 70, 50, 7, "f32", True, 3)
    wide, mwide = torch.full((7, 61), math.nan, device="cuda"), torch.full((7, 53), math.nan, device="cuda")
    wide[:, 3:53], mwide[:, 1:51] = gpu(X), gpu(M)
    out = torch.full((7, 90), 7.0, device="cuda")
    got = kb.table4_scores(t, wide[:, 3:53], M=mwide[:, 1:51], out=out[:, 5:75])
    x = X.astype(np.float64) * M
    assert (np.abs(got.double().cpu().numpy() - x @ rows.T) <= ref.scores_bound(x, rows, True)).all()
    assert bool((out[:, :5] == 7).all()) and bool((out[:, 75:] == 7).all())
    got = kb.table4_scores(t, wide[:, 3:53], fixed=gpu(fixed), M=mwide[:, 1:51])      # question q with M's row q
    x = X.astype(np.float64)[fixed] * M
    assert (np.abs(got.double().cpu().numpy() - x @ rows.T) <= ref.scores_bound(x, rows, True)).all()
    got = kb.table4_scores(t, wide[:, 3:53], M=mwide[:, 1:51], rel=gpu(r))
    x = X.astype(np.float64) * M[r]
    assert (np.abs(got.double().cpu().numpy() - x @ rows.T) <= ref.scores_bound(x, rows, True)).all()


@pytest.mark.parametrize("q", [3, 12, 40])
def test_ids_out_of_range(kb, q):  # noqa: F811
    t, rows, X, M, fixed, r = make(kb, 70, 50, q, "f32", True, 3)
    fixed[0], r[1] = -1, 7
    fixed[2] = len(X)
    got = kb.table4_scores(t, gpu(X), fixed=gpu(fixed), M=gpu(M), rel=gpu(r)).cpu().numpy()
    assert np.isnan(got[:3]).all() and np.isfinite(got[3:]).all()


@pytest.mark.parametrize("q", [2, 10])
def test_questions_of_all_sizes_of_numbers(kb, q):  # noqa: F811
    """A question whose numbers lie far apart keeps what each contributes; the largest number fp32 has, subnormal ones, infinities"""
    E = np.zeros((40, 64), np.float32)
    E[np.arange(40), np.arange(40)] = 6.0
    t = kb.table4_encode(gpu(E))
    X = np.zeros((q, 64), np.float32)
    X[0, :40] = 10.0 ** np.arange(-38, 2)
    X[1, :40] = 3.4028235e38 / 8 * (1 - np.arange(40) * 1e-7)
    got = kb.table4_scores(t, gpu(X)).cpu().numpy().astype(np.float64)
    want = X.astype(np.float64)[:, :40] * 6.0
    # one product of each sum is not zero; of a number below 2^-110 the last part is below the smallest bf16 number
    assert (np.abs(got - want) <= 4 * ref.U * np.abs(want) + 6 * 2.0 ** -133).all()
    X[0, 3], X[1, 5] = math.inf, math.nan
    got = kb.table4_scores(t, gpu(X)).cpu().numpy()
    assert math.isinf(got[0, 3]) and np.isnan(got[1]).all() and np.isnan(got[0, :32][np.arange(32) != 3]).all()


def test_captured_on_another_stream(kb):  # noqa: F811
    import torch
    t, rows, X, M, fixed, r = make(kb, 500, 72, 6, "f32", True, 9)
    X, M, fixed, r = gpu(X), gpu(M), gpu(fixed), gpu(r)
    out, dec = torch.empty((6, 500), device="cuda"), torch.empty((500, 72), device="cuda")
    E = torch.randn(500, 72, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())

    def calls(s=None):
        kb.table4_encode(E, table=t, stream=s)
        kb.table4_decode(t, out=dec, stream=s)
        kb.table4_scores(t, X, fixed=fixed, M=M, rel=r, out=out, stream=s)
    calls(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(3):
        E.copy_(torch.randn(500, 72, device="cuda") * (i + 1))
        fixed.copy_(torch.randint(0, len(X), (6,), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), dec.clone()
        out.zero_(), dec.zero_()
        calls(stream.cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], dec)


def test_offsets_past_32_bits(kb):  # noqa: F811
    """A table whose codes, and scores whose rows, lie more than 2^32 bytes apart"""
    import torch
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    n, d = 9_000_000, 1024
    t = kb.Table4(torch.zeros((n, 512), dtype=torch.uint8, device="cuda"), torch.zeros((n, 32), dtype=torch.bfloat16, device="cuda"), d)
    X = torch.randn(4, d, device="cuda")
    small = kb.table4_encode(X)
    for at in (0, 5_000_000, n - 4):
        t.codes[at:at + 4], t.scales[at:at + 4] = small.codes, small.scales
    want = kb.table4_scores(small, X)
    out = torch.full((4, 1_100_000_000), 7.0, device="cuda")[:, :n]
    kb.table4_scores(t, X, out=out)
    for at in (0, 5_000_000, n - 4):
        assert torch.equal(out[:, at:at + 4], want), at
    assert int((out != 0).sum()) == 3 * int((want != 0).sum())
    ids = torch.tensor([n - 4, n - 3, n - 2, n - 1], dtype=torch.int32, device="cuda")
    assert torch.equal(kb.table4_decode(t, rows=ids), kb.table4_decode(small))
