"""Calls of the answering operators and of gradient clipping that are refused, none of which needs a GPU, and the 64-bit forms that the GPU
tests measure against, checked against other forms of the same definitions."""
import ctypes as C
import itertools
import math
import os

import numpy as np
import pytest

import answer_ref as ref

EINVAL, ENOMEM, ERANGE = -1, -2, -4
P = C.c_void_p(1 << 12)          # an aligned address that is never used: every call below is refused before that
ODD = C.c_void_p((1 << 12) + 1)
N0 = C.c_void_p(0)


@pytest.fixture(scope="module")
def kb():
    from paper_2201_02791_amd import build, binding
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    binding.load()
    return binding


def test_struct_layouts(kb):
    assert C.sizeof(kb._GradTensor) == 2 * 8 + 2 * 8 + 4 + 4 and C.sizeof(kb._Table4) == 8 + 4 + 4 + 2 * 8
    assert C.sizeof(kb._Sampling) == 4 * 4 + 4 * 8


def said(kb, word):
    return word.encode() in kb.load().kge_last_error()


@pytest.mark.parametrize("change,status,word", [
    (dict(n=-1), EINVAL, "negative"), (dict(list=None), EINVAL, "NULL"), (dict(rows=-1), EINVAL, "negative"), (dict(dtype=2), EINVAL, "type"),
    (dict(rows=1 << 20, d=1 << 16), ERANGE, "2^36"), (dict(grad=0), EINVAL, "NULL"), (dict(grad=4098), EINVAL, "aligned"),
    (dict(dtype=1, grad=4097), EINVAL, "aligned"), (dict(most=-1.0), EINVAL, "max_norm"), (dict(most=math.nan), EINVAL, "max_norm"),
    (dict(ws=0), EINVAL, "workspace"), (dict(ws=64), EINVAL, "workspace"), (dict(size=8), ENOMEM, "workspace"), (dict(norm=2), EINVAL, "norm")])
@pytest.mark.parametrize("name", ["kge_grad_norm", "kge_clip_grads"])
def test_grad_norm(kb, name, change, status, word):
    a = dict(n=1, list=1, rows=4, d=4, dtype=0, grad=4096, most=1.0, ws=4096, size=1 << 20, norm=4096)
    a.update(change)
    t = (kb._GradTensor * 1)()
    t[0].grad, t[0].row_mask, t[0].n_rows, t[0].d, t[0].dtype = a["grad"] or None, None, a["rows"], a["d"], a["dtype"]
    rc = getattr(kb.load(), name)(t if a["list"] else None, a["n"], a["most"], a["norm"], 4096, a["ws"] or None, a["size"], None)
    assert rc == status and said(kb, word)


def test_grad_norm_places(kb):
    t = (kb._GradTensor * 1)()
    assert kb.load().kge_grad_norm(t, 1, 1.0, None, None, 4096, 1 << 20, None) == EINVAL and said(kb, "one of them")
    assert kb.load().kge_grad_norm_workspace_bytes(-1) == 0
    assert kb.grad_norm_workspace_bytes(1) <= kb.grad_norm_workspace_bytes(1000)


def test_adamw_factor(kb):
    assert kb.load().kge_adamw_step_scaled(C.byref(kb._AdamW(0.1, 0.9, 0.99, 1e-8, 1, None)), None, 0, None, None) == EINVAL and said(kb, "factor")
    assert kb.load().kge_adamw_step_scaled(C.byref(kb._AdamW(0.1, 0.9, 0.99, 1e-8, 1, None)), None, 0, ODD, None) == EINVAL
    assert kb.load().kge_adamw_step_scaled(C.byref(kb._AdamW(0.1, 1.0, 0.99, 1e-8, 1, None)), None, 0, P, None) == EINVAL and said(kb, "beta1")


TABLES = [(dict(d=0), EINVAL, "4096"), (dict(d=4097), EINVAL, "4096"), (dict(n=-1), EINVAL, "negative"), (dict(n=1 << 31), ERANGE, "2^31"),
          (dict(codes=None), EINVAL, "NULL"), (dict(scales=None), EINVAL, "NULL"), (dict(codes=4104), EINVAL, "aligned"), (dict(scales=4097), EINVAL, "aligned")]


def table(kb, a):
    return kb._Table4(a["n"], a["d"], a["codes"], a["scales"])


@pytest.mark.parametrize("change,status,word", TABLES + [
    (dict(X=0), EINVAL, "NULL"), (dict(X=4098), EINVAL, "aligned"), (dict(ldx=39), EINVAL, "stride"), (dict(dtype=2), EINVAL, "type")])
def test_table4_encode(kb, change, status, word):
    a = dict(n=10, d=40, codes=4096, scales=4096, X=4096, ldx=40, dtype=0)
    a.update(change)
    assert kb.load().kge_table4_encode(C.byref(table(kb, a)), a["dtype"], a["X"] or None, max(a["ldx"], a["d"]) if "d" in change else a["ldx"], None) == status
    assert said(kb, word)


@pytest.mark.parametrize("change,status,word", TABLES + [
    (dict(m=-1), EINVAL, "negative"), (dict(m=11), EINVAL, "more rows"), (dict(out=0), EINVAL, "NULL"), (dict(ldo=39), EINVAL, "stride"),
    (dict(dtype=7), EINVAL, "type")])
def test_table4_decode(kb, change, status, word):
    a = dict(n=10, d=40, codes=4096, scales=4096, out=4096, ldo=40, dtype=0, m=10)
    a.update(change)
    rc = kb.load().kge_table4_decode(C.byref(table(kb, a)), None, a["m"], a["dtype"], a["out"] or None, max(a["ldo"], a["d"]) if "d" in change else a["ldo"], None)
    assert rc == status and said(kb, word)


@pytest.mark.parametrize("change,status,word", TABLES + [
    (dict(X=None), EINVAL, "NULL"), (dict(ldx=39), EINVAL, "stride"), (dict(dtype=3), EINVAL, "type"), (dict(q=-1), EINVAL, "negative"),
    (dict(q=1 << 31), ERANGE, "2^31"), (dict(fixed=None, n_x=2), EINVAL, "fixed"), (dict(M=None), EINVAL, "rel"), (dict(rel=None, n_m=2), EINVAL, "rel"),
    (dict(ldm=39), EINVAL, "stride"), (dict(lds=9), EINVAL, "stride"), (dict(out=None), EINVAL, "scores"), (dict(out=4098), EINVAL, "scores"),
    (dict(fixed=4098), EINVAL, "aligned")])
def test_table4_scores(kb, change, status, word):
    a = dict(n=10, d=40, codes=4096, scales=4096, X=4096, ldx=40, n_x=5, dtype=0, fixed=4096, M=4096, ldm=40, n_m=5, rel=4096, q=3, out=4096, lds=10)
    a.update(change)
    if "d" in change or "n" in change:
        a["ldx"] = a["ldm"] = max(a["d"], 40)
    rc = kb.load().kge_table4_scores(C.byref(table(kb, a)), a["dtype"], a["X"], a["ldx"], a["n_x"], a["fixed"], a["M"], a["ldm"], a["n_m"], a["rel"], a["q"],
                                     a["out"], a["lds"], None)
    assert rc == status and said(kb, word)


@pytest.mark.parametrize("change,status,word", [
    (dict(rows=-1), EINVAL, "negative"), (dict(cols=-1), EINVAL, "negative"), (dict(rows=1 << 31), ERANGE, "2^31"), (dict(cols=1 << 31, lds=1 << 31), ERANGE, "2^31"),
    (dict(t=-1.0), EINVAL, "temperature"), (dict(t=math.nan), EINVAL, "temperature"), (dict(t=math.inf), EINVAL, "temperature"), (dict(k=-1), EINVAL, "top_k"),
    (dict(p=0.0), EINVAL, "top_p"), (dict(p=1.5), EINVAL, "top_p"), (dict(p=math.nan), EINVAL, "top_p"), (dict(m=-0.1), EINVAL, "min_p"), (dict(m=1.1), EINVAL, "min_p"),
    (dict(dtype=2), EINVAL, "type"), (dict(ub=16), EINVAL, "bits"), (dict(draws=-1), EINVAL, "draws"), (dict(lds=9), EINVAL, "stride"), (dict(s=None), EINVAL, "NULL"),
    (dict(u=None), EINVAL, "NULL"), (dict(choice=None), EINVAL, "NULL"), (dict(s=4098), EINVAL, "aligned"), (dict(u=4100, ub=64), EINVAL, "aligned"),
    (dict(ws=None, cols=65537, lds=65537), EINVAL, "workspace"), (dict(ws=64, cols=65537, lds=65537), EINVAL, "workspace"),
    (dict(size=0, cols=65537, lds=65537), ENOMEM, "workspace"), (dict(row_k=4098), EINVAL, "settings")])
def test_sample_scores(kb, change, status, word):
    a = dict(rows=3, cols=10, t=1.0, k=5, p=0.9, m=0.1, dtype=0, ub=32, draws=2, lds=10, s=4096, u=4096, choice=4096, ws=4096, size=1 << 30, row_k=None)
    a.update(change)
    how = kb._Sampling(a["t"], a["k"], a["p"], a["m"], None, a["row_k"], None, None)
    rc = kb.load().kge_sample_scores(C.byref(how), a["rows"], a["cols"], a["s"], a["dtype"], a["lds"], a["u"], a["ub"], a["draws"], a["choice"], None, a["ws"],
                                     a["size"], None)
    assert rc == status and said(kb, word)
    if set(change) & {"rows", "t", "k", "p", "m", "row_k"} or a["cols"] < 0 or a["cols"] >= 1 << 31:
        assert kb.load().kge_sample_workspace_bytes(C.byref(how), a["rows"], a["cols"]) == 0


def test_sample_settings_of_rows_replace_the_calls(kb):
    how = kb._Sampling(math.nan, 0, 9.0, -1.0, 4096, None, 4096, 4096)      # what rows have of their own is not looked at on the host
    assert kb.load().kge_sample_workspace_bytes(C.byref(how), 3, 10) > 0


def test_pick_negatives(kb):
    call = kb.load().kge_pick_negatives
    assert call(4096, 4096, -1, 4096, 3, 2, 4096, 4096, None) == EINVAL
    assert call(4096, 4096, 0, 4096, 3, 2, 4096, 4096, None) == EINVAL and said(kb, "candidates")
    assert call(None, 4096, 4, 4096, 3, 2, 4096, 4096, None) == EINVAL and call(4096, 4096, 4, 4096, 3, 2, 4096, None, None) == EINVAL
    assert call(4096, 4096, 4, 4096, 1 << 31, 2, 4096, 4096, None) == ERANGE
    assert call(None, None, 0, None, 0, 2, None, None, None) == 0 and call(None, None, 0, None, 3, 0, None, None, None) == 0


def test_hide_positives(kb):
    call = kb.load().kge_hide_positives
    assert call(None, 4096, 3, 4096, 4096, 4, 4096, 4, None) == EINVAL and said(kb, "partition")
    assert call(4096, 4096, -1, 4096, 4096, 4, 4096, 4, None) == EINVAL and call(4096, 4096, 3, 4096, 4096, 4, 4096, 3, None) == EINVAL
    assert call(4096, 4096, 1 << 31, 4096, 4096, 4, 4096, 4, None) == ERANGE
    assert call(4096, 4096, 3, 4096, None, 4, 4096, 4, None) == EINVAL and said(kb, "NULL array")
    assert call(4096, None, 0, None, None, 4, None, 4, None) == 0


def test_nothing_to_do_is_no_error(kb):
    lib = kb.load()
    t = kb._Table4(0, 40, None, None)
    assert lib.kge_table4_encode(C.byref(t), 0, None, 40, None) == 0 and lib.kge_table4_decode(C.byref(t), None, 0, 0, None, 40, None) == 0
    assert lib.kge_table4_scores(C.byref(t), 0, 4096, 40, 3, None, None, 0, 0, None, 3, None, 0, None) == 0
    full = kb._Table4(10, 40, 4096, 4096)
    assert lib.kge_table4_scores(C.byref(full), 0, None, 40, 0, None, None, 0, 0, None, 0, None, 10, None) == 0
    how = kb._Sampling(1.0, 0, 1.0, 0.0, None, None, None, None)
    assert lib.kge_sample_scores(C.byref(how), 0, 10, None, 0, 10, None, 32, 4, None, None, None, 0, None) == 0
    assert lib.kge_sample_scores(C.byref(how), 5, 10, None, 0, 10, None, 32, 0, None, None, None, 0, None) == 0


def test_python_checks(kb):
    import torch
    f = lambda *s: torch.zeros(*s)  # noqa: E731
    t = kb.Table4(torch.zeros(5, 32, dtype=torch.uint8), torch.zeros(5, 2, dtype=torch.bfloat16), 40)
    bad = [lambda: kb.Table4(torch.zeros(5, 31, dtype=torch.uint8), torch.zeros(5, 2, dtype=torch.bfloat16), 40),
           lambda: kb.Table4(torch.zeros(5, 32, dtype=torch.uint8), torch.zeros(5, 2), 40),
           lambda: kb.Table4(torch.zeros(5, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.bfloat16), 40),
           lambda: kb.table4_encode(f(5, 41), table=t), lambda: kb.table4_encode(f(4, 40), table=t), lambda: kb.table4_encode(f(5, 40).half()),
           lambda: kb.table4_encode(f(40)), lambda: kb.table4_decode(t, rows=f(3)), lambda: kb.table4_decode(t, out=f(5, 41)),
           lambda: kb.table4_scores(t, f(3, 41)), lambda: kb.table4_scores(t, f(3, 40), M=f(3, 39)), lambda: kb.table4_scores(t, f(3, 40), M=f(3, 40).bfloat16()),
           lambda: kb.table4_scores(t, f(3, 40), fixed=torch.zeros(2, dtype=torch.int32), M=f(3, 40), rel=torch.zeros(3, dtype=torch.int32)),
           lambda: kb.table4_scores(t, f(3, 40), fixed=torch.zeros(2, dtype=torch.int64)), lambda: kb.table4_scores(t, f(3, 40), out=f(3, 4)),
           lambda: kb.sample_scores(f(3, 9), f(2, 4)), lambda: kb.sample_scores(f(3, 9), f(3, 4).half()), lambda: kb.sample_scores(f(9, 3).T, f(3, 4)),
           lambda: kb.sample_scores(f(3, 9), f(3, 4), top_k=f(3)), lambda: kb.sample_scores(f(3, 9), f(3, 4), temperature=f(4)),
           lambda: kb.sample_scores(f(3, 9), f(3, 4), choice=f(3, 4)), lambda: kb.sample_scores(f(3, 9), f(3, 4), temperature=-1.0),
           lambda: kb.GradTensors([f(4, 6).T]), lambda: kb.GradTensors([f(4).half()]), lambda: kb.GradTensors([dict(grad=f(4, 6), row_mask=f(4))]),
           lambda: kb.GradTensors([dict(grad=f(4, 6), row_mask=torch.ones(6, dtype=torch.uint8))]), lambda: kb.grad_norm([]),
           lambda: kb.grad_norm([f(3)], norm=f(2)),
           lambda: kb.adamw_step([], factor=torch.zeros(2)), lambda: kb.adamw_step([], factor=torch.zeros(1, dtype=torch.float64)),
           # no call runs on the CPU
           lambda: kb.table4_encode(f(5, 40)), lambda: kb.table4_decode(t), lambda: kb.table4_scores(t, f(3, 40)), lambda: kb.sample_scores(f(3, 9), f(3, 4)),
           lambda: kb.grad_norm([f(3)]), lambda: kb.clip_grads([f(3)], 1.0)]
    for i, call in enumerate(bad):
        with pytest.raises(kb.KgeError) as e:
            call()
        assert e.value.status == EINVAL, i


def test_overlapping_gradients_are_refused(kb):
    import torch
    x = torch.zeros(100)
    kb.GradTensors([x[:50], x[50:]])
    kb.GradTensors([x[:0], x, x[100:]])
    for pair in ([x, x], [x[:51], x[50:]], [x, x[20:30]], [x[20:30], torch.zeros(3), x]):
        with pytest.raises(kb.KgeError, match="overlap"):
            kb.GradTensors(pair)


# ---- the 64-bit forms

def test_codes_are_the_nearest():
    rng = np.random.default_rng(0)
    X = rng.normal(0, 1, (40, 70)) * 10.0 ** rng.integers(-6, 6, (40, 1))
    X = X.astype(np.float32).astype(np.float64)
    codes, scales = ref.encode(X)
    Y = ref.decode(codes, scales, 70)
    s = np.repeat(scales, 32, 1)[:, :70]
    nearest = np.min(np.abs(np.abs(X)[:, :, None] - s[:, :, None] * ref.LEVELS), 2)
    assert np.array_equal(np.abs(X - Y), np.abs(np.abs(X) - np.abs(Y))) and np.allclose(np.abs(X - Y), nearest, rtol=1e-12, atol=0)
    assert (np.abs(X) <= 6 * s).all()
    most = np.abs(np.pad(X, ((0, 0), (0, 26)))).reshape(40, 3, 32).max(2)
    assert np.array_equal(ref.bf16(scales), scales) and (scales <= most / 6 * (1 + 2.0 ** -7)).all()
    assert np.array_equal(ref.unpack(ref.pack(codes)), codes)


def test_ties_go_to_the_even_code():
    x = np.array([[6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -5.0]])
    codes, scales = ref.encode(x)
    assert scales[0, 0] == 1.0 and codes[0, 0, :11].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 8, 10, 14]


def brute_force(s, u, t, k, p, m):
    """The same definition over sorted lists of Python numbers"""
    n = len(s)
    bits = ref.bits_of(n)
    most = max((x for x in s if x == x), default=-math.inf)
    w = [0 if x != x or x == -math.inf else 1 << bits if x == most else round(math.exp((x - most) / t) * 2.0 ** bits) for x in s]
    by_score = sorted(range(n), key=lambda i: (-(s[i] if s[i] == s[i] else -math.inf), i))
    left = by_score[:k] if k else by_score
    if p < 1.0:
        goal, sums, short = max(1, math.ceil(p * sum(w[i] for i in left))), 0, []
        for i in left:
            if sums >= goal:
                break
            short.append(i)
            sums += w[i]
        left = short
    left = sorted(i for i in left if w[i] >= m * 2.0 ** bits)
    total = sum(w[i] for i in left)
    out = []
    for x in u:
        goal, sums, got = min(int(x * float(total)), total - 1), 0, -1
        for i in left:
            sums += w[i]
            if sums > goal and total:
                got = i
                break
        out.append(got)
    return out


@pytest.mark.parametrize("t,k,p,m", list(itertools.product([0.5, 2.0], [0, 1, 3, 50], [1.0, 0.3, 0.9], [0.0, 0.2])))
def test_draws_against_lists(t, k, p, m):
    rng = np.random.default_rng(k)
    for n in (1, 2, 7, 40):
        s = np.round(rng.normal(0, 2, n), 1).astype(np.float32).astype(np.float64)
        s[rng.random(n) < 0.2] = -np.inf
        u = rng.random(30)
        f = lambda v: float(np.float32(v))  # noqa: E731
        cols, share = ref.sample_row(s, u, f(t), k, f(p), f(m))
        assert cols.tolist() == brute_force(s.tolist(), u.tolist(), f(t), k, f(p), f(m))
        if cols[0] >= 0:
            assert (share > 0).all()


def test_draws_follow_the_shares():
    """Many draws of a row come out in the shares of its softmax: within five standard deviations for every column"""
    s = np.array([0.0, 1.0, 2.0, 0.5, -1.0])
    u = (np.arange(20000) + 0.5) / 20000.0
    cols, _ = ref.sample_row(s, u)
    share = np.exp(s) / np.exp(s).sum()
    assert np.abs(np.bincount(cols, minlength=5) / 20000.0 - share).max() <= 1.0 / 20000.0 + 1e-9     # u is even: off by one at most


def test_factor():
    assert ref.factor(2.0, 1.0) == 0.5 and ref.factor(0.5, 1.0) == 1.0 and ref.factor(0.0, 0.0) == 1.0 and math.isnan(ref.factor(math.inf, 1.0))
