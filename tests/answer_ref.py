"""Plain 64-bit forms (NumPy) of the answering operators: tables of 4 bits, their scores, draws from scores, gradient norms.

Bounds count roundings: U = 2^-24 is half a step of fp32 relative to the number, H = 2^-8 that of bf16."""
import math

import numpy as np

U = 2.0 ** -24
H = 2.0 ** -8
GROUP = 32
LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def bf16(x):
    """float64 numbers of X rounded to bf16 (nearest even), as float64"""
    b = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    b = (b + 0x7FFF + ((b >> 16) & 1)) >> 16 << 16
    return b.astype(np.uint32).view(np.float32).astype(np.float64)


# ---- tables

def smallest_scale(most):
    """The smallest number of 8 significant bits, 2^-126 or more, six of which reach `most`: by trying them all in an octave; but six of which
    are a float"""
    if most == 0.0:
        return 0.0
    if not math.isfinite(most):
        return math.nan
    e = max(math.frexp(most / 6.0)[1] - 2, -126)
    while True:
        for m in range(128, 256):
            s = math.ldexp(m, e - 7)
            if 6.0 * s >= most:
                return s if 6.0 * s <= float(np.finfo(np.float32).max) else 170 * 2.0 ** 118
        e += 1


def encode(X):
    """(codes uint8 [n][groups][32], scales float64 [n][groups])"""
    X = np.asarray(X, np.float64)
    n, d = X.shape
    groups = -(-d // GROUP)
    x = np.zeros((n, groups * GROUP))
    x[:, :d] = X
    x = x.reshape(n, groups, GROUP)
    codes = np.zeros(x.shape, np.uint8)
    scales = np.zeros((n, groups))
    for i in range(n):
        for g in range(groups):
            a = np.abs(x[i, g])
            s = scales[i, g] = smallest_scale(math.nan if not np.isfinite(a).all() else a.max())
            if not s > 0.0:
                continue
            far = np.abs(a[:, None] / s - LEVELS[None, :])       # a and s are short enough for ties to be met exactly
            best = far.min(1)
            for k in range(GROUP):
                near = np.nonzero(far[k] == best[k])[0]
                codes[i, g, k] = near[0] if len(near) == 1 else near[near % 2 == 0][0]
            codes[i, g] += np.where(x[i, g] < 0, 8, 0).astype(np.uint8)
    return codes, scales


def pack(codes):
    n = len(codes)
    c = codes.reshape(n, -1, 2)
    return (c[:, :, 0] | c[:, :, 1] << 4).astype(np.uint8)


def unpack(packed):
    return np.stack([packed & 15, packed >> 4], 2).reshape(len(packed), -1, GROUP)


def decode(codes, scales, d):
    signed = np.concatenate([LEVELS, -LEVELS])
    return (signed[codes] * scales[:, :, None]).reshape(len(codes), -1)[:, :d]


def scores(q, rows):
    return q @ rows.T


def scores_bound(q, rows, product):
    """Products are exact.  A term passes through at most 3 x 32 additions of a group's sum (three parts), one product with the scale and an
    addition for each group, and three parts' sums may be added at the end; the rounding inside the matrix instruction may be by a whole step.
    With a relation the question itself is a rounded product."""
    groups = -(-q.shape[1] // GROUP)
    return (2.0 * (3 * GROUP + groups + 4) + (1.0 if product else 0.0)) * U * (np.abs(q) @ np.abs(rows).T)


# ---- draws

def bits_of(n):
    return min(40, 62 - max(n - 1, 0).bit_length())


def weights(s, temperature, bits):
    """Whole weights (Python ints in an object array would be slow: uint64) of a row of float64 scores"""
    s = np.where(np.isnan(s), -np.inf, s)
    most = s.max() if len(s) else -np.inf
    if most == -np.inf:
        return np.zeros(len(s), np.uint64)
    with np.errstate(invalid="ignore", over="ignore", under="ignore"):
        w = np.exp((s - most) / temperature)
    w[s == -np.inf] = 0.0
    w[s == most] = 1.0
    return np.rint(w * 2.0 ** bits).astype(np.uint64)


def sample_row(s, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, most_k=0):
    """(columns, shares) of one row's draws; settings as the library takes them from the device, out of range ones too"""
    s = np.asarray(s, np.float64)
    n, bits = len(s), bits_of(len(s))
    k = top_k if top_k > 0 else 0
    if most_k > 0:
        k = min(k, most_k) if k > 0 else most_k
    if not temperature > 0.0:
        temperature, k = 1.0, 1
    w = weights(s, temperature, bits)
    order = np.argsort(-np.where(np.isnan(s), -np.inf, s), kind="stable")
    v = w[order].copy()
    if 0 < k < n:
        v[k:] = 0
    if top_p < 1.0:
        total = int(v.sum(dtype=np.uint64))
        goal = min(math.ceil(max(1.0, float(top_p) * float(total))), total)
        before = np.cumsum(v, dtype=np.uint64) - v
        v[before >= np.uint64(goal)] = 0
    low = min(float(min_p), 1.0) if min_p > 0.0 else 0.0
    v[v.astype(np.float64) < low * 2.0 ** bits] = 0
    left = np.zeros(n, np.uint64)
    left[order] = v
    sums = np.cumsum(left, dtype=np.uint64)
    total = int(sums[-1]) if n else 0
    if total == 0:
        return np.full(len(u), -1), np.zeros(len(u))
    cols, share = [], []
    for x in u:
        x = float(x)
        reach = 0.0 if math.isnan(x) else x * float(total)
        goal = total - 1 if reach >= float(total) else min(int(reach), total - 1) if reach > 0.0 else 0
        c = int(np.searchsorted(sums, np.uint64(goal), side="right"))
        cols.append(c)
        share.append(float(left[c]) / float(total))
    return np.array(cols), np.array(share)


def sample(S, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, most_k=0):
    at = lambda v, r: v if np.isscalar(v) else v[r]  # noqa: E731
    f = lambda v: float(np.float32(v))  # noqa: E731
    rows = [sample_row(S[r], u[r], f(at(temperature, r)), int(at(top_k, r)), f(at(top_p, r)), f(at(min_p, r)), most_k) for r in range(len(S))]
    return np.array([c for c, _ in rows], np.int64).reshape(u.shape), np.array([p for _, p in rows]).reshape(u.shape)


# ---- gradients

def norm(grads):
    return math.sqrt(sum(float(np.square(np.asarray(g, np.float64)).sum()) for g in grads))


def factor(total, most):
    return math.nan if not math.isfinite(total) else 1.0 if total <= most or total == 0.0 else most / total
