"""Plain 64-bit forms (NumPy) of the vertex-feature block's operators, and how far a result of fp32 sums may be from them.

Bounds count roundings: U = 2^-24 is half a step of fp32 relative to the number, H = 2^-8 that of bf16."""
import numpy as np

U = 2.0 ** -24
H = 2.0 ** -8
HALF = {"f32": U, "bf16": H}

IDENTITY, RELU, SILU = 0, 1, 2


def sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def act(z, a):
    return np.maximum(z, 0.0) if a == RELU else z * sigmoid(z) if a == SILU else z


def act_grad(z, a):
    if a == RELU:
        return (z > 0).astype(np.float64)
    if a == SILU:
        s = sigmoid(z)
        return s * (1.0 + z * (1.0 - s))
    return np.ones_like(z)


def dense_forward(X, W, b, a, R=None):
    pre = X @ W + (0.0 if b is None else b)
    return act(pre, a) + (0.0 if R is None else R), pre


def dense_backward(X, W, pre, dY, a, add=None):
    dP = dY * act_grad(pre, a) if a != IDENTITY else dY
    return dP @ W.T + (0.0 if add is None else add), X.T @ dP, dP.sum(0)


def sum_bound(terms, absolute):
    """A sum of `terms` products in fp32: no term passes through more than terms + 8 additions, and the products that a
    three-way split leaves out are below 2^-24 of theirs; `absolute`: the sum of the products' magnitudes.  Twice that, since
    the rounding inside the matrix instruction may be by a whole step."""
    return 2.0 * (terms + 8) * U * absolute


def dense_forward_bound(X, W, b, a, R, kind):
    """(bound of Y, bound of pre), elementwise"""
    Y, pre = dense_forward(X, W, b, a, R)
    e = sum_bound(X.shape[1], np.abs(X) @ np.abs(W) + (0.0 if b is None else np.abs(b)))
    # |act'| <= 1.1; the exponential's argument and value are rounded a few times, relative (1 + |z|) U each
    soft = 8.0 * U * (1.0 + np.abs(pre)) * np.abs(act(pre, a)) if a == SILU else 0.0
    y = 1.1 * e + soft + 2.0 * U * (np.abs(Y) + (0.0 if R is None else np.abs(R)))
    h = HALF[kind]
    return y + h * (np.abs(Y) + y), e + h * (np.abs(pre) + e)


def dense_backward_bound(X, W, pre, dY, a, add, kind):
    g = act_grad(pre, a) if a != IDENTITY else np.ones_like(dY)
    dP = dY * g
    # act' itself, absolute: a few roundings of numbers up to 1 + |z|
    p = np.abs(dY) * (8.0 * U * (1.0 + np.abs(pre)) if a == SILU else 0.0) + 2.0 * U * np.abs(dP)
    dX, dW, db = dense_backward(X, W, pre, dY, a, add)
    x = sum_bound(W.shape[1], np.abs(dP) @ np.abs(W).T) + p @ np.abs(W).T + U * np.abs(dX)
    if kind == "bf16" and a == SILU:                 # two parts of dP
        x = x + 2.0 ** -17 * (np.abs(dP) @ np.abs(W).T)
    w = sum_bound(len(X), np.abs(X).T @ np.abs(dP)) + np.abs(X).T @ p
    c = sum_bound(len(X), np.abs(dP).sum(0)) + p.sum(0)
    return x + HALF[kind] * (np.abs(dX) + x), w, c


def norm_forward(X, gamma, beta, eps):
    mean = X.mean(1)
    rstd = 1.0 / np.sqrt(((X - mean[:, None]) ** 2).mean(1) + eps)
    return (X - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def norm_forward_bound(X, gamma, beta, eps, kind):
    """(Y, mean, rstd): a mean of d numbers is off by at most (d + 2) U of their mean magnitude; the deviations inherit that; the
    mean of their squares is off by (d + 4) U of itself and by the deviations' errors"""
    d = X.shape[1]
    Y, mean, rstd = norm_forward(X, gamma, beta, eps)
    em = (d + 2) * U * np.abs(X).mean(1)
    dev = np.abs(X - mean[:, None])
    ed = em[:, None] + U * (np.abs(X) + np.abs(mean)[:, None])
    ev = (d + 4) * U / rstd ** 2 + (2.0 * dev * ed + ed ** 2).mean(1)
    er = rstd * (0.5 * ev * rstd ** 2 * 1.1 + 4.0 * U)
    r = rstd[:, None]
    y = np.abs(gamma) * (ed * r + dev * er[:, None]) * 1.1 + 4.0 * U * (np.abs(Y) + np.abs(beta))
    return y + HALF[kind] * (np.abs(Y) + y), em, er


def norm_backward(X, gamma, mean, rstd, dY):
    xh = (X - mean[:, None]) * rstd[:, None]
    u = dY * gamma
    dX = rstd[:, None] * (u - u.mean(1, keepdims=True) - xh * (u * xh).mean(1, keepdims=True))
    return dX, (dY * xh).sum(0), dY.sum(0)


def norm_backward_bound(X, gamma, mean, rstd, dY, kind):
    n, d = X.shape
    r = rstd[:, None]
    xh = (X - mean[:, None]) * r
    ex = 2.0 * U * (np.abs(X) + np.abs(mean)[:, None]) * r + U * np.abs(xh)
    u = np.abs(dY * gamma)
    dX, dg, db = norm_backward(X, gamma, mean, rstd, dY)
    mu = u.mean(1, keepdims=True)
    mx = (u * np.abs(xh)).mean(1, keepdims=True)
    emx = (d + 4) * U * mx + (u * ex).mean(1, keepdims=True)
    e = r * (4.0 * U * u + (d + 4) * U * mu + ex * mx + np.abs(xh) * emx + 4.0 * U * (mu + np.abs(xh) * mx)) * 1.1
    eg = (n + 4) * U * (np.abs(dY * xh)).sum(0) + (np.abs(dY) * ex).sum(0)
    return e + HALF[kind] * (np.abs(dX) + e), eg, (n + 4) * U * np.abs(dY).sum(0)


# ---- AdamW with moments in 32 or in 8 bits --------------------------------------------------------

BLOCK = 256
E4M3 = dict(digits=3, least=-6, top=8, half=0)
E5M2 = dict(digits=2, least=-14, top=15, half=1)
f32 = np.float32


def moments(m, v, g, beta1, beta2):
    """New moments, every operation rounded to fp32 once, in the order of the definition."""
    b1, b2 = f32(beta1), f32(beta2)
    o1, o2 = f32(1.0 - float(b1)), f32(1.0 - float(b2))
    return b1 * m + o1 * g, b2 * v + (o2 * g) * g


def scales(a, form):
    """One power of two a block of BLOCK elements of a row (fp32 magnitudes a [n][d])."""
    n, d = a.shape
    pad = np.zeros((n, -(-d // BLOCK) * BLOCK), f32)
    pad[:, :d] = a
    most = pad.reshape(n, -1, BLOCK).max(2)
    f, e = np.frexp(most.astype(np.float64))
    k = np.maximum(e - 1 - form["top"] + (f > 0.875), -126)
    return np.where(most > 0, np.ldexp(1.0, k), 0.0).astype(f32)


def encode(x, form, t):
    """(numbers of the format with x's signs as float64, scales) that fp32 moments x [n][d] are held as at step t."""
    n, d = x.shape
    a = np.abs(x).astype(f32)
    s = scales(a, form)
    spread = np.repeat(s, BLOCK, 1)[:, :d].astype(np.float64)
    y = np.where(spread > 0, a.astype(np.float64) / np.where(spread > 0, spread, 1.0), 0.0)
    i = np.arange(n * d, dtype=np.uint64).reshape(n, d)
    w = np.uint64(0xFFFFFFFF)
    h = (i * np.uint64(0xC2B2AE35) + np.uint64((t * 0x9E3779B9) & 0xFFFFFFFF)) & w
    h = ((h ^ (h >> np.uint64(16))) * np.uint64(0x2C1B3C6D)) & w
    u = ((h >> np.uint64(16)) if form["half"] else (h & np.uint64(0xFFFF))).astype(f32) / f32(65536.0)
    e = np.maximum(np.frexp(y)[1] - 1, form["least"]) - form["digits"]
    q = np.ldexp(np.floor((np.ldexp(y, -e).astype(f32) + u).astype(np.float64)), e)      # the one addition is fp32's
    if form is E5M2:
        q = np.where(x > 0, np.maximum(q, 2.0 ** -16), q)
    return np.copysign(q, x), s


def adamw(p, m, v, g, t, lr, beta1, beta2, eps, wd):
    """(p, m, v) after a step, 64 bits; hyper-parameters as the fp32 numbers that the library takes"""
    lr, b1, b2, eps, wd = (float(f32(x)) for x in (lr, beta1, beta2, eps, wd))
    p, m, v, g = (np.asarray(x, np.float64) for x in (p, m, v, g))
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    return p - lr * (wd * p + (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + eps)), m, v
