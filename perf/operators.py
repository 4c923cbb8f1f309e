"""The operators of the vertex-feature block and of its update: inputs, one pass, its work and its exact result.

  dense   Y = act(X W + b) + R on the rows of a feature matrix, and its backward pass
  norm    layer norm of rows, and its backward pass with the gradients of gamma and beta
  adamw   one AdamW step over all tensors of a model, moments in 32 or in 8 bits

Sizes are those of the workloads of `paper_2201_02791_amd/synth.py` (the tiny graph, the 14,541-entity knowledge graph,
the citation-shaped graph with its 128 features a vertex, the large many-relation graph of a million entities and width
256) and of ranges around them.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)
BLOCK = 256                                                   # elements that share a scale of an 8-bit moment


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # features of one vertex that joins the graph after training
        dict(name="dense-one-row", kind="dense", back=False, dtype="bf16", n=1, d_in=1024, d_out=1024, act="silu", res=False, keep=False),
        # the citation graph's 128 features a vertex, all 2.9 M vertices: a residual block in fp32, training
        dict(name="dense-citation", kind="dense", back=False, dtype="f32", n=2900000, d_in=128, d_out=128, act="relu", res=True, keep=True),
        # a million entities at the large graph's width, bf16, training
        dict(name="dense-bigkg-bf16", kind="dense", back=False, dtype="bf16", n=1000000, d_in=256, d_out=256, act="silu", res=False, keep=True),
        # the mid-size graph with features of a width that is no multiple of anything, to a hidden layer
        dict(name="dense-ragged", kind="dense", back=False, dtype="f32", n=14541, d_in=203, d_out=517, act="silu", res=False, keep=True),
        # the paper's large-graph widths (fixed features, 128 to 32) on a tenth of the citation graph: weights' gradients only
        dict(name="dense-back-features", kind="dense", back=True, dtype="f32", n=290001, d_in=128, d_out=32, act="relu", res=False, need_dx=False),
        # backward pass of the million-row layer, with the gradient that reaches X past the layer
        dict(name="dense-back-bigkg-bf16", kind="dense", back=True, dtype="bf16", n=1000000, d_in=256, d_out=256, act="silu", res=True, need_dx=True),
        # backward pass of the ragged layer
        dict(name="dense-back-ragged", kind="dense", back=True, dtype="f32", n=14541, d_in=517, d_out=203, act="silu", res=False, need_dx=True),
        # rows of the citation graph's hidden layer on their way into the encoder, training
        dict(name="norm-citation", kind="norm", back=False, dtype="f32", out="f32", n=2900000, d=128),
        # backward pass of the million-row norm: bf16 rows, fp32 gradients from the encoder
        dict(name="norm-back-bigkg-bf16", kind="norm", back=True, dtype="bf16", out="f32", n=1000000, d=256),
        # the tiny graph's model: every tensor takes microseconds
        dict(name="adamw-tiny", kind="adamw", bits=32, n_ent=1000, n_rel=10, d=32, bases=4, rows="mask", read=0.8, copy=False),
        # the large graph's model (64 bases, 1000 relations, a million entities of which a batch reads most)
        dict(name="adamw-bigkg", kind="adamw", bits=32, n_ent=1000000, n_rel=1000, d=256, bases=64, rows="mask", read=0.9, copy=False),
        # the same with moments in 8 bits and bf16 copies of the weights
        dict(name="adamw-bigkg-8bit", kind="adamw", bits=8, n_ent=1000000, n_rel=1000, d=256, bases=64, rows="mask", read=0.9, copy=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["dense", "dense", "dense", "dense", "norm", "norm", "adamw", "adamw"])
    if kind == "dense":
        d_in, d_out = _log(rng, 8, 1024), _log(rng, 8, 1024)
        if rng.random() < 0.5:                                # half of the widths are multiples of 32
            d_in, d_out = -(-d_in // 32) * 32, -(-d_out // 32) * 32
        n = min(_log(rng, 1, 1000000), 60000000000 // (d_in * d_out), 400000000 // (d_in + d_out))
        c = dict(kind=kind, back=rng.random() < 0.5, dtype=rng.choice(["f32", "bf16"]), n=n, d_in=d_in, d_out=d_out,
                 act=rng.choice(["identity", "relu", "silu"]), res=rng.random() < 0.4)
        c["need_dx" if c["back"] else "keep"] = rng.random() < 0.7
        return c
    if kind == "norm":
        d = _log(rng, 16, 8192)
        return dict(kind=kind, back=rng.random() < 0.6, dtype=rng.choice(["f32", "bf16"]), out=rng.choice(["f32", "bf16"]),
                    n=min(_log(rng, 1, 2000000), 250000000 // d), d=d)
    d = _log(rng, 5, 300)
    return dict(kind=kind, bits=rng.choice([8, 32]), n_ent=_log(rng, 50, 400000), n_rel=_log(rng, 1, 1000), d=d,
                bases=rng.randint(1, 64), rows=rng.choice(["mask", "nonzero", "all"]), read=round(rng.uniform(0.05, 1.0), 2),
                copy=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _rand(shape, gen, std=1.0):
    return torch.randn(shape, generator=gen, device=DEV) * std


def _dense_inputs(case, seed):
    g, t = _gen(seed), TYPES[case["dtype"]]
    n, di, do = case["n"], case["d_in"], case["d_out"]
    x = dict(X=_rand((n, di), g).to(t), W=_rand((di, do), g, math.sqrt(2.0 / (di + do))).to(t), b=_rand((do,), g, 0.1))
    if not case["back"]:
        x["R"] = _rand((n, do), g).to(t) if case["res"] and di != do else x["X"] if case["res"] else None
        return x
    x["pre"] = (x["X"].float() @ x["W"].float() + x["b"]).to(t) if case["act"] != "identity" else None
    x["dY"] = _rand((n, do), g, 1e-2).to(t)
    x["add"] = _rand((n, di), g, 1e-2).to(t) if case["res"] and case["need_dx"] else None
    return x


def _norm_inputs(case, seed):
    g = _gen(seed)
    n, d = case["n"], case["d"]
    x = dict(X=(_rand((n, d), g) * (0.5 + torch.rand((n, 1), generator=g, device=DEV)) + _rand((n, 1), g, 0.5)).to(TYPES[case["dtype"]]),
             gamma=1.0 + _rand((d,), g, 0.1), beta=_rand((d,), g, 0.1))
    if case["back"]:
        f = x["X"].double() if d < 64 else x["X"].float()
        mean = f.mean(1)
        x["mean"], x["rstd"] = mean.float(), torch.rsqrt((f - mean[:, None]).square().mean(1) + EPS).float()
        x["dY"] = _rand((n, d), g, 1e-2).to(TYPES[case["out"]])
    return x


def _model(case):
    """(rows, columns, by rows, weight decay) of each tensor: the entity table, the score's relations, two layers, a norm."""
    d, R, B = case["d"], case["n_rel"], case["bases"]
    shapes = [(case["n_ent"], d, True, 0.0), (1, R * d, False, 0.01)]
    for _ in range(2):
        shapes += [(1, B * d * d, False, 0.01), (1, 2 * R * B, False, 0.01), (1, d * d, False, 0.01)]
    return shapes + [(1, d, False, 0.0), (1, d, False, 0.0)]


def _adamw_inputs(case, seed):
    g, tensors = _gen(seed), []
    for rows, d, by_rows, wd in _model(case):
        p = _rand((rows, d), g, 0.1)
        grad = _rand((rows, d), g, 1e-3) * torch.exp(_rand((rows, 1), g))
        m = _rand((rows, d), g, 3e-4)
        v = (_rand((rows, d), g, 1e-3)).square() + m.square()
        t = dict(param=p, grad=grad, weight_decay=wd, rows="all", row_mask=None, m_scale=None, v_scale=None, copy=None)
        if by_rows and case["rows"] != "all":
            read = torch.rand((rows,), generator=g, device=DEV) < case["read"]
            grad *= read[:, None]
            t.update(rows=case["rows"], row_mask=read.to(torch.uint8) if case["rows"] == "mask" else None)
        if case["bits"] == 8 and p.numel() >= 4096:           # small tensors keep moments of 32 bits
            i = torch.arange(rows * d, device=DEV).view(rows, d)
            m, t["m_scale"] = _encode(m, E4M3, _offset(i, 9, E4M3))
            v, t["v_scale"] = _encode(v, E5M2, _offset(i, 9, E5M2))
        if case["copy"] and not by_rows and wd:
            t["copy"] = p.to(torch.bfloat16)
        tensors.append(dict(t, m=m, v=v))
    return dict(tensors=tensors, t=10)


def prepare(case, seed):
    make = dict(dense=_dense_inputs, norm=_norm_inputs, adamw=_adamw_inputs)[case["kind"]]
    return dict(make(case, seed), case=case)


# ------------------------------------------------------------------------------------------------ plain forms

def _act(z, act):
    return torch.relu(z) if act == "relu" else z / (1.0 + torch.exp(-z)) if act == "silu" else z


def _act_grad(z, act):
    """act'(z)"""
    if act == "relu":
        return (z > 0).to(z.dtype)
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 + z * (1.0 - s))


def _dense(x):
    c, t = x["case"], x["X"].dtype
    if not c["back"]:
        z = x["X"].float() @ x["W"].float() + x["b"]
        y = _act(z, c["act"])
        if x["R"] is not None:
            y = y + x["R"].float()
        return dict(Y=y.to(t), pre=z.to(t)) if c["keep"] else dict(Y=y.to(t))
    dp = x["dY"].float()
    if c["act"] != "identity":
        dp = dp * _act_grad(x["pre"].float(), c["act"])
    out = dict(dW=x["X"].float().T @ dp, db=dp.sum(0))
    if c["need_dx"]:
        dx = dp @ x["W"].float().T
        out["dX"] = (dx if x["add"] is None else dx + x["add"].float()).to(t)
    return out


def _norm(x):
    c, f = x["case"], x["X"].float()
    if not c["back"]:
        mean = f.mean(1)
        f = f - mean[:, None]
        rstd = 1.0 / torch.sqrt(f.square().mean(1) + EPS)
        return dict(Y=(f * rstd[:, None] * x["gamma"] + x["beta"]).to(TYPES[c["out"]]), mean=mean, rstd=rstd)
    r = x["rstd"][:, None]
    xh = (f - x["mean"][:, None]) * r
    dy = x["dY"].float()
    u = dy * x["gamma"]
    dx = r * (u - u.mean(1, keepdim=True) - xh * (u * xh).mean(1, keepdim=True))
    return dict(dX=dx.to(x["X"].dtype), dgamma=(dy * xh).sum(0), dbeta=dy.sum(0))


# An 8-bit moment: a power of two per block of 256 elements of a row brings the block's largest magnitude to at most the
# format's largest number; a magnitude that lies a fraction f of their distance above the lower of two of the format's
# numbers goes to the upper one where f + u reaches one, u in [0, 1) from the element's index and the step.
E4M3 = dict(type=torch.float8_e4m3fn, digits=3, least=-6, top=8, shift=0)
E5M2 = dict(type=torch.float8_e5m2, digits=2, least=-14, top=15, shift=16)


def _offset(i, t, form):
    x = i * 0xC2B2AE35 + t * 0x9E3779B9 & 0xFFFFFFFF
    x = (x ^ x >> 16) * 0x2C1B3C6D & 0xFFFFFFFF
    return (x >> form["shift"] & 0xFFFF).float() * 2.0 ** -16


def _scale(most, form):
    """The power of two that brings `most` to between half the format's largest number and that number."""
    f, e = torch.frexp(most)                                  # f in [0.5, 1)
    k = (e - 1 - form["top"] + (f > 0.875)).clamp(min=-126)
    return torch.where(most > 0, torch.ldexp(torch.ones_like(most), k), torch.zeros_like(most))


def _spread(scale, d):
    return scale.repeat_interleave(BLOCK, 1)[:, :d]


def _round8(x, form, u):
    """Magnitudes x >= 0, scaled, to numbers of the format."""
    e = torch.clamp(torch.frexp(x)[1] - 1, min=form["least"]) - form["digits"]
    return torch.ldexp(torch.floor(torch.ldexp(x, -e) + u), e)


def _encode(x, form, u):
    rows, d = x.shape
    most = torch.nn.functional.pad(x.abs(), (0, -d % BLOCK)).view(rows, -1, BLOCK).amax(2)
    scale = _scale(most, form)
    s = _spread(scale, d)
    q = _round8(torch.where(s > 0, x.abs() / s, x.new_zeros(())), form, u)
    if form is E5M2:                                          # a second moment that is not zero stays above it
        q = torch.where(x > 0, torch.clamp(q, min=2.0 ** -16), q)
    return torch.copysign(q, x).to(form["type"]), scale


def _adamw(x):
    t, h = x["t"], HYPER
    x["t"] = t + 1
    c1, c2 = 1.0 - h["beta1"] ** t, 1.0 - h["beta2"] ** t
    return [_adamw_one(w, t, h, c1, c2) for w in x["tensors"]]


def _adamw_one(w, t, h, c1, c2):
    p, g, m, v, d = w["param"], w["grad"], w["m"].float(), w["v"].float(), w["param"].shape[1]
    b1, b2 = torch.tensor(h["beta1"]).item(), torch.tensor(h["beta2"]).item()      # as 32-bit numbers
    if w["m_scale"] is not None:
        m, v = m * _spread(w["m_scale"], d), v * _spread(w["v_scale"], d)
    m = m * b1 + g * (1.0 - b1)
    v = v * b2 + (g * (1.0 - b2)) * g
    new = p - h["lr"] * (w["weight_decay"] * p + m / c1 / (torch.sqrt(v / c2) + h["eps"]))
    on = (g != 0).any(1) if w["rows"] == "nonzero" else w["row_mask"] != 0 if w["rows"] == "mask" else None
    done = dict(param=new, m=m, v=v)
    if w["m_scale"] is not None:
        i = torch.arange(p.numel(), device=p.device).view_as(p)
        done["m"], done["m_scale"] = _encode(m, E4M3, _offset(i, t, E4M3))
        done["v"], done["v_scale"] = _encode(v, E5M2, _offset(i, t, E5M2))
    if w["copy"] is not None:
        done["copy"] = new.to(torch.bfloat16)
    for name, value in done.items():
        if on is None:
            w[name].copy_(value)
        else:                                                 # rows that the step did not reach stay as they are
            was, now = (z.view(torch.uint8) if z.element_size() == 1 else z for z in (w[name], value))
            was.copy_(torch.where(on[:, None], now, was))
    return {name: w[name] for name in done}


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    kind = state["case"]["kind"]
    if not own:
        return dict(dense=_dense, norm=_norm, adamw=_adamw)[kind](state)
    from paper_2201_02791_amd import binding as kb
    c = state["case"]
    if kind == "dense":
        layer = dict(W=state["W"], b=state["b"], act=dict(identity=kb.ACT_IDENTITY, relu=kb.ACT_RELU, silu=kb.ACT_SILU)[c["act"]])
        if not c["back"]:
            Y, pre = kb.dense_forward(layer, state["X"], R=state["R"], keep_pre=c["keep"])
            return dict(Y=Y, pre=pre) if c["keep"] else dict(Y=Y)
        grad = kb.dense_backward(layer, state["X"], state["pre"], state["dY"], add=state["add"], need_dX=c["need_dx"])
        return {name: grad[name] for name in (("dW", "db", "dX") if c["need_dx"] else ("dW", "db"))}
    if kind == "norm":
        norm = dict(gamma=state["gamma"], beta=state["beta"], eps=EPS)
        if not c["back"]:
            Y, mean, rstd = kb.layer_norm_forward(norm, state["X"], out_dtype=TYPES[c["out"]])
            return dict(Y=Y, mean=mean, rstd=rstd)
        return kb.layer_norm_backward(norm, state["X"], state["mean"], state["rstd"], state["dY"])
    if "plan" not in state:                                   # the addresses, which a training loop lays out once
        state["plan"] = kb.AdamWTensors(state["tensors"])
    kb.adamw_step(state["plan"], t=state["t"], **HYPER)
    state["t"] += 1
    return [{name: w[name] for name in ("param", "m", "v", "m_scale", "v_scale", "copy") if w[name] is not None} for w in state["tensors"]]


# ------------------------------------------------------------------------------------------------ work

def work(case):
    if case["kind"] == "dense":
        n, di, do, e = case["n"], case["d_in"], case["d_out"], 4 if case["dtype"] == "f32" else 2
        if not case["back"]:
            extra = (do if case["res"] and di != do else 0) + (do if case["keep"] else 0)
            return dict(bytes=e * (n * (di + do + extra) + di * do) + 4 * do, flops=2.0 * n * di * do)
        dx = (di if case["need_dx"] else 0) + (di if case["need_dx"] and case["res"] else 0)
        pre = do if case["act"] != "identity" else 0
        return dict(bytes=e * (n * (di + do + pre + dx) + (di * do if case["need_dx"] else 0)) + 4 * (di * do + do),
                    flops=(4.0 if case["need_dx"] else 2.0) * n * di * do)
    if case["kind"] == "norm":
        n, d, e, o = case["n"], case["d"], 4 if case["dtype"] == "f32" else 2, 4 if case["out"] == "f32" else 2
        if not case["back"]:
            return dict(bytes=n * d * (e + o) + 8 * n + 8 * d, flops=8.0 * n * d)
        return dict(bytes=n * d * (2 * e + o) + 8 * n + 12 * d, flops=14.0 * n * d)
    total, elements = 0.0, 0.0
    for rows, d, by_rows, wd in _model(case):
        part = case["read"] if by_rows and case["rows"] != "all" else 1.0
        small = case["bits"] == 32 or rows * d < 4096
        one = 28.0 if small else 16.0 + 16.0 * -(-d // BLOCK) / d
        if case["copy"] and not by_rows and wd:
            one += 2.0
        total += part * one * rows * d
        if by_rows and case["rows"] != "all":                 # a flag a row, or the gradients of the rows that are left out
            total += rows if case["rows"] == "mask" else (1.0 - part) * 4.0 * rows * d
        elements += part * rows * d
    return dict(bytes=total, flops=12.0 * elements)


# ------------------------------------------------------------------------------------------------ exact results

def _exact_dense(case, x):
    X, W = x["X"].double(), x["W"].double()
    if not case["back"]:
        out = dict(pre=torch.addmm(x["b"].double(), X, W))
        z = out["pre"]
        out["Y"] = z.clamp(min=0.0) if case["act"] == "relu" else z * torch.sigmoid(z) if case["act"] == "silu" else z.clone()
        if x["R"] is not None:
            out["Y"] += x["R"].double()
        return out if case["keep"] else dict(Y=out["Y"])
    G = x["dY"].double()
    if case["act"] == "relu":
        G = torch.where(x["pre"].double() > 0.0, G, torch.zeros_like(G))
    elif case["act"] == "silu":
        z = x["pre"].double()
        s = torch.sigmoid(z)
        G = G * (s + z * s * torch.sigmoid(-z))
    out = dict(dW=torch.mm(X.t(), G), db=torch.mv(G.t(), torch.ones(len(G), dtype=torch.float64, device=DEV)))
    if case["need_dx"]:
        out["dX"] = torch.mm(G, W.t())
        if x["add"] is not None:
            out["dX"] += x["add"].double()
    return out


def _exact_norm(case, x):
    X = x["X"].double()
    if not case["back"]:
        var, mean = torch.var_mean(X, 1, correction=0)
        rstd = (var + EPS).pow(-0.5)
        return dict(Y=torch.addcmul(x["beta"].double(), (X - mean[:, None]) * rstd[:, None], x["gamma"].double()), mean=mean, rstd=rstd)
    d, dy, r = case["d"], x["dY"].double(), x["rstd"].double()[:, None]
    X = (X - x["mean"].double()[:, None]) * r
    out = dict(dgamma=(dy * X).sum(0), dbeta=dy.sum(0))
    dy = dy * x["gamma"].double()
    dot = (dy * X).sum(1, keepdim=True)
    out["dX"] = r / d * (d * dy - dy.sum(1, keepdim=True) - X * dot)
    return out


def _exact_moment(x, digits, least, largest, half, t, scales):
    """(numbers, scales) that a moment x of 64 bits is held as; `half`: the half of the offset's 32 bits."""
    rows, d = x.shape
    blocks = scales.shape[1]
    a = torch.zeros((rows, blocks * BLOCK), dtype=torch.float64, device=DEV)
    a[:, :d] = x.abs()
    a = a.view(rows, blocks, BLOCK)
    most = a.amax(2)
    s = torch.exp2(torch.ceil(torch.log2(torch.where(most > 0, most, torch.ones_like(most)) / largest)))
    a = (a / s[:, :, None]).view(rows, -1)[:, :d]
    s = torch.where(most > 0, s, torch.zeros_like(s))
    e = torch.floor(torch.log2(torch.where(a > 0, a, torch.ones_like(a)))).clamp(min=least) - digits
    unit = torch.exp2(torch.where(a > 0, e, torch.full_like(e, least - digits)))
    i = torch.arange(rows * d, device=DEV).view(rows, d)
    w = torch.remainder(i * 3266489909 + t * 2654435769, 1 << 32)
    w = torch.remainder(torch.bitwise_xor(w, w.div(1 << 16, rounding_mode="floor")) * 739982445, 1 << 32)
    u = (w.div(1 << 16, rounding_mode="floor") if half else torch.remainder(w, 1 << 16)).double() / 65536.0
    return torch.floor(a / unit + u) * unit, s


def _exact_adamw(case, x):
    h, t, done = HYPER, x["t"], []
    f32 = lambda c: float(torch.tensor(c, dtype=torch.float32))  # noqa: E731
    b1, b2, lr, eps = f32(h["beta1"]), f32(h["beta2"]), f32(h["lr"]), f32(h["eps"])
    for w in x["tensors"]:
        p, g = w["param"].double(), w["grad"].double()
        m, v, d = w["m"].double(), w["v"].double(), p.shape[1]
        eight = w["m_scale"] is not None
        if eight:
            at = torch.arange(d, device=DEV) // BLOCK
            m, v = m * w["m_scale"].double()[:, at], v * w["v_scale"].double()[:, at]
        m.lerp_(g, 1.0 - b1)
        v.lerp_(g * g, 1.0 - b2)
        on = w["row_mask"].bool() if w["rows"] == "mask" else g.abs().amax(1) > 0 if w["rows"] == "nonzero" else None
        step = lr * (m / (1.0 - b1 ** t) / (eps + (v / (1.0 - b2 ** t)).sqrt()) + f32(w["weight_decay"]) * p)
        out = dict(param=p - step, m=m, v=v)
        if eight:
            del step
            q, out["m_scale"] = _exact_moment(m, 3, -6, 448.0, 0, t, w["m_scale"])
            out["m"] = torch.where(m < 0, -q, q)
            q, out["v_scale"] = _exact_moment(v, 2, -14, 57344.0, 1, t, w["v_scale"])
            out["v"] = torch.where(v > 0, q.clamp(min=2.0 ** -16), q)
        if w["copy"] is not None:
            out["copy"] = out["param"]
        done.append({k: y if on is None else torch.where(on[:, None], y, w[k].double()) for k, y in out.items()})
    return done


def exact(case, seed):
    make = dict(dense=_dense_inputs, norm=_norm_inputs, adamw=_adamw_inputs)[case["kind"]]
    return dict(dense=_exact_dense, norm=_exact_norm, adamw=_exact_adamw)[case["kind"]](case, make(case, seed))
