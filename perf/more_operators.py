"""Operators that answer from a trained model and train it further: inputs, one pass, its work and its exact result.

  table    an embedding table to 4 bits with a scale for each group of 32 elements of a row, and its rows back
  scores   DistMult scores of one query or a few against every row of such a table
  sample   draws from rows of scores, with temperature, top-k, top-p and min-p, from given random numbers
  clip     the norm of all gradients of a model, and the gradients scaled to a largest norm

Sizes are those of the workloads of `paper_2201_02791_amd/synth.py` (the tiny graph, the 14,541-entity knowledge graph,
the citation-shaped graph of 2.9 M vertices and 128 features, the large many-relation graph of a million entities and
width 256) and of ranges around them.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GROUP = 32                                                    # elements of a row that share a scale
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)             # magnitudes of the 4-bit numbers; the fourth bit is the sign


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # the mid-size graph's entities, whose width fills no whole number of groups
        dict(name="table-mid", kind="table", dtype="f32", n=14541, d=200),
        # the large graph's entities, after a training run
        dict(name="table-bigkg", kind="table", dtype="f32", n=1000000, d=256),
        # one question to the mid-size graph: latency counts
        dict(name="scores-one-mid", kind="scores", dtype="f32", q=1, n=14541, d=200, rel=True),
        # one question to the large graph
        dict(name="scores-one-bigkg", kind="scores", dtype="f32", q=1, n=1000000, d=256, rel=True),
        # a server's batch of questions to the large graph
        dict(name="scores-batch-bigkg", kind="scores", dtype="f32", q=16, n=1000000, d=256, rel=True),
        # similar papers: rows of the citation graph against all vertices, no relation between them
        dict(name="scores-citation-bf16", kind="scores", dtype="bf16", q=37, n=2900000, d=128, rel=False),
        # one answer out of the large graph's million scores
        dict(name="sample-one-bigkg", kind="sample", dtype="f32", rows=1, cols=1000000, draws=1, std=2.0, t=0.7, k=50, p=0.95, m=0.0, by_row=False, out=0.0),
        # a server's batch with settings of their own, without top-k, each question with known answers left out
        dict(name="sample-nucleus-citation", kind="sample", dtype="f32", rows=16, cols=2900000, draws=4, std=2.0, t=0.9, k=0, p=0.9, m=0.0, by_row=True, out=0.01),
        # negatives that the model takes for true: 64 of 256 candidates for each positive of the large graph's batch
        dict(name="sample-negatives-bigkg", kind="sample", dtype="f32", rows=65536, cols=256, draws=64, std=1.0, t=1.0, k=0, p=1.0, m=0.0, by_row=False, out=0.02),
        # the tiny graph's model: every tensor takes microseconds
        dict(name="clip-tiny", kind="clip", dtype="f32", n_ent=1000, n_rel=10, d=32, bases=4, read=0.8, most=0.5, scale=True),
        # the large graph's model, gradients that have to be scaled
        dict(name="clip-bigkg", kind="clip", dtype="f32", n_ent=1000000, n_rel=1000, d=256, bases=64, read=0.9, most=0.5, scale=True),
        # the same model before an update that takes the factor along: the norm and the factor alone
        dict(name="norm-bigkg", kind="clip", dtype="f32", n_ent=1000000, n_rel=1000, d=256, bases=64, read=0.9, most=0.5, scale=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["table", "scores", "scores", "sample", "sample", "sample", "clip"])
    if kind == "table":
        d = _log(rng, 4, 1024)
        return dict(kind=kind, dtype=rng.choice(["f32", "bf16"]), n=min(_log(rng, 1, 1000000), 200000000 // d), d=d)
    if kind == "scores":
        d, q = _log(rng, 4, 1024), rng.choice([1, rng.randint(2, 5), rng.randint(6, 16), rng.randint(17, 64)])
        n = min(_log(rng, 16, 2900000), 250000000 // d, 100000000 // q)
        return dict(kind=kind, dtype=rng.choice(["f32", "bf16"]), q=q, n=n, d=d, rel=rng.random() < 0.6)
    if kind == "sample":
        cols = _log(rng, 2, 2900000)
        rows = min(_log(rng, 1, 65536), 40000000 // cols)
        return dict(kind=kind, dtype=rng.choice(["f32", "f32", "bf16"]), rows=rows, cols=cols, draws=min(_log(rng, 1, 64), max(1, 4000000 // rows)),
                    std=round(rng.uniform(0.2, 6.0), 2), t=round(rng.uniform(0.2, 2.0), 2), k=rng.choice([0, 0, 1, _log(rng, 2, 500), _log(rng, 2, 100000)]),
                    p=rng.choice([1.0, round(rng.uniform(0.05, 0.999), 3)]), m=rng.choice([0.0, 0.0, round(rng.uniform(0.001, 0.5), 3)]),
                    by_row=rng.random() < 0.3, out=rng.choice([0.0, 0.05, 0.9]))
    return dict(kind=kind, dtype=rng.choice(["f32", "f32", "bf16"]), n_ent=_log(rng, 50, 500000), n_rel=_log(rng, 1, 1000), d=_log(rng, 5, 300),
                bases=rng.randint(1, 64), read=round(rng.uniform(0.05, 1.0), 2), most=rng.choice([0.1, 0.5, 2.0]), scale=rng.random() < 0.7)


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _rand(shape, gen, std=1.0):
    return torch.randn(shape, generator=gen, device=DEV) * std


def _embeddings(n, d, gen):
    """Rows of widely different lengths, as after training: entities of many edges grow."""
    return _rand((n, d), gen, 0.1) * torch.exp(_rand((n, 1), gen, 0.5))


def _table_inputs(case, seed):
    return dict(X=_embeddings(case["n"], case["d"], _gen(seed)).to(TYPES[case["dtype"]]))


def _scores_inputs(case, seed):
    g, q, n, d = _gen(seed), case["q"], case["n"], case["d"]
    codes, scales = _encode(_embeddings(n, d, g))
    near = min(n, 4096)
    x = dict(codes=codes, scales=scales, X=_embeddings(near, d, g).to(TYPES[case["dtype"]]), M=None, rel=None,
             fixed=torch.randint(0, near, (q,), generator=g, device=DEV, dtype=torch.int32))
    if case["rel"]:
        x["M"] = _rand((474, d), g)
        x["rel"] = torch.randint(0, 474, (q,), generator=g, device=DEV, dtype=torch.int32)
    return x


def _sample_inputs(case, seed):
    g, rows, cols = _gen(seed), case["rows"], case["cols"]
    s = _rand((rows, cols), g, case["std"])
    if case["out"]:                                           # answers that are left out
        s.masked_fill_(torch.rand((rows, cols), generator=g, device=DEV) < case["out"], -math.inf)
    x = dict(scores=s.to(TYPES[case["dtype"]]), u=torch.rand((rows, case["draws"]), generator=g, device=DEV, dtype=torch.float64),
             temperature=case["t"], top_k=case["k"], top_p=case["p"], min_p=case["m"])
    if case["by_row"]:
        r = torch.rand((3, rows), generator=g, device=DEV)
        x["temperature"] = case["t"] * (0.5 + r[0])
        x["top_p"] = case["p"] * (0.8 + 0.2 * r[1])
        x["min_p"] = case["m"] * r[2]
        if case["k"]:
            x["top_k"] = torch.randint(1, case["k"] + 1, (rows,), generator=g, device=DEV, dtype=torch.int32)
    return x


def _model(case):
    """(rows, columns, by rows) of each gradient: the entity table, the score's relations, two layers."""
    d, R, B = case["d"], case["n_rel"], case["bases"]
    return [(case["n_ent"], d, True), (R, d, False)] + [(B, d * d, False), (2 * R, B, False), (d, d, False)] * 2


def _clip_inputs(case, seed):
    g, grads, expected = _gen(seed), [], 0.0
    for rows, d, by_rows in _model(case):
        x = _rand((rows, d), g, 1e-3) * torch.exp(_rand((rows, 1), g, 0.5))
        expected += rows * d * 1e-6 * math.exp(0.5) * (case["read"] if by_rows else 1.0)
        mask = None
        if by_rows:                                           # what a batch does not read has no gradient
            on = torch.rand((rows,), generator=g, device=DEV) < case["read"]
            x *= on[:, None]
            mask = on.to(torch.uint8)
        grads.append(dict(grad=x.to(TYPES[case["dtype"]]), row_mask=mask))
    return dict(grads=grads, max_norm=case["most"] * math.sqrt(expected))


def prepare(case, seed):
    make = dict(table=_table_inputs, scores=_scores_inputs, sample=_sample_inputs, clip=_clip_inputs)[case["kind"]]
    return dict(make(case, seed), case=case)


# ------------------------------------------------------------------------------------------------ plain forms

# A group's scale s is the smallest bfloat16 number, 2^-126 or more, six of which reach the group's largest magnitude (0 for a
# group of zeros); an element is the number of LEVELS times s that is nearest to it, of two as near the one of the even code.
# A byte holds two elements, the first in its low half; rows are filled up to whole groups with zeros.

def _encode(X):
    """(codes uint8 [n][16 groups], scales bfloat16 [n][groups])"""
    n, d = X.shape
    groups = -(-d // GROUP)
    x = torch.nn.functional.pad(X.float(), (0, groups * GROUP - d)).view(n, groups, GROUP)
    a = x.abs()
    most = a.amax(2)
    s = ((most * (1.0 / 6.0)).view(torch.int32) & -65536).view(torch.float32).clamp(min=2.0 ** -126)
    for _ in range(2):                                        # the product was rounded, then cut: at most two steps short
        s = torch.where(6.0 * s < most, (s.view(torch.int32) + 65536).view(torch.float32), s)
    s = torch.where(most > 0, s, torch.zeros_like(s))
    t = s[:, :, None]
    code = torch.zeros_like(x, dtype=torch.uint8)
    for k in range(7):                                        # the borders lie half way; on them the even code's side wins
        border = t * (0.5 * (LEVELS[k] + LEVELS[k + 1]))
        code += (a > border) if k % 2 == 0 else (a >= border)
    code = torch.where(t > 0, code + 8 * (x < 0), torch.zeros_like(code)).view(n, -1, 2)
    return code[:, :, 0] + 16 * code[:, :, 1], s.to(torch.bfloat16)


def _decode(codes, scales, d):
    n = len(codes)
    signed = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=DEV)
    both = torch.stack([signed[(codes & 15).int()], signed[(codes >> 4).int()]], 2).view(n, -1, GROUP)
    return (both * scales.float()[:, :, None]).view(n, -1)[:, :d]


def _table(x):
    codes, scales = _encode(x["X"])
    return dict(rows=_decode(codes, scales, x["case"]["d"]).contiguous(), scales=scales)


def _scores(x):
    q = x["X"][x["fixed"].long()].float()
    if x["M"] is not None:
        q = q * x["M"][x["rel"].long()]
    return q @ _decode(x["codes"], x["scales"], x["case"]["d"]).T


# The weight of a score l in a row whose largest is m: e^((l - m) / temperature), rounded to a multiple of 2^-b with
# b = min(40, 62 - ceil(log2 columns)), so that sums of weights are exact; minus infinity and NaN have none.  In descending
# order of scores, equal ones in the order of their columns, top-k leaves the first k, top-p of those the shortest beginning
# whose weights reach top_p of theirs, min-p what has at least min_p times the largest weight.  The draw is the first column at
# which the sum of the weights left, in the order of columns, passes u times their total.

def _bits(cols):
    return min(40, 62 - (cols - 1).bit_length())


def _column(v, like, kind):
    return v.to(kind)[:, None] if torch.is_tensor(v) else torch.full((len(like), 1), v, dtype=kind, device=DEV)


def _sample(x):
    s = x["scores"].float()
    rows, cols = s.shape
    s = torch.where(torch.isnan(s), torch.full_like(s, -math.inf), s) + 0.0
    most = s.amax(1, keepdim=True)
    t, k = _column(x["temperature"], s, torch.float64), _column(x["top_k"], s, torch.int64)
    p, low = _column(x["top_p"], s, torch.float32).double(), _column(x["min_p"], s, torch.float32).double()
    if not torch.is_tensor(x["temperature"]):
        t = t.float().double()
    unit = 2.0 ** _bits(cols)
    w = torch.exp((s.double() - most.double()) / t)
    w = torch.where(s == most, torch.ones_like(w), w)
    w = torch.where(s == -math.inf, torch.zeros_like(w), torch.round(w * unit)).long()
    order = torch.sort(s, dim=1, descending=True, stable=True)[1]
    ranked = torch.gather(w, 1, order)
    place = torch.arange(cols, device=DEV)[None, :]
    ranked = torch.where((k <= 0) | (place < k), ranked, torch.zeros_like(ranked))
    before = torch.cumsum(ranked, 1)
    total = before[:, -1:]
    before = before - ranked
    goal = torch.minimum(torch.ceil(p * total.double()).long().clamp(min=1), total)
    keep = ((p >= 1.0) | (before < goal)) & (ranked.double() >= low * unit)
    ranked = torch.where(keep, ranked, torch.zeros_like(ranked))
    w = torch.zeros_like(w).scatter_(1, order, ranked)
    sums = torch.cumsum(w, 1)
    total = sums[:, -1:]
    at = torch.minimum((x["u"].double() * total.double()).long(), total - 1)
    choice = torch.searchsorted(sums, at, right=True)
    none = total == 0
    choice = torch.where(none, torch.full_like(choice, -1), choice)
    prob = torch.gather(w, 1, choice.clamp(min=0, max=cols - 1)).double() / total.clamp(min=1).double()
    return dict(choice=choice.int(), prob=torch.where(none, torch.zeros_like(prob), prob).float())


def _clip(x):
    total = sum((g["grad"] if g["row_mask"] is None else g["grad"] * g["row_mask"][:, None]).double().square().sum() for g in x["grads"])
    norm = torch.sqrt(total)
    factor = (x["max_norm"] / norm).clamp(max=1.0).float()
    out = dict(norm=norm.float(), factor=factor)
    if x["case"]["scale"]:
        for g in x["grads"]:
            g["grad"].copy_((g["grad"].float() * factor).to(g["grad"].dtype))
        out["grads"] = [g["grad"] for g in x["grads"]]
    return out


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    c = state["case"]
    kind = c["kind"]
    if kind == "clip" and c["scale"] and c["most"] < 1.0:     # the gradients of a pass are the scaled ones of the last: scaled again
        state["max_norm"] *= 0.999
    if not own:
        return dict(table=_table, scores=_scores, sample=_sample, clip=_clip)[kind](state)
    from paper_2201_02791_amd import binding as kb
    if kind == "table":
        table = kb.table4_encode(state["X"])
        return dict(rows=kb.table4_decode(table), scales=table.scales)
    if kind == "scores":
        if "table" not in state:                              # the codes as the bytes that a program holds them in
            state["table"] = kb.Table4(state["codes"].to(torch.uint8), state["scales"], c["d"])
        return kb.table4_scores(state["table"], state["X"], fixed=state["fixed"], M=state["M"], rel=state["rel"])
    if kind == "sample":
        choice, prob = kb.sample_scores(state["scores"], state["u"], temperature=state["temperature"], top_k=state["top_k"],
                                        top_p=state["top_p"], min_p=state["min_p"], want_prob=True)
        return dict(choice=choice, prob=prob)
    if "plan" not in state:                                   # the addresses, which a training loop lays out once
        state["plan"] = kb.GradTensors(state["grads"])
    norm, factor = (kb.clip_grads if c["scale"] else kb.grad_norm)(state["plan"], state["max_norm"])
    out = dict(norm=norm, factor=factor)
    if c["scale"]:
        out["grads"] = [g["grad"] for g in state["grads"]]
    return out


# ------------------------------------------------------------------------------------------------ work

def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] in ("table", "scores"):
        n, d = case["n"], case["d"]
        groups = -(-d // GROUP)
        if case["kind"] == "table":                           # rows in, codes and scales out and in again, rows out
            return dict(bytes=n * (d * (e + 4.0) + 36.0 * groups), flops=3.0 * n * d)
        q = case["q"]
        return dict(bytes=18.0 * n * groups + q * (d * (e + (4 if case["rel"] else 0)) + 4.0 * n), flops=2.0 * q * n * d)
    if case["kind"] == "sample":
        cells = case["rows"] * case["cols"]
        return dict(bytes=e * cells + 16.0 * case["rows"] * case["draws"], flops=4.0 * cells)
    numbers = sum(r * d * (case["read"] if by_rows else 1.0) for r, d, by_rows in _model(case))
    again = case["scale"] and case["most"] < 1.0              # read once and, where they change, written
    return dict(bytes=numbers * e * (2 if again else 1) + case["n_ent"], flops=numbers * (3.0 if again else 2.0))


# ------------------------------------------------------------------------------------------------ exact results

def _exact_scale(most):
    """The smallest 8-bit mantissa times a power of two that is a sixth of `most` or more."""
    sixth = torch.where(most > 0, most, torch.ones_like(most)) / 6.0
    step = torch.exp2(torch.floor(torch.log2(sixth)) - 7.0)
    s = torch.ceil(sixth / step) * step
    s = torch.where((s - step) * 6.0 >= most, s - step, s)
    s = torch.where(s * 6.0 < most, s + step, s)
    return torch.where(most > 0, s.clamp(min=2.0 ** -126), torch.zeros_like(s))


def _exact_table(case, x):
    X, d = x["X"].double(), case["d"]
    at = torch.arange(d, device=DEV) // GROUP
    groups = -(-d // GROUP)
    s = torch.stack([_exact_scale(X[:, g * GROUP:(g + 1) * GROUP].abs().amax(1)) for g in range(groups)], 1)
    rows = X
    for lo in range(0, len(X), 1 << 18):                      # by parts: the distances to all numbers take eight times the rows
        y, t = X[lo:lo + (1 << 18)], s[lo:lo + (1 << 18)][:, at]
        z = torch.where(t > 0, y.abs() / t, torch.zeros_like(y))
        exponent = torch.floor(torch.log2(z.clamp(min=1.0)))
        unit = torch.exp2(exponent - 1.0)
        rows[lo:lo + (1 << 18)] = torch.copysign(torch.round(z / unit) * unit * t, y)
    return dict(rows=rows, scales=s)


def _exact_scores(case, x):
    d = case["d"]
    q = x["X"].double().index_select(0, x["fixed"].long())
    if x["M"] is not None:
        q = torch.mul(q, x["M"].double().index_select(0, x["rel"].long()))
    low = torch.bitwise_and(x["codes"], 15)
    nibbles = torch.stack([low, torch.bitwise_right_shift(x["codes"], 4)], -1).flatten(1)[:, :d]
    e, f = torch.bitwise_and(nibbles >> 1, 3).double(), torch.bitwise_and(nibbles, 1).double()
    value = torch.where(e > 0, (1.0 + 0.5 * f) * torch.exp2(e - 1.0), 0.5 * f)
    value = torch.where(nibbles >= 8, -value, value)
    value *= x["scales"].double().repeat_interleave(GROUP, 1)[:, :d]
    return torch.mm(q, value.t().contiguous())


def _exact_sample(case, x):
    rows, cols = x["scores"].shape
    bits = min(40, 62 - math.ceil(math.log2(cols)))
    f32 = lambda v: v.double() if torch.is_tensor(v) else torch.full((rows,), float(torch.tensor(v, dtype=torch.float32)), dtype=torch.float64, device=DEV)  # noqa: E731
    t, p, low = f32(x["temperature"]), f32(x["top_p"]), f32(x["min_p"])
    k = x["top_k"].long() if torch.is_tensor(x["top_k"]) else torch.full((rows,), x["top_k"], device=DEV)
    prob = torch.zeros((rows, case["draws"]), dtype=torch.float64, device=DEV)
    step = max(1, (1 << 24) // cols)
    for lo in range(0, rows, step):
        at = slice(lo, lo + step)
        s = torch.nan_to_num(x["scores"][at].double(), nan=-math.inf, posinf=math.inf, neginf=-math.inf)
        w = torch.exp((s - s.max(1).values[:, None]) / t[at, None])
        w = (w * 2.0 ** bits).round().nan_to_num(nan=0.0)     # a row of nothing but minus infinity
        key = torch.argsort(-s, dim=1, stable=True)
        w = w.gather(1, key)
        place = torch.arange(cols, device=DEV)
        limit = torch.where(k[at] > 0, k[at], torch.full_like(k[at], cols))
        w *= place < limit[:, None]
        whole = w.long()
        sums = whole.cumsum(1)
        goal = (p[at] * sums[:, -1].double()).ceil().long()
        short = (sums < goal[:, None]).sum(1) + 1             # entries of the beginning that top-p leaves
        short = torch.where(p[at] >= 1.0, torch.full_like(short, cols), short)
        whole *= place < short[:, None]
        whole *= w >= (low[at] * 2.0 ** bits)[:, None]
        back = torch.empty_like(whole).scatter_(1, key, whole)
        sums = back.cumsum(1)
        total = sums[:, -1:]
        goal = torch.minimum((x["u"][at] * total.double()).long(), total - 1)
        j = torch.searchsorted(sums, goal + 1).clamp(max=cols - 1)
        prob[at] = torch.where(total > 0, back.gather(1, j).double() / total.double().clamp(min=1.0), torch.zeros_like(prob[at]))
    return dict(choice=None, prob=prob)


def _exact_clip(case, x):
    most, squares = x["max_norm"] * (0.999 if case["scale"] and case["most"] < 1.0 else 1.0), 0.0
    for g in x["grads"]:
        y = g["grad"].double()
        if g["row_mask"] is not None:
            y = y[g["row_mask"].bool()]
        squares += float(torch.linalg.vector_norm(y)) ** 2
    norm = math.sqrt(squares)
    factor = min(1.0, most / norm)
    one = lambda v: torch.tensor(v, dtype=torch.float64, device=DEV)  # noqa: E731
    out = dict(norm=one(norm), factor=one(factor))
    if case["scale"]:
        out["grads"] = [g["grad"].double() * factor for g in x["grads"]]
    return out


def exact(case, seed):
    make = dict(table=_table_inputs, scores=_scores_inputs, sample=_sample_inputs, clip=_clip_inputs)[case["kind"]]
    at = dict(table=_exact_table, scores=_exact_scores, sample=_exact_sample, clip=_exact_clip)[case["kind"]]
    return at(case, make(case, seed))
