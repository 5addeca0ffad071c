"""Performance cases of the operators between a block's Q/K/V projection and its output projection.

The rows that the projections give are heads of queries, keys and values.  Their operators:

  heads        cq_head_norm: norms of queries and keys for each head, with the position rotation, one pass
  heads_grad   cq_head_norm_grad: the gradients of the above, those of the norms' weights among them
  append       cq_cache_append: keys and values into the pages of a cache (norm and rotation on the way, of the queries too)
  attention    cq_cache_attention: attention of one new token per sequence over that cache

  listed()               the cases that are always timed
  draw(rng)              one more case of the same ranges
  prepare(case, seed)    inputs on the GPU
  run(state)             one call: in plain torch operations, or (own) by the library
  work(case)             bytes and operations that it cannot do without
  exact(case, seed)      what run returns, in float64
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}
EPS = 1e-6
BASE = 1e6              # of the rotation's frequencies
MOST_E4M3 = 448.0

# the dearest of each kind that is drawn: no more than the largest listed one
MAX_HEADS = 4096 * 40 * 128        # values of queries and keys
MAX_GRAD = 8192 * 40 * 128
MAX_APPEND = 4096 * 48 * 128       # values of queries, keys and values
MAX_CACHED = 48 * 4096 * 8 * 128   # keys that a batch's sequences may hold


def _heads(op, T, Hq, Hk, D, rot, interleaved, norm, x, out, weight, name=None):
    """x: type of the projection's rows; out: of the heads; rot of each head's D values are rotated."""
    c = {"op": op, "T": T, "Hq": Hq, "Hk": Hk, "D": D, "rot": rot, "interleaved": interleaved, "norm": norm, "x": x, "out": out,
         "weight": weight}
    return {"name": name, **c} if name else c


def _append(T, seqs, Hq, Hk, D, rot, interleaved, norm, page, past, x, cache, name=None):
    """T new tokens of `seqs` sequences, each with up to `past` tokens in the cache before."""
    c = {"op": "append", "T": T, "seqs": seqs, "Hq": Hq, "Hk": Hk, "D": D, "rot": rot, "interleaved": interleaved, "norm": norm,
         "page": page, "past": past, "x": x, "cache": cache}
    return {"name": name, **c} if name else c


def _attention(seqs, longest, ragged, Hq, Hk, D, page, q, cache, out, window, softcap, sinks, name=None):
    """One new token of each sequence; ragged: the sequences hold 1 to `longest` tokens.  window 0: all of them."""
    c = {"op": "attention", "seqs": seqs, "longest": longest, "ragged": ragged, "Hq": Hq, "Hk": Hk, "D": D, "page": page, "q": q,
         "cache": cache, "out": out, "window": window, "softcap": softcap, "sinks": sinks}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one token of one user, 32 query and 8 key heads on a hidden size of 4096: launch and latency
        _heads("heads", 1, 32, 8, 128, 128, False, True, "bf16", "bf16", "bf16", "heads-token"),
        # an odd batch of small heads, a quarter of each rotated in neighbouring pairs, no norms
        _heads("heads", 515, 12, 3, 80, 20, True, False, "f16", "f16", "f32", "heads-odd"),
        # a prefill: fp32 rows of a clustered projection become the heads of a 16-bit attention
        _heads("heads", 4096, 32, 8, 128, 128, False, True, "f32", "bf16", "f32", "heads-prefill"),
        # a small training step, and the largest: a long batch
        _heads("heads_grad", 512, 16, 4, 128, 128, False, True, "f32", "f32", "f32", "heads_grad-512"),
        _heads("heads_grad", 8192, 32, 8, 128, 128, False, True, "bf16", "bf16", "bf16", "heads_grad-8192"),
        # a decode step of one user
        _append(1, 1, 32, 8, 128, 128, False, True, 16, 100, "bf16", "bf16", "append-token"),
        # a decode step of 64 users into a cache of 8 bits
        _append(64, 64, 32, 8, 128, 128, False, True, 32, 250, "f32", "e4m3", "append-decode"),
        # nine prompts, half of each head rotated
        _append(4096, 9, 32, 8, 128, 64, True, False, 64, 0, "f16", "f16", "append-prefill"),
        # one user's first answers
        _attention(1, 777, False, 32, 8, 128, 16, "bf16", "bf16", "bf16", 0, 0.0, False, "attention-token"),
        # a decode step of 48 users with contexts of all lengths
        _attention(48, 4096, True, 32, 8, 128, 16, "bf16", "bf16", "bf16", 0, 0.0, False, "attention-decode"),
        # one user with a long document
        _attention(1, 131071, False, 32, 4, 128, 64, "f16", "f16", "f32", 0, 0.0, False, "attention-long"),
        # small heads over a cache of 8 bits, the last tokens only, capped scores and sinks
        _attention(61, 4500, True, 40, 8, 64, 48, "bf16", "e4m3", "bf16", 2000, 30.0, True, "attention-e4m3"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _draw_heads(rng):
    """Query heads, key heads, values of a head, and whether pairs are neighbours."""
    Hk = rng.choice([1, 2, 4, 8, _log(rng, 1, 16)])
    Hq = Hk * rng.choice([1, 2, 4, 5, 8, _log(rng, 1, 16)])
    return Hq, Hk, rng.choice([64, 128, 128, 256, 16 * _log(rng, 2, 16)]), rng.random() < 0.3


def draw(rng):
    op = rng.choice(["heads", "heads_grad", "append", "attention", "attention"])
    Hq, Hk, D, interleaved = _draw_heads(rng)
    x = rng.choice(["f32", "f16", "bf16", "bf16"])
    if op in ("heads", "heads_grad"):
        if rng.random() < 0.3:
            D = _log(rng, 8, 256)
        rot = rng.choice([D // 2 * 2, D // 4 * 2, 2 * rng.randint(0, D // 2)])
        T = _log(rng, 1, min(8192, (MAX_HEADS if op == "heads" else MAX_GRAD) // ((Hq + Hk) * D)))
        return _heads(op, T, Hq, Hk, D, rot, interleaved, rng.random() < 0.7, x, rng.choice([x, "bf16"]) if x == "f32" else x,
                      rng.choice(["f32", x]))
    if op == "append":
        rot = rng.choice([D, D // 4 * 2, 2 * rng.randint(0, D // 2)])
        T = _log(rng, 1, min(4096, MAX_APPEND // ((Hq + 2 * Hk) * D)))
        seqs = T if T <= 256 and rng.random() < 0.5 else _log(rng, 1, min(T, 64))
        past = _log(rng, 1, 300) if seqs * Hk * D <= 1 << 17 else 0
        return _append(T, seqs, Hq, Hk, D, rot, interleaved, rng.random() < 0.7, rng.choice([16, 64, _log(rng, 1, 256)]), past, x,
                       rng.choice(["e4m3", "f16" if x == "f16" else "bf16"]))
    longest = _log(rng, 1, min(131072, MAX_CACHED // (Hk * D)))
    seqs = _log(rng, 1, max(1, min(256, MAX_CACHED // (Hk * D * longest))))
    q = rng.choice(["f32", "f16", "bf16", "bf16"])
    return _attention(seqs, longest, rng.random() < 0.7, Hq, Hk, D, rng.choice([16, 64, _log(rng, 1, 256)]), q,
                      rng.choice(["e4m3", "f16", "bf16", "bf16"]), rng.choice(["f32", q]),
                      rng.choice([0, 0, _log(rng, 1, longest)]), rng.choice([0.0, 0.0, 30.0]), rng.random() < 0.3)


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _randn(g, shape, dtype, scale=1.0, mean=0.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale + mean).to(dtype)


def _cuts(T, parts, seed):
    """parts lengths of at least one that add up to T."""
    cuts = sorted(random.Random(seed).sample(range(1, T), parts - 1)) if parts > 1 else []
    return [0, *cuts, T]


def _frequencies(rot):
    return BASE ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / max(1, rot))


def _weights(g, c, wt):
    one = lambda: _randn(g, (c["D"],), wt, 0.2, 1.0) if c["norm"] else None  # noqa: E731
    return {"w_q": one(), "w_k": one(), "freq": _frequencies(c["rot"])}


def _projection(g, T, c, dtype):
    """Rows as a fused projection leaves them: queries, keys and values of a token side by side."""
    Hq, Hk, D = c["Hq"], c["Hk"], c["D"]
    rows = _randn(g, (T, Hq + 2 * Hk, D), dtype, 1.5)
    return {"q": rows[:, :Hq], "k": rows[:, Hq:Hq + Hk], "v": rows[:, Hq + Hk:]}


def _heads_inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, o, wt = (DTYPES[c[n]] for n in ("x", "out", "weight"))
    s = {**_projection(g, c["T"], c, x), **_weights(g, c, wt)}
    start = random.Random(seed).randrange(1 << 17)
    s["positions"] = torch.arange(start, start + c["T"], dtype=torch.int32, device="cuda")
    if c["op"] == "heads_grad":
        s["dq"], s["dk"] = _randn(g, (c["T"], c["Hq"], c["D"]), o, 0.05), _randn(g, (c["T"], c["Hk"], c["D"]), o, 0.05)
    return s


def _cache(g, c, lengths, tokens, seed):
    """Pages for sequences of these lengths, of up to `tokens` in all, handed out in any order; a table's unused entries hold -1."""
    page, Hk, D, kind = c["page"], c["Hk"], c["D"], DTYPES[c["cache"]]
    need = [-(-n // page) for n in lengths]
    pages = tokens // page + len(lengths) + 2
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((len(lengths), max(1, max(need))), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    s = {"lengths": torch.tensor(lengths, dtype=torch.int32).cuda(), "table": table.cuda(), "k_scale": None, "v_scale": None}
    for n in ("k_cache", "v_cache"):
        s[n] = torch.empty((pages, page, Hk, D), dtype=kind, device="cuda")
        for a in range(0, pages, 4096):
            s[n][a:a + 4096] = _randn(g, s[n][a:a + 4096].shape, torch.float32).to(kind)
    if c["cache"] == "e4m3":
        for n in ("k_scale", "v_scale"):
            s[n] = torch.rand(Hk, generator=g, device="cuda") * 0.5 + 0.5
    return s


def _append_inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    cuts = _cuts(c["T"], c["seqs"], seed)
    r = random.Random(seed)
    lengths = [b - a + r.randint(0, c["past"]) for a, b in zip(cuts, cuts[1:])]
    s = {**_projection(g, c["T"], c, DTYPES[c["x"]]), **_weights(g, c, DTYPES[c["x"]]),
         **_cache(g, c, lengths, c["T"] + c["seqs"] * c["past"], seed)}
    if c["cache"] == "e4m3":
        s["k_scale"], s["v_scale"] = s["k_scale"] * 0.02, s["v_scale"] * 0.02
    # (one new token of every sequence needs no offsets)
    s["offsets"] = None if c["T"] == c["seqs"] else torch.tensor(cuts, dtype=torch.int32).cuda()
    return s


def _attention_inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = random.Random(seed)
    lengths = [r.randint(1, c["longest"]) if c["ragged"] else c["longest"] for _ in range(c["seqs"])]
    s = {"q": _randn(g, (c["seqs"], c["Hq"], c["D"]), DTYPES[c["q"]], 1.5), **_cache(g, c, lengths, sum(lengths), seed)}
    s["sinks"] = torch.randn(c["Hq"], generator=g, device="cuda") * 2 if c["sinks"] else None
    return s


def _inputs(case, seed):
    return {"heads": _heads_inputs, "heads_grad": _heads_inputs, "append": _append_inputs, "attention": _attention_inputs}[case["op"]](
        case, seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = dict(case)
    if own:
        from paper_2604_10496_amd import binding as cq
        if case["op"] != "attention":
            s["norm"] = cq.HeadNorm(case["D"], s["w_q"], s["w_k"], eps=EPS, freq=s["freq"], interleaved=case["interleaved"])
        if "k_cache" in s:
            s["cache"] = cq.PagedCache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s["case"]["op"], s)


def _run_own(op, s):
    from paper_2604_10496_amd import binding as cq
    c = s["case"]
    if op == "heads":
        return cq.cq_head_norm(s["norm"], s["q"], s["k"], s["positions"], out_dtype=DTYPES[c["out"]])
    if op == "heads_grad":
        out = cq.cq_head_norm_grad(s["norm"], s["q"], s["k"], s["positions"], s["dq"], s["dk"])
        return {name: v for name, v in out.items() if v is not None}
    if op == "append":
        q = cq.cq_cache_append(s["cache"], s["k"], s["v"], s["table"], s["lengths"], s["offsets"], norm=s["norm"], q=s["q"])
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    return cq.cq_cache_attention(s["cache"], s["q"], s["table"], s["lengths"], scale=c["D"] ** -0.5, max_length=c["longest"],
                                 window=c["window"], softcap=c["softcap"], sinks=s["sinks"], out_dtype=DTYPES[c["out"]])


def _run_plain(op, s):
    return {"heads": _plain_heads, "heads_grad": _plain_heads_grad, "append": _plain_append, "attention": _plain_attention}[op](s)


def _turn(s, positions):
    """Cosines and sines [T, 1, rot / 2] of the rotation; the angles of far positions need 64 bits."""
    angle = positions.double()[:, None, None] * s["freq"]
    return torch.cos(angle).float(), torch.sin(angle).float()


def _pairs(x, c):
    """The two halves of the rotated values of [T, heads, D], and the values that stay."""
    rot = c["rot"]
    if c["interleaved"]:
        return x[..., 0:rot:2], x[..., 1:rot:2], x[..., rot:]
    return x[..., :rot // 2], x[..., rot // 2:rot], x[..., rot:]


def _unpair(a, b, rest, c):
    both = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([both, rest], -1)


def _plain_norm_turn(x, w, turn, c):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    a, b, rest = _pairs(x, c)
    cos, sin = turn
    return _unpair(a * cos - b * sin, b * cos + a * sin, rest, c)


def _plain_heads(s):
    c = s["case"]
    turn = _turn(s, s["positions"])
    return {n: _plain_norm_turn(s[n], s["w_" + n], turn, c).to(DTYPES[c["out"]]) for n in ("q", "k")}


def _plain_grad(x, w, dy, turn, c):
    x = x.float()
    a, b, rest = _pairs(dy.float(), c)
    cos, sin = turn
    d = _unpair(a * cos + b * sin, b * cos - a * sin, rest, c)
    if w is None:
        return d.to(DTYPES[c["x"]]), None
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    dw = (d * n).sum((0, 1))
    d = d * w.float()
    return (r * (d - n * (d * n).mean(-1, keepdim=True))).to(DTYPES[c["x"]]), dw.to(w.dtype)


def _plain_heads_grad(s):
    c = s["case"]
    turn = _turn(s, s["positions"])
    dq, dw_q = _plain_grad(s["q"], s["w_q"], s["dq"], turn, c)
    dk, dw_k = _plain_grad(s["k"], s["w_k"], s["dk"], turn, c)
    out = {"dq": dq, "dk": dk, "dw_q": dw_q, "dw_k": dw_k}
    return {name: v for name, v in out.items() if v is not None}


def _slots(s):
    """Every new token's position, page and slot in it."""
    page, T = s["case"]["page"], s["k"].shape[0]
    at = torch.arange(T, device="cuda")
    if s["offsets"] is None:
        seq, position = at, s["lengths"].long() - 1
    else:
        off = s["offsets"].long()
        seq = torch.bucketize(at, off[1:-1], right=True)
        position = s["lengths"].long()[seq] - off[seq + 1] + at
    return position, s["table"].long()[seq, position // page], position % page


def _stored(x, scale, kind):
    if scale is not None:
        x = (x / scale[:, None]).clamp(-MOST_E4M3, MOST_E4M3)
    return x.to(kind)


def _plain_append(s):
    c = s["case"]
    position, page, slot = _slots(s)
    turn = _turn(s, position)
    k = _plain_norm_turn(s["k"], s["w_k"], turn, c)
    s["k_cache"][page, slot] = _stored(k, s["k_scale"], DTYPES[c["cache"]])
    s["v_cache"][page, slot] = _stored(s["v"].float(), s["v_scale"], DTYPES[c["cache"]])
    return {"q": _plain_norm_turn(s["q"], s["w_q"], turn, c).to(DTYPES[c["x"]]), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attention(s):
    """All sequences at once, padded to the longest."""
    c = s["case"]
    S, Hq, Hk, D, page = c["seqs"], c["Hq"], c["Hk"], c["D"], c["page"]
    lengths = s["lengths"].long()[:, None]
    at = torch.arange(s["table"].shape[1] * page, device="cuda")[None, :]
    seen = at < lengths
    if c["window"]:
        seen = seen & (at >= lengths - c["window"])
    pages = s["table"].long().clamp(min=0)
    k = s["k_cache"][pages].float().view(S, -1, Hk, D)
    if s["k_scale"] is not None:
        k = k * s["k_scale"][:, None]
    q = s["q"].float().view(S, Hk, Hq // Hk, D)
    z = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) * D ** -0.5
    del k
    if c["softcap"]:
        z = c["softcap"] * torch.tanh(z / c["softcap"])
    z = torch.where(seen[:, None, None, :], z, torch.full((), -math.inf, device="cuda"))
    top = z.amax(-1, keepdim=True)
    sink = None if s["sinks"] is None else s["sinks"].view(1, Hk, Hq // Hk, 1)
    if sink is not None:
        top = torch.maximum(top, sink)
    p = torch.exp(z - top)
    total = p.sum(-1, keepdim=True)
    if sink is not None:
        total = total + torch.exp(sink - top)
    v = s["v_cache"][pages].float().view(S, -1, Hk, D)
    if s["v_scale"] is not None:
        v = v * s["v_scale"][:, None]
    o = torch.matmul(p / total, v.permute(0, 2, 1, 3).contiguous())
    return {"out": o.reshape(S, Hq, D).to(DTYPES[c["out"]]), "lse": (top + torch.log(total)).view(S, Hq)}


# ------------------------------------------------------------------------------------------------
# floors
# ------------------------------------------------------------------------------------------------
def work(c):
    Hq, Hk, D = c["Hq"], c["Hk"], c["D"]
    if c["op"] == "attention":
        # (a ragged batch's sequences are half as long as the longest on the average)
        mean = (c["longest"] + 1) / 2 if c["ragged"] else c["longest"]
        if c["window"]:
            w = min(c["window"], c["longest"])
            mean = w - w * (w - 1) / (2 * c["longest"]) if c["ragged"] else w
        keys = int(c["seqs"] * mean)
        ends = c["seqs"] * Hq * (D * (SIZE[c["q"]] + SIZE[c["out"]]) + 4) + 4 * keys // c["page"]
        return {"bytes": 2 * keys * Hk * D * SIZE[c["cache"]] + ends, "flops": 4 * keys * Hq * D}
    T, x = c["T"], SIZE[c["x"]]
    if c["op"] == "append":
        return {"bytes": T * D * (Hq * 2 * x + 2 * Hk * (x + SIZE[c["cache"]])) + 4 * T, "flops": 8 * T * (Hq + Hk) * D}
    values, weights = T * (Hq + Hk) * D, 2 * D * SIZE[c["weight"]] if c["norm"] else 0
    if c["op"] == "heads":
        return {"bytes": values * (x + SIZE[c["out"]]) + 4 * T + weights, "flops": 8 * values}
    # rows and gradients in, gradients out; without norms the rows are not needed
    return {"bytes": values * ((2 if c["norm"] else 1) * x + SIZE[c["out"]]) + 4 * T + 2 * weights,
            "flops": (20 if c["norm"] else 6) * values}


# ------------------------------------------------------------------------------------------------
# float64
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    """The definitions in float64: rotations as complex products, gradients by differentiating the forward formula, attention
    sequence by sequence."""
    s = _inputs(case, seed)
    return {"heads": _exact_heads, "heads_grad": _exact_heads_grad, "append": _exact_append, "attention": _exact_attention}[case["op"]](
        case, s)


def _exact_head(c, x, w, freq, positions):
    if w is not None:
        x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / c["D"] + EPS) * w
    if c["rot"] == 0:
        return x
    turned, rest = x.split([c["rot"], c["D"] - c["rot"]], dim=-1)
    shape = turned.shape
    if c["interleaved"]:
        z = turned.unflatten(-1, (c["rot"] // 2, 2))
    else:
        z = turned.unflatten(-1, (2, c["rot"] // 2)).transpose(-1, -2)
    angle = torch.outer(positions.double(), freq)
    z = torch.view_as_complex(z.contiguous()) * torch.polar(torch.ones_like(angle), angle).unsqueeze(1)
    z = torch.view_as_real(z)
    if not c["interleaved"]:
        z = z.transpose(-1, -2)
    return torch.cat([z.reshape(shape), rest], -1)


def _double(t):
    return None if t is None else t.double()


def _exact_heads(c, s):
    return {n: _exact_head(c, s[n].double(), _double(s["w_" + n]), s["freq"], s["positions"]) for n in ("q", "k")}


def _exact_heads_grad(c, s):
    out = {}
    for n in ("q", "k"):
        x = s[n].double().requires_grad_()
        leaves = [x]
        if c["norm"]:
            leaves.append(s["w_" + n].double().requires_grad_())
        y = _exact_head(c, x, leaves[1] if c["norm"] else None, s["freq"], s["positions"])
        for name, d in zip(("d" + n, "dw_" + n), torch.autograd.grad((y * s["d" + n].double()).sum(), leaves)):
            out[name] = d
    return {n: out[n] for n in ("dq", "dk", "dw_q", "dw_k") if n in out}


def _exact_append(c, s):
    lengths, table = s["lengths"].tolist(), s["table"].tolist()
    cuts = list(range(c["T"] + 1)) if s["offsets"] is None else s["offsets"].tolist()
    position, page = [], []
    for i, (a, b) in enumerate(zip(cuts, cuts[1:])):
        for t in range(a, b):
            position.append(lengths[i] - (b - t))
            page.append(table[i][position[-1] // c["page"]])
    position = torch.tensor(position, device="cuda")
    page = torch.tensor(page, device="cuda")
    q, k = (_exact_head(c, s[n].double(), _double(s["w_" + n]), s["freq"], position) for n in ("q", "k"))
    out = {"q": q}
    for n, x in (("k", k), ("v", s["v"].double())):
        whole = s[n + "_cache"].double()
        if c["cache"] == "e4m3":
            x = torch.clamp(x / s[n + "_scale"].double().view(1, -1, 1), -MOST_E4M3, MOST_E4M3)
        whole.view(-1, c["Hk"], c["D"])[page * c["page"] + position % c["page"]] = x
        out[n + "_cache"] = whole
    return out


def _exact_attention(c, s):
    S, Hq, Hk, D, page = c["seqs"], c["Hq"], c["Hk"], c["D"], c["page"]
    outs, sums = [], []
    for i, n in enumerate(s["lengths"].tolist()):
        first = max(0, n - c["window"]) if c["window"] else 0
        at = torch.arange(first, n, device="cuda")
        rows = s["table"][i].long()[at // page], at % page
        k, v = (s[x + "_cache"][rows].double() for x in ("k", "v"))            # [n, Hk, D]
        if c["cache"] == "e4m3":
            k, v = k * s["k_scale"].double().view(1, Hk, 1), v * s["v_scale"].double().view(1, Hk, 1)
        q = s["q"][i].double().view(Hk, Hq // Hk, D)
        z = torch.bmm(q, k.permute(1, 2, 0).contiguous()) / math.sqrt(D)
        if c["softcap"]:
            z = torch.tanh(z / c["softcap"]) * c["softcap"]
        all_z = z if s["sinks"] is None else torch.cat([z, s["sinks"].double().view(Hk, -1, 1)], -1)
        lse = torch.logsumexp(all_z, -1)
        outs.append(torch.bmm(torch.exp(z - lse.unsqueeze(-1)), v.permute(1, 0, 2).contiguous()).view(Hq, D))
        sums.append(lse.view(Hq))
    return {"out": torch.stack(outs), "lse": torch.stack(sums)}
