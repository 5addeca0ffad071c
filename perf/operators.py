"""Performance cases of the operators that stand around the MoE expert layer in a model.

A block of a model is  norm -> layer -> gate, norm and residual -> norm of the next block.  Its operators:

  norm           cq_block_norm: residual stream and next block's input from the block's output, one pass
  norm_grad      cq_block_norm_grad: the gradients of the above, those of gates and weights among them
  balance        cq_balance_loss: load-balancing loss of the router, per-expert counts, mean probabilities, by sequence
  balance_grad   cq_balance_loss_grad: its gradient with respect to the router's logits
  adapter        cq_adapter_apply: every request's own low-rank adapter beside a projection that all of them share

  listed()               the cases that are always timed
  draw(rng)              one more case of the same ranges
  prepare(case, seed)    inputs on the GPU
  run(state)             one call: in plain torch operations, or (own) by the library
  work(case)             bytes and operations that it cannot do without
  exact(case, seed)      what run returns, in float64
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6
ALPHA = 1e-2

# the dearest of each kind that is drawn: no more than the largest listed one
MAX_NORM = 4096 * 4096            # values of the residual stream (of up to 32 bits; the largest listed one has twice as many of 16)
MAX_LOGITS = 65536 * 128          # router logits
MAX_ADAPTER_IO = 4096 * 8192      # values of the projection's rows, input and output
MAX_ADAPTER_W = 64 * 64 * 8192    # values of all adapters


def _norm(op, T, H, stream, block, weight, post, gate, sigmoid, name=None):
    """gate: none, row (one per token) or elem (one per value); post: a norm on the block's output."""
    c = {"op": op, "T": T, "H": H, "stream": stream, "block": block, "weight": weight, "post": post, "gate": gate,
         "sigmoid": sigmoid}
    return {"name": name, **c} if name else c


def _balance(op, T, E, k, seqs, padded, logits, name=None):
    """padded: every sequence ends in tokens that are left out."""
    c = {"op": op, "T": T, "E": E, "k": k, "seqs": seqs, "padded": padded, "logits": logits}
    return {"name": name, **c} if name else c


def _adapter(T, K, N, rank, adapters, requests, ragged, x, w, out, name=None):
    """Request i uses adapter i % adapters, every eighth none; ragged: ranks of rank, rank / 2 and rank / 4."""
    c = {"op": "adapter", "T": T, "K": K, "N": N, "rank": rank, "adapters": adapters, "requests": requests,
         "ragged": ragged, "x": x, "w": w, "out": out}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one token of one user through a Mixtral-shaped block: launch and latency
        _norm("norm", 1, 4096, "bf16", "f32", "bf16", False, "none", False, "norm-token"),
        # a prefill of the same width with norms on both sides and a gate per token; the layer takes and gives fp32
        _norm("norm", 4096, 4096, "bf16", "f32", "f32", True, "row", True, "norm-prefill"),
        # an odd width and batch with a gate per value, all fp16
        _norm("norm", 515, 1111, "f16", "f16", "f16", True, "elem", False, "norm-odd"),
        # a training step at the width of the DeepSeek-V2-Lite and Qwen3 shapes
        _norm("norm_grad", 2048, 2048, "bf16", "bf16", "f32", True, "row", True, "norm_grad-2048"),
        # the largest: a long training batch with a gate per value
        _norm("norm_grad", 8192, 4096, "bf16", "bf16", "bf16", True, "elem", False, "norm_grad-8192"),
        # the tiny layer's router
        _balance("balance", 64, 4, 2, 1, False, "f32", "balance-64x4"),
        # the DeepSeek-V2-Lite router over sequences of different lengths, each balanced by itself
        _balance("balance", 8192, 64, 6, 13, True, "f32", "balance-8192x64"),
        # the same router's gradient in a small step, and the Qwen3 router's over a long batch
        _balance("balance_grad", 512, 64, 6, 3, True, "f32", "balance_grad-512x64"),
        _balance("balance_grad", 65536, 128, 8, 1, False, "f32", "balance_grad-65536x128"),
        # one token of one request beside a 4096 x 4096 projection
        _adapter(1, 4096, 4096, 16, 8, 1, False, "f32", "bf16", "f32", "adapter-token"),
        # a decode step of 64 requests with adapters of their own beside a shared expert's gate/up product
        _adapter(64, 2048, 2816, 64, 64, 64, True, "bf16", "bf16", "f32", "adapter-decode"),
        # a prefill of a few prompts
        _adapter(4096, 4096, 4096, 32, 8, 9, False, "bf16", "bf16", "bf16", "adapter-prefill"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "balance", "balance_grad", "adapter"])
    if op in ("norm", "norm_grad"):
        H = rng.choice([_log(rng, 64, 8192), 64 * _log(rng, 1, 128), 2048, 4096])
        T = _log(rng, 1, min(8192, MAX_NORM // H))
        stream = rng.choice(["f32", "f16", "bf16", "bf16"])
        return _norm(op, T, H, stream, rng.choice(["f32", stream]), rng.choice(["f32", stream]), rng.random() < 0.5,
                     rng.choice(["none", "row", "elem"]), rng.random() < 0.5)
    if op in ("balance", "balance_grad"):
        E = rng.choice([_log(rng, 2, 512), 8, 64, 128])
        T = _log(rng, 1, min(65536, MAX_LOGITS // E))
        return _balance(op, T, E, rng.randint(1, max(1, min(8, E // 2))), rng.choice([1, _log(rng, 1, min(T, 64))]),
                        rng.random() < 0.5, rng.choice(["f32", "f32", "bf16", "f16"]))
    K, N = (rng.choice([_log(rng, 64, 8192), 64 * _log(rng, 1, 128)]) for _ in range(2))
    rank = rng.choice([4, 8, 16, 32, 64, _log(rng, 1, 128)])
    adapters = _log(rng, 1, max(1, min(64, MAX_ADAPTER_W // (rank * (K + N)))))
    T = _log(rng, 1, max(1, min(8192, MAX_ADAPTER_IO // (K + N))))
    requests = T if T <= 256 and rng.random() < 0.5 else _log(rng, 1, min(T, 64))
    x = rng.choice(["f32", "f16", "bf16", "bf16"])
    w = rng.choice([x, "bf16"]) if x == "f32" else x
    return _adapter(T, K, N, rank, adapters, requests, rng.random() < 0.5, x, w, rng.choice(["f32", x]))


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _randn(g, shape, dtype, scale=1.0, mean=0.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale + mean).to(dtype)


def _cuts(T, parts, seed):
    """parts lengths of at least one that add up to T."""
    g = torch.Generator().manual_seed(seed)
    cuts = (torch.randperm(T - 1, generator=g)[:parts - 1] + 1).sort().values.tolist() if parts > 1 else []
    return [0, *cuts, T]


def _norm_inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, H = c["T"], c["H"]
    st, bl, wt = DTYPES[c["stream"]], DTYPES[c["block"]], DTYPES[c["weight"]]
    channel = torch.ones(H, device="cuda")
    channel[torch.randperm(H, generator=g, device="cuda")[:max(1, H // 512)]] = 20.0   # the stream's outlier channels
    s = {"h": (torch.randn((T, H), generator=g, device="cuda") * channel).to(st), "y": _randn(g, (T, H), bl, 0.7),
         "w_pre": _randn(g, (H,), wt, 0.2, 1.0), "w_post": _randn(g, (H,), wt, 0.2, 1.0) if c["post"] else None}
    s["gate"] = {"none": None, "row": (T,), "elem": (T, H)}[c["gate"]]
    if s["gate"] is not None:
        s["gate"] = _randn(g, s["gate"], bl, 1.0, 0.3)
    s["rho"], s["beta"] = 0.9, 1.25
    if c["op"] == "norm_grad":
        s["dh"], s["dx"] = _randn(g, (T, H), st, 0.05), _randn(g, (T, H), bl, 0.05)
    return s


def _balance_inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, E = c["T"], c["E"]
    z = torch.randn((T, E), generator=g, device="cuda") + torch.randn(E, generator=g, device="cuda")
    z = z.to(DTYPES[c["logits"]])
    cuts = _cuts(T, c["seqs"], seed)
    mask = None
    if c["padded"]:
        host = torch.ones(T, dtype=torch.bool)
        for a, b in zip(cuts, cuts[1:]):
            host[b - (b - a) // 5:b] = False
        mask = host.cuda()
    s = {"z": z, "ids": z.float().topk(c["k"], dim=1).indices.to(torch.int32),
         "offsets": torch.tensor(cuts, dtype=torch.int32).cuda(), "mask": mask}
    if c["op"] == "balance_grad":
        # counts and tokens as the forward pass leaves them
        seq = torch.bucketize(torch.arange(T, device="cuda"), s["offsets"][1:-1].long(), right=True)
        keep = torch.ones(T, dtype=torch.bool, device="cuda") if mask is None else mask
        slot = (seq[:, None] * E + s["ids"].long())[keep].reshape(-1)
        s["counts"] = torch.bincount(slot, minlength=c["seqs"] * E).view(c["seqs"], E).to(torch.int32)
        n = torch.bincount(seq[keep], minlength=c["seqs"]).to(torch.int32)
        s["tokens"] = torch.cat([n, (n > 0).sum().to(torch.int32)[None]])
        s["dloss"] = torch.rand(1, generator=g, device="cuda") + 0.5
    return s


def _adapter_inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, K, N, R, M = c["T"], c["K"], c["N"], c["rank"], c["adapters"]
    x, w, o = DTYPES[c["x"]], DTYPES[c["w"]], DTYPES[c["out"]]
    cuts = _cuts(T, c["requests"], seed)
    ids = torch.empty(T, dtype=torch.int32)
    for i, (a, b) in enumerate(zip(cuts, cuts[1:])):
        ids[a:b] = -1 if i % 8 == 7 else i % M
    ranks = torch.tensor([max(1, R >> (a % 3)) for a in range(M)], dtype=torch.int32).cuda() if c["ragged"] else None
    return {"X": _randn(g, (T, K), x), "ids": ids.cuda(), "A": _randn(g, (M, R, K), w, K ** -0.5),
            "B": _randn(g, (M, N, R), w, 0.1), "scale": torch.rand(M, generator=g, device="cuda") + 0.5, "ranks": ranks,
            "base": _randn(g, (T, N), o)}


def _inputs(case, seed):
    return {"n": _norm_inputs, "b": _balance_inputs, "a": _adapter_inputs}[case["op"][0]](case, seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = dict(case)
    if own:
        from paper_2604_10496_amd import binding as cq
        if "norm" in case["op"]:
            s["norm"] = cq.BlockNorm(s["w_pre"], s["w_post"], eps=EPS, residual_scale=s["rho"], branch_scale=s["beta"],
                                     gate_sigmoid=case["sigmoid"], block_dtype=DTYPES[case["block"]])
        elif case["op"] == "adapter":
            s["adapters"] = cq.DeviceAdapters(s["A"], s["B"], s["scale"], s["ranks"])
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s["case"]["op"], s)


def _run_own(op, s):
    from paper_2604_10496_amd import binding as cq
    if op == "norm":
        return cq.cq_block_norm(s["norm"], s["h"], s["y"], s["gate"])
    if op == "norm_grad":
        out = cq.cq_block_norm_grad(s["norm"], s["h"], s["y"], s["gate"], dh=s["dh"], dx=s["dx"])
        return {name: v for name, v in out.items() if v is not None}
    if op == "balance":
        return cq.cq_balance_loss(s["z"], s["ids"], ALPHA, s["offsets"], s["mask"])
    if op == "balance_grad":
        return cq.cq_balance_loss_grad(s["z"], s["counts"], s["tokens"], s["case"]["k"], ALPHA, s["offsets"], s["mask"],
                                       s["dloss"])
    return cq.cq_adapter_apply(s["adapters"], s["X"], s["ids"], base=s["base"])


def _run_plain(op, s):
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "balance": _plain_balance,
            "balance_grad": _plain_balance_grad, "adapter": _plain_adapter}[op](s)


def _gate(s):
    """The gate as a factor of [T, H] values, None without one."""
    if s["gate"] is None:
        return None
    a = s["gate"].float()
    if s["case"]["sigmoid"]:
        a = 1.0 / (1.0 + torch.exp(-a))
    return a[:, None] if a.dim() == 1 else a


def _plain_norm(s):
    c = s["case"]
    u = s["y"].float()
    if s["w_post"] is not None:
        u = u * torch.rsqrt((u * u).mean(1, keepdim=True) + EPS) * s["w_post"].float()
    a = _gate(s)
    h = s["rho"] * s["h"].float() + s["beta"] * (u if a is None else a * u)
    x = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["w_pre"].float()
    return {"h": h.to(DTYPES[c["stream"]]), "x": x.to(DTYPES[c["block"]])}


def _plain_norm_grad(s):
    """s["h"] is the residual stream that the forward pass wrote."""
    c = s["case"]
    st, bl, wt = DTYPES[c["stream"]], DTYPES[c["block"]], DTYPES[c["weight"]]
    h, dx = s["h"].float(), s["dx"].float()
    r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    n = h * r
    dn = dx * s["w_pre"].float()
    total = s["dh"].float() + r * (dn - n * (dn * n).mean(1, keepdim=True))
    out = {"dh": (s["rho"] * total).to(st), "dw_pre": (dx * n).sum(0).to(wt)}
    e = s["beta"] * total
    y = s["y"].float()
    if s["w_post"] is not None:
        q = torch.rsqrt((y * y).mean(1, keepdim=True) + EPS)
        m = y * q
        u = m * s["w_post"].float()
    else:
        u = y
    a = _gate(s)
    if a is not None:
        da = e * u
        if c["gate"] == "row":
            da = da.sum(1, keepdim=True)
        if c["sigmoid"]:
            da = da * a * (1.0 - a)
        out["dgate"] = (da[:, 0] if c["gate"] == "row" else da).to(bl)
        e = a * e
    if s["w_post"] is not None:
        out["dw_post"] = (e * m).sum(0).to(wt)
        dm = e * s["w_post"].float()
        e = q * (dm - m * (dm * m).mean(1, keepdim=True))
    out["dy"] = e.to(bl)
    return out


def _sequences(s):
    """Every token's sequence, and which tokens count."""
    T = s["z"].shape[0]
    seq = torch.bucketize(torch.arange(T, device="cuda"), s["offsets"][1:-1].long(), right=True)
    keep = torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"]
    return seq, keep


def _softmax(z):
    p = torch.exp(z - z.amax(1, keepdim=True))
    return p / p.sum(1, keepdim=True)


def _plain_balance(s):
    c = s["case"]
    S, E = c["seqs"], c["E"]
    seq, keep = _sequences(s)
    member = (seq[None, :] == torch.arange(S, device="cuda")[:, None]) & keep[None, :]
    n = member.sum(1)
    hot = torch.zeros((c["T"], E), dtype=torch.float64, device="cuda").scatter_(1, s["ids"].long(), 1.0)
    counts = member.double() @ hot            # (whole numbers)
    probs = (member.double() @ _softmax(s["z"].float()).double()) / n.clamp(min=1)[:, None]
    used = (n > 0).sum()
    f = counts / (c["k"] * n.clamp(min=1))[:, None]
    loss = ALPHA * E * (f * probs).sum() / used.clamp(min=1)
    return {"loss": loss.float().view(1), "counts": counts.to(torch.int32), "probs": probs.float(),
            "tokens": torch.cat([n, used[None]]).to(torch.int32)}


def _plain_balance_grad(s):
    c = s["case"]
    seq, keep = _sequences(s)
    n = s["tokens"][:-1].float().clamp(min=1)
    f = s["counts"].float() / (c["k"] * n)[:, None]
    p = _softmax(s["z"].float())
    ft = f[seq]
    w = s["dloss"] * ALPHA * c["E"] / (s["tokens"][-1].float().clamp(min=1) * n)
    d = w[seq][:, None] * p * (ft - (ft * p).sum(1, keepdim=True))
    return torch.where(keep[:, None], d, torch.zeros((), device="cuda")).to(s["z"].dtype)


def _plain_adapter(s):
    """All adapters' products at once, with those of other requests' adapters left out."""
    c = s["case"]
    M, R, K, N = c["adapters"], c["rank"], c["K"], c["N"]
    v = (s["X"].float() @ s["A"].float().view(M * R, K).t()).view(-1, M, R)
    mine = s["ids"][:, None, None] == torch.arange(M, device="cuda")[None, :, None]
    if s["ranks"] is not None:
        mine = mine & (torch.arange(R, device="cuda")[None, None, :] < s["ranks"][None, :, None])
    v = torch.where(mine, v * s["scale"][None, :, None], torch.zeros((), device="cuda"))
    y = v.view(-1, M * R) @ s["B"].float().permute(0, 2, 1).reshape(M * R, N)
    return (s["base"].float() + y).to(DTYPES[c["out"]])


# ------------------------------------------------------------------------------------------------
# floors
# ------------------------------------------------------------------------------------------------
def work(c):
    T = c["T"]
    if "norm" in c["op"]:
        H = c["H"]
        st, bl, wt = (SIZE[c[x]] for x in ("stream", "block", "weight"))
        gate = {"none": 0, "row": T, "elem": T * H}[c["gate"]] * bl
        weights = H * wt * (2 if c["post"] else 1)
        if c["op"] == "norm":   # h, y and gate in, h' and x out
            return {"bytes": T * H * 2 * (st + bl) + gate + weights, "flops": T * H * (12 if c["post"] else 8)}
        # h', its gradient, the input's gradient, y and gate in; gradients of h, y and gate out
        return {"bytes": T * H * (3 * st + 3 * bl) + 2 * gate + 2 * weights, "flops": T * H * (30 if c["post"] else 16)}
    if "balance" in c["op"]:
        E, S, z = c["E"], c["seqs"], SIZE[c["logits"]]
        side = T * (1 if c["padded"] else 0) + S * E * 4
        if c["op"] == "balance":
            return {"bytes": T * E * z + T * c["k"] * 4 + side + S * E * 4, "flops": 5 * T * E}
        return {"bytes": 2 * T * E * z + side, "flops": 9 * T * E}
    K, N, R = c["K"], c["N"], c["rank"]
    used = sorted({i % c["adapters"] for i in range(c["requests"]) if i % 8 != 7})
    ranks = [max(1, R >> (a % 3)) if c["ragged"] else R for a in used]
    x, w, o = (SIZE[c[n]] for n in ("x", "w", "out"))
    mean = sum(ranks) / max(1, len(ranks))
    return {"bytes": T * K * x + sum(ranks) * (K + N) * w + 2 * T * N * o + T * 4, "flops": int(2 * T * mean * (K + N))}


# ------------------------------------------------------------------------------------------------
# float64
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    """The definitions in float64; gradients by differentiating the forward formula."""
    s = _inputs(case, seed)
    return {"n": _exact_norm, "b": _exact_balance, "a": _exact_adapter}[case["op"][0]](case, s)


def _exact_rms(v, w):
    return w * v / torch.sqrt(v.pow(2).sum(-1, keepdim=True) / v.shape[-1] + EPS)


def _exact_norm(c, s):
    d = {k: v.double() for k, v in s.items() if torch.is_tensor(v)}

    def branch(y, gate, w_post):
        u = y if w_post is None else _exact_rms(y, w_post)
        if gate is not None:
            a = torch.sigmoid(gate) if c["sigmoid"] else gate
            u = u * (a.unsqueeze(-1) if a.dim() == 1 else a)
        return s["beta"] * u
    if c["op"] == "norm":
        h = branch(d["y"], d.get("gate"), d.get("w_post")) + s["rho"] * d["h"]
        return {"h": h, "x": _exact_rms(h, d["w_pre"])}
    # h' is given: the gradient that reaches it goes on to h by rho and to the branch as it is
    h, w_pre = d["h"].requires_grad_(), d["w_pre"].requires_grad_()
    x = _exact_rms(h, w_pre)
    through, dw_pre = torch.autograd.grad((x * d["dx"]).sum(), [h, w_pre])
    total = through + d["dh"]
    leaves = {k: d[k].requires_grad_() for k in ("y", "gate", "w_post") if k in d}
    grads = torch.autograd.grad((branch(leaves["y"], leaves.get("gate"), leaves.get("w_post")) * total).sum(),
                                list(leaves.values()))
    out = {"dh": s["rho"] * total, "dw_pre": dw_pre}
    out.update({"d" + k: v for k, v in zip(leaves, grads)})
    # (laid out as run lays them out)
    return {k: out[k].detach() for k in ("dh", "dw_pre", "dgate", "dw_post", "dy") if k in out}


def _exact_balance(c, s):
    E, k = c["E"], c["k"]
    z = s["z"].double().requires_grad_()
    cuts = s["offsets"].tolist()
    keep = s["mask"].tolist() if s["mask"] is not None else [True] * c["T"]
    loss, rows, probs, tokens = z.sum() * 0.0, [], [], []
    for a, b in zip(cuts, cuts[1:]):
        at = torch.tensor([t for t in range(a, b) if keep[t]], dtype=torch.long, device="cuda")
        tokens.append(len(at))
        p = torch.log_softmax(z[at], dim=1).exp().sum(0) / max(1, len(at))
        cnt = (s["ids"][at].reshape(-1, 1) == torch.arange(E, device="cuda")).sum(0)
        loss = loss + E * (cnt.double() / (k * max(1, len(at))) * p).sum()
        rows.append(cnt)
        probs.append(p.detach())
    used = sum(n > 0 for n in tokens)
    loss = ALPHA * loss / max(1, used)
    if c["op"] == "balance":
        return {"loss": loss.detach().view(1), "counts": torch.stack(rows).to(torch.int32), "probs": torch.stack(probs),
                "tokens": torch.tensor(tokens + [used], dtype=torch.int32).cuda()}
    (dz,) = torch.autograd.grad(loss * s["dloss"].double().view(()), [z])
    return dz


def _exact_adapter(c, s):
    out = s["base"].double()
    for a in range(c["adapters"]):
        at = (s["ids"] == a).nonzero().view(-1)
        r = c["rank"] if s["ranks"] is None else int(s["ranks"][a])
        low = torch.matmul(s["A"][a, :r].double(), s["X"][at].double().t().contiguous())       # [r, tokens]
        out[at] += float(s["scale"][a].double()) * torch.matmul(s["B"][a, :, :r].double().contiguous(), low).t()
    return out
