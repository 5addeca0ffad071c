"""Heads with norm and rotation, the paged cache, and attention of single tokens, against the float64 oracle.

Bounds.  A rounding costs half a step: H(t) = 2^-8 (bf16), 2^-11 (f16), 2^-24 (fp32), 2^-4 (e4m3) of the value, counted against the
magnitudes (sums of |terms|) that the oracle returns.  U = 2^-24.
  heads: a sum of 256 squares, 8 in a lane, then a tree of at most 6: 14 U, halved by the root, 3 for root, quotient and eps; two
    products; an angle that is off by 2^-25 of a half revolution and sine and cosine by 2 U: 6; a product and a sum: under 32 U of the pair's
    magnitude |a| + |b| (which an error of the angle is counted against), then the output's rounding.
  gradients: the same for the rotation; two row sums, three products: under 64 U of the magnitude; a weight's gradient adds up to N rows one after
    another and a tree: (64 + N) U of the sum of |terms|.
  attention: scores are off by dz = (D + 16) U sum |q| |k| scale + 8 U |z| (fp32 sums, factor, log2 e) + 2^-22 sum |q| |k| scale (queries in
    parts); weights by 2 dz and 2^-16 (two parts of 8 bits and the exponential), sums over n positions by (n / 8 + 64) U: together of
    sum p |v|.  lse: dz + (n / 8 + 64) U + 2 U |lse|.
"""
import numpy as np
import pytest

from oracle import heads_oracle as O

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8, "e4m3": 2.0 ** -4}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -133, "e4m3": 2.0 ** -10}


@pytest.fixture(scope="module")
def cq():
    import torch  # noqa: F401
    from paper_2604_10496_amd import binding
    return binding


def _t(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[name]


def _np(x):
    return None if x is None else x.double().cpu().numpy()


def _close(got, ref, mag, rel, kind, what):
    err, bar = np.abs(_np(got) - ref), rel * mag + HALF[kind] * (np.abs(ref) + rel * mag) + TINY[kind]
    assert np.isfinite(_np(got)).all(), what
    worst = (err / bar).max() if err.size else 0
    assert worst <= 1, f"{what}: {worst:.3g} of the bound"


def _freq(rot, base=1e4):
    import torch
    return base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1)).cuda() if rot else None


def _rows(g, T, n, D, kind, scale=1.5):
    import torch
    return (torch.randn((T, n, D), generator=g) * scale).to(_t(kind)).cuda()


SHAPES = [  # D, rot, interleaved
    (128, 128, False), (64, 32, True), (80, 20, True), (80, 20, False), (1, 0, False), (7, 2, False), (33, 10, True), (256, 256, False),
    (256, 2, False), (250, 6, True), (96, 96, True), (2, 2, False), (13, 12, False), (128, 0, False), (8, 2, False),
    (9, 6, False), (9, 6, True), (15, 8, False), (15, 10, True), (20, 18, False), (200, 198, False), (255, 30, True), (254, 12, False)]
KINDS = [("bf16", "bf16", "bf16"), ("f16", "f16", "f32"), ("f32", "f32", "f32"), ("f32", "bf16", "bf16"), ("f32", "f16", "f16"),
         ("bf16", "bf16", "f32")]


def _norm(cq, g, D, rot, inter, weight, q=True, k=True, scale=1.0):
    import torch
    w = lambda on: (torch.randn(D, generator=g) * 0.3 + 1).to(_t(weight)).cuda() if on else None  # noqa: E731
    return cq.HeadNorm(D, w(q), w(k), eps=1e-5, freq=_freq(rot), interleaved=inter, rot_scale=scale)


def _ref(norm, x, w, pos, dy=None):
    freq = np.zeros(0) if norm.freq is None else _np(norm.freq)
    if dy is None:
        return O.head_norm(_np(x), _np(w), norm.eps, freq, norm.interleaved, norm.rot_scale, pos)
    return O.head_norm_grad(_np(x), _np(w), _np(dy), norm.eps, freq, norm.interleaved, norm.rot_scale, pos)


@pytest.mark.parametrize("D,rot,inter", SHAPES)
@pytest.mark.parametrize("kind,out,weight", KINDS)
def test_head_norm_and_gradients(cq, D, rot, inter, kind, out, weight):
    import torch
    g = torch.Generator().manual_seed(D + rot)
    T, Hq, Hk = 5, 6, 3
    norm = _norm(cq, g, D, rot, inter, weight, scale=1.25 if D == 96 else 1.0)
    rows = _rows(g, T, Hq + 2 * Hk, D, kind)
    q, k = rows[:, :Hq], rows[:, Hq:Hq + Hk]          # slices of a fused projection
    pos = [0, 1, 70001, -3, 2 ** 31 - 1]
    positions = torch.tensor(pos, dtype=torch.int32).cuda() if rot else None
    got = cq.cq_head_norm(norm, q, k, positions, out_dtype=_t(out))
    for n, x, w in (("q", q, norm.w_q), ("k", k, norm.w_k)):
        ref, mag = _ref(norm, x, w, pos)
        assert got[n].dtype == _t(out)
        _close(got[n], ref, mag, 32 * U, out, n)
    dq, dk = _rows(g, T, Hq, D, out, 0.1), _rows(g, T, Hk, D, out, 0.1)
    grads = cq.cq_head_norm_grad(norm, q, k, positions, dq, dk)
    for n, x, w, dy in (("q", q, norm.w_q, dq), ("k", k, norm.w_k, dk)):
        dx, dw, mx, mw = _ref(norm, x, w, pos, dy)
        _close(grads["d" + n], dx, mx, 64 * U, kind, "d" + n)
        _close(grads["dw_" + n], dw, mw, (64 + T * x.shape[1]) * U, weight, "dw_" + n)


@pytest.mark.parametrize("T,Hq,Hk", [(1, 1, 1), (12, 32, 8), (13, 32, 8), (40, 3, 1), (1, 71, 1), (2, 32, 8), (300, 5, 0), (0, 3, 1), (4099, 2, 1),
                                     (700, 0, 16)])
@pytest.mark.parametrize("norms", [(True, True), (True, False), (False, True), (False, False)])
def test_batches_heads_and_missing_norms(cq, T, Hq, Hk, norms):
    import torch
    g = torch.Generator().manual_seed(T + Hq)
    D, rot = 64, 48
    norm = _norm(cq, g, D, rot, False, "f32", *norms)
    q, k = (_rows(g, T, n, D, "bf16") if n else None for n in (Hq, Hk))
    pos = np.arange(T) * 3 + 5
    positions = torch.from_numpy(pos.astype(np.int32)).cuda()
    got = cq.cq_head_norm(norm, q, k, positions)
    dq, dk = (None if x is None else _rows(g, T, x.shape[1], D, "bf16", 0.1) for x in (q, k))
    grads = cq.cq_head_norm_grad(norm, q, k, positions, dq, dk)
    for n, x, w, dy in (("q", q, norm.w_q, dq), ("k", k, norm.w_k, dk)):
        if x is None:
            assert got[n] is None and grads["d" + n] is None and grads["dw_" + n] is None
            continue
        ref, mag = _ref(norm, x, w, pos)
        _close(got[n], ref, mag, 32 * U, "bf16", n)
        dx, dw, mx, mw = _ref(norm, x, w, pos, dy)
        _close(grads["d" + n], dx, mx, 64 * U, "bf16", "d" + n)
        if w is None:
            assert grads["dw_" + n] is None
        else:
            _close(grads["dw_" + n], dw, mw, (64 + T * x.shape[1]) * U, "f32", "dw_" + n)


def test_gradients_match_differences(cq):
    """The gradient along a direction against a central difference of the forward pass in fp32: step h = 2^-6 leaves h^2 / 6 of the third
    derivative and 32 U / h of the sum's magnitude from the roundings; both are under 2^-9 of the sum of |terms| here (rows of size 1, direction
    of size 1: the norm's third derivative is under 15)."""
    import torch
    g = torch.Generator().manual_seed(9)
    T, n, D = 4, 3, 32
    norm = _norm(cq, g, D, 16, False, "f32", True, False)
    x, c, d = (_rows(g, T, n, D, "f32", 1.0) for _ in range(3))
    pos = torch.arange(T, dtype=torch.int32).cuda()
    f = lambda x: (cq.cq_head_norm(norm, x, None, pos)["q"].double() * c.double()).sum().item()  # noqa: E731
    h = 2.0 ** -6
    grad = cq.cq_head_norm_grad(norm, x, None, pos, c)
    want = (f(x + h * d) - f(x - h * d)) / (2 * h)
    terms = grad["dq"].double() * d.double()
    assert abs(terms.sum().item() - want) <= 2.0 ** -9 * terms.abs().sum().item()
    w, dw = norm.w_q, torch.randn(D, generator=g).cuda()
    norm.w_q = w + h * dw
    up = f(x)
    norm.w_q = w - h * dw
    want = (up - f(x)) / (2 * h)      # (linear in the weights: no third derivative)
    terms = grad["dw_q"].double() * dw.double()
    assert abs(terms.sum().item() - want) <= 2.0 ** -9 * terms.abs().sum().item()


def test_in_place_broadcast_and_unaligned_rows(cq):
    import torch
    g = torch.Generator().manual_seed(1)
    D = 80
    norm = _norm(cq, g, D, 40, False, "bf16")
    wide = _rows(g, 7, 4, D + 3, "bf16")
    q = wide[:, :3, 3:]                                        # rows that start on odd elements
    k = wide[:, 3:, :D]
    pos = torch.arange(7, dtype=torch.int32).cuda()
    want = cq.cq_head_norm(norm, q.contiguous(), k.contiguous(), pos)
    before = wide.clone()
    got = cq.cq_head_norm(norm, q, k, pos, q_out=q, k_out=k)
    assert got["q"] is q and torch.equal(q, want["q"]) and torch.equal(k, want["k"])
    assert torch.equal(wide[:, :3, :3], before[:, :3, :3]) and torch.equal(wide[:, 3:, D:], before[:, 3:, D:])
    one = _rows(g, 1, 1, D, "bf16")
    many = cq.cq_head_norm(norm, one.expand(7, 3, D), None, pos)["q"]     # one row for all tokens and heads
    assert torch.equal(many, cq.cq_head_norm(norm, one.expand(7, 3, D).contiguous(), None, pos)["q"])
    dy = _rows(g, 7, 3, D, "bf16")
    a, b = (cq.cq_head_norm_grad(norm, x, None, pos, dy) for x in (one.expand(7, 3, D), one.expand(7, 3, D).contiguous()))
    assert torch.equal(a["dq"], b["dq"]) and torch.equal(a["dw_q"], b["dw_q"])
    with pytest.raises(ValueError, match="overlap"):
        cq.cq_head_norm(norm, dy, None, pos, q_out=one.expand(7, 3, D))


def test_special_rows(cq):
    """Rows of zeros, infinities and NaN stay their own affair."""
    import torch
    g = torch.Generator().manual_seed(2)
    norm = _norm(cq, g, 64, 64, False, "f32")
    q = _rows(g, 4, 5, 64, "f32")
    q[0, 1] = 0
    q[1, 2, 3] = float("inf")
    q[2, 0, 60] = float("nan")
    pos = torch.arange(4, dtype=torch.int32).cuda()
    got = cq.cq_head_norm(norm, q, None, pos)["q"]
    assert not got[0, 1].any() and torch.isnan(got[1, 2]).any() and torch.isnan(got[2, 0]).all()
    rest = torch.ones(4, 5, dtype=torch.bool)
    rest[1, 2] = rest[2, 0] = False
    ref, mag = _ref(norm, torch.nan_to_num(q, 0, 0, 0), norm.w_q, range(4))
    _close(got[rest.cuda()], ref[rest.numpy()], mag[rest.numpy()], 32 * U, "f32", "rows beside special ones")


def test_rows_beyond_32_bit_offsets(cq):
    import torch
    g = torch.Generator().manual_seed(3)
    D, T, step = 64, 5, (1 << 29) + 8
    buf = torch.zeros(step * (T - 1) + 2 * D, dtype=torch.bfloat16, device="cuda")
    q = buf.as_strided((T, 2, D), (step, D, 1))
    q.copy_(_rows(g, T, 2, D, "bf16"))
    norm = _norm(cq, g, D, 64, False, "f32")
    pos = torch.arange(T, dtype=torch.int32).cuda()
    want = cq.cq_head_norm(norm, q.contiguous(), None, pos)["q"]
    dy = _rows(g, T, 2, D, "bf16")
    a, b = (cq.cq_head_norm_grad(norm, x, None, pos, dy) for x in (q, q.contiguous()))
    assert torch.equal(a["dq"], b["dq"]) and torch.equal(a["dw_q"], b["dw_q"])
    cq.cq_head_norm(norm, q, None, pos, q_out=q)
    assert torch.equal(q, want)


def test_batches_beyond_one_launch(cq):
    """2^25 + 5 tokens: a launch has 2^31 threads, 64 for each.  Against the same rows in two calls."""
    import torch
    T, D = (1 << 25) + 5, 8
    x = torch.randn((T, 1, D), device="cuda", dtype=torch.bfloat16)
    norm = _norm(cq, torch.Generator().manual_seed(4), D, D, False, "f32")
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    got = cq.cq_head_norm(norm, x, None, pos)["q"]
    half = T // 2
    for a, b in ((0, half), (half, T)):
        assert torch.equal(got[a:b], cq.cq_head_norm(norm, x[a:b], None, pos[a:b])["q"])
    page = 1 << 14
    pages = -(-T // page)
    cache = cq.PagedCache(*(torch.zeros((pages, page, 1, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1)
    off = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    cq.cq_cache_append(cache, x, x, table, off[1:].clone(), off, norm=norm)
    k, v = (c.view(-1, 1, D)[:T] for c in (cache.k, cache.v))
    assert torch.equal(v, x) and torch.equal(k, cq.cq_head_norm(norm, None, x, pos)["k"])


# ------------------------------------------------------------------------------------------------
# the cache
# ------------------------------------------------------------------------------------------------
def _paged(cq, g, lengths, page, Hk, D, kind, scales=None, head_major=False, spare=2):
    """A cache of noise, pages of the sequences in any order; unused entries of the table are outside of it."""
    import torch
    need = [-(-max(n, 0) // page) for n in lengths]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((len(lengths), max([1] + need) + 1), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    shape = (pages, Hk, page, D) if head_major else (pages, page, Hk, D)
    k, v = (torch.randn(shape, generator=g).to(_t(kind)).cuda() for _ in range(2))
    if head_major:
        k, v = k.permute(0, 2, 1, 3), v.permute(0, 2, 1, 3)
    ks, vs = (None, None) if scales is None else ((torch.rand(Hk, generator=g) + scales).cuda() for _ in range(2))
    return cq.PagedCache(k, v, ks, vs), table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda()


def _bits(x):
    import torch
    return x.contiguous().view(torch.uint8)


@pytest.mark.parametrize("kind,cache_kind,scales", [("bf16", "bf16", None), ("f32", "f16", None), ("f16", "e4m3", 0.5), ("f32", "e4m3", None),
                                                    ("bf16", "f16", None)])
@pytest.mark.parametrize("page,head_major", [(1, False), (16, False), (7, True)])
@pytest.mark.parametrize("case", ["decode", "prompts", "one", "none"])
def test_append(cq, kind, cache_kind, scales, page, head_major, case):
    import torch
    g = torch.Generator().manual_seed(page + len(case))
    D, Hq, Hk, rot = 64, 6, 2, 32
    new = {"decode": [1] * 9, "prompts": [5, 0, 40, 1, 0, 17], "one": [1], "none": [0, 0]}[case]
    lengths = [n + 3 * i for i, n in enumerate(new)]
    T = sum(new) + (4 if case == "prompts" else 0)              # (four rows of padding)
    offsets = None if case in ("decode", "one") else np.concatenate([[0], np.cumsum(new)])
    cache, table, lens = _paged(cq, g, lengths, page, Hk, D, cache_kind, scales, head_major)
    if case == "decode":
        table[4, (lengths[4] - 1) // page] = 10 ** 6              # a page that is not there
        lens[5] = 0                                             # a token before position 0
        lens[6] = 10 ** 5                                       # and one beyond the table
    norm = _norm(cq, g, D, rot, True, "f32")
    rows = _rows(g, T, Hq + 2 * Hk, D, kind)
    q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hk], rows[:, Hq + Hk:]
    before_k, before_v = cache.k.clone(), cache.v.clone()
    q_out = torch.full((T, Hq, D), 7.0, dtype=_t(kind), device="cuda")
    off = None if offsets is None else torch.tensor(offsets, dtype=torch.int32).cuda()
    cq.cq_cache_append(cache, k, v, table, lens, off, norm=norm, q=q, q_out=q_out)
    places = O.slots(table.cpu().numpy(), lens.tolist(), offsets, page, cache.k.shape[0], T)
    pos = [0 if p is None else p[1] for p in places]
    ref_q, mag_q = _ref(norm, q, norm.w_q, pos)
    ref_k, mag_k = _ref(norm, k, norm.w_k, pos)
    sk, sv = (np.ones(Hk) if s is None else _np(s) for s in (cache.k_scale, cache.v_scale))
    touched = torch.zeros(cache.k.shape[:2], dtype=torch.bool)
    for t, p in enumerate(places):
        if p is None:
            assert (q_out[t] == 7).all()
            continue
        _close(q_out[t], ref_q[t], mag_q[t], 32 * U, kind, f"q of token {t}")
        if p[2] is None:
            continue
        touched[p[2], p[3]] = True
        _close(cache.k[p[2], p[3]], ref_k[t] / sk[:, None], mag_k[t] / sk[:, None], 33 * U, cache_kind, f"k of token {t}")
        want = v[t].float().cpu()
        if cache.v_scale is not None:
            want = want / cache.v_scale.cpu()[:, None]
        if cache_kind == "e4m3":
            want = want.clamp(-448, 448)
        assert torch.equal(_bits(cache.v[p[2], p[3]]).cpu(), _bits(want.to(_t(cache_kind)))), f"v of token {t}"
    rest = ~touched.cuda()
    assert torch.equal(_bits(cache.k[rest]), _bits(before_k[rest])) and torch.equal(_bits(cache.v[rest]), _bits(before_v[rest]))


def test_append_as_it_is_and_other_positions(cq):
    """Without a norm handle keys are stored as they are; positions of the caller's replace those of the cache; e4m3 saturates, NaN stays."""
    import torch
    g = torch.Generator().manual_seed(5)
    D, Hk = 128, 3
    cache, table, lens = _paged(cq, g, [4, 9], 4, Hk, D, "e4m3")
    k, v = _rows(g, 2, Hk, D, "f32", 300.0), _rows(g, 2, Hk, D, "f32", 300.0)
    v[0, 0, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), 464.1])
    assert cq.cq_cache_append(cache, k, v, table, lens) is None
    for s, n in enumerate((4, 9)):
        page, slot = int(table[s, (n - 1) // 4]), (n - 1) % 4
        for x, c in ((k, cache.k), (v, cache.v)):
            got, want = c[page, slot].float().cpu(), x[s].float().cpu().clamp(-448, 448).to(_t("e4m3")).float()
            assert torch.equal(torch.nan_to_num(got, 9.0), torch.nan_to_num(want, 9.0)) and torch.equal(torch.isnan(got), torch.isnan(want))
    norm = cq.HeadNorm(D, freq=_freq(D))
    cache, table, lens = _paged(cq, g, [4, 9], 4, Hk, D, "bf16")
    pos = torch.tensor([100, 7], dtype=torch.int32).cuda()
    cq.cq_cache_append(cache, k, v, table, lens, positions=pos, norm=norm)
    want = cq.cq_head_norm(norm, None, k, pos, out_dtype=_t("bf16"))["k"]
    assert torch.equal(cache.k[table[0, 0].long(), 3], want[0]) and torch.equal(cache.k[table[1, 2].long(), 0], want[1])


def test_append_many_sequences_finds_each(cq):
    """Offsets of 5000 sequences, many of them empty: three rounds of the search."""
    import torch
    g = torch.Generator().manual_seed(6)
    S, D = 5000, 16
    new = torch.randint(0, 3, (S,), generator=g)
    new[1000:1200] = 0
    cache, table, lens = _paged(cq, g, new.tolist(), 2, 1, D, "bf16")
    off = torch.cat([torch.zeros(1, dtype=torch.long), new.cumsum(0)]).to(torch.int32).cuda()
    T = int(new.sum())
    k, v = _rows(g, T, 1, D, "bf16"), _rows(g, T, 1, D, "bf16")
    cq.cq_cache_append(cache, k, v, table, lens, off)
    seq = torch.repeat_interleave(torch.arange(S), new).cuda()
    p = torch.arange(T).cuda() - off.long()[seq]
    assert torch.equal(cache.k[table.long()[seq, p // 2], p % 2], k) and torch.equal(cache.v[table.long()[seq, p // 2], p % 2], v)


# ------------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------------
def _check_attention(cq, cache, q, table, lens, out_kind=None, sample=None, **kw):
    import torch
    kind = {v: k for k, v in ((n, _t(n)) for n in HALF)}[q.dtype]
    out_kind = out_kind or kind
    S, Hq, D = q.shape
    k, v = (_np(x) if s is None else _np(x) * _np(s)[:, None] for x, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
    scale = D ** -0.5 if kw.get("scale") is None else kw["scale"]
    # expected lengths decide whether a workgroup takes a sequence or wavefronts take shares of all: both ways
    ways = [cq.cq_cache_attention(cache, q, table, lens, out_dtype=_t(out_kind), **{**kw, "max_length": n})
            for n in (kw.get("max_length"), 1 << 20)]
    out, lse, mag, dot, top = O.attention(_np(q), k, v, table.cpu().numpy(), lens.cpu().numpy(), scale, kw.get("window", 0),
                                          kw.get("softcap", 0.0), _np(kw.get("sinks")))
    n = max(1, int(lens.max()))
    dz = ((D + 16) * U + 2.0 ** -22) * dot + 8 * U * (top + kw.get("softcap", 0.0))
    rel = 2 * dz + 2.0 ** -16 + (n / 8 + 64) * U
    empty = lse == -np.inf
    bar = dz[~empty] + (n / 8 + 64) * U + 2 * U * np.abs(lse[~empty])
    for got in ways:
        _close(got["out"], out, mag * rel[:, :, None], 1.0, out_kind, "out")
        g = _np(got["lse"])
        assert (g[empty] == -np.inf).all()
        assert (np.abs(g[~empty] - lse[~empty]) <= bar).all(), "lse"
    return ways[0]


KIND_SETS = [("bf16", "bf16", "bf16"), ("f16", "f16", "f16"), ("f32", "bf16", "f32"), ("f32", "f16", "f32"), ("f32", "e4m3", "f32"),
             ("bf16", "e4m3", "bf16"), ("f16", "bf16", "f16"), ("bf16", "f16", "bf16"), ("f16", "e4m3", "f32")]


@pytest.mark.parametrize("D", [16, 48, 64, 80, 128, 144, 256])
@pytest.mark.parametrize("kind,cache_kind,out", KIND_SETS)
def test_attention_types_and_widths(cq, D, kind, cache_kind, out):
    import torch
    g = torch.Generator().manual_seed(D)
    lengths = [1, 31, 100, 0, 33, 517]
    cache, table, lens = _paged(cq, g, lengths, 16, 2, D, cache_kind, 0.5 if cache_kind == "e4m3" else None)
    q = _rows(g, len(lengths), 6, D, kind)
    _check_attention(cq, cache, q, table, lens, out)


@pytest.mark.parametrize("D", [8, 24, 136])
def test_attention_widths_of_eight(cq, D):
    import torch
    g = torch.Generator().manual_seed(D)
    cache, table, lens = _paged(cq, g, [70, 3], 5, 1, D, "bf16")
    _check_attention(cq, cache, _rows(g, 2, 3, D, "bf16"), table, lens)


@pytest.mark.parametrize("Hq,Hk", [(1, 1), (8, 8), (16, 1), (17, 1), (71, 1), (40, 2), (48, 3), (64, 8)])
@pytest.mark.parametrize("page,head_major", [(1, False), (16, True), (48, False), (256, False)])
def test_attention_heads_and_pages(cq, Hq, Hk, page, head_major):
    import torch
    g = torch.Generator().manual_seed(Hq + page)
    cache, table, lens = _paged(cq, g, [130, 1, 64, 300], page, Hk, 64, "bf16", None, head_major)
    _check_attention(cq, cache, _rows(g, 4, Hq, 64, "bf16"), table, lens)


@pytest.mark.parametrize("window", [0, 1, 17, 32, 200, 10 ** 6])
@pytest.mark.parametrize("softcap", [0.0, 5.0])
@pytest.mark.parametrize("sinks", [False, True])
def test_attention_window_softcap_sinks(cq, window, softcap, sinks):
    import torch
    g = torch.Generator().manual_seed(window % 1000)
    cache, table, lens = _paged(cq, g, [400, 0, 1, 33, 199, 200, 201, 1234], 16, 2, 128, "bf16")
    kw = {"sinks": torch.randn(8, generator=g).cuda()} if sinks else {}
    got = _check_attention(cq, cache, _rows(g, 8, 8, 128, "bf16"), table, lens, window=window, softcap=softcap, **kw)
    assert not got["out"][1].any()
    if sinks:
        assert (got["lse"][1] - kw["sinks"]).abs().max() <= 4 * U * kw["sinks"].abs().max()


@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-44, 3.0])
@pytest.mark.parametrize("softcap", [0.0, 5.0])
@pytest.mark.parametrize("cache_kind", ["bf16", "f16", "e4m3"])
def test_attention_scales(cq, scale, softcap, cache_kind):
    import torch
    g = torch.Generator().manual_seed(25)
    cache, table, lens = _paged(cq, g, [70, 0, 1, 40], 16, 2, 64, cache_kind, 0.5 if cache_kind == "e4m3" else None)
    if cache.k_scale is not None:
        cache.k_scale[1] *= -1
    sinks = torch.randn(4, generator=g).cuda()
    for kw in ({}, {"sinks": sinks}):
        got = _check_attention(cq, cache, _rows(g, 4, 4, 64, "bf16"), table, lens, scale=scale, softcap=softcap, **kw)
        assert not got["out"][1].any()


@pytest.mark.parametrize("softcap", [1e-42, 1e-3, 0.05, 1.0, 30.0, 64.0, 65.0, 1e4, 1e30])
@pytest.mark.parametrize("kind,cache_kind", [("f32", "bf16"), ("bf16", "e4m3")])
def test_attention_caps_keep_scores(cq, softcap, kind, cache_kind):
    import torch
    g = torch.Generator().manual_seed(26)
    cache, table, lens = _paged(cq, g, [70, 3, 1, 16], 16, 2, 64, cache_kind, 0.5 if cache_kind == "e4m3" else None)
    q = _rows(g, 4, 4, 64, kind)
    k, v = (_np(x) if s is None else _np(x) * _np(s)[:, None] for x, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
    _, lse, _, dot, top = O.attention(_np(q), k, v, table.cpu().numpy(), lens.cpu().numpy(), 0.01, 0, softcap, None)
    # tanh's argument is off by at most 8 U of itself (five products, the last rounded once more, a constant), which is no more of the
    # tanh; the exponential's form by 11 U of it above 5/8 (e^(2x) 2.5 U, the sum 1, its reciprocal 2, of which 1.6 / 0.55 remain), the
    # cap by 1.5; the exponent in units of ln 2 by 2 again.  16-bit results under caps up to 64: by 6 U of the cap instead
    bar = ((64 + 16) * U + 2.0 ** -22) * dot + 24 * U * top + (70 / 8 + 64) * U + 2 * U * np.abs(lse)
    if kind != "f32" and softcap <= 64:
        bar += 6 * U * softcap
    for n in (None, 1 << 20):
        got = cq.cq_cache_attention(cache, q, table, lens, scale=0.01, softcap=softcap, max_length=n)
        assert (np.abs(_np(got["lse"]) - lse) <= bar).all()


@pytest.mark.parametrize("max_length", [1, 100, 5000, 1 << 20, None])
def test_attention_lengths_beyond_what_was_expected(cq, max_length):
    import torch
    g = torch.Generator().manual_seed(11)
    cache, table, lens = _paged(cq, g, [5000, 700, 1, 0], 64, 2, 64, "f16")
    _check_attention(cq, cache, _rows(g, 4, 4, 64, "f16"), table, lens, max_length=max_length)


@pytest.mark.parametrize("S,longest,Hk", [(64, 40, 1), (65, 300, 2), (200, 70, 1), (1000, 90, 1), (130, 2000, 1)])
def test_attention_many_sequences(cq, S, longest, Hk):
    """More sequences than a wavefront has lanes, many of them empty, in shares that hold several."""
    import torch
    g = torch.Generator().manual_seed(S)
    lengths = torch.randint(0, longest + 1, (S,), generator=g)
    lengths[torch.rand(S, generator=g) < 0.3] = 0
    lengths[:3] = lengths[-2:] = 0
    cache, table, lens = _paged(cq, g, lengths.tolist(), 16, Hk, 64, "bf16")
    for window in (0, 50):
        got = _check_attention(cq, cache, _rows(g, S, 2 * Hk, 64, "bf16"), table, lens, window=window, max_length=longest)
        assert not got["out"][lens == 0].any()


def test_attention_of_thousands_and_of_several_tokens_of_one(cq):
    """3000 sequences; then the last tokens of a sequence at once, by one row of the table for all of them."""
    import torch
    g = torch.Generator().manual_seed(27)
    lengths = torch.randint(0, 40, (3000,), generator=g)
    cache, table, lens = _paged(cq, g, lengths.tolist(), 16, 1, 16, "bf16")
    _check_attention(cq, cache, _rows(g, 3000, 2, 16, "bf16"), table, lens)
    cache, table, lens = _paged(cq, g, [90], 16, 2, 64, "bf16")
    q = _rows(g, 5, 4, 64, "bf16")
    lens = torch.arange(86, 91, dtype=torch.int32).cuda()
    _check_attention(cq, cache, q, table.expand(5, -1), lens)


def test_attention_all_empty(cq):
    import torch
    g = torch.Generator().manual_seed(24)
    cache, table, lens = _paged(cq, g, [0, 0, 0], 16, 1, 64, "bf16")
    _check_attention(cq, cache, _rows(g, 3, 2, 64, "bf16"), table, lens)
    none = cq.PagedCache(cache.k[:0], cache.v[:0])                       # a cache without pages
    _check_attention(cq, none, _rows(g, 3, 2, 64, "bf16"), table, torch.full_like(lens, 9))
    out = cq.cq_cache_attention(cache, _rows(g, 0, 2, 64, "bf16"), table[:0], lens[:0])
    assert out["out"].shape == (0, 2, 64) and out["lse"].shape == (0, 2)


def test_attention_long(cq):
    import torch
    g = torch.Generator().manual_seed(12)
    cache, table, lens = _paged(cq, g, [40000], 64, 1, 128, "bf16")
    _check_attention(cq, cache, _rows(g, 1, 4, 128, "f32"), table, lens)


def test_attention_large_scores(cq):
    """Scores of some hundreds: one position takes all of the weight; the running maximum rises again and again."""
    import torch
    g = torch.Generator().manual_seed(13)
    cache, table, lens = _paged(cq, g, [600, 600], 16, 1, 64, "bf16")
    at = torch.arange(600)
    for s in range(2):
        order = at if s == 0 else at.flip(0)
        cache.k[table[s].long()[at // 16], at % 16, 0] = (order[:, None] / 100 * torch.ones(64)).bfloat16().cuda()
    q = torch.full((2, 4, 64), 1.0, device="cuda")
    _check_attention(cq, cache, q, table, lens, scale=1.0)


def test_attention_pages_that_are_not_there(cq):
    import torch
    g = torch.Generator().manual_seed(14)
    cache, table, lens = _paged(cq, g, [100, 100, 100, 50], 16, 2, 64, "bf16")
    table[0, 2] = -1
    table[1, 6] = cache.k.shape[0]
    table[2, :] = 2 ** 31 - 1
    lens[3] = 10 ** 9                                    # far beyond the table
    _check_attention(cq, cache, _rows(g, 4, 4, 64, "bf16"), table, lens)
    lens[3] = -5
    got = _check_attention(cq, cache, _rows(g, 4, 4, 64, "bf16"), table, lens)
    assert not got["out"][2:].any()


def test_attention_does_not_read_behind_the_length(cq):
    """NaN and infinities in slots behind the length, in pages of others and before the window change nothing."""
    import torch
    g = torch.Generator().manual_seed(15)
    for kind in ("bf16", "f16", "e4m3"):
        cache, table, lens = _paged(cq, g, [45, 16, 3], 16, 2, 64, kind)
        q = _rows(g, 3, 4, 64, "bf16")
        want = [cq.cq_cache_attention(cache, q, table, lens, window=w) for w in (0, 10)]
        for w, first in ((0, [0, 0, 0]), (10, [35, 6, 0])):
            k, v = cache.k.clone(), cache.v.clone()
            keep = torch.zeros(k.shape[:2], dtype=torch.bool)
            for s, n in enumerate([45, 16, 3]):
                p = torch.arange(first[s], n)
                keep[table[s].cpu().long()[p // 16], p % 16] = True
            for x in (k, v):          # (all bits set is a NaN in each of the types)
                x.view(torch.uint8)[~keep.cuda()] = 0xff
            got = cq.cq_cache_attention(cq.PagedCache(k, v), q, table, lens, window=w)
            assert torch.equal(got["out"], want[w // 10]["out"]) and torch.equal(got["lse"], want[w // 10]["lse"])


def test_attention_special_values(cq):
    """A key of -inf leaves its position out; a row all of whose keys are -inf gives zeros; NaN in a key gives NaN in its rows alone."""
    import torch
    g = torch.Generator().manual_seed(16)
    cache, table, lens = _paged(cq, g, [40, 40, 40], 16, 1, 64, "bf16")
    q = _rows(g, 3, 2, 64, "bf16").abs()
    slot = lambda s, p: (int(table[s, p // 16]), p % 16)  # noqa: E731
    want = cq.cq_cache_attention(cache, q, table, torch.tensor([40, 39, 40], dtype=torch.int32).cuda())
    cache.k[slot(1, 39)] = -float("inf")
    got = cq.cq_cache_attention(cache, q, table, lens)
    # (a position of weight zero in place of one that is not there: the same sums)
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
    for p in range(40):
        cache.k[slot(0, p)] = -float("inf")
    cache.k[slot(2, 7)] = float("nan")
    got = cq.cq_cache_attention(cache, q, table, lens)
    assert not got["out"][0].any() and (got["lse"][0] == -float("inf")).all()
    assert torch.isnan(got["out"][2]).all() and torch.equal(got["out"][1], want["out"][1])


def test_attention_far_pages(cq):
    """Pages whose rows lie beyond 2^31 values."""
    import torch
    g = torch.Generator().manual_seed(17)
    page = 64 * 2 * 64
    pages = (1 << 32) // page // 2 + 40
    k, v = (torch.zeros((pages, 64, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    far = cq.PagedCache(k, v)
    near, table, lens = _paged(cq, g, [150, 40], 64, 2, 64, "bf16", spare=0)
    shift = pages - near.k.shape[0]
    k[shift:], v[shift:] = near.k, near.v
    q = _rows(g, 2, 4, 64, "bf16")
    moved = torch.where(table >= 0, table + shift, table)
    a, b = cq.cq_cache_attention(near, q, table, lens), cq.cq_cache_attention(far, q, moved, lens)
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])
    nk, nv = _rows(g, 2, 2, 64, "bf16"), _rows(g, 2, 2, 64, "bf16")
    for c, t in ((near, table), (far, moved)):
        cq.cq_cache_append(c, nk, nv, t, lens)
    assert torch.equal(k[shift:], near.k) and torch.equal(v[shift:], near.v) and not k[:shift].any() and not v[:shift].any()


def test_attention_strided_queries_and_outputs(cq):
    import torch
    g = torch.Generator().manual_seed(18)
    cache, table, lens = _paged(cq, g, [90, 14], 16, 2, 64, "bf16")
    wide = torch.randn((2, 9, 64), generator=g).bfloat16().cuda()
    q = wide[:, 1:7]
    want = cq.cq_cache_attention(cache, q.contiguous(), table, lens)
    room = torch.full((6, 2, 70), 3.0, device="cuda", dtype=torch.bfloat16)
    out = room.permute(1, 0, 2)[..., 5:69]
    got = cq.cq_cache_attention(cache, q, table, lens, out=out, want_lse=False)
    assert got["lse"] is None and torch.equal(out, want["out"]) and (room[..., :5] == 3).all() and (room[..., 69:] == 3).all()
    wider = torch.full((2, table.shape[1] + 5), 0, dtype=torch.int32, device="cuda")
    wider[:, :table.shape[1]] = table
    got = cq.cq_cache_attention(cache, q, wider[:, :table.shape[1]], lens)
    assert torch.equal(got["out"], want["out"])


# ------------------------------------------------------------------------------------------------
# together, on streams and in graphs
# ------------------------------------------------------------------------------------------------
def _decode_step(cq, norm, cache, rows, table, lens, Hq, Hk):
    q = cq.cq_cache_append(cache, rows[:, Hq:Hq + Hk], rows[:, Hq + Hk:], table, lens, norm=norm, q=rows[:, :Hq])
    return cq.cq_cache_attention(cache, q, table, lens)["out"]


def test_prompts_then_tokens_match_the_definition(cq):
    """Three prompts are appended, then four tokens each; every step's attention against the oracle on the cache as it stands."""
    import torch
    g = torch.Generator().manual_seed(20)
    Hq, Hk, D, page = 8, 2, 64, 16
    norm = _norm(cq, g, D, D, False, "f32")
    prompts = [21, 1, 40]
    cache, table, lens = _paged(cq, g, [n + 4 for n in prompts], page, Hk, D, "bf16")
    lens.copy_(torch.tensor(prompts))
    rows = _rows(g, sum(prompts), Hq + 2 * Hk, D, "f32")
    off = torch.tensor(np.concatenate([[0], np.cumsum(prompts)]), dtype=torch.int32).cuda()
    q = cq.cq_cache_append(cache, rows[:, Hq:Hq + Hk], rows[:, Hq + Hk:], table, lens, off, norm=norm, q=rows[:, :Hq])
    heads = cq.cq_head_norm(norm, rows[:, :Hq], rows[:, Hq:Hq + Hk], torch.cat([torch.arange(n) for n in prompts]).to(torch.int32).cuda())
    assert torch.equal(q, heads["q"])                      # the same norm and rotation, bit for bit
    t = 0
    for s, n in enumerate(prompts):
        p = torch.arange(n).cuda()
        assert torch.equal(cache.k[table[s].long()[p // page], p % page], heads["k"][t:t + n].bfloat16())
        t += n
    for step in range(4):
        lens += 1
        rows = _rows(g, 3, Hq + 2 * Hk, D, "f32")
        q = cq.cq_cache_append(cache, rows[:, Hq:Hq + Hk], rows[:, Hq + Hk:], table, lens, norm=norm, q=rows[:, :Hq])
        _check_attention(cq, cache, q, table, lens)


def test_graph_of_a_decode_step_and_other_streams(cq):
    """A captured step replayed with eager work between; each replay matches the eager step bit for bit.  Two graphs of their own workspaces."""
    import torch
    g = torch.Generator().manual_seed(21)
    Hq, Hk, D = 8, 2, 128
    norm = _norm(cq, g, D, D, False, "f32")
    cache, table, lens = _paged(cq, g, [3000, 700, 40], 16, Hk, D, "bf16")
    lens -= 8
    rows = _rows(g, 3, Hq + 2 * Hk, D, "f32")
    step = lambda c: _decode_step(cq, norm, c, rows, table, lens, Hq, Hk)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cache)
    torch.cuda.current_stream().wait_stream(side)
    other = cq.PagedCache(cache.k.clone(), cache.v.clone())     # (behind the step above, which has written a token)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(cache)
        graphs.append((graph, out))
    for n in range(5):
        lens += 1
        rows.copy_(_rows(g, 3, Hq + 2 * Hk, D, "f32"))
        want = step(other)
        torch.cuda.synchronize()
        for graph, out in graphs:
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), n
        assert torch.equal(cache.k, other.k) and torch.equal(cache.v, other.v)


def test_gradient_in_a_graph(cq):
    import torch
    g = torch.Generator().manual_seed(22)
    norm = _norm(cq, g, 64, 64, False, "f32")
    q, k, dq, dk = (_rows(g, 300, n, 64, "bf16") for n in (6, 2, 6, 2))
    pos = torch.arange(300, dtype=torch.int32).cuda()
    run = lambda: cq.cq_head_norm_grad(norm, q, k, pos, dq, dk)  # noqa: E731
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for n in range(4):
        q.copy_(_rows(g, 300, 6, 64, "bf16"))
        want = run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[x], want[x]) for x in out), n


def test_results_do_not_depend_on_timing(cq):
    import torch
    g = torch.Generator().manual_seed(23)
    cache, table, lens = _paged(cq, g, [9000, 4000, 100], 16, 2, 128, "bf16")
    q = _rows(g, 3, 8, 128, "bf16")
    norm = _norm(cq, g, 128, 128, False, "f32")
    x, dy = _rows(g, 900, 8, 128, "bf16"), _rows(g, 900, 8, 128, "bf16")
    pos = torch.arange(900, dtype=torch.int32).cuda()
    first = cq.cq_cache_attention(cache, q, table, lens), cq.cq_head_norm_grad(norm, x, None, pos, dy)
    for _ in range(5):
        a, b = cq.cq_cache_attention(cache, q, table, lens), cq.cq_head_norm_grad(norm, x, None, pos, dy)
        assert torch.equal(a["out"], first[0]["out"]) and torch.equal(a["lse"], first[0]["lse"])
        assert torch.equal(b["dq"], first[1]["dq"]) and torch.equal(b["dw_q"], first[1]["dw_q"])


def test_handles_look_at_their_tensors_at_every_call(cq):
    import torch
    g = torch.Generator().manual_seed(26)
    norm = _norm(cq, g, 64, 64, False, "f32")
    q = _rows(g, 3, 2, 64, "bf16")
    pos = torch.arange(3, dtype=torch.int32).cuda()
    want = cq.cq_head_norm(norm, q, None, pos)["q"]
    kept = norm.w_q
    for bad in (kept.bfloat16(), kept[:32], kept.cpu(), torch.stack([kept, kept], 1)[:, 0]):
        norm.w_q = bad
        with pytest.raises(ValueError, match="w_q|w_k"):
            cq.cq_head_norm(norm, q, q, pos)
    norm.w_q = kept * 2                                     # another weight is taken as it is
    assert torch.equal(cq.cq_head_norm(norm, q, None, pos)["q"], want * 2)
    norm.w_q, norm.freq = kept, norm.freq.float()
    with pytest.raises(ValueError, match="freq"):
        cq.cq_head_norm(norm, q, None, pos)
    cache, table, lens = _paged(cq, g, [20, 3], 16, 2, 64, "bf16")
    q = _rows(g, 2, 4, 64, "bf16")
    want = cq.cq_cache_attention(cache, q, table, lens)["out"]
    k, v = cache.k, cache.v
    for bad_k, bad_v in ((k.half(), v), (k, v[:1]), (k.permute(0, 2, 1, 3), v), (k[..., ::2], v[..., ::2])):
        cache.k, cache.v = bad_k, bad_v
        with pytest.raises(ValueError, match="pages of one layout"):
            cq.cq_cache_attention(cache, q, table, lens)
    cache.k, cache.v = k.clone(), v.clone()
    k.zero_()
    assert torch.equal(cq.cq_cache_attention(cache, q, table, lens)["out"], want)
    for bad in (dict(q=q[:1]), dict(q=q[..., :32]), dict(lengths=lens[:1]), dict(lengths=lens.long()), dict(page_table=table.long()),
                dict(page_table=table[0]), dict(sinks=torch.zeros(3, device="cuda")), dict(window=1 << 31), dict(window=-1),
                dict(max_length=1 << 31), dict(q=q.cpu())):
        with pytest.raises((ValueError, cq.CqError)):
            cq.cq_cache_attention(cache, **{"q": q, "page_table": table, "lengths": lens, **bad})
