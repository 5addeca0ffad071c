"""The operators around the expert layer on the GPU, against the float64 oracle on the same inputs.

Bounds.  u = 2^-24 is fp32's rounding; a result of type t is rounded once more, by at most finfo(t).eps / 2 of its value (a
subnormal by half of its step).  Before that it is a fixed chain of fp32 operations: its error is a number of roundings times
the sum of its terms' absolute values (the oracle's magnitudes).  Row sums of H <= 32768 values take at most 32 additions in a
thread, 6 in a wavefront and 16 across, and enter through a square root and a quotient; the number below covers each chain with
room for the few products around it."""
import numpy as np
import pytest

from oracle import around_oracle as O

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2604_10496_amd import binding
    binding.load_library()
    return binding


def _dt(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def _put(rng, shape, dtype, scale=1.0, mean=0.0):
    """A GPU tensor of the type and its values in float64."""
    import torch
    t = torch.from_numpy(rng.standard_normal(shape) * scale + mean).to(dtype)
    return t.cuda(), t.double().numpy()


def _close(got, ref, mag, roundings, what):
    import torch
    info = torch.finfo(got.dtype)
    half = 0.0 if got.dtype == torch.float32 else info.eps / 2
    err = np.abs(got.detach().double().cpu().numpy() - ref)
    bound = roundings * U * mag
    bound = bound + half * (np.abs(ref) + bound) + info.tiny * info.eps
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, worst {np.nanmax(err / np.maximum(bound, 1e-300)):.3g} of the bound"


# ------------------------------------------------------------------------------------------------
# norms before and after a block
# ------------------------------------------------------------------------------------------------
NORM_ROUNDINGS = 128        # of a value behind one or two row sums
EPS = 1e-5


class _Norm:
    def __init__(self, B, rng, T, H, stream, block, weight, post, gate, use_sigmoid, rho=0.9, beta=1.25, pre=True):
        st, bl, wt = _dt(stream), _dt(block), _dt(weight)
        self.h, self.h64 = _put(rng, (T, H), st)
        self.y, self.y64 = _put(rng, (T, H), bl, 0.7)
        self.dh, self.dh64 = _put(rng, (T, H), st, 0.5)
        self.dx, self.dx64 = _put(rng, (T, H), bl, 0.5)
        self.w_pre, self.w_pre64 = _put(rng, (H,), wt, 0.3, 1.0) if pre else (None, None)
        self.w_post, self.w_post64 = _put(rng, (H,), wt, 0.3, 1.0) if post else (None, None)
        self.gate, self.gate64 = {"none": lambda: (None, None), "row": lambda: _put(rng, (T,), bl),
                                  "elem": lambda: _put(rng, (T, H), bl)}[gate]()
        self.tail = (EPS, rho, beta, use_sigmoid)
        self.norm = B.BlockNorm(self.w_pre, self.w_post, EPS, rho, beta, use_sigmoid, bl)

    def forward(self):
        return O.block_norm(self.h64, self.y64, self.gate64, self.w_pre64, self.w_post64, *self.tail)

    def backward(self, h64, dh=True, dx=True):
        return O.block_norm_grad(h64, self.y64, self.gate64, self.dh64 if dh else None, self.dx64 if dx else None, self.w_pre64,
                                 self.w_post64, *self.tail)


def _check_norm(got, want, T, what):
    ref, mag = want
    assert {k for k, v in got.items() if v is not None} == set(ref), what
    for name, v in ref.items():
        n = NORM_ROUNDINGS + (T if name.startswith("dw") else 0)
        if name == "dgate":
            n += 64
        _close(got[name], v, mag[name], n, f"{what} {name}")


KINDS = [("f32", "f32", "f32"), ("bf16", "f32", "bf16"), ("bf16", "bf16", "f32"), ("f16", "f16", "f16"), ("f16", "f32", "f32"),
         ("bf16", "bf16", "bf16")]
SHAPES = [(1, 1), (3, 7), (5, 64), (2, 512), (67, 513), (4, 1111), (130, 2048), (3, 2049), (70, 4096), (2, 4104), (1, 8192),
          (5, 8200), (2, 16383), (3, 16384), (2, 20001), (1, 32768)]


@pytest.mark.parametrize("T,H", SHAPES)
@pytest.mark.parametrize("post,gate,use_sigmoid", [(False, "none", False), (True, "row", True), (True, "elem", False), (False, "elem", True),
                                                   (False, "row", False), (True, "none", False)])
def test_block_norm_and_its_gradients(B, T, H, post, gate, use_sigmoid):
    at = SHAPES.index((T, H)) + (3 if post else 0) + len(gate)
    for kinds in (KINDS[at % len(KINDS)], KINDS[(at + 3) % len(KINDS)]):
        rng = np.random.default_rng(1000 * T + H)
        c = _Norm(B, rng, T, H, *kinds, post, gate, use_sigmoid)
        what = f"T={T} H={H} {kinds} post={post} gate={gate}"
        print(what, flush=True)
        out = B.cq_block_norm(c.norm, c.h, c.y, c.gate)
        _check_norm(out, c.forward(), T, what)
        h64 = out["h"].double().cpu().numpy()
        _check_norm(B.cq_block_norm_grad(c.norm, out["h"], c.y, c.gate, dh=c.dh, dx=c.dx), c.backward(h64), T, what)


@pytest.mark.parametrize("H", [96, 1025])
@pytest.mark.parametrize("kinds", KINDS)
def test_block_norm_many_rows(B, kinds, H):
    """More rows than a gradient's workgroups have at once: several rows each, in turn."""
    c = _Norm(B, np.random.default_rng(H), 1501, H, *kinds, True, "row", True)
    out = B.cq_block_norm(c.norm, c.h, c.y, c.gate)
    _check_norm(out, c.forward(), 1501, "forward")
    got = B.cq_block_norm_grad(c.norm, out["h"], c.y, c.gate, dh=c.dh, dx=c.dx)
    _check_norm(got, c.backward(out["h"].double().cpu().numpy()), 1501, "backward")
    again = B.cq_block_norm_grad(c.norm, out["h"], c.y, c.gate, dh=c.dh, dx=c.dx)
    for name in got:
        assert got[name].equal(again[name]), name     # nothing depends on timing


@pytest.mark.parametrize("T,H", [(1, 64), (9, 511), (300, 2048)])
def test_block_norm_parts(B, T, H):
    """The norm in front of the first block alone, the sum behind the last one alone, and gradients of either kind alone."""
    rng = np.random.default_rng(H)
    c = _Norm(B, rng, T, H, "bf16", "f32", "f32", True, "row", True)
    first = B.cq_block_norm(c.norm, c.h)
    assert first["h"] is c.h
    ref, mag = O.block_norm(c.h64, None, None, c.w_pre64, None, *c.tail)
    _close(first["x"], ref["x"], mag["x"], NORM_ROUNDINGS, "x")
    got = B.cq_block_norm_grad(c.norm, c.h, dh=c.dh, dx=c.dx)
    want = O.block_norm_grad(c.h64, None, None, c.dh64, c.dx64, c.w_pre64, None, *c.tail)
    _check_norm(got, want, T, "first block")
    # without a norm in front of a next block
    last = _Norm(B, rng, T, H, "bf16", "f32", "f32", True, "elem", False, pre=False)
    out = B.cq_block_norm(last.norm, last.h, last.y, last.gate)
    assert out["x"] is None
    _check_norm(out, last.forward(), T, "last block")
    h64 = out["h"].double().cpu().numpy()
    _check_norm(B.cq_block_norm_grad(last.norm, out["h"], last.y, last.gate, dh=last.dh), last.backward(h64, dx=False), T, "last block")
    # a residual stream that nothing reads but the norm
    h64 = c.h64
    _check_norm(B.cq_block_norm_grad(c.norm, c.h, c.y, c.gate, dx=c.dx), c.backward(h64, dh=False), T, "dx alone")
    frozen = B.cq_block_norm_grad(c.norm, c.h, c.y, c.gate, dh=c.dh, dx=c.dx, want_weights=False)
    full = B.cq_block_norm_grad(c.norm, c.h, c.y, c.gate, dh=c.dh, dx=c.dx)
    assert frozen["dw_pre"] is None and frozen["dw_post"] is None
    for name in ("dh", "dy", "dgate"):
        assert frozen[name].equal(full[name])


def test_block_norm_in_place_and_unaligned(B):
    """h' over h, x over y, a gradient over the incoming one; rows that start on any element."""
    import torch
    rng = np.random.default_rng(8)
    for H, off in ((256, 0), (256, 1), (255, 0), (1000, 3)):
        c = _Norm(B, rng, 33, H, "bf16", "bf16", "bf16", True, "elem", True)
        want = B.cq_block_norm(c.norm, c.h, c.y, c.gate)

        def moved(t):
            buf = torch.zeros(t.numel() + 8, dtype=t.dtype, device="cuda")
            v = buf[off:off + t.numel()].view(t.shape)
            v.copy_(t)
            return v
        h, y = moved(c.h), moved(c.y)
        out = B.cq_block_norm(c.norm, h, y, c.gate, h_out=h, x_out=y)
        assert out["h"] is h and out["x"] is y
        if off == 0:
            assert h.equal(want["h"]) and y.equal(want["x"])
        _check_norm(out, c.forward(), 33, f"H={H} off={off}")


def test_block_norm_rows_of_special_values(B):
    """A row of zeros has a norm of zeros; NaN and infinities stay in their own rows."""
    import torch
    c = _Norm(B, np.random.default_rng(2), 40, 200, "f32", "f32", "f32", True, "row", False)
    clean = B.cq_block_norm(c.norm, c.h, c.y, c.gate)
    c.h[3] = 0
    c.y[3] = 0
    c.h[7, 11] = float("nan")
    c.y[9, 0] = float("inf")
    c.gate[12] = float("nan")
    out = B.cq_block_norm(c.norm, c.h, c.y, c.gate)
    assert not out["h"][3].any() and not out["x"][3].any()
    assert out["x"][7].isnan().all() and out["h"][9].isnan().any() and out["h"][12].isnan().all()
    good = [t for t in range(40) if t not in (3, 7, 9, 12)]
    assert out["h"][good].equal(clean["h"][good]) and out["x"][good].equal(clean["x"][good])
    g = B.cq_block_norm_grad(c.norm, clean["h"], torch.zeros_like(c.y), c.gate.nan_to_num(), dh=c.dh, dx=c.dx)   # y = 0: m = 0
    assert torch.isfinite(g["dy"]).all() and not g["dw_post"].any() and not g["dgate"].any()


def test_block_norm_without_tokens(B):
    import torch
    w = torch.ones(64, device="cuda")
    norm = B.BlockNorm(w, w)
    h = torch.empty((0, 64), device="cuda")
    assert B.cq_block_norm(norm, h, h)["x"].shape == (0, 64)
    g = B.cq_block_norm_grad(norm, h, h, dh=h, dx=h)
    assert not g["dw_pre"].any() and not g["dw_post"].any() and g["dw_pre"].shape == (64,)


def test_block_norm_gradient_against_differences_of_the_kernel(B):
    """<gradient, v> against (L(h + s v) - L(h - s v)) / 2s of the forward kernel in fp32, L = <c, h'> + <e, x>.  The difference is
    off by its truncation, s^2 / 6 of a third derivative of about |c| + |e|, and by the forward's roundings over s."""
    T, H, step = 6, 300, 2.0 ** -6
    rng = np.random.default_rng(11)
    c = _Norm(B, rng, T, H, "f32", "f32", "f32", True, "row", True)
    out = B.cq_block_norm(c.norm, c.h, c.y, c.gate)
    g = B.cq_block_norm_grad(c.norm, out["h"], c.y, c.gate, dh=c.dh, dx=c.dx)

    def loss(h, y, gate):
        o = B.cq_block_norm(c.norm, h, y, gate)
        return float((o["h"].double() * c.dh.double()).sum() + (o["x"].double() * c.dx.double()).sum())
    for name, at in (("dh", 0), ("dy", 1), ("dgate", 2)):
        args = [c.h, c.y, c.gate]
        v, _ = _put(rng, tuple(args[at].shape), _dt("f32"))
        v = v / float(v.double().norm())
        plus, minus = list(args), list(args)
        plus[at], minus[at] = args[at] + step * v, args[at] - step * v
        diff = (loss(*plus) - loss(*minus)) / (2 * step)
        got = float((g[name].double() * v.double()).sum())
        size = float(c.dh.double().norm() + c.dx.double().norm()) * 4      # of the derivatives along a unit vector
        assert abs(diff - got) <= size * (step ** 2 + 64 * U / step), (name, diff, got)


# ------------------------------------------------------------------------------------------------
# balance loss
# ------------------------------------------------------------------------------------------------
def _routing(rng, T, E, k, dtype):
    import torch
    z = torch.from_numpy(rng.standard_normal((T, E)) * 1.5 + rng.standard_normal(E)).to(dtype)
    z64 = z.double().numpy()
    ids = np.argsort(-z64, axis=1, kind="stable")[:, :k].astype(np.int32)
    return z.cuda(), z64, ids


def _offsets(rng, T, S):
    return np.concatenate([[0], np.sort(rng.integers(0, T + 1, S - 1)), [T]]).astype(np.int32)


def _check_balance(B, z, z64, ids, alpha, offsets=None, mask=None, dloss=None, what=""):
    import torch
    T, E = z64.shape
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    t_ids, t_off, t_mask = dev(ids), dev(offsets), dev(mask)
    out = B.cq_balance_loss(z, t_ids, alpha, t_off, t_mask)
    ref = O.balance_loss(z64, ids, alpha, offsets, mask)
    assert np.array_equal(out["counts"].cpu().numpy(), ref["counts"]), what
    assert np.array_equal(out["tokens"].cpu().numpy(), ref["tokens"]), what
    # a probability: an exponential (4 roundings, and its argument's own rounding times |z - max| <= 32), a sum over E / 64 values
    # a lane and 6 exchanges, a quotient; a mean over a tile's 64 tokens at most in sequence and the tiles after each other
    n = 64 + E // 64 + 64 + T // 64
    _close(out["probs"], ref["probs"], ref["probs"], n, f"{what} probs")
    _close(out["loss"], np.array([ref["loss"]]), np.array([abs(ref["loss"])]), n + 64 + len(ref["tokens"]), f"{what} loss")
    w = None if dloss is None else torch.tensor([dloss], dtype=torch.float32, device="cuda")
    got = B.cq_balance_loss_grad(z, out["counts"], out["tokens"], ids.shape[1], alpha, t_off, t_mask, w)
    grad, mag = O.balance_loss_grad(z64, ids, alpha, 1.0 if dloss is None else float(np.float32(dloss)), offsets, mask)
    _close(got, grad, mag, 128 + E // 64, f"{what} gradient")
    return out, got


@pytest.mark.parametrize("T,E,k,S", [(1, 1, 1, 1), (1, 8, 2, 1), (3, 2, 1, 2), (64, 4, 2, 1), (65, 5, 3, 4), (200, 8, 2, 7), (129, 60, 6, 3),
                                     (512, 64, 6, 1), (777, 65, 4, 40), (300, 100, 8, 2), (1000, 128, 8, 5), (257, 160, 6, 3),
                                     (90, 256, 8, 90), (70, 257, 8, 2), (33, 500, 10, 3), (40, 1000, 64, 2), (20, 1024, 64, 4),
                                     (5000, 16, 4, 3), (4099, 7, 2, 300)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_balance_loss_and_its_gradient(B, T, E, k, S, kind):
    rng = np.random.default_rng(T * 1000 + E)
    z, z64, ids = _routing(rng, T, E, k, _dt(kind))
    print(f"T={T} E={E} k={k} S={S} {kind}", flush=True)
    _check_balance(B, z, z64, ids, 0.01, what="one sequence")
    _check_balance(B, z, z64, ids, 0.5, _offsets(rng, T, S), None, 1.75, "sequences")
    _check_balance(B, z, z64, ids, 1.0, _offsets(rng, T, S), rng.random(T) < 0.7, 0.5, "sequences with padding")


def test_balance_loss_of_left_out_tokens(B):
    """Padded tokens hold anything; tokens in no sequence, sequences without tokens, assignments that were dropped."""
    import torch
    rng = np.random.default_rng(21)
    T, E, k = 150, 12, 3
    z, z64, ids = _routing(rng, T, E, k, torch.float32)
    mask = np.ones(T, dtype=bool)
    mask[[0, 70, 71, 149]] = False
    z[0], z[70, 3], z[71], z[149] = float("nan"), float("inf"), -float("inf"), float("-inf")
    z64[~mask] = 0.0
    ids[0] = 2 ** 31 - 1
    ids[5, 0], ids[6, 2], ids[7] = -1, E, [-5, 1 << 30, -2 ** 31]
    offsets = np.array([10, 10, 64, 64, 64, 120, 140], dtype=np.int32)
    _check_balance(B, z, z64, ids, 0.3, offsets, mask, 2.0, "offsets inside")
    _check_balance(B, z, z64, ids, 0.3, None, mask, 2.0, "one sequence")
    nothing = np.zeros(T, dtype=bool)
    out, grad = _check_balance(B, z, z64, ids, 0.3, offsets, nothing, None, "nothing left")
    assert float(out["loss"]) == 0.0 and not out["probs"].any() and not grad.any()
    empty = B.cq_balance_loss(z[:0], torch.from_numpy(ids[:0]).cuda(), 0.3)
    assert float(empty["loss"]) == 0.0 and empty["tokens"].tolist() == [0, 0] and not empty["counts"].any()


def test_balance_loss_of_masked_experts(B):
    """Logits of -inf and of the type's lowest value: no probability, no gradient; rows of nothing else."""
    import torch
    rng = np.random.default_rng(22)
    T, E, k = 70, 20, 2
    for kind in ("f32", "bf16", "f16"):
        z, z64, ids = _routing(rng, T, E, k, _dt(kind))
        low = torch.finfo(_dt(kind)).min
        z[:, 4], z64[:, 4] = -float("inf"), -np.inf
        z[:, 9], z64[:, 9] = low, float(low)
        z[13], z64[13] = -float("inf"), -np.inf         # a row without any logit
        z[14], z64[14] = low, float(low)                # a row of lowest values: all the same
        ids = np.where((ids == 4) | (ids == 9), 0, ids).astype(np.int32)
        _, grad = _check_balance(B, z, z64, ids, 0.3, None, None, None, kind)
        assert not grad[:14, 4].any() and not grad[13].any() and torch.isfinite(grad).all()


def test_balance_loss_offsets_out_of_range_stay_in_bounds(B):
    """Offsets are clamped to the batch: beyond it there is nothing to read."""
    import torch
    rng = np.random.default_rng(23)
    z, z64, ids = _routing(rng, 100, 8, 2, torch.float32)
    off = torch.tensor([-7, 40, 1 << 30], dtype=torch.int32, device="cuda")
    got = B.cq_balance_loss(z, torch.from_numpy(ids).cuda(), 0.1, off)
    ref = O.balance_loss(z64, ids, 0.1, [0, 40, 100])
    assert np.array_equal(got["counts"].cpu().numpy(), ref["counts"])


def test_balance_gradient_against_differences_of_the_kernel(B):
    """As for the norms: the loss is of size alpha E max f, its third derivative along a unit vector no larger than that over the
    tokens; probabilities carry 64 roundings."""
    import torch
    rng = np.random.default_rng(24)
    T, E, k, alpha, step = 50, 9, 2, 3.0, 0.25
    z, z64, ids = _routing(rng, T, E, k, torch.float32)
    t_ids = torch.from_numpy(ids).cuda()
    out = B.cq_balance_loss(z, t_ids, alpha)
    g = B.cq_balance_loss_grad(z, out["counts"], out["tokens"], k, alpha)
    for _ in range(3):
        v, _ = _put(rng, (T, E), torch.float32)
        v = v / float(v.double().norm())
        f = lambda s: float(B.cq_balance_loss(z + s * v, t_ids, alpha)["loss"])
        diff, got = (f(step) - f(-step)) / (2 * step), float((g.double() * v.double()).sum())
        size = alpha * E / T
        assert abs(diff - got) <= size * step ** 2 + 64 * U * float(out["loss"]) / step


# ------------------------------------------------------------------------------------------------
# adapters
# ------------------------------------------------------------------------------------------------
def _adapter_inputs(rng, T, K, N, R, n, x, w, o, ragged):
    A, A64 = _put(rng, (n, R, K), _dt(w), K ** -0.5)
    Bm, B64 = _put(rng, (n, N, R), _dt(w), 0.2)
    X, X64 = _put(rng, (T, K), _dt(x))
    base, base64 = _put(rng, (T, N), _dt(o))
    scale, scale64 = _put(rng, (n,), _dt("f32"), 0.5, 1.0)
    ids = rng.integers(-1, n, T).astype(np.int32)
    ranks = rng.integers(0, R + 1, n).astype(np.int32) if ragged else None
    return A, A64, Bm, B64, X, X64, base, base64, scale, scale64, ids, ranks


def _adapter_roundings(K, R):
    """Errors of a sum of K products have either sign: 2 sqrt(K) roundings of the sum of absolute values, the same for the second
    sum, and a few for partial sums, scale and base."""
    return 2 * K ** 0.5 + 2 * R ** 0.5 + 16


def _check_adapter(got, ref, mag, base64, K, R, what):
    _close(got, ref, mag + (0 if base64 is None else np.abs(base64)), _adapter_roundings(K, R), what)


@pytest.mark.parametrize("T,K,N,R,n", [(1, 1, 1, 1, 1), (1, 64, 64, 4, 2), (1, 4096, 512, 16, 3), (2, 257, 33, 5, 2), (7, 512, 1000, 8, 3),
                                       (16, 1408, 256, 16, 20), (17, 100, 31, 17, 4), (33, 2048, 130, 64, 40), (64, 300, 2816, 24, 64),
                                       (65, 768, 96, 128, 3), (100, 1111, 77, 100, 5), (128, 256, 4096, 32, 1), (200, 96, 160, 256, 2),
                                       (300, 640, 64, 12, 100), (515, 513, 515, 33, 7), (1025, 256, 200, 16, 9), (1500, 72, 1024, 40, 500)])
@pytest.mark.parametrize("x,w,o", [("f32", "bf16", "f32"), ("bf16", "bf16", "bf16"), ("f16", "f16", "f32"), ("f32", "f32", "f32"),
                                   ("bf16", "f32", "f16"), ("f16", "bf16", "bf16")])
def test_adapter_apply(B, T, K, N, R, n, x, w, o):
    import torch
    rng = np.random.default_rng(T + 10 * K + R)
    ragged = (T + K) % 2 == 1
    A, A64, Bm, B64, X, X64, base, base64, scale, scale64, ids, ranks = _adapter_inputs(rng, T, K, N, R, n, x, w, o, ragged)
    print(f"T={T} K={K} N={N} R={R} n={n} {x} {w} {o}", flush=True)
    t_ids = torch.from_numpy(ids).cuda()
    ad = B.DeviceAdapters(A, Bm, scale, None if ranks is None else torch.from_numpy(ranks).cuda())
    got = B.cq_adapter_apply(ad, X, t_ids, base=base)
    ref, mag = O.adapter_apply(X64, ids, A64, B64, scale64, ranks, base64)
    _check_adapter(got, ref, mag, base64, K, R, "mixed")
    none = torch.from_numpy(ids < 0).cuda()
    assert got[none].equal(base[none])
    # prompts: neighbours share an adapter
    runs = np.sort(ids)
    got = B.cq_adapter_apply(ad, X, torch.from_numpy(runs).cuda(), base=base)
    ref, mag = O.adapter_apply(X64, runs, A64, B64, scale64, ranks, base64)
    _check_adapter(got, ref, mag, base64, K, R, "runs")
    # a row's result does not depend on its neighbours (where the kernel is the same: the same batch in another order)
    perm = rng.permutation(T)
    p = torch.from_numpy(perm).cuda()
    one, two = B.cq_adapter_apply(ad, X, t_ids, base=base), B.cq_adapter_apply(ad, X[p], t_ids[p], base=base[p])
    assert two.equal(one[p])


@pytest.mark.parametrize("T,K,N,R,n", [(1040, 1152, 80, 24, 5), (1100, 2304, 64, 16, 3), (1030, 4224, 40, 40, 4), (1090, 1024, 130, 8, 2), (1026, 1000, 96, 70, 3),
                                       (30, 4300, 96, 48, 9), (900, 1500, 64, 32, 4), (20, 4096, 600, 12, 20), (3, 2049, 1024, 32, 3),
                                       (384, 640, 1100, 16, 30), (385, 640, 1100, 16, 30), (383, 200, 2100, 40, 2)])
@pytest.mark.parametrize("x,w,o", [("f32", "bf16", "f32"), ("bf16", "bf16", "bf16"), ("f16", "f16", "f16"), ("f32", "f32", "f32")])
def test_adapter_widths_around_the_rounds_of_the_sum(B, T, K, N, R, n, x, w, o):
    """K of whole rounds, of rounds and units, of units and a rest; several adapters within a tile share the values of X."""
    import torch
    rng = np.random.default_rng(T + K)
    A, A64, Bm, B64, X, X64, base, base64, scale, scale64, ids, _ = _adapter_inputs(rng, T, K, N, R, n, x, w, o, False)
    print(f"T={T} K={K} N={N} R={R} n={n} {x} {w} {o}", flush=True)
    ids[:T // 2] = np.sort(ids[:T // 2])
    got = B.cq_adapter_apply(B.DeviceAdapters(A, Bm, scale), X, torch.from_numpy(ids).cuda(), base=base)
    ref, mag = O.adapter_apply(X64, ids, A64, B64, scale64, None, base64)
    _check_adapter(got, ref, mag, base64, K, R, f"K={K}")


def test_adapter_rows_in_wider_rows_and_in_place(B):
    import torch
    rng = np.random.default_rng(31)
    T, K, N, R, n = 40, 192, 96, 16, 6
    for x, o, cut in (("bf16", "f32", 8), ("bf16", "bf16", 3), ("f32", "f32", 1), ("f32", "bf16", 16)):
        A, A64, Bm, B64, X, X64, base, base64, scale, scale64, ids, ranks = _adapter_inputs(rng, T, K, N, R, n, x, "bf16", o, True)
        ad = B.DeviceAdapters(A, Bm, scale, torch.from_numpy(ranks).cuda())
        t_ids = torch.from_numpy(ids).cuda()
        ref, mag = O.adapter_apply(X64, ids, A64, B64, scale64, ranks, base64)
        wide_x = torch.full((T, K + 2 * cut), float("nan"), dtype=X.dtype, device="cuda")
        wide_o = torch.full((T, N + 2 * cut), 7.0, dtype=base.dtype, device="cuda")
        wide_x[:, cut:cut + K], wide_o[:, cut:cut + N] = X, base
        view = wide_o[:, cut:cut + N]
        out = B.cq_adapter_apply(ad, wide_x[:, cut:cut + K], t_ids, base=view, out=view)
        assert out is view
        _check_adapter(view, ref, mag, base64, K, R, "in place")
        assert (wide_o[:, :cut] == 7).all() and (wide_o[:, cut + N:] == 7).all()
        # without a base, and without scales
        got = B.cq_adapter_apply(B.DeviceAdapters(A, Bm), X, t_ids, out_dtype=_dt(o))
        ref, mag = O.adapter_apply(X64, ids, A64, B64)
        _check_adapter(got, ref, mag, None, K, R, "no base")
        assert not got[t_ids < 0].any()


@pytest.mark.parametrize("T", [5, 80, 1100])
def test_adapter_values_that_are_not_used_do_not_matter(B, T):
    """Rows beyond an adapter's rank, adapters of nobody, ids of no adapter, a token with NaN beside others."""
    import torch
    rng = np.random.default_rng(32)
    K, N, R, n = 160, 70, 24, 5
    for x, w in (("f32", "bf16"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "f32")):
        A, A64, Bm, B64, X, X64, base, base64, scale, scale64, ids, _ = _adapter_inputs(rng, T, K, N, R, n, x, w, "f32", False)
        ranks = np.array([24, 16, 3, 0, 7], dtype=np.int32)
        ids[ids == 4] = 0
        ids[T // 2] = [1 << 30, -(1 << 31), n, -1][T % 4]
        ids[1] = 2
        for a in range(n):
            A[a, ranks[a]:] = float("nan")
            Bm[a, :, ranks[a]:] = float("inf")
        A[4], Bm[4] = float("nan"), float("nan")
        scale[3] = float("nan")          # of an adapter of rank 0 ...
        scale64[3] = 0.0
        ids[ids == 3] = -1               # ... that nobody asks for
        X[1] = float("nan")
        ad = B.DeviceAdapters(A, Bm, scale, torch.from_numpy(ranks).cuda())
        got = B.cq_adapter_apply(ad, X, torch.from_numpy(ids).cuda(), base=base)
        X64[1] = 0.0
        ref, mag = O.adapter_apply(X64, ids, np.nan_to_num(A64), np.nan_to_num(B64), scale64, ranks, base64)
        assert got[1].isnan().all()
        rest = [t for t in range(T) if t != 1]
        _check_adapter(got[rest], ref[rest], mag[rest], base64[rest], K, R, f"{x} {w}")


def test_adapter_of_rank_zero_and_empty_batches(B):
    import torch
    rng = np.random.default_rng(33)
    A, _, Bm, _, X, _, base, _, scale, _, ids, _ = _adapter_inputs(rng, 20, 64, 48, 8, 2, "bf16", "bf16", "bf16", False)
    ad = B.DeviceAdapters(A, Bm, scale, torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert B.cq_adapter_apply(ad, X, torch.from_numpy(ids).cuda(), base=base).equal(base)
    over = B.DeviceAdapters(A, Bm, scale, torch.tensor([99, -4], dtype=torch.int32, device="cuda"))   # clamped to [0, rank]
    want = B.DeviceAdapters(A, Bm, scale, torch.tensor([8, 0], dtype=torch.int32, device="cuda"))
    t_ids = torch.from_numpy(ids).cuda()
    assert B.cq_adapter_apply(over, X, t_ids, base=base).equal(B.cq_adapter_apply(want, X, t_ids, base=base))
    assert B.cq_adapter_apply(ad, X[:0], t_ids[:0], base=base[:0]).shape == (0, 48)


# ------------------------------------------------------------------------------------------------
# streams, graphs, refusals of the binding
# ------------------------------------------------------------------------------------------------
def _everything(B, rng):
    """One call of each operator as a closure that writes into tensors of its own."""
    import torch
    c = _Norm(B, rng, 70, 520, "bf16", "f32", "f32", True, "row", True)
    z, _, ids = _routing(rng, 300, 24, 4, torch.float32)
    t_ids = torch.from_numpy(ids).cuda()
    off = torch.from_numpy(_offsets(rng, 300, 4)).cuda()
    A, _, Bm, _, X, _, base, _, scale, _, aid, _ = _adapter_inputs(rng, 50, 256, 96, 16, 5, "f32", "bf16", "f32", False)
    ad = B.DeviceAdapters(A, Bm, scale)
    a_ids = torch.from_numpy(aid).cuda()

    def call():
        f = B.cq_block_norm(c.norm, c.h, c.y, c.gate)
        g = B.cq_block_norm_grad(c.norm, f["h"], c.y, c.gate, dh=c.dh, dx=c.dx)
        b = B.cq_balance_loss(z, t_ids, 0.1, off)
        d = B.cq_balance_loss_grad(z, b["counts"], b["tokens"], 4, 0.1, off)
        return [f["h"], f["x"], *g.values(), *b.values(), d, B.cq_adapter_apply(ad, X, a_ids, base=base)]
    return call, (c.h, c.y, z, X)


def test_operators_on_a_stream_of_their_own(B):
    import torch
    call, _ = _everything(B, np.random.default_rng(41))
    want = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call()
    side.synchronize()
    assert all(a.equal(b) for a, b in zip(got, want))


def test_operators_replayed_from_a_captured_graph(B):
    """Several replays with new inputs and eager work in between, each compared with the eager call bit for bit."""
    import torch
    call, inputs = _everything(B, np.random.default_rng(42))
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for rep in range(4):
        for t in inputs:
            t.mul_(1.0 - 0.1 * rep)
        want = [v.clone() for v in call()]
        torch.cuda.synchronize()
        for v in held:
            v.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        assert all(a.equal(b) for a, b in zip(held, want)), rep


def test_binding_refuses_what_the_kernels_cannot_take(B):
    import torch
    w = torch.ones(32, device="cuda")
    norm = B.BlockNorm(w, w)
    h = torch.ones((4, 32), device="cuda")
    for bad in (lambda: B.cq_block_norm(norm, h.t(), h), lambda: B.cq_block_norm(norm, h, h.half()), lambda: B.cq_block_norm(norm, h.cpu()),
                lambda: B.cq_block_norm(norm, h[:, :16]), lambda: B.cq_block_norm(norm, h, None, w[:4]), lambda: B.cq_block_norm(norm, h.double()),
                lambda: B.cq_block_norm(norm, h, h, w[:5]), lambda: B.BlockNorm(w, w[:8]), lambda: B.BlockNorm(w.double()),
                lambda: B.cq_block_norm_grad(B.BlockNorm(None, w), h, h, dx=h), lambda: B.cq_block_norm_grad(norm, h, h, dh=h.half())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.CqError) as e:
        B.cq_block_norm(B.BlockNorm(w.half(), None), h)          # f16 weights beside an fp32 stream
    assert e.value.status == 3
    z, ids = torch.zeros((4, 8), device="cuda"), torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    for bad in (lambda: B.cq_balance_loss(z, ids.long(), 0.1), lambda: B.cq_balance_loss(z, ids[:3], 0.1), lambda: B.cq_balance_loss(z.t(), ids, 0.1),
                lambda: B.cq_balance_loss(z, ids, 0.1, ids[0].long()), lambda: B.cq_balance_loss(z, ids, 0.1, None, z[:, 0]),
                lambda: B.cq_balance_loss_grad(z, ids, ids[:2, 0], 2, 0.1)):
        with pytest.raises(ValueError):
            bad()
    A, Bm = torch.zeros((2, 4, 16), device="cuda"), torch.zeros((2, 8, 4), device="cuda")
    ad = B.DeviceAdapters(A, Bm)
    X, aid = torch.zeros((3, 16), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    for bad in (lambda: B.DeviceAdapters(A, Bm.half()), lambda: B.DeviceAdapters(A, Bm[:, :, :2]), lambda: B.DeviceAdapters(A, Bm, aid[:2].float().cpu()),
                lambda: B.cq_adapter_apply(ad, X[:, :8], aid), lambda: B.cq_adapter_apply(ad, X.t().contiguous().t(), aid),
                lambda: B.cq_adapter_apply(ad, X, aid.long()), lambda: B.cq_adapter_apply(ad, X, aid, base=torch.zeros((3, 7), device="cuda")),
                lambda: B.cq_adapter_apply(ad, X[:1].expand(3, 16), aid)):
        with pytest.raises(ValueError):
            bad()


def test_tensors_of_a_handle_may_be_replaced(B):
    """A training step gives the norm and the adapters new tensors: the next call reads those."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(6)
    h = torch.randn((5, 64), generator=g, device="cuda")
    norm = B.BlockNorm(torch.ones(64, device="cuda"))
    first = B.cq_block_norm(norm, h)["x"]
    norm.w_pre = torch.full((64,), 2.0, device="cuda")
    assert B.cq_block_norm(norm, h)["x"].equal(2 * first)
    A, Bm = torch.randn((2, 4, 64), generator=g, device="cuda"), torch.randn((2, 32, 4), generator=g, device="cuda")
    ad, ids = B.DeviceAdapters(A, Bm), torch.tensor([0, 1, 0, -1, 1], dtype=torch.int32, device="cuda")
    first = B.cq_adapter_apply(ad, h, ids)
    ad.B = 2 * Bm
    assert B.cq_adapter_apply(ad, h, ids).equal(2 * first)


def test_rows_beyond_32_bit_offsets(B):
    """More than 2^31 values: the rows at the end equal those of a call on them alone."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(5)
    T, H, n = 70000, 32768, 3
    w = torch.rand(H, generator=g, device="cuda") + 0.5
    norm = B.BlockNorm(w, w, block_dtype=torch.bfloat16)
    h = torch.ones((T, H), dtype=torch.bfloat16, device="cuda")
    tail = torch.randn((n, H), generator=g, device="cuda").bfloat16()
    h[T - n:] = tail
    print("norm", flush=True)
    out = B.cq_block_norm(norm, h, h)
    want = B.cq_block_norm(norm, tail, tail)
    assert out["h"][T - n:].equal(want["h"]) and out["x"][T - n:].equal(want["x"])
    got = B.cq_block_norm_grad(norm, h, h, dh=h, dx=h, want_weights=False)
    want = B.cq_block_norm_grad(norm, tail, tail, dh=tail, dx=tail, want_weights=False)
    assert got["dh"][T - n:].equal(want["dh"]) and got["dy"][T - n:].equal(want["dy"])
    del out, got, h
    print("balance", flush=True)
    T, E = 2200000, 1024
    z = torch.zeros((T, E), dtype=torch.float16, device="cuda")
    z[T - n:] = torch.randn((n, E), generator=g, device="cuda").half()
    ids = torch.zeros((T, 1), dtype=torch.int32, device="cuda")
    ids[T - n:, 0] = torch.arange(n, device="cuda")
    off = torch.tensor([0, T - n, T], dtype=torch.int32, device="cuda")
    bal = B.cq_balance_loss(z, ids, 1.0, off)
    alone = B.cq_balance_loss(z[T - n:].clone(), ids[T - n:].clone(), 1.0)
    assert bal["counts"][1].equal(alone["counts"][0]) and bal["tokens"].tolist() == [T - n, n, 2]
    assert (bal["probs"][1] - alone["probs"][0]).abs().max() <= 200 * U * alone["probs"].max()
    one = torch.tensor([T - n, n, 1], dtype=torch.int32, device="cuda")
    grad = B.cq_balance_loss_grad(z, bal["counts"], one, 1, 1.0, off)
    assert grad[T - n:].equal(B.cq_balance_loss_grad(z[T - n:].clone(), alone["counts"], alone["tokens"], 1, 1.0))
    del z, grad, ids
    print("adapters", flush=True)
    T, K = 1100, 1 << 21
    X = torch.ones((T, K), dtype=torch.bfloat16, device="cuda")
    X[T - n:] = torch.randn((n, K), generator=g, device="cuda").bfloat16()
    A = (torch.randn((2, 8, K), generator=g, device="cuda") * K ** -0.5).bfloat16()
    Bm = torch.randn((2, 64, 8), generator=g, device="cuda").bfloat16()
    ad = B.DeviceAdapters(A, Bm)
    ids = torch.ones(T, dtype=torch.int32, device="cuda")
    got = B.cq_adapter_apply(ad, X, ids)[T - n:].double()
    low = X[T - n:].double() @ A[1].double().t()
    mag = X[T - n:].double().abs() @ A[1].double().abs().t() @ Bm[1].double().abs().t()
    assert ((got - low @ Bm[1].double().t()).abs() <= _adapter_roundings(K, 8) * U * mag).all()
