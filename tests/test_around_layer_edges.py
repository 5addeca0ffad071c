"""The operators around the layer on the GPU where fp32 arithmetic or the launch can go wrong although ordinary values and sizes come out
right.  Bounds as in test_around_layer: a number of fp32 roundings times the oracle's magnitudes, and one rounding to the result's type."""
import numpy as np
import pytest

from oracle import around_oracle as O
from tests import test_around_layer as A
from tests.test_around_layer import B  # noqa: F401  (the library, a fixture)

pytestmark = pytest.mark.gpu

U = A.U


# ------------------------------------------------------------------------------------------------
# gates that are nearly open or shut
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("stream,block", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("gate,H", [("row", 64), ("elem", 64), ("row", 1111), ("elem", 1111), ("elem", 8192), ("elem", 9000), ("row", 16384)])
def test_gradients_of_gates_far_from_zero(B, stream, block, gate, H):  # noqa: F811
    """sigmoid' = s (1 - s) is as exact at |z| = 20 or 80 as at 0: the oracle's magnitude of a gate's gradient has the slope as a
    factor, so that a difference of nearly equal numbers does not pass."""
    import torch
    T = 12
    rng = np.random.default_rng(H)
    c = A._Norm(B, rng, T, H, stream, block, "f32", True, gate, True)
    z = np.resize(np.array([8.0, -8.0, 12.0, -12.0, 15.0, 16.0, -16.0, 17.0, 20.0, -20.0, 80.0, -80.0]), T)
    z = z if gate == "row" else np.stack([np.roll(np.resize(z, H), t) for t in range(T)])
    c.gate = torch.from_numpy(z).to(A._dt(block)).cuda()
    c.gate64 = c.gate.double().cpu().numpy()
    print(f"{stream} {block} {gate} H={H}", flush=True)
    out = B.cq_block_norm(c.norm, c.h, c.y, c.gate)
    A._check_norm(out, c.forward(), T, "forward")
    got = B.cq_block_norm_grad(c.norm, out["h"], c.y, c.gate, dh=c.dh, dx=c.dx)
    A._check_norm(got, c.backward(out["h"].double().cpu().numpy()), T, "backward")
    near = c.gate.abs() <= 20          # (at 80 a value may lie below a type's smallest)
    assert (got["dgate"][near] != 0).all()


# ------------------------------------------------------------------------------------------------
# the balance loss along its gradient
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T,E,k,S,padded", [(50, 9, 2, 1, False), (120, 16, 3, 5, True), (700, 64, 6, 3, True), (60, 300, 8, 2, False)])
def test_balance_gradient_along_itself(B, T, E, k, S, padded):  # noqa: F811
    """(L(z + s v) - L(z - s v)) / 2s of the forward kernel against |gradient|, v the gradient's direction, and against the gradient
    along the part of it that each sequence has.  Truncation: along v a token's sum of f p has the third derivative
    E[f' v'^3] - 3 E[f' v'] E[v'^2] (f', v' centred, expectations under p), at most 4 F V^3 with F and V the ranges of f and v over the
    experts.  Rounding: both losses by the roundings that test_around_layer derives, and z + s v by half a step of fp32 times the
    gradient.  The bound is small beside what it is held against: a gradient of zero, of the wrong sign or off by a tenth fails."""
    import torch
    rng = np.random.default_rng(T)
    alpha, step = 3.0, 2.0 ** -4
    z, z64, ids = A._routing(rng, T, E, k, torch.float32)
    off = A._offsets(rng, T, S) if S > 1 else None
    mask = rng.random(T) < 0.8 if padded else None
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    t_ids, t_off, t_mask = dev(ids), dev(off), dev(mask)
    out = B.cq_balance_loss(z, t_ids, alpha, t_off, t_mask)
    g = B.cq_balance_loss_grad(z, out["counts"], out["tokens"], k, alpha, t_off, t_mask).double().cpu().numpy()
    seqs = [m for m in O.members(T, off, mask) if len(m)]
    counts = [c for c, n in zip(out["counts"].cpu().numpy(), out["tokens"].cpu().numpy()[:-1]) if n]
    loss = lambda s, v: float(B.cq_balance_loss(z + dev((s * v).astype(np.float32)), t_ids, alpha, t_off, t_mask)["loss"])
    parts = [np.arange(T)] + (seqs if len(seqs) > 1 else [])
    for part in parts:
        v = np.zeros((T, E))
        v[part] = g[part]
        v = (v / np.linalg.norm(v)).astype(np.float32).astype(np.float64)
        diff, got = (loss(step, v) - loss(-step, v)) / (2 * step), float((g * v).sum())
        cut = 0.0
        for at, c in zip(seqs, counts):
            F, V = np.ptp(c) / (k * len(at)), np.ptp(v[at], axis=1)
            cut += alpha * E / (len(seqs) * len(at)) * 4 * F * (V ** 3).sum() * step ** 2 / 6
        roundings = 256 + T // 64 + S
        bound = cut + roundings * U * float(out["loss"]) / step + U * (np.abs(g) * (np.abs(z64) + 1)).sum() / step
        print(f"{diff:.6g} {got:.6g} bound {bound:.3g}", flush=True)
        assert bound < 0.1 * got
        assert abs(diff - got) <= bound


# ------------------------------------------------------------------------------------------------
# batches beyond one launch, whose threads along a dimension are counted in 32 bits
# ------------------------------------------------------------------------------------------------
def _around(step, T):
    """Rows on either side of every boundary between launches, and the last ones."""
    import torch
    at = [t + d for t in range(0, T, step) for d in (-1, 0, 1)] + [T - 2, T - 1]
    return torch.tensor(sorted({t for t in at if 0 <= t < T}), device="cuda")


def test_norm_of_more_rows_than_one_launch_takes(B):  # noqa: F811
    import torch
    T, H = (1 << 26) + 3, 2
    g = torch.Generator(device="cuda").manual_seed(1)
    h = torch.randn((T, H), generator=g, device="cuda").bfloat16()
    y = torch.randn((T, H), generator=g, device="cuda").bfloat16()
    gate = torch.randn(T, generator=g, device="cuda").bfloat16()
    w = torch.tensor([0.5, 2.0], device="cuda")
    norm = B.BlockNorm(w, w, gate_sigmoid=True, block_dtype=torch.bfloat16)
    h_out, x_out = torch.full_like(h, float("nan")), torch.full_like(h, float("nan"))
    print("rows", flush=True)
    B.cq_block_norm(norm, h, y, gate, h_out=h_out, x_out=x_out)
    assert h_out.isfinite().all() and x_out.isfinite().all()
    at = _around(1 << 21, T)
    for gates in (gate, y):
        if gates is y:
            print("a gate per value", flush=True)
            B.cq_block_norm(norm, h, y, y, h_out=h_out, x_out=x_out)
        want = B.cq_block_norm(norm, h[at], y[at], gates[at])
        assert h_out[at].equal(want["h"]) and x_out[at].equal(want["x"])
    print("without a block", flush=True)
    assert B.cq_block_norm(norm, h, x_out=x_out)["x"][at].equal(B.cq_block_norm(norm, h[at])["x"])


def test_balance_gradient_of_more_tokens_than_one_launch_takes(B):  # noqa: F811
    import torch
    T, E = (1 << 26) + 5, 257
    g = torch.Generator(device="cuda").manual_seed(2)
    at = _around(1 << 25, T)
    z = torch.zeros((T, E), dtype=torch.float16, device="cuda")
    z[at] = torch.randn((len(at), E), generator=g, device="cuda").half()
    counts = torch.randint(0, 1000, (1, E), generator=g, device="cuda", dtype=torch.int32)
    tokens = torch.tensor([100, 1], dtype=torch.int32, device="cuda")
    print("gradient", flush=True)
    got = B.cq_balance_loss_grad(z, counts, tokens, 2, 1.0)
    assert got[at].equal(B.cq_balance_loss_grad(z[at], counts, tokens, 2, 1.0))
    assert got[12345].equal(got[T - 12345])
    del z, got
    torch.cuda.empty_cache()


def test_balance_loss_of_more_sequences_than_one_launch_takes(B):  # noqa: F811
    """One token each, and one sequence without any."""
    import torch
    T, E = (1 << 22) + 2, 4
    g = torch.Generator(device="cuda").manual_seed(3)
    z = torch.randn((T, E), generator=g, device="cuda")
    ids = torch.randint(0, E, (T, 1), generator=g, device="cuda", dtype=torch.int32)
    off = torch.cat([torch.arange(T + 1, device="cuda"), torch.tensor([T], device="cuda")]).int()
    print("loss", flush=True)
    out = B.cq_balance_loss(z, ids, 1.0, off)
    p = torch.softmax(z.double(), dim=1)
    one = torch.nn.functional.one_hot(ids[:, 0].long(), E)
    assert out["counts"][:T].equal(one.int()) and not out["counts"][T].any()
    assert out["tokens"][:T].eq(1).all() and out["tokens"][T:].tolist() == [0, T]
    assert ((out["probs"][:T].double() - p).abs() <= 128 * U * p).all() and not out["probs"][T].any()
    want = E * (p * one).sum().item() / T
    assert abs(out["loss"].item() - want) <= (256 + T // 1024) * U * want


def test_adapters_of_more_tokens_than_one_launch_takes(B):  # noqa: F811
    import torch
    T, K, N, n = (1 << 27) + 40, 2, 3, 5
    g = torch.Generator(device="cuda").manual_seed(4)
    A_, Bm = torch.randn((n, 1, K), generator=g, device="cuda").bfloat16(), torch.randn((n, N, 1), generator=g, device="cuda").bfloat16()
    X = torch.randn((T, K), generator=g, device="cuda").bfloat16()
    base = torch.randn((T, N), generator=g, device="cuda").bfloat16()
    ids = torch.randint(-1, n, (T,), generator=g, device="cuda", dtype=torch.int32)
    print("adapters", flush=True)
    got = B.cq_adapter_apply(B.DeviceAdapters(A_, Bm), X, ids, base=base)
    for t in range(0, T, 1 << 24):
        a = ids[t:t + (1 << 24)].long()
        on, a = (a >= 0)[:, None], a.clamp(min=0)
        x, b = X[t:t + (1 << 24)].double(), base[t:t + (1 << 24)].double()
        up = Bm[a, :, 0].double()
        want = b + on * (A_[a, 0].double() * x).sum(1, keepdim=True) * up
        mag = b.abs() + (A_[a, 0].double() * x).abs().sum(1, keepdim=True) * up.abs()
        bound = A._adapter_roundings(K, 1) * U * mag
        bound = bound + torch.finfo(torch.bfloat16).eps / 2 * (want.abs() + bound) + 1e-40
        assert ((got[t:t + (1 << 24)].double() - want).abs() <= bound).all(), t


# ------------------------------------------------------------------------------------------------
# adapters with infinite weights
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T", [1, 5, 80, 1100])
@pytest.mark.parametrize("R,K", [(8, 64), (12, 300), (16, 4096), (40, 1111), (100, 640)])
@pytest.mark.parametrize("x,w,o", [("f32", "bf16", "f32"), ("f32", "bf16", "bf16"), ("bf16", "bf16", "bf16"), ("f16", "f16", "f32"), ("f32", "f32", "f32"),
                                   ("bf16", "f32", "f16")])
def test_adapters_with_infinite_weights(B, T, R, K, x, w, o):  # noqa: F811
    """An infinite weight makes the infinities that the definition gives, and NaN only where that has 0 times infinity or a difference of
    infinities.  Small whole numbers: every sum is exact, so everything else is equal to the last bit."""
    import torch
    rng = np.random.default_rng(R + K)
    n, N = 5, 70
    A_, Bm = rng.integers(-2, 3, (n, R, K)).astype(float), rng.integers(-1, 2, (n, N, R)).astype(float)
    A_[:, :, rng.random(K) < 0.9] = 0.0                # (sums stay small enough for every type)
    X, base = rng.integers(-1, 2, (T, K)).astype(float), rng.integers(-3, 4, (T, N)).astype(float)
    ids = rng.integers(-1, n, T).astype(np.int32)
    ids[0] = 0
    ranks = np.array([R, R, max(1, R - 3), R, 1], dtype=np.int32)
    for a, k in ((0, K - 1), (1, 0), (2, K // 2)):
        A_[a, ranks[a] - 1, k] = np.inf if a else -np.inf
    Bm[1, 3, 0], Bm[3, N - 1, R - 1], Bm[3, 5, 0], Bm[4, 0, 0] = np.inf, -np.inf, np.inf, np.inf
    X[1::7, K - 1], X[0, K - 1] = 0.0, 1.0
    with np.errstate(invalid="ignore"):
        want, _ = O.adapter_apply(X, ids, A_, Bm, None, ranks, base)
    put = lambda v, d: torch.from_numpy(v).to(A._dt(d)).cuda()
    print(f"T={T} R={R} K={K} {x} {w} {o}", flush=True)
    ad = B.DeviceAdapters(put(A_, w), put(Bm, w), None, torch.from_numpy(ranks).cuda())
    for order in (np.arange(T), np.argsort(ids, kind="stable")):
        got = B.cq_adapter_apply(ad, put(X[order], x), torch.from_numpy(ids[order]).cuda(), base=put(base[order], o))
        ref = torch.from_numpy(want[order]).to(A._dt(o))
        assert ((got.cpu() == ref) | (got.cpu().isnan() & ref.isnan())).all()
