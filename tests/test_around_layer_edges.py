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
