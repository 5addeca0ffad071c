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
