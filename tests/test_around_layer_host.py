"""The operators around the expert layer without a GPU: the oracle's gradients against differences, the refusals of the C
entry points (arguments are checked before any device call), and the workspace queries."""
import ctypes

import numpy as np
import pytest

from oracle import around_oracle as O
from paper_2604_10496_amd import binding as B

ONE = ctypes.c_void_p(256)   # a non-null dummy that must never be dereferenced
F16, F32, BF16 = B.CQ_A_F16, B.CQ_A_F32, B.CQ_A_BF16


# ------------------------------------------------------------------------------------------------
# the oracle's gradients against central differences of its forward pass, in float64
# ------------------------------------------------------------------------------------------------
def _difference(f, x, d, step=1e-5):
    return (f(x + step * d) - f(x - step * d)) / (2 * step)


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate", ["none", "row", "elem"])
@pytest.mark.parametrize("use_sigmoid", [False, True])
def test_oracle_block_norm_gradients_match_differences(post, gate, use_sigmoid):
    rng = np.random.default_rng(3)
    T, H, eps, rho, beta = 4, 9, 1e-3, 0.8, 1.3
    h, y = rng.standard_normal((T, H)), rng.standard_normal((T, H))
    g = {"none": None, "row": rng.standard_normal(T), "elem": rng.standard_normal((T, H))}[gate]
    w_pre, w_post = rng.standard_normal(H), rng.standard_normal(H) if post else None
    ch, cx = rng.standard_normal((T, H)), rng.standard_normal((T, H))

    def loss(**over):
        a = dict(h=h, y=y, gate=g, w_pre=w_pre, w_post=w_post)
        a.update(over)
        out, _ = O.block_norm(a["h"], a["y"], a["gate"], a["w_pre"], a["w_post"], eps, rho, beta, use_sigmoid)
        return (out["h"] * ch).sum() + (out["x"] * cx).sum()
    new = O.block_norm(h, y, g, w_pre, w_post, eps, rho, beta, use_sigmoid)[0]["h"]
    grads, _ = O.block_norm_grad(new, y, g, ch, cx, w_pre, w_post, eps, rho, beta, use_sigmoid)
    names = {"dh": ("h", h), "dy": ("y", y), "dw_pre": ("w_pre", w_pre), "dgate": ("gate", g), "dw_post": ("w_post", w_post)}
    assert set(grads) == {k for k, (_, v) in names.items() if v is not None}
    for name, got in grads.items():
        arg, at = names[name]
        for _ in range(3):
            d = rng.standard_normal(at.shape)
            want = _difference(lambda v: loss(**{arg: v}), at, d)
            assert abs((got * d).sum() - want) <= 1e-7 * (1 + np.abs(got * d).sum()), name


def test_oracle_pre_norm_alone_matches_differences():
    rng = np.random.default_rng(4)
    h, w, ch, cx = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal((3, 7)), rng.standard_normal((3, 7))
    f = lambda v: (v * ch).sum() + (O.block_norm(v, None, None, w, None, 1e-3, 0.5, 2.0, False)[0]["x"] * cx).sum()
    grads, _ = O.block_norm_grad(h, None, None, ch, cx, w, None, 1e-3, 0.5, 2.0, False)
    d = rng.standard_normal(h.shape)
    assert abs((grads["dh"] * d).sum() - _difference(f, h, d)) <= 1e-7 * np.abs(grads["dh"] * d).sum()


def test_oracle_balance_gradient_matches_differences():
    rng = np.random.default_rng(5)
    T, E, k = 23, 6, 2
    z = rng.standard_normal((T, E))
    ids = np.argsort(-z, axis=1)[:, :k]
    ids[3, 1] = -1
    mask = rng.random(T) < 0.8
    offsets = [0, 5, 5, 17, 22]
    grad, _ = O.balance_loss_grad(z, ids, 0.3, 1.7, offsets, mask)
    f = lambda v: 1.7 * O.balance_loss(v, ids, 0.3, offsets, mask)["loss"]
    for _ in range(4):
        d = rng.standard_normal(z.shape)
        assert abs((grad * d).sum() - _difference(f, z, d)) <= 1e-8
    assert not grad[22].any() and not grad[~mask].any()


def test_oracle_balance_by_hand():
    """Two experts, top-1, all tokens to expert 0 with even probabilities: alpha * 2 * (1 * 1/2 + 0 * 1/2) = alpha."""
    out = O.balance_loss(np.zeros((4, 2)), np.zeros((4, 1), dtype=np.int64), 0.25)
    assert out["loss"] == 0.25 and out["counts"].tolist() == [[4, 0]] and out["tokens"].tolist() == [4, 1]


# ------------------------------------------------------------------------------------------------
# refusals
# ------------------------------------------------------------------------------------------------
def _spec(**k):
    a = dict(H=64, stream_kind=BF16, block_kind=F32, weight_kind=F32, gate_kind=0, gate_sigmoid=0, eps=1e-6, residual_scale=1.0,
             branch_scale=1.0, w_pre=256, w_post=256)
    a.update(k)
    return B.BlockNormSpec(*[a[n] for n, _ in B.BlockNormSpec._fields_])


def test_block_norm_refusals():
    lib = B.load_library()

    def call(T=4, h=ONE, y=ONE, gate=None, h_out=ONE, x_out=ONE, **k):
        return lib.cq_block_norm(ctypes.byref(_spec(**k)), h, y, gate, T, h_out, x_out, None)
    assert lib.cq_block_norm(None, ONE, ONE, None, 4, ONE, ONE, None) == 1
    assert call(h=None) == 1 and call(h_out=None) == 1 and call(y=None, x_out=None) == 1 and call(w_pre=None) == 1
    assert call(gate_kind=1) == 1 and call(gate_kind=2) == 1
    assert call(T=-1) == 2 and call(T=(1 << 30) + 1) == 2 and call(H=0) == 2 and call(H=32769) == 2
    assert call(eps=0.0) == 2 and call(eps=-1.0) == 2 and call(eps=float("nan")) == 2 and call(eps=float("inf")) == 2
    assert call(stream_kind=0) == 3 and call(stream_kind=9) == 3 and call(block_kind=F16) == 3 and call(weight_kind=F16) == 3
    assert call(stream_kind=F32, block_kind=BF16) == 3 and call(gate_kind=3) == 3
    assert call(T=0) == 0 and call(T=0, h=None, y=None, h_out=None, x_out=None) == 0


def test_block_norm_grad_refusals():
    lib = B.load_library()

    def call(T=4, h=ONE, y=ONE, gate=None, dh=ONE, dx=ONE, o_dh=ONE, o_dy=ONE, o_dg=None, o_pre=ONE, o_post=ONE, ws=ONE, n=1 << 30, **k):
        return lib.cq_block_norm_grad(ctypes.byref(_spec(**k)), h, y, gate, dh, dx, T, o_dh, o_dy, o_dg, o_pre, o_post, ws, n, None)
    assert lib.cq_block_norm_grad(None, ONE, ONE, None, ONE, ONE, 4, ONE, ONE, None, None, None, ONE, 1 << 30, None) == 1
    assert call(dh=None, dx=None) == 1 and call(o_dh=None) == 1 and call(o_dy=None) == 1 and call(h=None) == 1
    assert call(w_pre=None) == 1 and call(dx=None) == 1          # a weight's gradient without the gradient that it comes from
    assert call(w_post=None) == 1 and call(y=None) == 1
    assert call(gate_kind=1) == 1
    assert call(T=-1) == 2 and call(H=40000) == 2 and call(eps=0.0) == 2
    assert call(stream_kind=7) == 3 and call(block_kind=F16) == 3
    need = lib.cq_block_norm_grad_workspace_bytes(ctypes.byref(_spec()), 4)
    assert need > 0 and call(n=need - 1) == 4 and call(ws=None) == 4
    assert lib.cq_block_norm_grad_workspace_bytes(ctypes.byref(_spec(H=0)), 4) == 0
    assert call(T=0, o_pre=None, o_post=None) == 0


def test_balance_refusals():
    lib = B.load_library()

    def call(z=ONE, kind=F32, ids=ONE, off=ONE, S=3, mask=None, T=8, E=16, k=2, loss=ONE, counts=ONE, probs=ONE, tokens=ONE, ws=ONE,
             n=1 << 30):
        return lib.cq_balance_loss(z, kind, ids, off, S, mask, T, E, k, 0.1, loss, counts, probs, tokens, ws, n, None)
    for name in ("z", "ids", "off", "loss", "counts", "probs", "tokens"):
        assert call(**{name: None}) == 1, name
    assert call(T=-1) == 2 and call(E=0) == 2 and call(E=1025) == 2 and call(k=0) == 2 and call(k=17) == 2 and call(S=0) == 2
    assert call(E=100, k=65) == 2 and call(T=(1 << 30) + 1, k=1) == 2 and call(T=1 << 30, k=2) == 2
    assert call(kind=0) == 3 and call(kind=4) == 3
    need = lib.cq_balance_loss_workspace_bytes(4096, 16, 3)
    assert need > 0 and call(T=4096, n=need - 1) == 4 and call(T=4096, ws=None) == 4
    assert lib.cq_balance_loss_workspace_bytes(8, 16, 1) == 0      # few logits: one workgroup, no workspace
    assert lib.cq_balance_loss_workspace_bytes(8, 0, 3) == 0

    def grad(z=ONE, kind=F32, counts=ONE, tokens=ONE, off=ONE, S=3, T=8, E=16, k=2, out=ONE):
        return lib.cq_balance_loss_grad(z, kind, counts, tokens, off, S, None, T, E, k, 0.1, None, out, None)
    for name in ("z", "counts", "tokens", "off", "out"):
        assert grad(**{name: None}) == 1, name
    assert grad(T=-1) == 2 and grad(E=1025) == 2 and grad(k=17) == 2 and grad(S=0) == 2 and grad(kind=0) == 3
    assert grad(T=0, z=None, counts=None, tokens=None, out=None) == 0


def _adapters(**k):
    a = dict(n=4, rank=8, K=64, N=32, kind=BF16, A=256, B=256, scale=None, ranks=None)
    a.update(k)
    return B.Adapters(*[a[n] for n, _ in B.Adapters._fields_])


def test_adapter_refusals():
    lib = B.load_library()

    def call(X=ONE, xk=F32, ldx=64, ids=ONE, T=5, base=ONE, ldb=32, out=ONE, ok=F32, ldo=32, ws=ONE, n=1 << 30, **k):
        return lib.cq_adapter_apply(ctypes.byref(_adapters(**k)), X, xk, ldx, ids, T, base, ldb, out, ok, ldo, ws, n, None)
    assert lib.cq_adapter_apply(None, ONE, F32, 64, ONE, 5, ONE, 32, ONE, F32, 32, ONE, 1 << 30, None) == 1
    assert call(X=None) == 1 and call(ids=None) == 1 and call(out=None) == 1 and call(A=None) == 1 and call(B=None) == 1
    assert call(T=-1) == 2 and call(T=(1 << 30) + 1) == 2
    for k in (dict(rank=0), dict(rank=257), dict(K=0), dict(N=0)):
        assert call(**k) == 2, k
    assert lib.cq_adapter_apply(ctypes.byref(_adapters(n=0)), ONE, F32, 64, ONE, 5, ONE, 32, ONE, F32, 32, ONE, 1 << 30, None) == 2
    assert call(ldx=63) == 2 and call(ldb=31) == 2 and call(ldo=31) == 2
    assert call(kind=0) == 3 and call(xk=0) == 3 and call(ok=5) == 3
    s = _adapters(rank=40)
    need = lib.cq_adapter_workspace_bytes(ctypes.byref(s), F32, 5)
    assert need > 0 and call(rank=40, n=need - 1) == 4 and call(rank=40, ws=None) == 4
    assert lib.cq_adapter_workspace_bytes(ctypes.byref(_adapters()), F32, 5) == 0      # few tokens of low rank: no workspace
    assert lib.cq_adapter_workspace_bytes(ctypes.byref(_adapters(rank=300)), F32, 5) == 0
    assert call(T=0, X=None, ids=None, out=None, ws=None) == 0


def test_workspaces_never_fall_as_the_batch_grows():
    lib = B.load_library()
    T = [*range(0, 700), 4000, 4096, 4097, 70000]
    for s in (_spec(), _spec(H=1111), _spec(H=8192)):
        sizes = [lib.cq_block_norm_grad_workspace_bytes(ctypes.byref(s), t) for t in T]
        assert sizes == sorted(sizes)
    for s in (_adapters(), _adapters(rank=200, n=100, K=4096, N=4096)):
        for kind in (F32, BF16):
            sizes = [lib.cq_adapter_workspace_bytes(ctypes.byref(s), kind, t) for t in T]
            assert sizes == sorted(sizes)
    for E, S in ((60, 5), (4, 1), (128, 3), (1000, 2)):
        sizes = [lib.cq_balance_loss_workspace_bytes(t, E, S) for t in T]
        assert sizes == sorted(sizes)
