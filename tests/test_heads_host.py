"""Heads, paged cache and attention without a GPU: the oracle against differences and hand-made values, the refusals of the C entry
points (arguments are checked before any device call), the workspace queries, the binding's checks."""
import ctypes

import numpy as np
import pytest

from oracle import heads_oracle as O
from paper_2604_10496_amd import binding as B

ONE = ctypes.c_void_p(256)   # a non-null dummy that must never be dereferenced
F16, F32, BF16, E4M3 = B.CQ_A_F16, B.CQ_A_F32, B.CQ_A_BF16, B.CQ_C_E4M3


# ------------------------------------------------------------------------------------------------
# the oracle
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_oracle_head_gradients_match_differences(norm, interleaved):
    rng = np.random.default_rng(3)
    T, n, D = 3, 2, 10
    x, c = rng.standard_normal((T, n, D)), rng.standard_normal((T, n, D))
    w = rng.standard_normal(D) if norm else None
    freq, pos = rng.random(3), [0, 5, -7]
    f = lambda x, w: (O.head_norm(x, w, 1e-3, freq, interleaved, 1.2, pos)[0] * c).sum()  # noqa: E731
    dx, dw, _, _ = O.head_norm_grad(x, w, c, 1e-3, freq, interleaved, 1.2, pos)
    step = 1e-5
    for _ in range(4):
        d = rng.standard_normal(x.shape)
        want = (f(x + step * d, w) - f(x - step * d, w)) / (2 * step)
        assert abs((dx * d).sum() - want) <= 1e-7 * (1 + np.abs(dx * d).sum())
        if norm:
            d = rng.standard_normal(D)
            want = (f(x, w + step * d) - f(x, w - step * d)) / (2 * step)
            assert abs((dw * d).sum() - want) <= 1e-7 * (1 + np.abs(dw * d).sum())


def test_oracle_rotation_by_hand():
    """A quarter revolution per position: (a, b) -> (-b, a); rows keep their length, values beyond `rot` stay."""
    freq = [np.pi / 2]
    x = np.array([[[1.0, 2.0, 3.0]]])
    for inter in (False, True):
        out, _ = O.head_norm(x, None, 0, freq, inter, 1.0, [1])
        assert np.allclose(out[0, 0], [-2, 1, 3])
    x = np.arange(1.0, 7).reshape(1, 1, 6)
    out, _ = O.head_norm(x, None, 0, [np.pi / 2, 0.0], False, 1.0, [1])
    assert np.allclose(out[0, 0], [-3, 2, 1, 4, 5, 6])
    out, _ = O.head_norm(x, None, 0, [np.pi / 2, 0.0], True, 1.0, [1])
    assert np.allclose(out[0, 0], [-2, 1, 3, 4, 5, 6])


def test_oracle_attention_by_hand():
    """Two positions with equal scores: the mean of their values; a window of one leaves the last, a sink of the same score a third of the sum."""
    k = np.zeros((2, 1, 1, 2))
    v = np.array([[1.0, 3.0], [5.0, 7.0]]).reshape(2, 1, 1, 2)
    q = np.ones((1, 1, 2))
    run = lambda **kw: O.attention(q, k, v, [[1, 0]], [2], 1.0, **kw)[:2]  # noqa: E731
    out, lse = run()
    assert np.allclose(out[0, 0], [3, 5]) and np.isclose(lse[0, 0], np.log(2))
    out, lse = run(window=1)
    assert np.allclose(out[0, 0], [1, 3]) and np.isclose(lse[0, 0], 0)
    out, lse = run(sinks=np.zeros(1))
    assert np.allclose(out[0, 0], [2, 10 / 3]) and np.isclose(lse[0, 0], np.log(3))
    out, lse, *_ = O.attention(q, k, v, [[-1, 9]], [2], 1.0)
    assert not out.any() and lse[0, 0] == -np.inf


def test_oracle_slots():
    table = [[3, 1], [0, 7]]
    got = O.slots(table, [3, 4], [0, 2, 4], 2, 4, 5)
    assert got == [(0, 1, 3, 1), (0, 2, 1, 0), (1, 2, None, 0), (1, 3, None, 1), None]
    assert O.slots(table, [1, 5], None, 2, 8, 2) == [(0, 0, 3, 0), None]


# ------------------------------------------------------------------------------------------------
# refusals of the entry points
# ------------------------------------------------------------------------------------------------
def _heads(p=256, kind=BF16, n=2, token=256, head=64):
    return B.Heads(p, kind, n, token, head)


def _spec(**k):
    a = dict(D=64, rot=64, interleaved=0, weight_kind=F32, eps=1e-6, rot_scale=1.0, freq=256, w_q=256, w_k=256)
    a.update(k)
    return B.HeadSpec(*[a[n] for n, _ in B.HeadSpec._fields_])


def _cache(**k):
    a = dict(kind=BF16, heads=2, D=64, page_size=16, pages=8, page_stride=2048, slot_stride=128, head_stride=64, k=256, v=256, k_scale=None,
             v_scale=None)
    a.update(k)
    return B.Cache(*[a[n] for n, _ in B.Cache._fields_])


def _seqs(**k):
    a = dict(n=4, width=4, stride=4, page_table=256, lengths=256)
    a.update(k)
    return B.Sequences(*[a[n] for n, _ in B.Sequences._fields_])


H = _heads()
NONE = object()


def test_head_norm_refusals():
    lib = B.load_library()

    def call(T=4, q=H, k=H, pos=ONE, qo=H, ko=H, spec=None, **s):
        return lib.cq_head_norm(None if spec is NONE else _spec(**s), q, k, pos, T, qo, ko, None)
    assert call(spec=NONE) == 1 and call(q=None, k=None) == 1 and call(qo=None) == 1 and call(ko=None) == 1 and call(pos=None) == 1
    assert call(q=_heads(p=None)) == 1 and call(qo=_heads(p=None)) == 1 and call(freq=None) == 1
    assert call(T=-1) == 2 and call(T=(1 << 30) + 1) == 2
    assert call(D=0) == 2 and call(D=257) == 2 and call(rot=66) == 2 and call(rot=63) == 2 and call(rot=-2) == 2
    assert call(eps=0.0) == 2 and call(eps=float("nan")) == 2 and call(eps=float("inf")) == 2 and call(rot_scale=float("inf")) == 2
    assert call(q=_heads(n=0)) == 2 and call(q=_heads(n=20000)) == 2 and call(q=_heads(n=3)) == 2
    assert call(qo=_heads(head=63)) == 2 and call(ko=_heads(token=63)) == 2        # rows on another's place
    assert call(qo=_heads(token=64, head=64)) == 2 and call(qo=_heads(token=64, head=192)) == 2
    assert call(q=_heads(kind=7)) == 3 and call(weight_kind=9) == 3 and call(k=_heads(kind=F16)) == 3
    assert call(qo=_heads(kind=F32), ko=_heads(kind=F32)) == 3                     # 16-bit rows stay what they are
    assert call(qo=_heads(kind=F16)) == 3 and call(q=_heads(kind=E4M3)) == 3
    assert call(T=0) == 0 and call(T=0, q=_heads(p=None), pos=None) == 0


def test_head_norm_grad_refusals():
    lib = B.load_library()

    def call(T=4, q=H, k=H, pos=ONE, dqo=H, dko=H, dq=H, dk=H, wq=ONE, wk=ONE, ws=ONE, n=1 << 30, **s):
        return lib.cq_head_norm_grad(_spec(**s), q, k, pos, T, dqo, dko, dq, dk, wq, wk, ws, n, None)
    assert lib.cq_head_norm_grad(None, H, H, ONE, 4, H, H, H, H, ONE, ONE, ONE, 1 << 30, None) == 1
    assert call(dqo=None, dko=None, wq=None, wk=None) == 1 and call(dq=None) == 1 and call(dk=None) == 1
    assert call(q=None) == 1 and call(k=None) == 1 and call(pos=None) == 1
    assert call(w_q=None) == 1 and call(dko=None) == 1                             # a weight's gradient without what it comes from
    assert call(T=-1) == 2 and call(D=300) == 2 and call(dq=_heads(n=3)) == 2 and call(q=_heads(n=3)) == 2 and call(dq=_heads(head=8)) == 2
    assert call(dqo=_heads(kind=F32)) == 3 and call(q=_heads(kind=F16)) == 3 and call(dk=_heads(kind=F32)) == 3
    need = lib.cq_head_norm_grad_workspace_bytes(_spec(), 4, 4000)
    assert need > 0 and call(T=4000, n=need - 1) == 4 and call(T=4000, ws=None) == 4
    assert lib.cq_head_norm_grad_workspace_bytes(_spec(D=0), 4, 4000) == 0
    assert lib.cq_head_norm_grad_workspace_bytes(_spec(), 40, 1) == 0              # few rows need none
    sizes = [lib.cq_head_norm_grad_workspace_bytes(_spec(), 40, T) for T in (0, 1, 2, 20, 100, 255, 256, 300, 1 << 20)]
    assert sizes == sorted(sizes)
    assert call(T=0, wq=None, wk=None, ws=None, n=0) == 0


def test_cache_append_refusals():
    lib = B.load_library()

    def call(T=4, q=H, k=H, v=H, off=None, pos=None, qo=H, spec=None, c=None, s=None):
        return lib.cq_cache_append(_cache(**(c or {})), _seqs(**(s or {})), _spec(**(spec or {})), q, k, v, off, pos, T, qo, None)
    assert lib.cq_cache_append(None, _seqs(), None, None, H, H, None, None, 4, None, None) == 1
    assert lib.cq_cache_append(_cache(), None, None, None, H, H, None, None, 4, None, None) == 1
    assert call(k=None) == 1 and call(v=None) == 1 and call(qo=None) == 1 and call(c=dict(k=None)) == 1 and call(k=_heads(p=None)) == 1
    assert call(s=dict(page_table=None)) == 1 and call(s=dict(lengths=None)) == 1
    assert call(T=3) == 2 and call(T=-1, off=ONE) == 2                              # without offsets: one token of every sequence
    assert call(k=_heads(n=3)) == 2 and call(v=_heads(n=1)) == 2 and call(spec=dict(D=32, rot=32)) == 2
    for bad in (dict(D=60), dict(D=264), dict(D=0), dict(heads=0), dict(page_size=0), dict(pages=-1), dict(page_stride=2044),
                dict(slot_stride=56), dict(slot_stride=132), dict(head_stride=32), dict(k=264), dict(kind=E4M3, D=72)):
        assert call(c=bad) == 2, bad
    for bad in (dict(n=-1), dict(width=-1), dict(stride=-1), dict(width=1 << 27, stride=1 << 27)):
        assert call(s=bad, off=ONE) == 2, bad
    assert call(c=dict(kind=F32)) == 3 and call(c=dict(k_scale=256)) == 3 and call(v=_heads(kind=F16)) == 3 and call(q=_heads(kind=F16)) == 3
    assert call(qo=_heads(kind=F16)) == 3
    assert call(T=0, off=ONE) == 0 and call(T=0, s=dict(n=0, page_table=None, lengths=None)) == 0


def test_cache_attention_refusals():
    lib = B.load_library()

    def call(q=H, o=H, lse=ONE, ws=ONE, n=1 << 30, c=None, s=None, spec=NONE, **a):
        p = dict(scale=0.1, softcap=0.0, window=0, max_length=64, sinks=None)
        p.update(a)
        p = None if spec is None else B.AttentionSpec(*[p[x] for x, _ in B.AttentionSpec._fields_])
        return lib.cq_cache_attention(_cache(**(c or {})), _seqs(**(s or {})), p, q, o, lse, ws, n, None)
    assert call(q=None) == 1 and call(o=None) == 1 and call(spec=None) == 1 and call(q=_heads(p=None)) == 1 and call(o=_heads(p=None)) == 1
    assert call(q=_heads(n=3), o=_heads(n=3)) == 2 and call(o=_heads(n=4)) == 2 and call(o=_heads(head=8)) == 2
    assert call(scale=float("nan")) == 2 and call(scale=float("inf")) == 2 and call(softcap=-1.0) == 2 and call(softcap=float("inf")) == 2
    assert call(window=-1) == 2 and call(max_length=-1) == 2 and call(max_length=(1 << 30) + 1) == 2
    assert call(c=dict(kind=F32)) == 3 and call(q=_heads(kind=E4M3)) == 3 and call(o=_heads(kind=E4M3)) == 3
    need = lib.cq_cache_attention_workspace_bytes(_cache(), 4, 2, 1 << 16, 0)
    assert need > 0 and call(max_length=1 << 16, n=need - 1) == 4 and call(max_length=1 << 16, ws=None) == 4
    assert lib.cq_cache_attention_workspace_bytes(_cache(D=60), 4, 2, 1 << 16, 0) == 0
    assert lib.cq_cache_attention_workspace_bytes(_cache(), 0, 2, 1 << 16, 0) == 0
    assert call(c=dict(pages=1 << 30, page_stride=1 << 20)) == 2                          # rows beyond 64 GB
    assert call(s=dict(n=1 << 30, width=1, stride=1)) == 2
    assert call(s=dict(n=0, page_table=None, lengths=None)) == 0


# ------------------------------------------------------------------------------------------------
# the binding's checks
# ------------------------------------------------------------------------------------------------
def test_binding_refuses_what_is_not_on_the_gpu():
    import torch
    x = torch.zeros(2, 3, 64)
    with pytest.raises(ValueError, match="freq"):
        B.HeadNorm(64, freq=torch.ones(4, dtype=torch.float64))
    with pytest.raises(ValueError, match="q: not on the GPU"):
        B.cq_head_norm(B.HeadNorm(64), x)
    with pytest.raises(ValueError, match="neither"):
        B.cq_head_norm(B.HeadNorm(64))
    with pytest.raises(ValueError, match="no gradients"):
        B.cq_head_norm_grad(B.HeadNorm(64))
    with pytest.raises(ValueError, match="k: not on the GPU"):
        B.PagedCache(torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16), torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="float16, bfloat16"):
        B.PagedCache(torch.zeros(2, 16, 2, 64), torch.zeros(2, 16, 2, 64))
