"""The handles and the binding of the operators around the layer without a GPU: CPU tensors that call themselves GPU tensors, and a
library whose launches are written down instead of made (arguments and workspace sizes are checked by the real one)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2604_10496_amd import binding as B


class OnCard(torch.Tensor):
    is_cuda = property(lambda self: True)


def card(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnCard)


class Recorder:
    """Workspace queries of the library; its calls only keep their arguments.  A norm's gradient answers as the library does: a
    specification that the query refuses is refused, and a workspace below the query's size."""

    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        if name.endswith("_workspace_bytes"):
            return getattr(self.real, name)
        return lambda *args: self._call(name, args)

    def _call(self, name, args):
        handle = args[0]
        if isinstance(handle, ctypes.Structure):
            handle = type(handle).from_buffer_copy(handle)
        self.calls.append((name, handle, args[1:]))
        if name == "cq_block_norm_grad":
            need = self.real.cq_block_norm_grad_workspace_bytes(handle, args[6])
            return 3 if need == 0 else 4 if args[13] < need else 0
        return 0


@pytest.fixture
def lib(monkeypatch):
    rec = Recorder(B.load_library())
    monkeypatch.setattr(B, "_lib", rec)
    monkeypatch.setattr(B, "_raw_stream", lambda t: 0)
    yield rec


def test_a_refused_call_leaves_later_ones_alone(lib, monkeypatch):
    monkeypatch.setattr(B, "CqError", type("CqError", (RuntimeError,), {"__init__": lambda self, st: setattr(self, "status", st)}))
    h = card(5, 72)
    refused = B.BlockNorm(card(72, dtype=torch.float16))          # f16 weights beside an fp32 stream
    with pytest.raises(B.CqError) as e:
        B.cq_block_norm_grad(refused, h, dx=h)
    assert e.value.status == 3
    valid = B.BlockNorm(card(72))
    assert B.cq_block_norm_grad(valid, h, dx=h)["dw_pre"].shape == (72,)
    assert lib.calls[-1][2][12] == lib.real.cq_block_norm_grad_workspace_bytes(valid.struct(h), 5) > 0


def test_batch_sizes_leave_nothing_behind(lib):
    ad, norm, w = B.DeviceAdapters(card(2, 40, 8), card(2, 16, 40)), B.BlockNorm(card(8)), B.__dict__
    sizes = lambda: [len(v) for holder in (w, vars(ad), vars(norm)) for v in holder.values() if isinstance(v, dict)]
    ids = lambda T: card(T, dtype=torch.int32)

    def calls(T):
        B.cq_adapter_apply(ad, card(T, 8), ids(T))
        B.cq_block_norm_grad(norm, card(T, 8), dx=card(T, 8))
        B.cq_balance_loss(card(T, 4), card(T, 1, dtype=torch.int32), 0.1)
    calls(3)
    before = sizes()
    for T in range(4, 40):
        calls(T)
    assert sizes() == before


def _norm_calls(norm, h, y, gate):
    return (lambda: B.cq_block_norm(norm, h, y, gate), lambda: B.cq_block_norm_grad(norm, h, y, gate, dh=h, dx=y))


@pytest.mark.parametrize("bad", [card(64, dtype=torch.bfloat16), card(63), card(65), card(1), card(1, 64), card(64, 2)[:, 0], torch.zeros(64)])
@pytest.mark.parametrize("name", ["w_pre", "w_post"])
def test_replaced_weights_are_checked(lib, name, bad):
    """By another tensor, and by other contents of the same one."""
    h, y, gate = card(3, 64, dtype=torch.bfloat16), card(3, 64), card(3)
    norm = B.BlockNorm(card(64), card(64))
    for call in _norm_calls(norm, h, y, gate):
        call()
        with pytest.raises(ValueError):
            setattr(norm, name, bad)
            call()
        setattr(norm, name, card(64))
        call()
    norm = B.BlockNorm(card(64), card(64))
    if bad.is_cuda:
        getattr(norm, name).data = bad
        for call in _norm_calls(norm, h, y, gate):
            with pytest.raises(ValueError):
                call()
    assert all(handle.w_pre and handle.w_post for _, handle, _ in lib.calls)


def test_a_handle_without_weights_takes_those_that_fit(lib):
    h, y = card(3, 64, dtype=torch.bfloat16), card(3, 64)
    norm = B.BlockNorm()
    assert B.cq_block_norm(norm, h, y)["x"] is None
    norm.w_pre = card(64)
    assert B.cq_block_norm(norm, h, y)["x"].shape == (3, 64)
    norm.w_pre = None
    assert B.cq_block_norm(norm, h, y)["x"] is None
    norm.w_pre = card(32)
    with pytest.raises(ValueError):
        B.cq_block_norm(norm, h, y)


def test_changed_numbers_of_a_norm_take_effect(lib):
    h, y = card(3, 64, dtype=torch.bfloat16), card(3, 64)
    norm = B.BlockNorm(card(64), eps=1.0, residual_scale=2.0, branch_scale=3.0)
    for call in _norm_calls(norm, h, y, None):
        call()
        got = lib.calls[-1][1]
        assert (got.eps, got.residual_scale, got.branch_scale, got.gate_sigmoid, got.block_kind) == (1.0, 2.0, 3.0, 0, B.CQ_A_F32)
        norm.eps, norm.residual_scale, norm.branch_scale, norm.gate_sigmoid = 0.5, 4.0, 0.25, True
        call()
        got = lib.calls[-1][1]
        assert (got.eps, got.residual_scale, got.branch_scale, got.gate_sigmoid) == (0.5, 4.0, 0.25, 1)
        norm.eps, norm.residual_scale, norm.branch_scale, norm.gate_sigmoid = 1.0, 2.0, 3.0, False
    norm.block_dtype = torch.bfloat16
    with pytest.raises(ValueError):
        B.cq_block_norm(norm, h, y)
    B.cq_block_norm(norm, h, y.bfloat16())
    assert lib.calls[-1][1].block_kind == B.CQ_A_BF16


@pytest.mark.parametrize("name,bad", [("A", card(3, 4, 16, dtype=torch.bfloat16)), ("A", card(2, 4, 16)), ("A", card(4, 4, 16)), ("A", card(3, 8, 16)),
                                      ("A", card(3, 4, 8)), ("A", card(3, 16, 4).transpose(1, 2)), ("A", torch.zeros(3, 4, 16)),
                                      ("B", card(3, 10, 4, dtype=torch.float16)), ("B", card(2, 10, 4)), ("B", card(3, 9, 4)), ("B", card(3, 10, 2)),
                                      ("B", card(3, 4, 10).transpose(1, 2)), ("scale", card(2)), ("scale", card(3, dtype=torch.float64)),
                                      ("scale", torch.zeros(3)), ("ranks", card(3)), ("ranks", card(2, dtype=torch.int32)),
                                      ("ranks", card(3, dtype=torch.int64))])
def test_replaced_adapters_are_checked(lib, name, bad):
    def handle():
        return B.DeviceAdapters(card(3, 4, 16), card(3, 10, 4), card(3), card(3, dtype=torch.int32))
    X, ids = card(5, 16), card(5, dtype=torch.int32)
    ad = handle()
    B.cq_adapter_apply(ad, X, ids)
    with pytest.raises(ValueError):
        setattr(ad, name, bad)
        B.cq_adapter_apply(ad, X, ids)
    ad = handle()
    if bad.is_cuda:
        getattr(ad, name).data = bad
        with pytest.raises(ValueError):
            B.cq_adapter_apply(ad, X, ids)
    assert len(lib.calls) == 1
    ad = handle()
    ad.scale = ad.ranks = None
    B.cq_adapter_apply(ad, X, ids)
    got = lib.calls[-1][1]
    assert (got.n, got.rank, got.K, got.N, got.scale, got.ranks) == (3, 4, 16, 10, None, None)


def test_outputs_of_adapters_are_laid_out_like_rows(lib):
    """What the call allocates is contiguous, whatever the base's rows are."""
    ad, X, ids = B.DeviceAdapters(card(3, 4, 16), card(3, 10, 4)), card(5, 16), card(5, dtype=torch.int32)
    wide = card(5, 30, dtype=torch.bfloat16)
    for base, ldb in ((wide[:, 3:13], 30), (card(5, 10, dtype=torch.bfloat16), 10)):
        out = B.cq_adapter_apply(ad, X, ids, base=base)
        args = lib.calls[-1][2]
        assert out.is_contiguous() and out.dtype == torch.bfloat16 and (args[6], args[9]) == (ldb, 10)
        assert B.cq_adapter_apply(ad, X, ids, base=base, out=base) is base and (lib.calls[-1][2][6], lib.calls[-1][2][9]) == (ldb, ldb)
    assert B.cq_adapter_apply(ad, X, ids).dtype == torch.float32
    with pytest.raises(ValueError):
        B.cq_adapter_apply(ad, X, ids, base=wide[:, :10], out=card(5, 10))


def test_sequences_beyond_those_that_can_be_counted_are_refused():
    real = B.load_library()
    one = ctypes.c_void_p(256)     # a non-null dummy that must never be dereferenced
    S = (1 << 26) + 1
    assert real.cq_balance_loss(one, B.CQ_A_F32, one, one, S, None, 8, 4, 1, 0.1, one, one, one, one, one, 1 << 60, None) == 2
    assert real.cq_balance_loss_grad(one, B.CQ_A_F32, one, one, one, S, None, 8, 4, 1, 0.1, None, one, None) == 2
    assert real.cq_balance_loss_workspace_bytes(8, 4, S) == 0 and real.cq_balance_loss_workspace_bytes(8, 4, S - 1) > 0


def test_workspace_of_adapters_ends_with_the_longest_launch():
    real = B.load_library()
    for N, most in ((3, 1 << 26), (256, 1 << 26), (1 << 23, 8192)):
        s = B.Adapters(2, 16, 8, N, B.CQ_A_BF16, 256, 256, None, None)
        at = lambda T: real.cq_adapter_workspace_bytes(ctypes.byref(s), B.CQ_A_BF16, T)
        assert at(most - 1) <= at(most) == at(most + 1) == at(1 << 30) == most * 16 * 4


def test_few_tokens_take_one_launch_where_it_is_the_faster_form():
    """No workspace: one launch.  A's products are repeated by every workgroup of it, and cost the more the wider the types."""
    real = B.load_library()
    F16, F32, BF16 = B.CQ_A_F16, B.CQ_A_F32, B.CQ_A_BF16

    def one(x, w, T, K, N, R):
        s = B.Adapters(4, R, K, N, w, 256, 256, None, None)
        return real.cq_adapter_workspace_bytes(ctypes.byref(s), x, T) == 0
    for same in (F16, BF16):
        assert one(same, same, 1, 4096, 4096, 16) and one(same, same, 1, 8192, 2048, 8) and one(same, same, 16, 2048, 2048, 32)
        assert not one(same, same, 1, 16384, 2048, 4)
    assert one(F32, BF16, 1, 4096, 4096, 16) and one(F32, BF16, 16, 2048, 2048, 32) and not one(F32, BF16, 1, 5120, 2048, 8)
    for x, w in ((F32, F32), (BF16, F32), (F16, BF16), (F32, F16)):
        assert one(x, w, 1, 2048, 2048, 16) and not one(x, w, 1, 2048, 2048, 32) and not one(x, w, 1, 4096, 4096, 16)
    assert not one(BF16, BF16, 400, 2048, 2048, 16) and not one(BF16, BF16, 1, 512, 512, 33)
