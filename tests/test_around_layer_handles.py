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
