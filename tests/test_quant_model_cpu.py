"""Buffers that the model keeps for steps on 8-bit and other pools (no GPU: sizes and quantisation are stand-ins)."""
import pytest
import torch

from paper_2608_29809_amd import abi, quant
from paper_2608_29809_amd.runtime import RegionCacheModel


@pytest.fixture
def model(monkeypatch):
    """A model of two blocks without a context."""
    monkeypatch.setattr(abi, "rc_workspace_bytes", lambda ctx, rows, batch: 1000 * rows)
    monkeypatch.setattr(abi, "rc_quant_workspace_bytes", lambda ctx, rows, batch: 1700 * rows)
    monkeypatch.setattr(RegionCacheModel, "__init__", lambda self: None)
    m = RegionCacheModel()
    m.ctx, m.device, m.L, m._ws, m._quant = None, "cpu", 2, {}, None
    m._quantizable = [{f: torch.zeros(4, 4) for f in ("qkv_w", "fc1_w", "fc2_w")} for _ in range(2)]
    return m


def test_pools_have_workspaces_of_their_own(model):
    """Steps on one pool leave the other's workspace where a captured step has it, whichever comes first and is larger."""
    plain, eight = model.workspace(10, 1), model.workspace(10, 1, 8)
    assert plain.numel() == 10000 and eight.numel() == 17000
    assert model.workspace(10, 1) is plain and model.workspace(3, 1) is plain
    more = model.workspace(40, 1)
    assert more.numel() == 40000 and model.workspace(10, 1, 8) is eight
    model.workspace(90, 1, 8)
    assert model.workspace(40, 1) is more


def test_weights_stay_where_captured_steps_read_them(model, monkeypatch):
    """Made once, made anew in place, and kept while the bf16 weights are in use."""
    calls, given = [], []

    class Matrix:
        def struct(self):
            return abi.rc_qmat(id(self))

    def quantize(t, block_rows=1, out=None):
        calls.append(out)
        return out or Matrix()

    def put(ctx, layers):
        given.append(layers and [[getattr(layer, f).data for f, _ in abi.rc_quant_layer._fields_] for layer in layers])

    monkeypatch.setattr(quant, "quantize", quantize)
    monkeypatch.setattr(abi, "rc_set_quant_weights", put)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: None)
    for enable in (True, True, False, True):
        model.quantize_weights(enable)
    assert given[0] == given[1] == given[3] and given[2] is None
    assert len({p for layer in given[0] for p in layer}) == 6
    assert calls[:6] == [None] * 6 and len(calls) == 18 and {id(c) for c in calls[6:]} == {p for layer in given[0] for p in layer}


def test_without_private_names_of_torch(monkeypatch):
    """The module's stream and device lookups fall back to PyTorch's public ones."""
    import importlib.util
    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        monkeypatch.delattr(torch._C, name, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index: type("S", (), {"cuda_stream": 100 + index})())
    spec = importlib.util.spec_from_file_location("paper_2608_29809_amd._quant_again", quant.__file__)
    again = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(again)
    got = []
    again._call(lambda *args: got.append(args), 3, "x")
    assert got == [("x", 103)]
