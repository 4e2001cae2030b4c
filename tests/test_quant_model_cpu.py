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
    m.ctx, m.device, m.L, m._ws = None, "cpu", 2, {}
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
