"""Workspaces of the 4-bit cache that are smaller than they look, or in host
memory, are refused before anything is launched."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_workspaces():
    from paper_2609_36757_gb300 import fastvr as FV
    cfg = FV.make_config(1, 2, 64, 1, 1, 3)
    need = FV.fastvr_q4_workspace_bytes(cfg, 2)
    one = torch.zeros(1, dtype=torch.uint8, device="cuda")
    for bad in (one.expand(need), torch.zeros(need, dtype=torch.uint8)):
        with pytest.raises(ValueError):
            FV.StreamingAttention4(cfg, workspace=bad)
    with pytest.raises(FV.FastVRError):
        FV.StreamingAttention4(cfg, workspace=one)
