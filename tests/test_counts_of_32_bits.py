"""Numbers that do not fit the 32 bits of an entry point are refused by the binding: ctypes would pass their lower half."""
import pytest
import torch

from paper_2206_07882_amd import qrnnt

DEV = "cuda:0"


@pytest.mark.parametrize("far", [1 << 32, -(1 << 32), 1 << 31, 1 << 40])
def test_workspaces(far):
    m = qrnnt.QMat(torch.zeros(2048, dtype=torch.uint8), torch.zeros(64), 64, 8192, qrnnt.LAYOUT_TILED, 8)
    with pytest.raises(ValueError):
        qrnnt.linear_tokens_workspace(m, far + 300)
    for at in range(4):
        sizes = [2, 4, 100, 4]
        sizes[at] += far
        with pytest.raises(ValueError):
            qrnnt.beam_select_workspace(*sizes)


@pytest.mark.gpu
def test_end_tokens(gpu_lib):
    score, logits = torch.zeros((1, 2), device=DEV), torch.zeros((2, 8), device=DEV)
    finished = torch.ones((1, 2), dtype=torch.bool, device=DEV)
    for token in ((1 << 32) + 3, 3 - (1 << 32), 1 << 31):
        for through in (None, finished):
            with pytest.raises(ValueError):
                gpu_lib.beam_select(score, logits, finished=through, end_token=token)
