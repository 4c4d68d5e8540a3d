"""One workspace, made for the largest call, for all smaller ones: the bits of calls with a workspace of their own, and nothing
written behind it."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


@pytest.mark.parametrize("W,V,n,batches", [(32, 1000, 32, (40, 33, 32, 31, 7, 1)), (25, 2048, 7, (41, 40, 3)), (64, 600, 64, (17, 16, 2, 1)), (4, 20000, 4, (9, 2))])
def test_a_search_whose_batch_shrinks(gpu_lib, W, V, n, batches):
    q = gpu_lib
    need = q.beam_select_workspace(batches[0], W, V, n)
    ws = torch.full((need + 4096,), 99, dtype=torch.uint8, device=DEV)
    logits = 3 * torch.randn((batches[0] * W, V), device=DEV, generator=gen(V))
    score = -torch.rand((batches[0], W), device=DEV, generator=gen(W))
    for B in batches:
        args = (score[:B].contiguous(), logits[:B * W], n)
        got, want = q.beam_select(*args, workspace=ws[:need]), q.beam_select(*args)
        assert all(torch.equal(a, b) for a, b in zip(got[:3], want[:3]))
        assert bool((ws[need:] == 99).all())
