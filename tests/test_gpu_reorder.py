"""Reordering of states: byte for byte, in place and into other arrays, several arrays in one launch."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gather(x, parent, W):
    """Host oracle: rows of x [B*W, ...] named by parent [B, W_out]; None where the parent is negative."""
    B = parent.shape[0]
    return [None if p < 0 else x[b * W + min(int(p), W - 1)] for b in range(B) for p in parent[b]]


def check(got, want, old):
    for j, w in enumerate(want):
        assert torch.equal(got[j].cpu(), (old[j] if w is None else w).cpu()), j


def random_parent(seed, B, W_out, W):
    g = torch.Generator().manual_seed(seed)
    p = torch.randint(-1, W + 1, (B, W_out), generator=g, dtype=torch.int32)   # -1: stays as it was, W: clamped
    return p


def states(seed, n):
    g = torch.Generator().manual_seed(seed)
    ints = lambda *s: torch.randint(-128, 128, s, generator=g, dtype=torch.int8).to(DEV)
    return [ints(n, 640), torch.randn((n, 640), generator=g).to(DEV), ints(n, 1), ints(n, 17), ints(n, 3, 50),
            torch.randint(0, 1000, (n, 7), generator=g, dtype=torch.int32).to(DEV), torch.randn((n, 2, 3, 4), generator=g).to(torch.bfloat16).to(DEV)]


@pytest.mark.parametrize("B,W", [(1, 1), (1, 2), (3, 4), (2, 5), (64, 16), (5, 17), (2, 32), (3, 64)])
def test_in_place(gpu_lib, B, W):
    parent = random_parent(B * 100 + W, B, W, W)
    xs = states(B + W, B * W)
    old = [x.clone() for x in xs]
    gpu_lib.reorder_states(xs, parent.to(DEV))
    for x, o in zip(xs, old):
        check(x, gather(o, parent, W), o)


@pytest.mark.parametrize("B,W,W_out", [(1, 1, 1), (3, 4, 4), (2, 5, 3), (7, 3, 10), (64, 16, 16), (2, 16, 32), (3, 64, 64), (2, 1, 64)])
def test_into_other_arrays(gpu_lib, B, W, W_out):
    parent = random_parent(B * 100 + W + W_out, B, W_out, W)
    src = states(B + W, B * W)
    dst = states(1000 + B, B * W_out)
    old_src, old = [x.clone() for x in src], [x.clone() for x in dst]
    group = gpu_lib.StateGroup(list(zip(src, dst)), B, W, W_out)
    group.reorder(parent.to(DEV))
    for s, d, o, os in zip(src, dst, old, old_src):
        check(d, gather(s, parent, W), o)
        assert torch.equal(s, os)


def test_rows_apart_odd_places_and_neighbours(gpu_lib):
    """Columns of one matrix as several states, at odd bytes; in place beside arrays that are not."""
    B, W = 4, 6
    g = torch.Generator().manual_seed(3)
    big = torch.randint(-128, 128, (B * W, 301), generator=g, dtype=torch.int8).to(DEV)
    other = torch.randint(-128, 128, (B * W + 1, 100), generator=g, dtype=torch.int8).to(DEV)
    to = torch.zeros((B * W, 90), dtype=torch.int8, device=DEV)
    old, old_other = big.clone(), other.clone()
    parent = random_parent(4, B, W, W)
    gpu_lib.reorder_states([big[:, 1:50], big[:, 50:131], (other[1:, 3:93], to)], parent.to(DEV))
    check(big[:, 1:131], gather(old[:, 1:131], parent, W), old[:, 1:131])
    assert torch.equal(big[:, :1], old[:, :1]) and torch.equal(big[:, 131:], old[:, 131:]) and torch.equal(other, old_other)
    check(to, gather(old_other[1:, 3:93], parent, W), torch.zeros_like(to))


def test_the_same_parent_for_all_and_no_utterances(gpu_lib):
    x = torch.arange(12, dtype=torch.float32, device=DEV).reshape(6, 2)
    gpu_lib.reorder_states([x], torch.tensor([[2, 2, 2], [0, 0, 0]], dtype=torch.int32, device=DEV))
    assert x.cpu().tolist() == [[4, 5]] * 3 + [[6, 7]] * 3
    gpu_lib.reorder_states([torch.empty((0, 5), device=DEV)], torch.empty((0, 3), dtype=torch.int32, device=DEV))


def test_most_states_of_a_call(gpu_lib):
    xs = [torch.full((4, k + 1), k, dtype=torch.int8, device=DEV) + torch.arange(4, dtype=torch.int8, device=DEV)[:, None] for k in range(32)]
    gpu_lib.reorder_states(xs, torch.tensor([[3, 2, 1, 0]], dtype=torch.int32, device=DEV))
    for k, x in enumerate(xs):
        assert x[:, 0].cpu().tolist() == [k + 3, k + 2, k + 1, k]
