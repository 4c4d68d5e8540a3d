"""One workspace, made for the largest call, for all smaller ones: the bits of calls with a workspace of their own, and nothing
written behind it."""
from concurrent.futures import ThreadPoolExecutor

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


@pytest.mark.parametrize("N,K,tokens", [(4096, 4096, (700, 400, 77, 65, 64, 40, 20, 1)), (1024, 8192, (2000, 1024, 512, 300, 65, 33, 3)),
                                        (8192, 8192, (300, 65, 64, 33, 17)), (130, 131071, (600, 100, 33)), (1000, 1283, (3000, 77, 5)),
                                        (2600, 2500, (7215, 4494, 1412, 130))])
def test_a_layer_whose_tokens_become_fewer(gpu_lib, N, K, tokens):
    q, width = gpu_lib, (K + 15) // 16 * 16
    m = q.pack_int8(torch.randint(-127, 128, (N, K), dtype=torch.int8, device=DEV, generator=gen(1)), q.LAYOUT_TILED,
                    torch.rand(N, device=DEV, generator=gen(2)))
    a = torch.randint(-127, 128, (tokens[0], width), dtype=torch.int8, device=DEV, generator=gen(3))
    scale = torch.rand(tokens[0], device=DEV, generator=gen(4))
    need = q.linear_tokens_workspace(m, tokens[0])
    ws = torch.full((need + 4096,), 99, dtype=torch.uint8, device=DEV)
    whole = None
    for M in tokens:
        y = q.linear_tokens(m, a[:M], scale[:M], workspace=ws[:need])
        assert bool((ws[need:] == 99).all())
        whole = y if whole is None else whole
        assert torch.equal(y, whole[:M])   # (sums of whole numbers: the same in every way)
        assert torch.equal(y, q.linear_tokens(m, a[:M], scale[:M]))


def test_first_calls_of_several_threads(gpu_lib):
    """Every size of tile in every type, from four threads at once, each on a stream and with a workspace of its own."""
    q, K = gpu_lib, 2048
    sizes = [(70, 500), (700, 1000), (3000, 4200)]
    ins = []
    for M, N in sizes:
        m = q.pack_int8(torch.randint(-127, 128, (N, K), dtype=torch.int8, device=DEV, generator=gen(N)), q.LAYOUT_TILED)
        a = torch.randint(-127, 128, (M, K), dtype=torch.int8, device=DEV, generator=gen(M))
        ins.append((m, a, torch.rand(M, device=DEV, generator=gen(5))))
    torch.cuda.synchronize()

    def work():
        stream, out = torch.cuda.Stream(), []
        with torch.cuda.stream(stream):
            for i in ins:
                out += [q.linear_tokens(*i, dtype=t) for t in (torch.float32, torch.float16, torch.bfloat16)]
        stream.synchronize()
        return out

    with ThreadPoolExecutor(4) as pool:
        got = [f.result() for f in [pool.submit(work) for _ in range(4)]]
    want = work()
    for out in got:
        assert all(torch.equal(a, b) for a, b in zip(out, want))
