"""Rows so far apart that offsets pass 32 bits, in bytes and in elements: every call gives the bits that it gives for the same
rows side by side (which the operators' own tests hold against 64 bits)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()   # up to 50 GB a test


def gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def apart(t, pitch):
    """The rows of t in a larger matrix."""
    far = torch.empty((t.shape[0], pitch), dtype=t.dtype, device=DEV)[:, :t.shape[1]]
    far.copy_(t)
    assert (t.shape[0] - 1) * pitch > 1 << 32
    return far


@pytest.mark.parametrize("rows,cols,pitch", [(1030, 200, 1 << 22), (70, 9000, 1 << 26)])
def test_tokens(gpu_lib, rows, cols, pitch):
    q, width = gpu_lib, (cols + 15) // 16 * 16
    x = torch.randn((rows, cols), device=DEV, generator=gen(1)).bfloat16()
    res = torch.randn((rows, cols), device=DEV, generator=gen(2)).bfloat16()
    codes, scale = q.quantize_tokens(x)
    far = apart(x, pitch)
    out = apart(torch.zeros((rows, width), dtype=torch.int8, device=DEV), pitch)
    _, far_scale = q.quantize_tokens(far, out)
    assert torch.equal(out, codes) and torch.equal(far_scale, scale)
    codes, scale, total = q.rms_norm_quant(x, residual=res)
    far_res = apart(res, pitch)
    _, far_scale, far_total = q.rms_norm_quant(far, residual=far_res, sum_out=far_res, codes=out)
    assert torch.equal(out, codes) and torch.equal(far_scale, scale) and torch.equal(far_total, total)


@pytest.mark.parametrize("M,N,K,pitch", [(16, 300, 200, 1 << 30), (60, 300, 200, 1 << 27), (1100, 70, 300, 1 << 22), (1100, 70, 3000, 1 << 22),
                                         (4096, 1024, 520, 1 << 21), (8192, 2056, 1024, 1 << 20)])
def test_linear(gpu_lib, M, N, K, pitch):
    """(few tokens in two ways, small tiles, small tiles of a cut sum, larger tiles)"""
    q, width = gpu_lib, (K + 15) // 16 * 16
    w = q.pack_int8(torch.randn((N, K), device=DEV, generator=gen(3)), q.LAYOUT_TILED)
    a = torch.randint(-127, 128, (M, width), dtype=torch.int8, device=DEV, generator=gen(4))
    s = torch.rand(M, device=DEV, generator=gen(5))
    y = q.linear_tokens(w, a, s, dtype=torch.bfloat16)
    out = torch.empty((M, pitch), dtype=torch.bfloat16, device=DEV)[:, :N]
    q.linear_tokens(w, apart(a, pitch), s, out=out)
    assert torch.equal(out, y)


@pytest.mark.parametrize("V,pitch", [(300, 1 << 22), (3000, 1 << 22), (40000, (1 << 22) + 1)])
def test_selection(gpu_lib, V, pitch):
    q = gpu_lib
    logits = torch.randn((64 * 17, V), device=DEV, generator=gen(6)).half()
    score = -torch.rand((64, 17), device=DEV, generator=gen(7))
    near, far = q.beam_select(score, logits, 20), q.beam_select(score, apart(logits, pitch), 20)
    assert all(torch.equal(a, b) for a, b in zip(near[:3], far[:3]))


@pytest.mark.parametrize("W", [16, 32])
def test_reordering(gpu_lib, W):
    q, B, pitch = gpu_lib, 1056 // W, 1 << 22
    parent = torch.randint(0, W, (B, W), dtype=torch.int32, device=DEV, generator=gen(8))
    rows = torch.randint(0, 256, (B * W, 1003), dtype=torch.uint8, device=DEV, generator=gen(9))
    want = rows[(parent.long() + W * torch.arange(B, device=DEV)[:, None]).view(-1)]
    src, dst = apart(rows, pitch), torch.empty((B * W, pitch), dtype=torch.uint8, device=DEV)[:, :1003]
    q.reorder_states([(src, dst)], parent)
    assert torch.equal(dst, want)
    q.reorder_states([src], parent)
    assert torch.equal(src, want)
