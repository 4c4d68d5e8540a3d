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
def test_quantizer_and_values(gpu_lib, rows, cols, pitch):
    q = gpu_lib
    x = torch.randn((rows, cols), device=DEV, generator=gen(1)).bfloat16()
    codes, scale = q.quantize_mx4(x)
    out, out_scale = apart(torch.zeros_like(codes), pitch), apart(torch.zeros_like(scale), pitch)
    far = apart(x, pitch)
    q.quantize_mx4(far, out, out_scale)
    assert torch.equal(out, codes) and torch.equal(out_scale, scale)
    q.dequantize_mx4(out, out_scale, cols, out=far)
    assert torch.equal(far, q.dequantize_mx4(codes, scale, cols, dtype=torch.bfloat16))


@pytest.mark.parametrize("M,N,K,pitch", [(16, 300, 200, 1 << 30), (60, 300, 200, 1 << 27), (1100, 70, 300, 1 << 22), (1100, 70, 5000, 1 << 22),
                                         (4096, 1024, 520, 1 << 21), (8192, 2056, 1024, 1 << 20)])
def test_linear(gpu_lib, M, N, K, pitch):
    """(few tokens in two ways, small tiles, small tiles of a cut sum, larger tiles)"""
    q = gpu_lib
    w, w_scale = q.quantize_mx4(torch.randn((N, K), device=DEV, generator=gen(3)))
    mat = q.pack_mx4(w, w_scale, K)
    a, s = q.quantize_mx4(torch.randn((M, K), device=DEV, generator=gen(4)))
    y = q.linear_mx4(mat, a, s, dtype=torch.bfloat16)
    far_a, far_s = apart(a, pitch), apart(s, pitch)
    out = torch.empty((M, pitch), dtype=torch.bfloat16, device=DEV)[:, :N]
    q.linear_mx4(mat, far_a, far_s, out=out)
    assert torch.equal(out, y)


def test_packing(gpu_lib):
    q = gpu_lib
    w, w_scale = q.quantize_mx4(torch.randn((1100, 300), device=DEV, generator=gen(3)))
    assert torch.equal(q.pack_mx4(apart(w, 1 << 22), apart(w_scale, 1 << 22), 300).packed, q.pack_mx4(w, w_scale, 300).packed)


@pytest.mark.parametrize("rows,V,pitch", [(1088, 300, 1 << 22), (1088, 3000, 1 << 22), (1088, 40000, (1 << 22) + 1), (9000, 500, 1 << 19), (40, 140000, 1 << 27)])
def test_scores(gpu_lib, rows, V, pitch):
    q = gpu_lib
    logits = torch.randn((rows, V), device=DEV, generator=gen(6)).half()
    token = torch.randint(0, V, (rows,), dtype=torch.int32, device=DEV, generator=gen(7))
    near, far = q.token_scores(logits, token, n_top=20), q.token_scores(apart(logits, pitch), token, n_top=20)
    assert all(torch.equal(a, b) for a, b in zip(near, far))
