"""Microscaled 4-bit floats: quantizer, values, packed weights and their linear layer against 64 bits.

Quantizer and values are exact.  The linear layer is exact where scales lie close together: all partial sums are then multiples of
2^-4 below 2^20 and so held by fp32 in any order; one rounding to fp32 with the bias and one to the type of y remain, and
these are the reference's, too.  With scales far apart the sums are rounded; what by is derived at the test."""
import numpy as np
import pytest
import torch

from tests import plain_mx4 as plain
from tests.plain64 import HALF_STEP

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def rows_of(seed, rows, cols, dtype):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g) * torch.exp(2.0 * torch.randn((rows, cols), generator=g))
    return x.to(dtype)


def check_codes(x, codes, scale):
    want, want_scale = plain.quantize(x.double().cpu().numpy())
    rows, cols = x.shape
    n = want_scale.shape[1]
    assert np.array_equal(codes.cpu().numpy()[:, :16 * n], plain.join(want))
    assert np.array_equal(scale.cpu().numpy()[:, :n], want_scale)
    width = (n + 7) // 8 * 8
    assert (scale.cpu().numpy()[:, n:width] == 127).all()
    return want, want_scale


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (3, 32), (2, 33), (5, 64), (300, 255), (7, 256), (4, 257), (33, 1283), (2, 8192), (4097, 40), (1500, 1280), (9, 16411)])
def test_quantizer(gpu_lib, dtype, rows, cols):
    x = rows_of(rows + cols, rows, cols, dtype).to(DEV)
    codes, scale = gpu_lib.quantize_mx4(x)
    assert codes.shape == (rows, gpu_lib.mx4_pitch(cols)) and scale.shape == (rows, gpu_lib.mx4_scale_pitch(cols))
    want, want_scale = check_codes(x, codes, scale)
    for out in TYPES:
        got = gpu_lib.dequantize_mx4(codes, scale, cols, dtype=out)
        ref = torch.from_numpy(plain.values(want, want_scale)[:, :cols]).to(out)
        assert torch.equal(got.cpu(), ref)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lead,pitch", [(0, 70), (1, 71), (3, 96), (8, 101)])
def test_quantizer_of_rows_at_odd_places(gpu_lib, dtype, lead, pitch):
    rows, cols = 37, 67
    store = rows_of(5, rows, pitch + 16, dtype).to(DEV).flatten()
    x = store[lead:lead + rows * pitch].view(rows, pitch)[:, :cols]
    q = torch.full((rows, 64), 77, dtype=torch.uint8, device=DEV)
    s = torch.full((rows, 16), 77, dtype=torch.uint8, device=DEV)
    gpu_lib.quantize_mx4(x, q, s)
    check_codes(x, q, s)
    assert bool((q[:, 48:] == 77).all()) and bool((s[:, 8:] == 77).all())   # behind the row: left as they are
    out = torch.full((rows * pitch + 16,), 3.0, dtype=dtype, device=DEV)
    y = out[lead:lead + rows * pitch].view(rows, pitch)[:, :cols]
    gpu_lib.dequantize_mx4(q, s, cols, out=y)
    assert torch.equal(y, gpu_lib.dequantize_mx4(q, s, cols, dtype=dtype))
    keep = torch.ones_like(out, dtype=torch.bool)
    keep[lead:lead + rows * pitch].view(rows, pitch)[:, :cols] = False
    assert bool((out[keep] == 3.0).all())


def test_quantizer_next_to_every_border(gpu_lib):
    """Values on the borders of two codes and next to them, at every exponent that fp32 has."""
    near = []
    for b in list(plain.BORDERS) + [6.0, 7.0, 7.5]:
        b = np.float32(b)
        near += [b, np.nextafter(b, np.float32(9)), np.nextafter(b, np.float32(0))]
    near = np.array(near, np.float32)
    block = np.zeros(32, np.float32)
    block[0], block[1:16] = 4.0, near[:15]
    block2 = np.zeros(32, np.float32)
    block2[0], block2[1:16] = 7.999, near[15:]
    rows = []
    for e in range(-149, 125):
        with np.errstate(all="ignore"):
            rows.append(np.concatenate([np.ldexp(block, e), -np.ldexp(block2, e)]))
    x = torch.from_numpy(np.array(rows, np.float32)).to(DEV)
    codes, scale = gpu_lib.quantize_mx4(x)
    want, want_scale = check_codes(x, codes, scale)
    assert want_scale.min() == 0 and want_scale.max() == 251
    assert np.array_equal(gpu_lib.dequantize_mx4(codes, scale, 64).cpu().double().numpy(), plain.values(want, want_scale))


@pytest.mark.parametrize("dtype", TYPES)
def test_blocks_of_zeros_and_blocks_that_are_not_finite(gpu_lib, dtype):
    x = torch.ones((6, 96), dtype=dtype)
    x[0, :32] = 0.0
    x[1, 32:64] = -0.0
    x[2, 40] = float("nan")
    x[3, 95] = float("inf")
    x[4, 0] = -float("inf")
    x[5, 64:] = torch.finfo(dtype).max
    x = x.to(DEV)
    codes, scale = gpu_lib.quantize_mx4(x)
    check_codes(x, codes, scale)
    s = scale.cpu()
    assert s[0, 0] == 127 and s[1, 1] == 127 and s[2, 1] == 255 and s[3, 2] == 255 and s[4, 0] == 255 and int((s[:, :3] == 255).sum()) == 3
    back = gpu_lib.dequantize_mx4(codes, scale, 96).cpu()
    assert int(back.isnan().sum()) == 96 and bool(back[2, 32:64].isnan().all())
    assert bool((codes[2, 16:32] == 0).all())


def codes_of(seed, rows, cols, low=126, high=128):
    """Random codes and scales [rows, ...] with anything in the bits behind column cols."""
    rng = np.random.default_rng(seed)
    n = (cols + 31) // 32
    code = rng.integers(0, 16, (rows, n * 32)).astype(np.uint8)
    scale = np.full((rows, (n + 7) // 8 * 8), 127, np.uint8)
    scale[:, :n] = rng.integers(low, high + 1, (rows, n))
    return code, scale


def exact(code, scale, cols):
    return plain.values(code, scale[:, :code.shape[1] // 32])[:, :cols]


def run(q, M, N, K, dtype, seed, bias=True, low=126, high=128, **more):
    a, sa = codes_of(seed, M, K, low, high)
    w, sw = codes_of(seed + 1, N, K, low, high)
    b = torch.from_numpy(np.random.default_rng(seed + 2).standard_normal(N).astype(np.float32)).to(DEV) if bias else None
    dev = lambda x: torch.from_numpy(x).to(DEV)
    mat = q.pack_mx4(dev(plain.join(w)), dev(sw), K)
    y = q.linear_mx4(mat, dev(plain.join(a)), dev(sa), bias=b, dtype=dtype, **more)
    ref = exact(a, sa, K) @ exact(w, sw, K).T
    mag = np.abs(exact(a, sa, K)) @ np.abs(exact(w, sw, K)).T
    return y, ref, mag, b


def assert_same(y, ref, b, dtype):
    """Held to the last bit: magnitudes below 2^20 and multiples of 2^-4 lie within 2^27 of each other."""
    r = torch.from_numpy(ref.astype(np.float32))   # exact
    r = (r if b is None else r + b.cpu()).to(dtype)
    assert torch.equal(y.cpu(), r)


# few tokens in every form, small, middle and large tiles, cut sums, whole rounds and a rest; odd numbers of everything
SIZES = [(1, 1, 1), (1, 16, 32), (2, 17, 33), (16, 100, 257), (5, 5000, 300), (16, 13000, 96), (17, 64, 256), (32, 8200, 100), (33, 48, 1000), (64, 130, 2048),
         (65, 64, 512), (80, 65, 31), (129, 130, 255), (100, 70, 5000), (300, 260, 769), (40, 64, 16500), (777, 515, 129), (1030, 2050, 640), (2100, 8192, 300), (4100, 4200, 512)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_linear(gpu_lib, M, N, K, dtype):
    y, ref, _, b = run(gpu_lib, M, N, K, dtype, M + N + K)
    assert_same(y, ref, b, dtype)


@pytest.mark.parametrize("M,dtype", [(15001, torch.float32), (29001, torch.bfloat16)])
def test_results_that_no_cache_holds(gpu_lib, M, dtype):
    """All sums are exact, so the bits are those of calls for a part of the tokens."""
    q, N, K = gpu_lib, 4096, 700
    (a, sa), (w, sw) = codes_of(4, M, K), codes_of(5, N, K)
    dev = lambda x: torch.from_numpy(x).to(DEV)
    mat, a, sa = q.pack_mx4(dev(plain.join(w)), dev(sw), K), dev(plain.join(a)), dev(sa)
    y = q.linear_mx4(mat, a, sa, dtype=dtype)
    for m in range(0, M, 3000):
        assert torch.equal(y[m:m + 3000], q.linear_mx4(mat, a[m:m + 3000], sa[m:m + 3000], dtype=dtype))


@pytest.mark.parametrize("M,N,K", [(3, 40, 300), (70, 200, 300), (300, 300, 600), (1000, 1000, 260)])
def test_linear_without_bias_into_rows_that_lie_apart(gpu_lib, M, N, K):
    for lead, pitch, dtype in ((0, N + 5, torch.float32), (1, N + 16, torch.bfloat16), (4, N + 128 - N % 128, torch.float16), (0, N, torch.bfloat16)):
        store = torch.full((lead + M * pitch + 8,), 9.0, dtype=dtype, device=DEV)
        out = store[lead:lead + M * pitch].view(M, pitch)[:, :N]
        y, ref, _, b = run(gpu_lib, M, N, K, dtype, 3, bias=False, out=out)
        assert y is out
        assert_same(y, ref, b, dtype)
        keep = torch.ones_like(store, dtype=torch.bool)
        keep[lead:lead + M * pitch].view(M, pitch)[:, :N] = False
        assert bool((store[keep] == 9.0).all())


@pytest.mark.parametrize("M,N,K", [(4, 60, 260), (90, 130, 700), (400, 300, 530), (600, 64, 4100)])
def test_codes_at_wide_pitches_with_anything_behind_them(gpu_lib, M, N, K):
    """Bytes behind the rows of codes and bits behind the last column reach no result, nor do scales behind the last (but NaN)."""
    q = gpu_lib
    a, sa = codes_of(1, M, K)
    w, sw = codes_of(2, N, K)
    n = (K + 31) // 32
    g = np.random.default_rng(3)
    wide = g.integers(0, 256, (M, 16 * n + 48)).astype(np.uint8)
    wide[:, :16 * n] = plain.join(a)
    scales = g.integers(0, 255, (M, (n + 7) // 8 * 8 + 8)).astype(np.uint8)
    scales[:, :n] = sa[:, :n]
    dev = lambda x: torch.from_numpy(x).to(DEV)
    w_wide = g.integers(0, 256, (N, 16 * n + 32)).astype(np.uint8)
    w_wide[:, :16 * n] = plain.join(w)
    w_scales = np.full((N, n + 3), 255, np.uint8)
    w_scales[:, :n] = sw[:, :n]
    mat = q.pack_mx4(dev(w_wide), dev(w_scales), K)
    y = q.linear_mx4(mat, dev(wide), dev(scales))
    assert_same(y, exact(a, sa, K) @ exact(w, sw, K).T, None, torch.float32)


@pytest.mark.parametrize("M,N,K", [(8, 50, 640), (200, 150, 1000), (500, 600, 2000), (130, 64, 6000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_with_scales_far_apart(gpu_lib, M, N, K, dtype):
    """The sums are off by plain.sum_tolerance, the bias costs half a step of fp32 and the result half a step of its type."""
    y, ref, mag, b = run(gpu_lib, M, N, K, dtype, 9, low=117, high=130)
    want = ref + b.double().cpu().numpy()
    bound = plain.sum_tolerance(K, mag) + 2.0 ** -24 * np.abs(want) + (np.abs(want) * HALF_STEP[dtype] + float(torch.finfo(dtype).smallest_normal) * 2.0 ** -9) * (1 + 2.0 ** -10)
    got = y.double().cpu().numpy()
    if dtype == torch.float16:   # beyond its range
        far = np.abs(want) > 65000
        got, want, bound = np.where(far, 0, got), np.where(far, 0, want), np.where(far, 1, bound)
    assert (np.abs(got - want) <= bound).all()


@pytest.mark.parametrize("M,N,K", [(9, 40, 300), (100, 100, 600), (300, 600, 300)])
def test_rows_with_a_nan_scale(gpu_lib, M, N, K):
    q = gpu_lib
    a, sa = codes_of(1, M, K)
    w, sw = codes_of(2, N, K)
    ref = exact(a, sa, K) @ exact(w, sw, K).T
    sa[3, 2] = 255
    sw[N - 1, 0] = 255
    dev = lambda x: torch.from_numpy(x).to(DEV)
    y = q.linear_mx4(q.pack_mx4(dev(plain.join(w)), dev(sw), K), dev(plain.join(a)), dev(sa)).cpu().double().numpy()
    assert np.isnan(y[3]).all() and np.isnan(y[:, N - 1]).all()
    keep = np.ones_like(y, bool)
    keep[3], keep[:, N - 1] = False, False
    assert np.array_equal(y[keep], ref[keep].astype(np.float32))


@pytest.mark.parametrize("N,K", [(1, 1), (15, 31), (16, 256), (33, 257), (100, 1000)])
def test_packed_weights_column_by_column(gpu_lib, N, K):
    """Activations that are 1 in one column and 0 elsewhere read the weights back."""
    q = gpu_lib
    w, sw = codes_of(7, N, K, 100, 140)
    eye = torch.eye(K, device=DEV)
    codes, scale = q.quantize_mx4(eye)
    dev = lambda x: torch.from_numpy(x).to(DEV)
    y = q.linear_mx4(q.pack_mx4(dev(plain.join(w)), dev(sw), K), codes, scale)
    assert np.array_equal(y.t().cpu().double().numpy(), exact(w, sw, K))


def test_no_rows(gpu_lib):
    q = gpu_lib
    codes, scale = q.quantize_mx4(torch.empty((0, 40), device=DEV))
    assert codes.shape == (0, 32) and scale.shape == (0, 8)
    assert q.dequantize_mx4(codes, scale, 40).shape == (0, 40)
    mat = q.pack_mx4(*q.quantize_mx4(torch.ones((4, 40), device=DEV)), 40)
    assert q.linear_mx4(mat, codes, scale).shape == (0, 4)


def test_a_workspace_for_many_tokens_serves_fewer(gpu_lib):
    q = gpu_lib
    N, K = 100, 9000
    w, sw = codes_of(1, N, K)
    dev = lambda x: torch.from_numpy(x).to(DEV)
    mat = q.pack_mx4(dev(plain.join(w)), dev(sw), K)
    ws = torch.empty(q.linear_mx4_workspace(mat, 500), dtype=torch.uint8, device=DEV)
    for M in (500, 200, 70, 33, 3):
        a, sa = codes_of(M, M, K)
        y = q.linear_mx4(mat, dev(plain.join(a)), dev(sa), workspace=ws)
        assert_same(y, exact(a, sa, K) @ exact(w, sw, K).T, None, torch.float32)


@pytest.mark.parametrize("M,N,K", [(5, 20, 384), (70, 100, 384), (300, 300, 640)])
def test_sums_of_one_large_and_many_small_products(gpu_lib, M, N, K):
    """The first block's scale makes its products larger than the others by up to 2^44: what is cut off stays within the bound."""
    q = gpu_lib
    for d in (20, 27, 28, 31, 44):
        code = np.full((M, (K + 31) // 32 * 32), 3, np.uint8)   # 1.5
        code[:, 1:32] = 0
        scale = np.full((M, (K + 255) // 256 * 8), 127, np.uint8)
        scale[:, 0] = 127 + d // 2
        w, sw = np.resize(code[:1], (N, code.shape[1])).copy(), np.resize(scale[:1], (N, scale.shape[1])).copy()
        w[1::2, 32:] |= 8   # every second row's small products are negative
        dev = lambda x: torch.from_numpy(x).to(DEV)
        y = q.linear_mx4(q.pack_mx4(dev(plain.join(w)), dev(sw), K), dev(plain.join(code)), dev(scale)).double().cpu().numpy()
        a, b = exact(code, scale, K), exact(w, sw, K)
        want, largest = a @ b.T, (np.abs(a[:, 0])[:, None] * np.abs(b[:, 0])[None, :])
        steps = 2 * ((K + 255) // 256)
        assert (np.abs(y - want) <= steps * 2.0 ** -19 * (largest + np.abs(want))).all()
        if d < 24:
            assert np.array_equal(y, want.astype(np.float32))
