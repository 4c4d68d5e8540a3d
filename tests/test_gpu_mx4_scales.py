"""The linear layer of microscaled 4-bit floats with every scale byte: from 2^-127 to 2^127 on either side, alone and against each other."""
import numpy as np
import pytest
import torch

from tests import plain_mx4 as plain
from tests.test_gpu_mx4 import DEV, TYPES, exact

pytestmark = pytest.mark.gpu
TINY = 2.0 ** -149   # the step of fp32 below 2^-126
# few tokens in two forms, small tiles, small tiles of a cut sum, and what larger results take
SIZES = [(7, 40, 160), (45, 100, 700), (90, 130, 1283), (70, 64, 9000), (1030, 2050, 640), (4200, 4100, 300)]


def dev(x):
    return torch.from_numpy(x).to(DEV)


def layer(q, a, sa, w, sw, **more):
    """Codes [., 32 * blocks] and scales [., blocks]."""
    wide = lambda s: np.pad(s, ((0, 0), (0, -s.shape[1] % 8)), constant_values=127)
    return q.linear_mx4(q.pack_mx4(dev(plain.join(w)), dev(wide(sw)), w.shape[1]), dev(plain.join(a)), dev(wide(sa)), **more)


@pytest.mark.parametrize("M,K,at", [(16, 32, 0), (255, 32, 0), (255, 96, 70), (40, 544, 300), (255, 4640, 4400), (4335, 64, 33)])
def test_one_product_of_any_two_scales(gpu_lib, M, K, at):
    """255 x 255 scales: the product as fp32 holds it, subnormal or infinite ones too.  The other codes are zeros of the same scales."""
    e = np.arange(255, dtype=np.uint8)
    for ca, cw in ((2, 2), (7, 7), (15, 1), (0, 7), (1, 1)):
        w, a = np.zeros((255, K), np.uint8), np.zeros((M, K), np.uint8)
        w[:, at], a[:, at] = cw, ca
        for first in range(0, 255 if M < 255 else 1, M):
            ea = np.resize(np.roll(e, -first), M)
            y = layer(gpu_lib, a, np.repeat(ea[:, None], K // 32, 1), w, np.repeat(e[:, None], K // 32, 1))
            value = np.outer(np.ldexp(plain.VALUES[ca & 7] * (-1.0 if ca & 8 else 1.0), ea.astype(np.int64) - 127),
                             np.ldexp(plain.VALUES[cw & 7], e.astype(np.int64) - 127))
            with np.errstate(over="ignore"):
                assert torch.equal(y.cpu(), torch.from_numpy(value.astype(np.float32)))


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_scales_at_the_ends_against_each_other(gpu_lib, M, N, K, dtype):
    """Blocks of activations with scales from 2^-127 to 2^127 meet weights with the others: all products are ordinary, multiples of 2^-4 whose
    sums' magnitudes stay below 2^20, so fp32 holds every sum."""
    rng = np.random.default_rng(M + K)
    n = (K + 31) // 32
    mid = np.where(np.arange(n) % 3 == 0, rng.choice([0, 1, 2, 127, 252, 253, 254], n), rng.integers(0, 255, n))
    a, w = rng.integers(0, 16, (M, n * 32)).astype(np.uint8), rng.integers(0, 16, (N, n * 32)).astype(np.uint8)
    a[:, K:] = 0
    one = lambda rows, e: np.clip(e[None, :] - rng.integers(0, 2, (rows, n)), 0, 254).astype(np.uint8)
    sa, sw = one(M, mid), one(N, 254 - mid)
    va, vw = plain.values(a, sa), plain.values(w, sw)
    want = (torch.from_numpy(va).to(DEV) @ torch.from_numpy(vw).to(DEV).t()).cpu().numpy()   # (exact in 64 bits)
    assert torch.equal(layer(gpu_lib, a, sa, w, sw, dtype=dtype).cpu(), torch.from_numpy(want.astype(np.float32)).to(dtype))


@pytest.mark.parametrize("M,N,K", SIZES[:4])
def test_sums_that_fp32_holds_as_subnormals(gpu_lib, M, N, K):
    """A block's sum is rounded to 2^-149 (half of that, and half again for the result), and may be cut as others are."""
    rng = np.random.default_rng(K)
    n = (K + 31) // 32
    a, w = rng.integers(0, 16, (M, n * 32)).astype(np.uint8), rng.integers(0, 16, (N, n * 32)).astype(np.uint8)
    a[:, K:] = 0
    sa, sw = np.full((M, n), 3, np.uint8), np.repeat(rng.integers(85, 130, (N, 1)).astype(np.uint8), n, 1)
    va, vw = plain.values(a, sa), plain.values(w, sw)
    want, mag = va @ vw.T, np.abs(va) @ np.abs(vw).T
    got = layer(gpu_lib, a, sa, w, sw).double().cpu().numpy()
    assert (np.abs(got - want) <= (n + 1) * TINY / 2 + plain.sum_tolerance(K, mag) + 2.0 ** -24 * np.abs(want)).all()
    assert (got != 0).any() and (np.abs(want) < 2.0 ** -126).any()


@pytest.mark.parametrize("M,N,K", SIZES[:4])
def test_sums_that_pass_fp32_are_not_finite(gpu_lib, M, N, K):
    """Whether they come back or not; other rows and columns of the result are what they are."""
    n = (K + 31) // 32
    a, w = np.full((M, n * 32), 2, np.uint8), np.full((N, n * 32), 2, np.uint8)
    a[:, K:] = 0
    sa, sw = np.full((M, n), 127, np.uint8), np.full((N, n), 127, np.uint8)
    sa[3, 1], sw[5, 1] = 254, 253
    w[:, 32:64] = 0
    w[5, 32:64] = 2                 # 32 products of 2^253 in row 3, of 2^126 in the others: 2^131, too much
    w[6, 32:64], w[6, :32] = 2, 10  # 32 of 2^127 in row 3
    w[7, 40] = 2                    # one of them: not too much
    y = layer(gpu_lib, a, sa, w, sw).cpu().double().numpy()
    va, vw = exact(a, sa, n * 32), exact(w, sw, n * 32)
    over = np.zeros(y.shape, bool)
    for b in range(0, n * 32, 32):
        over |= np.abs(va[:, b:b + 32] @ vw[:, b:b + 32].T) >= 2.0 ** 128
    assert int(over.sum()) == M + 1 and np.array_equal(np.isfinite(y), ~over)
    want, mag = va @ vw.T, np.abs(va) @ np.abs(vw).T
    assert (np.abs(y - want)[~over] <= (plain.sum_tolerance(K, mag) + 2.0 ** -24 * np.abs(want))[~over]).all()


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_not_finite_when_quantized_makes_its_row_nan(gpu_lib, M, N, K, dtype):
    """The quantizer writes such a block as zeros with a NaN scale; its products are NaN, whatever they meet, zeros too."""
    q = gpu_lib
    g = torch.Generator().manual_seed(M)
    x, w = torch.randn((M, K), generator=g), torch.randn((N, K), generator=g)
    w[:, :64] = 0.0
    want = q.linear_mx4(q.pack_mx4(*q.quantize_mx4(w.to(DEV)), K), *q.quantize_mx4(x.to(DEV)), dtype=dtype)
    x[2, 40], x[M - 1, K - 1], w[N - 1, 3] = float("nan"), float("inf"), -float("inf")
    y = q.linear_mx4(q.pack_mx4(*q.quantize_mx4(w.to(DEV)), K), *q.quantize_mx4(x.to(DEV)), dtype=dtype)
    assert bool(y[2].isnan().all()) and bool(y[M - 1].isnan().all()) and bool(y[:, N - 1].isnan().all())
    rows = [m for m in range(M) if m not in (2, M - 1)]
    assert torch.equal(y[rows, :N - 1], want[rows, :N - 1])
