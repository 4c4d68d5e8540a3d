"""8-bit activations with a range for each row against 64 bits: the codes are those of the exact quotients, the sums those of
their type, the scales within the roundings counted below."""
import numpy as np
import pytest
import torch

from . import plain64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def scale_tolerance(cols, dtype):
    """Relative.  The squares of a row: a chain of at most `chain` fused additions in a thread, 6 over a wave, 16 over a
    workgroup, each half a step of fp32 and halved by the root; mean, eps, root, reciprocal, product, quotient: 1 + 1
    (halved), then 4 of them."""
    V = 4 if dtype == torch.float32 else 8
    chain = V * max(5, -(-cols // (1024 * V)))
    return ((chain + 6 + 16 + 2) / 2 + 4) * 2.0 ** -24


def check(codes, scale, want, cols, dtype, norm):
    got, s = codes.cpu().numpy(), scale.cpu().numpy()
    w_codes, w_scale = want
    assert got.shape[1] == (cols + 15) // 16 * 16
    np.testing.assert_array_equal(got[:, :cols], w_codes)
    assert (got[:, cols:] == 0).all()
    tol = scale_tolerance(cols, dtype) if norm else 2.0 ** -24
    np.testing.assert_array_equal(np.isnan(s), np.isnan(w_scale))
    ok = ~np.isnan(w_scale)
    assert (np.abs(s[ok] - w_scale[ok]) <= tol * np.abs(w_scale[ok]) * (1 + 1e-6) + 2.0 ** -150).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 8), (2, 15), (4, 16), (1, 33), (7, 255), (9, 512), (2, 513), (3, 1024),
                                       (2, 1027), (1, 2049), (3, 4096), (2, 4101), (2, 8192), (2, 8200), (1, 16385), (2, 33000), (1, 70001)])
def test_codes_of_every_row_length(gpu_lib, dtype, rows, cols):
    q = gpu_lib
    x = (randn(rows * 100003 + cols, rows, cols) * torch.exp(randn(5, rows, 1))).to(dtype)
    res, w = randn(6 + cols, rows, cols).to(dtype), (1 + 0.3 * randn(7, cols)).to(dtype)
    codes, scale = q.quantize_tokens(x.to(DEV))
    check(codes, scale, plain64.token_codes(x.double().numpy()), cols, dtype, False)
    for residual, weight in ((res, w), (None, w), (res, None), (None, None)):
        on = lambda t: None if t is None else t.to(DEV)
        codes, scale, total = q.rms_norm_quant(on(x), on(weight), 1e-5, residual=on(residual))
        want = plain64.rms_norm_quant(x, weight, 1e-5, residual)
        check(codes, scale, want[:2], cols, dtype, True)
        assert torch.equal(total.cpu(), want[2])


@pytest.mark.parametrize("dtype", TYPES)
def test_borders_between_codes_go_by_the_exact_quotient(gpu_lib, dtype):
    """Rows whose largest value is 127 (or 127 / 2^7) and whose others lie at, just below and just above the half codes."""
    q = gpu_lib
    k = torch.arange(-126, 127).double()
    at = torch.cat([k + 0.5, k + 0.5 + 1e-5, k + 0.5 - 1e-5, torch.tensor([127.0]).double()])
    x = torch.stack([at, at / 128, -at * 3.0]).to(dtype)
    codes, scale = q.quantize_tokens(x.to(DEV))
    check(codes, scale, plain64.token_codes(x.double().numpy()), x.shape[1], dtype, False)
    w = (1 + 0.1 * randn(3, x.shape[1])).to(dtype)
    codes, scale, _ = q.rms_norm_quant(x.to(DEV), w.to(DEV), 0.0)
    check(codes, scale, plain64.rms_norm_quant(x, w, 0.0)[:2], x.shape[1], dtype, True)


@pytest.mark.parametrize("cols", [5, 300, 1500, 5000, 40000])
def test_rows_out_of_the_ordinary(gpu_lib, cols):
    """Zeros, NaN, infinities, values whose squares overflow or vanish, denormal values: each row by itself."""
    q = gpu_lib
    base = randn(11, 1, cols)
    rows = [torch.zeros(1, cols), base, base * 1e30, base * 1e-30, base * 3e37, base * 1e-42, -base * 2.0 ** 70, base * 2.0 ** -59]
    bad = [base.clone() for _ in range(3)]
    bad[0][0, cols - 1] = float("nan")
    bad[1][0, 0] = float("inf")
    bad[2][0, cols // 2] = float("-inf")
    one = torch.zeros(1, cols)
    one[0, cols // 3] = 1e-45
    x = torch.cat(rows + bad + [one])
    codes, scale = q.quantize_tokens(x.to(DEV))
    check(codes, scale, plain64.token_codes(np.where(np.isfinite(x.double().numpy()), x.double().numpy(), np.nan)), cols, torch.float32, False)
    for weight in (None, torch.full((cols,), 1e30), torch.zeros(cols), 1 + 0.1 * randn(12, cols)):
        for eps in (0.0, 1e-5):
            codes, scale, _ = q.rms_norm_quant(x.to(DEV), None if weight is None else weight.to(DEV), eps)
            want = plain64.rms_norm_quant(x, weight, eps)
            with np.errstate(over="ignore"):
                s = np.where(np.isnan(want[1]), np.nan, want[1].astype(np.float32).astype(np.float64))
            got = scale.cpu().numpy().astype(np.float64)
            np.testing.assert_array_equal(codes.cpu().numpy()[:, :cols], want[0])
            np.testing.assert_array_equal(np.isnan(got), np.isnan(s))
            np.testing.assert_array_equal(np.isinf(got), np.isinf(s))
            ok = np.isfinite(s)
            assert (np.abs(got[ok] - s[ok]) <= (scale_tolerance(cols, torch.float32) + 2.0 ** -23) * s[ok] + 2.0 ** -149).all()


def test_sixteen_bit_rows_that_overflow_their_sum(gpu_lib):
    q = gpu_lib
    x = torch.full((2, 40), 60000.0, dtype=torch.float16)
    x[1] = 1.0
    codes, scale, total = q.rms_norm_quant(x.to(DEV), None, 1e-5, residual=x.to(DEV))
    assert torch.isinf(total[0]).all() and torch.isnan(scale[0]) and bool((codes[0] == 0).all())
    assert bool((codes[1, :40] == 127).all()) and bool((total[1] == 2).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_places_and_neighbours(gpu_lib, dtype):
    """Inputs and outputs inside larger matrices at odd places; the sum in place of the residual or of x; what lies around
    the outputs stays."""
    q = gpu_lib
    rows, cols = 37, 333
    big = randn(21, rows, cols + 29).to(dtype).to(DEV)
    x = big[:, 3:3 + cols]
    res_big = randn(22, rows, 2 * cols + 5).to(dtype).to(DEV)
    res = res_big[:, cols + 1:2 * cols + 1]
    w = (1 + 0.2 * randn(23, cols + 1)).to(dtype).to(DEV)[1:]
    want = plain64.rms_norm_quant(x.cpu(), w.cpu(), 1e-6, res.cpu())
    code_big = torch.full((rows + 2, 400), 77, dtype=torch.int8, device=DEV)
    codes, scale_big = code_big[1:rows + 1, 16:16 + 336], torch.full((rows + 2,), 5.0, device=DEV)
    before = res_big.clone()
    got, scale, total = q.rms_norm_quant(x, w, 1e-6, residual=res, sum_out=res, codes=codes, scale=scale_big[1:rows + 1])
    assert total.data_ptr() == res.data_ptr()
    check(got.contiguous(), scale, want[:2], cols, dtype, True)
    assert torch.equal(res.cpu(), want[2])
    assert torch.equal(res_big[:, :cols + 1], before[:, :cols + 1]) and torch.equal(res_big[:, 2 * cols + 1:], before[:, 2 * cols + 1:])
    assert bool((code_big[0] == 77).all()) and bool((code_big[-1] == 77).all()) and bool((code_big[:, :16] == 77).all()) and bool((code_big[1:-1, 352:] == 77).all())
    assert scale_big[0] == 5 and scale_big[-1] == 5
    x2, res2 = big.clone()[:, 3:3 + cols], before[:, cols + 1:2 * cols + 1]
    _, _, total = q.rms_norm_quant(x2, w, 1e-6, residual=res2, sum_out=x2)
    assert total.data_ptr() == x2.data_ptr() and torch.equal(total.cpu(), want[2])
    wide = torch.full((rows, 512), 9, dtype=torch.int8, device=DEV)   # a wide pitch: the padding ends at the next 16 bytes
    q.quantize_tokens(x, codes=wide)
    assert bool((wide[:, cols:336] == 0).all()) and bool((wide[:, 336:] == 9).all())


def test_no_rows(gpu_lib):
    q = gpu_lib
    codes, scale = q.quantize_tokens(torch.empty((0, 64), device=DEV))
    assert codes.shape == (0, 64) and scale.shape == (0,)
    codes, scale, total = q.rms_norm_quant(torch.empty((0, 20), device=DEV), None, 1e-5, residual=torch.empty((0, 20), device=DEV))
    assert codes.shape == (0, 32) and total.shape == (0, 20)


def test_many_rows(gpu_lib):
    """More rows than a grid's y extent, the last ones checked."""
    q = gpu_lib
    x = randn(31, 70003, 24).to(DEV)
    codes, scale = q.quantize_tokens(x)
    tail = x[-50:].cpu()
    check(codes[-50:], scale[-50:], plain64.token_codes(tail.double().numpy()), 24, torch.float32, False)


@pytest.mark.parametrize("rows", [(1 << 26) + 70, (1 << 27) + 70])
def test_more_rows_than_a_launch_takes(gpu_lib, rows):
    """Rows of 16 threads: 2^31 threads, 2^27 rows, to a launch; the last ones, and those of the second launch, as all others."""
    q = gpu_lib
    x = torch.randn((rows, 1), device=DEV, dtype=torch.float16, generator=torch.Generator(DEV).manual_seed(1))
    codes, scale = q.quantize_tokens(x)
    at = torch.cat([torch.arange(5), torch.arange(1 << 25, (1 << 25) + 5), torch.arange(rows - 140, rows)]).to(DEV)
    want = plain64.token_codes(x[at].cpu().double().numpy())
    check(codes[at], scale[at], want, 1, torch.float16, False)
    assert torch.equal(codes[:, 0].float(), 127.0 * torch.sign(x[:, 0].float()))
    assert not codes[:, 1:].any()


@pytest.mark.parametrize("value", [1.1, 1.3330078125, 0.7])
def test_long_rows_of_equal_values(gpu_lib, value):
    """Sums of very many equal squares, which fp32 would round to the same side for long stretches: a vector's squares are added
    in fp32, vectors in fp64, 6 + 16 sums of fp32 join them."""
    q, cols = gpu_lib, (1 << 24) + 5
    x = torch.full((1, cols), value, dtype=torch.float32)
    codes, scale, _ = q.rms_norm_quant(x.to(DEV), None, 0.0)
    h = float(x[0, 0])
    want = h / np.sqrt(h * h) / 127.0
    # 4 + 1 + 6 + 16 + 2 roundings halved by the root, 4 behind it; the count of columns itself is rounded to fp32: half of one
    assert abs(float(scale[0]) - want) <= ((4 + 1 + 6 + 16 + 2) / 2 + 4 + 0.5) * 2.0 ** -24 * want
    assert bool((codes[0, :cols] == 127).all()) and not bool(codes[0, cols:].any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 9, 60, 64, 65, 100, 127, 128, 129, 250, 256])
def test_short_rows_of_every_kind_side_by_side(gpu_lib, dtype, cols):
    """Several rows to a wave: rows that are ordinary, all zero, not finite, tiny or huge next to one another, a last wave that is
    not full."""
    q, rows = gpu_lib, 77
    x = randn(cols, rows, cols).double()
    big = 3e38 if dtype != torch.float16 else 6e4
    x[3::8] = 0.0
    x[4::8, cols // 2] = float("inf")
    x[5::8, cols - 1] = float("nan")
    x[6::8] *= 1e-30 if dtype != torch.float16 else 1e-6
    x[7::8] = x[7::8].sign() * big
    x = x.to(dtype)
    codes, scale = q.quantize_tokens(x.to(DEV))
    values = x.double().numpy()
    check(codes, scale, plain64.token_codes(np.where(np.isfinite(values), values, np.nan)), cols, dtype, False)
    w = (1 + 0.3 * randn(7, cols)).to(dtype)
    codes, scale, _ = q.rms_norm_quant(x.to(DEV), w.to(DEV), 1e-5)
    check(codes, scale, plain64.rms_norm_quant(x, w, 1e-5, None)[:2], cols, dtype, True)
