"""Rows of fp32 with a weight for which 64 bits do not decide: products of two fp32 values have 48 bits, 127 times them 55, and
a quotient may lie so near the border of two codes that fp64 rounds onto it.  The expected codes come from whole numbers."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# value, its weight, the row's largest value, its weight: 127 * value * weight / (largest * weight) is within 2^-53 of a half
NEAR = [(13584009, 8509953, 12290083, 9518320), (11023329, 13666381, 12793516, 15659458), (15642983, 9019847, 15225983, 16012155),
        (15642983, 9019847, 15225983, 13764835), (13227203, 13173249, 14272204, 12867274), (14618029, 8953173, 11915842, 11871536),
        (10582359, 10850585, 11730093, 10316939), (9958251, 13467876, 14051179, 15641249), (11146650, 11784417, 14200113, 15560281),
        (10299142, 12322864, 13548638, 16409025), (10299142, 12322864, 13548638, 10574705), (14706544, 8708158, 10176483, 15746241),
        (9934616, 13880719, 13732198, 12817509), (13163666, 15079352, 13965955, 16636535), (9649961, 13171371, 13289237, 16304367),
        (12936874, 9737182, 11304771, 11842317), (11145924, 14358381, 15563013, 15455209), (8892439, 16257012, 15127853, 9827003)]


def code(value, largest):
    """rne(127 value / largest) of whole numbers."""
    two, rest = divmod(254 * abs(value), largest)   # in half codes
    k = two // 2
    up = two % 2 and (rest or k % 2)
    return (1 if value > 0 else -1) * (k + (1 if up else 0))


def case(pad, scale, sign):
    """A row for each entry, zeros but for two columns of its own, and one with an exact half: (x, weight, codes)."""
    rows = NEAR + [(15, 1 << 20, 254, 1 << 20)]   # 127 * 15 / 254 = 7.5
    cols = 2 * len(rows) + pad
    x, w, want = torch.zeros((len(rows), cols)), torch.ones(cols), np.zeros((len(rows), cols), np.int8)
    for r, (h, hw, p, pw) in enumerate(rows):
        at = cols - 2 * len(rows) + 2 * r
        x[r, at], w[at], x[r, at + 1], w[at + 1] = sign * h, hw, p, pw
        want[r, at], want[r, at + 1] = code(sign * h * hw, p * pw), 127
    return x * scale, w * scale, want


@pytest.mark.parametrize("scale", [2.0 ** -23, 1.0, 2.0 ** -50, 2.0 ** 40])   # the latter two in the way of rows out of the ordinary
@pytest.mark.parametrize("pad", [0, 3, 300, 5000, 20000])
def test_codes_that_64_bits_do_not_decide(gpu_lib, pad, scale):
    for sign in (1, -1):
        x, w, want = case(pad, scale, sign)
        codes, _, _ = gpu_lib.rms_norm_quant(x.to(DEV), w.to(DEV), 0.0)
        np.testing.assert_array_equal(codes.cpu().numpy()[:, :x.shape[1]], want)


def test_the_expected_codes_are_not_those_of_64_bits():
    for h, hw, p, pw in NEAR:
        assert int(np.rint(127.0 * float(h * hw) / float(p * pw))) != code(h * hw, p * pw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [4, 200, 5000])
def test_scales_of_rows_whose_largest_value_passes_fp32(gpu_lib, dtype, cols):
    """One value of 2^-30 among zeros times 2^127: normalised it is 2^127 sqrt(cols), and a 127th of it fits fp32."""
    x = torch.zeros((2, cols))
    x[0, 1] = x[1, cols - 1] = 2.0 ** -30
    w = torch.full((cols,), 2.0 ** 127)
    codes, scale, _ = gpu_lib.rms_norm_quant(x.to(dtype).to(DEV), w.to(dtype).to(DEV), 0.0)
    want = 2.0 ** 127 * np.sqrt(cols) / 127.0
    # quotient, mean, its root and reciprocal, product: 5 roundings, the mean's halved by the root
    assert (np.abs(scale.cpu().numpy().astype(np.float64) - want) <= 5 * 2.0 ** -24 * want).all()
    assert codes[0, 1] == 127 and codes[1, cols - 1] == 127 and int(codes.float().sum()) == 254


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_the_sum_beside_its_inputs_in_one_matrix(gpu_lib, dtype):
    """x, residual and sum as columns of one matrix: their rows lie between one another and share no byte."""
    q, rows, cols = gpu_lib, 9, 75
    big = torch.randn((rows, 3 * cols), generator=torch.Generator().manual_seed(1)).to(dtype).to(DEV)
    x, res = big[:, :cols], big[:, 2 * cols:]
    want = q.rms_norm_quant(x.contiguous(), None, 1e-5, residual=res.contiguous())
    before = big.clone()
    got = q.rms_norm_quant(x, None, 1e-5, residual=res, sum_out=big[:, cols:2 * cols])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(x, before[:, :cols]) and torch.equal(res, before[:, 2 * cols:])
    with pytest.raises(RuntimeError):   # a column of x among the sum's
        q.rms_norm_quant(x, None, 1e-5, residual=res, sum_out=big[:, cols - 1:2 * cols - 1])
    with pytest.raises(RuntimeError):
        q.rms_norm_quant(x, None, 1e-5, residual=res, sum_out=big[:, cols + 1:2 * cols + 1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_row_in_place_by_views_of_different_pitch(gpu_lib, dtype):
    """A single row has no pitch: two views of it are the same row."""
    q, cols = gpu_lib, 75
    big = torch.randn((6, 100), generator=torch.Generator().manual_seed(2)).to(dtype).to(DEV)
    res = torch.randn((1, cols), generator=torch.Generator().manual_seed(3)).to(dtype).to(DEV)
    for a, b in ((big[3:4, :cols], big[3, :cols].unsqueeze(0)), (big[4, :cols].unsqueeze(0), big[4:5, :cols])):
        want, before = q.rms_norm_quant(a.clone(), None, 1e-5, residual=res), big.clone()
        assert a.stride(0) != b.stride(0)
        got = q.rms_norm_quant(a, None, 1e-5, residual=res, sum_out=b)
        assert all(torch.equal(x, y) for x, y in zip(got, want)) and torch.equal(a, want[2])
        assert torch.equal(big[:3], before[:3]) and torch.equal(big[5:], before[5:]) and torch.equal(big[:, cols:], before[:, cols:])
    with pytest.raises(RuntimeError):
        q.rms_norm_quant(big[3:4, :cols], None, 1e-5, residual=res, sum_out=big[3:4, 1:cols + 1])
