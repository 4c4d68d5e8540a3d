"""8-bit linear layers of rows with a scale each against 64 bits."""
import numpy as np
import pytest
import torch

from . import plain64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def make(seed, M, N, K, full=False):
    r = np.random.RandomState(seed)
    lo, hi = (-128, 128) if full else (-127, 128)
    return dict(a=r.randint(lo, hi, (M, K)).astype(np.int8), w=r.randint(lo, hi, (N, K)).astype(np.int8),
                sa=np.exp(r.randn(M)).astype(np.float32) / 100, sw=np.exp(r.randn(N)).astype(np.float32) / 100,
                bias=r.randn(N).astype(np.float32))


def pad(a, pitch, fill=0):
    out = np.full((a.shape[0], pitch), fill, np.int8)
    out[:, :a.shape[1]] = a
    return torch.from_numpy(out).to(DEV)


def weights(q, d):
    return q.pack_int8(torch.from_numpy(d["w"]).to(DEV), q.LAYOUT_TILED, torch.from_numpy(d["sw"]).to(DEV))


def tolerance(y, p, dtype):
    """The sum is rounded to fp32, multiplied by the row's scale (two roundings of the product), by the token's in one
    operation with the bias's addition (one rounding of the result), and rounded to its type."""
    return 2.01 * 2.0 ** -24 * p + (2.0 ** -24 + plain64.HALF_STEP[dtype]) * np.abs(y) * (1 + 2.0 ** -8) + 2.0 ** -25


def check(got, d, dtype, with_bias=True):
    y, p = plain64.linear(d["a"], d["sa"], d["w"], d["sw"], d["bias"] if with_bias else None)
    off = np.abs(got.float().cpu().numpy().astype(np.float64) - y) - tolerance(y, p, dtype)
    assert off.max() <= 0, np.unravel_index(off.argmax(), off.shape)


SIZES = [(1, 1, 1), (1, 16, 16), (1, 1000, 129), (2, 17, 63), (5, 64, 64), (16, 250, 300), (17, 256, 1280), (31, 130, 4100), (33, 48, 127), (63, 1000, 640),
         (64, 512, 1024), (65, 100, 257), (77, 333, 1283), (128, 128, 128), (129, 257, 400), (200, 640, 272), (255, 255, 255),
         (256, 256, 256), (257, 513, 129), (300, 1100, 2064), (513, 300, 96), (700, 768, 1536), (1025, 1031, 515)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_sizes(gpu_lib, dtype, M, N, K):
    q = gpu_lib
    d = make(M + 7 * N + 13 * K, M, N, K)
    a = pad(d["a"], (K + 15) // 16 * 16, fill=113)   # what lies behind the columns may be anything
    sa, bias = torch.from_numpy(d["sa"]).to(DEV), torch.from_numpy(d["bias"]).to(DEV)
    m = weights(q, d)
    check(q.linear_tokens(m, a, sa, bias=bias, dtype=dtype), d, dtype)
    check(q.linear_tokens(m, a, sa, dtype=dtype), d, dtype, with_bias=False)


@pytest.mark.parametrize("M", [1, 40, 300])
def test_largest_sums_are_exact(gpu_lib, M):
    """Codes of -128 throughout, the longest sum: 131071 * 2^14 is just below 2^31."""
    q = gpu_lib
    K, N = 131071, 20
    a = torch.full((M, K + 1), -128, dtype=torch.int8, device=DEV)
    m = q.pack_int8(torch.full((N, K), -128, dtype=torch.int8, device=DEV), q.LAYOUT_TILED)
    y = q.linear_tokens(m, a, torch.ones(M, device=DEV))
    assert bool((y == float(np.float32(131071 * 2 ** 14))).all())


@pytest.mark.parametrize("M", [3, 130, 600])
def test_rows_apart_and_neighbours(gpu_lib, M):
    """Codes and results inside larger matrices, results at an odd element; what lies around them stays."""
    q = gpu_lib
    N, K = 203, 150
    d = make(5, M, N, K)
    a = pad(d["a"], 400, fill=-7)[:, :160]
    sa, m = torch.from_numpy(d["sa"]).to(DEV), weights(q, d)
    for dtype in TYPES:
        big = torch.full((M + 2, 3 * N), 42.0, dtype=dtype, device=DEV)
        out = big[1:M + 1, N + 1:2 * N + 1]
        y = q.linear_tokens(m, a, sa, out=out)
        assert y.data_ptr() == out.data_ptr()
        check(out, d, dtype, with_bias=False)
        assert bool((big[0] == 42).all()) and bool((big[-1] == 42).all())
        assert bool((big[:, :N + 1] == 42).all()) and bool((big[:, 2 * N + 1:] == 42).all())


def test_no_tokens_and_scales_that_are_not_finite(gpu_lib):
    q = gpu_lib
    d = make(9, 20, 40, 64)
    m = weights(q, d)
    assert q.linear_tokens(m, torch.empty((0, 64), dtype=torch.int8, device=DEV), torch.empty(0, device=DEV)).shape == (0, 40)
    sa = torch.from_numpy(d["sa"]).to(DEV)
    sa[3] = float("nan")
    y = q.linear_tokens(m, pad(d["a"], 64), sa)
    assert bool(torch.isnan(y[3]).all()) and not bool(torch.isnan(torch.cat([y[:3], y[4:]])).any())


def test_the_same_call_gives_the_same_bits_whatever_the_workspace_held(gpu_lib):
    q = gpu_lib
    for M, N, K in ((16, 96, 8192), (100, 200, 4096), (300, 64, 6000)):
        d = make(M, M, N, K)
        a, sa, m = pad(d["a"], (K + 15) // 16 * 16), torch.from_numpy(d["sa"]).to(DEV), weights(q, d)
        need = q.linear_tokens_workspace(m, M)
        first = q.linear_tokens(m, a, sa)
        check(first, d, torch.float32, with_bias=False)
        for fill in (0, 255, 77):
            ws = torch.full((need + 256,), fill, dtype=torch.uint8, device=DEV)
            assert torch.equal(q.linear_tokens(m, a, sa, workspace=ws), first)
            assert bool((ws[need:] == fill).all())


def test_every_way_captured_and_replayed(gpu_lib):
    """Few tokens, each size of tile, a sum in parts: replays on new inputs in the captured places against eager calls."""
    q = gpu_lib
    for M, N, K in ((7, 100, 300), (90, 700, 640), (700, 2600, 300), (3000, 4200, 256), (300, 64, 8192)):
        d = [make(M + i, M, N, K) for i in range(3)]
        a, sa, m = pad(d[0]["a"], (K + 15) // 16 * 16), torch.from_numpy(d[0]["sa"]).to(DEV), weights(q, d[0])
        ws = torch.empty(max(1, q.linear_tokens_workspace(m, M)), dtype=torch.uint8, device=DEV)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = q.linear_tokens(m, a, sa, dtype=torch.float16, workspace=ws)
        for e in d[1:]:
            a[:, :K] = torch.from_numpy(e["a"]).to(DEV)
            sa.copy_(torch.from_numpy(e["sa"]))
            graph.replay()
            torch.cuda.synchronize()
            check(y, dict(d[0], a=e["a"], sa=e["sa"]), torch.float16, with_bias=False)
            assert torch.equal(q.linear_tokens(m, a, sa, dtype=torch.float16), y)
            ws.fill_(255)


def test_two_streams_at_once(gpu_lib):
    """Calls that overlap, each with a workspace of its own."""
    q = gpu_lib
    d = [make(i, M, 64, 8192) for i, M in enumerate((300, 200))]
    ins = [(weights(q, e), pad(e["a"], 8192), torch.from_numpy(e["sa"]).to(DEV)) for e in d]
    want = [q.linear_tokens(*i) for i in ins]
    streams = [torch.cuda.Stream() for _ in ins]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(5):
        for k, (s, i) in enumerate(zip(streams, ins)):
            with torch.cuda.stream(s):
                outs[k].append(q.linear_tokens(*i))
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(o, want[k]) for o in outs[k])


# Large tiles alone, in rounds, with small or middle ones behind them; middle and small ones in one round and in several; one, two,
# three and more chunks of columns; edges in every dimension.
WAYS = [(10941, 132, 40), (11403, 142, 200), (295, 10943, 520), (9991, 267, 40), (10302, 263, 200), (270, 10248, 257), (835, 11970, 40),
        (10794, 1290, 200), (1291, 11271, 257), (9295, 1552, 520), (8899, 1313, 40), (10158, 773, 200), (10975, 727, 257), (729, 10918, 520),
        (10960, 1448, 257), (2200, 9190, 520), (1412, 11042, 700), (11928, 2602, 700), (9927, 2823, 200), (2050, 11715, 257), (2693, 8875, 520),
        (7215, 4494, 257), (5162, 6769, 520), (2954, 11036, 520), (4922, 9842, 520), (4608, 4096, 1920)]


@pytest.mark.parametrize("M,N,K", WAYS)
def test_every_way_of_larger_products(gpu_lib, M, N, K):
    """Against 64 bits on the GPU; results in aligned rows, in rows at odd places, and with what lies beside them left as it was."""
    q, g = gpu_lib, torch.Generator(DEV).manual_seed(M + N + K)
    width = (K + 15) // 16 * 16
    a = torch.randint(-127, 128, (M, width), dtype=torch.int8, device=DEV, generator=g)
    w = torch.randint(-127, 128, (N, K), dtype=torch.int8, device=DEV, generator=g)
    sa, sw = (torch.exp(torch.randn(n, device=DEV, generator=g)) / 100 for n in (M, N))
    bias = torch.randn(N, device=DEV, generator=g)
    p = torch.matmul(a[:, :K].double(), w.double().t().contiguous()) * sa.double()[:, None] * sw.double()[None, :]
    m = q.pack_int8(w, q.LAYOUT_TILED, sw)
    for dtype, pad_to, with_bias in ((torch.float32, 8, True), (torch.bfloat16, 8, False), (torch.float16, 1, True), (torch.bfloat16, 1, True)):
        pitch = (N + 1 + 7) // 8 * 8 if pad_to == 8 else (N + 1) | 1
        base = torch.full((M + 1, pitch), 3.0, dtype=dtype, device=DEV)
        out = base[:M, :N]
        q.linear_tokens(m, a, sa, bias=bias if with_bias else None, out=out)
        y = p + bias.double() if with_bias else p
        off = (out.double() - y).abs() - (2.01 * 2.0 ** -24 * p.abs() + (2.0 ** -24 + plain64.HALF_STEP[dtype]) * y.abs() * (1 + 2.0 ** -8) + 2.0 ** -25)
        assert off.max().item() <= 0, (dtype, divmod(off.argmax().item(), N))
        assert bool((base[M] == 3).all()) and bool((base[:, N:] == 3).all())
