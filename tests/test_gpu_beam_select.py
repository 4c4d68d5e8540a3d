"""Selection over beams and vocabulary from logits, against 64 bits.  Where values are sums of small whole numbers (no
log-softmax) every comparison is exact, ties included; with log-softmax picks have to be the reference's wherever its values
lie further apart than the roundings counted in `tolerance`."""
import numpy as np
import pytest
import torch

from . import plain64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def tolerance(V, v):
    """A row's sum of exponentials: 32 fp32 additions in a thread; each term exp2(d log2 e) with two roundings of its argument
    and one step of exp2, which weigh d exp(-d) on average at most log V.  The result is rounded to fp32."""
    return (16 + np.log(V) + 2) * 2.0 ** -23 + np.where(np.isfinite(v), np.abs(v), 0.0) * 2.0 ** -24


def grid_case(seed, B, W, V, dtype, spread=6):
    """Logits and scores on a coarse grid: many ties, all sums exact in every type."""
    r = np.random.RandomState(seed)
    logits = r.randint(-spread, spread + 1, (B * W, V)).astype(np.float32) / 4
    logits[r.rand(B * W, V) < 0.2] = -np.inf
    score = (-r.randint(0, 9, (B, W)) / 4).astype(np.float32)
    return torch.from_numpy(score), torch.from_numpy(logits).to(dtype)


def run(q, score, logits, n, **kw):
    on = {k: (v.to(DEV) if torch.is_tensor(v) else v) for k, v in kw.items()}
    par, tok, val, done = q.beam_select(score.to(DEV), logits.to(DEV), n, **on)
    return par.cpu().numpy(), tok.cpu().numpy(), val.cpu().numpy(), None if done is None else done.cpu().numpy()


def check_exact(got, v, n):
    parent, token, value = plain64.select(v, n)
    np.testing.assert_array_equal(got[0], parent)
    np.testing.assert_array_equal(got[1], token)
    np.testing.assert_array_equal(got[2], value.astype(np.float32))


def check_near(got, v, n):
    B, W, V = v.shape
    parent, token, value = plain64.select(v, n)
    tol = tolerance(V, value)
    np.testing.assert_array_equal(np.isfinite(got[2]), np.isfinite(value))
    fine = np.isfinite(value)
    assert (np.abs(got[2].astype(np.float64)[fine] - value[fine]) <= tol[fine]).all()
    more = plain64.select(v, n + 1)[2]   # with the first value that is left out
    for b in range(B):
        assert len({(p, t) for p, t in zip(got[0][b], got[1][b]) if p >= 0}) == (got[0][b] >= 0).sum()
        for j in range(n):
            if not fine[b, j]:
                assert got[0][b, j] == -1 and got[1][b, j] == -1
                continue
            assert abs(v[b, got[0][b, j], got[1][b, j]] - value[b, j]) <= 2 * tol[b, j]
            alone = (j == 0 or value[b, j - 1] - value[b, j] > 2 * tol[b, j]) and value[b, j] - more[b, j + 1] > 2 * tol[b, j]
            if alone:
                assert got[0][b, j] == parent[b, j] and got[1][b, j] == token[b, j]


SIZES = [(1, 1, 1, 1), (1, 1, 1, 5), (2, 1, 3, 2), (1, 2, 46, 2), (3, 4, 46, 8), (2, 16, 46, 16), (1, 4, 1000, 4), (5, 3, 1031, 6), (2, 5, 2048, 5),
         (2, 8, 2049, 16), (1, 16, 4096, 32), (3, 2, 8193, 64), (1, 64, 300, 64), (2, 33, 77, 40), (1, 16, 32000, 16), (40, 8, 9000, 8),
         (1, 2, 131072, 4), (1, 1, 262145, 64)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,W,V,n", SIZES)
def test_sums_of_whole_numbers_ties_included(gpu_lib, dtype, B, W, V, n):
    score, logits = grid_case(B + W + V + n, B, W, V, dtype)
    v = plain64.candidates(score.numpy(), logits.float().numpy(), False)
    check_exact(run(gpu_lib, score, logits, n, log_softmax=False), v, n)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,W,V,n", SIZES)
def test_log_softmax(gpu_lib, dtype, B, W, V, n):
    g = torch.Generator().manual_seed(B + 2 * W + 3 * V + n)
    logits = (3 * torch.randn((B * W, V), generator=g)).to(dtype)
    logits[torch.rand((B * W, V), generator=g) < 0.1] = -INF
    score = torch.sort(-6 * torch.rand((B, W), generator=g), dim=1, descending=True).values
    v = plain64.candidates(score.numpy(), logits.float().numpy(), True)
    check_near(run(gpu_lib, score, logits, n), v, n)


@pytest.mark.parametrize("V", [50, 3000, 20000])
def test_all_logits_equal(gpu_lib, V):
    """Every candidate ties: the lowest hypotheses and tokens win, whatever the list in between holds."""
    B, W, n = 2, 6, 40
    score = torch.tensor([[-1.0, -1.0, -2.0, -1.0, -3.0, -1.0]] * B)
    for value in (0.0, -3.5, 1e-40):
        logits = torch.full((B * W, V), value)
        for soft in (False, True):
            got = run(gpu_lib, score, logits, n, log_softmax=soft)
            order = [(w, k) for s in (-1.0, -2.0, -3.0) for w in range(W) if score[0, w] == s for k in range(V)][:n]
            assert [(p, t) for p, t in zip(got[0][1], got[1][1])] == order


@pytest.mark.parametrize("V", [60, 2500])
def test_equal_hypotheses_in_rows_that_start_at_different_bytes(gpu_lib, V):
    """Identical rows at odd places: their sums have to come out the same, or a tie would be broken by rounding."""
    W, n = 8, 24
    row = torch.randn(V, generator=torch.Generator().manual_seed(V)) * 3
    for dtype in TYPES:
        big = torch.empty((W, V + 3), dtype=dtype, device=DEV)
        big[:, 1:V + 1] = row.to(dtype).to(DEV)
        par, tok, val, _ = gpu_lib.beam_select(torch.zeros((1, W), device=DEV), big[:, 1:V + 1], n)
        first = tok[0, ::8].cpu().tolist()
        assert par[0].cpu().tolist() == list(range(W)) * 3
        assert tok[0].cpu().tolist() == [t for t in first for _ in range(W)] and len(set(first)) == 3


@pytest.mark.parametrize("V", [40, 5000])
def test_rows_without_candidates(gpu_lib, V):
    """Dead hypotheses, masks that leave nothing or one token, NaN and +inf logits, masks of the type's lowest value."""
    W, n = 9, 12
    for dtype in TYPES:
        low = torch.finfo(dtype).min
        logits = torch.full((W, V), -INF, dtype=dtype)
        score = torch.tensor([[-1.0, -INF, -2.0, -3.0, -4.0, float("nan"), -5.0, -0.5, -7.0]])
        logits[1] = 1.0                      # score -inf
        logits[2, V - 1] = 2.0               # one token
        logits[3] = 0.0
        logits[3, 7] = float("nan")
        logits[4] = 0.0
        logits[4, V - 2] = INF
        logits[5] = 1.0                      # score NaN
        logits[6] = low                      # masked by the lowest value throughout: all alike
        logits[7] = low
        logits[7, 5] = 3.0
        got = run(gpu_lib, score, logits, n)
        assert (got[0][0, 0], got[1][0, 0], got[2][0, 0]) == (7, 5, -0.5)
        assert (got[0][0, 1], got[1][0, 1], got[2][0, 1]) == (2, V - 1, -2.0)
        assert got[0][0, 2:12].tolist() == [6] * 10 and got[1][0, 2:12].tolist() == list(range(10))
        assert np.abs(got[2][0, 2:12] - (-5.0 - np.log(V))).max() <= tolerance(V, np.float64(12.0))
        # nothing anywhere
        got = run(gpu_lib, score[:, :1], logits[:1], 4, end_token=3)
        assert (got[0] == -1).all() and (got[1] == -1).all() and (got[2] == -np.inf).all() and not got[3].any()
        # without log-softmax NaN is passed over and +inf is the best
        got = run(gpu_lib, score[:, 3:5], logits[3:5], 3, log_softmax=False)
        assert got[0][0].tolist() == [1, 0, 0] and got[1][0].tolist() == [V - 2, 0, 1] and got[2][0, 0] == INF


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,W,V,n", [(3, 5, 70, 5), (2, 16, 3000, 20), (1, 64, 65, 64)])
def test_finished_hypotheses(gpu_lib, dtype, B, W, V, n):
    r = np.random.RandomState(V)
    score, logits = grid_case(V, B, W, V, dtype)
    finished = torch.from_numpy(r.rand(B, W) < 0.4)
    logits[finished.reshape(-1)] = float("nan")   # what they hold is not read
    end = V - 3
    v = plain64.candidates(score.numpy(), logits.float().numpy(), False, finished.numpy(), end)
    for kind in (finished, finished.to(torch.uint8) * 3):
        got = run(gpu_lib, score, logits, n, log_softmax=False, finished=kind, end_token=end)
        check_exact(got, v, n)
        parent = got[0]
        was = np.take_along_axis(finished.numpy(), np.maximum(parent, 0), axis=1)
        np.testing.assert_array_equal(got[3], (parent >= 0) & (was | (got[1] == end)))
    everyone = torch.ones((B, W), dtype=torch.bool)
    got = run(gpu_lib, score, logits, n, finished=everyone, end_token=end)
    check_exact(got, plain64.candidates(score.numpy(), logits.float().numpy(), True, everyone.numpy(), end), n)


def test_many_utterances(gpu_lib):
    """More rows than a grid's y extent."""
    B, W, V, n = 33000, 2, 33, 2
    score, logits = grid_case(8, B, W, V, torch.float32)
    check_exact(run(gpu_lib, score, logits, n, log_softmax=False), plain64.candidates(score.numpy(), logits.numpy(), False), n)


def test_no_utterances_and_what_the_workspace_held(gpu_lib):
    q = gpu_lib
    par, tok, val, done = q.beam_select(torch.empty((0, 4), device=DEV), torch.empty((0, 50), device=DEV), 3, end_token=1)
    assert par.shape == tok.shape == val.shape == done.shape == (0, 3)
    for B, W, V, n in ((2, 4, 300, 6), (2, 4, 9001, 6)):
        score, logits = grid_case(1, B, W, V, torch.float32)
        need = q.beam_select_workspace(B, W, V, n)
        v = plain64.candidates(score.numpy(), logits.numpy(), False)
        for fill in (0, 255, 64):
            ws = torch.full((need + 256,), fill, dtype=torch.uint8, device=DEV)
            check_exact(run(q, score, logits, n, log_softmax=False, workspace=ws), v, n)
            # (run() moves the workspace to the device it is on already)
            assert bool((ws[need:] == fill).all())


# Wide beams on both sides of the choice between one launch and two, lists that fit the second one's registers and that do not.
WIDE = [(1, 64, 2000, 64), (16, 32, 600, 32), (33, 32, 600, 32), (3, 25, 513, 25), (41, 25, 1025, 7), (1, 64, 20000, 64), (2, 64, 3000, 64), (1, 25, 2048, 64),
        (1, 3, 50001, 64), (2, 17, 16385, 33)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,W,V,n", WIDE)
def test_wide_beams(gpu_lib, dtype, B, W, V, n):
    score, logits = grid_case(B + W + V + n, B, W, V, dtype, spread=40)
    finished = torch.from_numpy(np.random.RandomState(V).rand(B, W) < 0.2)
    v = plain64.candidates(score.numpy(), logits.float().numpy(), False, finished.numpy(), 3)
    check_exact(run(gpu_lib, score, logits, n, log_softmax=False, finished=finished, end_token=3), v, n)
    g = torch.Generator().manual_seed(B + 2 * W + 3 * V + n)
    logits = (3 * torch.randn((B * W, V), generator=g)).to(dtype)
    v = plain64.candidates(score.numpy(), logits.float().numpy(), True)
    check_near(run(gpu_lib, score, logits, n), v, n)
