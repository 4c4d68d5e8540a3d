"""Scores of given tokens from logits, against 64 bits: tokens are exact, log probabilities and entropies within what is derived in
plain_mx4.scores_tolerance (and their own rounding to fp32)."""
import numpy as np
import pytest
import torch

from tests import plain_mx4 as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def close(got, want, tolerance):
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    with np.errstate(invalid="ignore"):
        near = (got == want) | (np.abs(got - want) <= tolerance + np.abs(want) * 2.0 ** -24)
    assert (near | np.isnan(want)).all()


def check(q, x, token, n, **more):
    rows, V = x.shape
    logp, entropy, tokens, values = q.token_scores(x, token, n_top=n, **more)
    want = plain.scores(x.double().cpu().numpy(), None if token is None else token.cpu().numpy(), n)
    lse, ent = plain.scores_tolerance(V)
    if token is None:
        assert logp is None
    else:
        close(logp, want[0], lse)
    close(entropy, want[1], ent)
    if n == 0:
        assert tokens is None and values is None
        return
    assert np.array_equal(tokens.cpu().numpy(), want[2])
    close(values, want[3], lse)


def logits(seed, rows, V, dtype, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    return (spread * torch.randn((rows, V), generator=g)).to(dtype).to(DEV)


def some_tokens(seed, rows, V):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, V, (rows,), generator=g, dtype=torch.int32).to(DEV)


# a wave, four and sixteen waves to a row, rows in parts; lengths around vectors, groups, chunks and parts
SIZES = [(1, 1), (3, 2), (5, 7), (2, 46), (9, 64), (4, 65), (7, 1023), (3, 1025), (6, 2048), (5, 2049), (2, 4097), (3, 8192), (2, 8193), (4, 16385), (1, 32000), (3, 32777),
         (1, 131075), (2, 262144), (300, 9001), (1025, 2500), (4100, 3000), (257, 17000)]


@pytest.mark.parametrize("rows,V", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_scores(gpu_lib, rows, V, dtype):
    x = logits(rows + V, rows, V, dtype)
    if V > 40:
        x[:, 5] = float("-inf")
    t = some_tokens(V, rows, V)
    for n in (0, 1, 5, 20, 64):
        check(gpu_lib, x, t, n)


@pytest.mark.parametrize("rows,V", [(3, 100), (2, 3000), (3, 9000), (2, 20000), (1, 70000), (1100, 2500), (4100, 2500)])
def test_equal_logits_go_by_the_lowest_token(gpu_lib, rows, V):
    g = torch.Generator().manual_seed(V)
    for values in ([0.5], [1.0, 2.0], list(range(8))):
        x = torch.tensor(values)[torch.randint(0, len(values), (rows, V), generator=g)].to(torch.bfloat16).to(DEV)
        for n in (1, 16, 64):
            check(gpu_lib, x, some_tokens(1, rows, V), n)
    x = torch.zeros((rows, V), device=DEV)
    x[:, ::2] = -0.0   # equal to 0
    check(gpu_lib, x, None, 40)


@pytest.mark.parametrize("rows,V", [(2, 6000), (3, 40000), (1, 140000), (4100, 2600)])
@pytest.mark.parametrize("dtype", TYPES)
def test_rising_and_falling_rows(gpu_lib, rows, V, dtype):
    """Rising rows raise the bound and move the sums with every piece that is read."""
    ramp = torch.linspace(-40.0, 40.0, V)
    for r in (ramp, ramp.flip(0), 0.01 * ramp, 0.01 * ramp.flip(0)):
        x = r.expand(rows, V).to(dtype).to(DEV)
        check(gpu_lib, x.contiguous(), some_tokens(3, rows, V), 64)
        check(gpu_lib, x.contiguous(), some_tokens(3, rows, V), 3)


@pytest.mark.parametrize("rows,V", [(3, 9001), (2, 24500), (3, 48999), (70, 140001)])
@pytest.mark.parametrize("dtype", TYPES)
def test_many_large_logits_among_small_ones(gpu_lib, rows, V, dtype):
    """As many as fill the lists of candidates by half, nearly, and over; different or equal, in what is read first or later."""
    base = logits(V, rows, V, dtype, 0.1)
    for many in (250, 300, 513, 700, 1000) if rows < 70 else (300, 700):
        for start in (0, 17000, V - 16 * many) if rows < 70 else (40000,):
            if start < 0 or start + 16 * many > V:
                continue
            x = base.clone()
            at = start + 16 * torch.arange(many, device=DEV)
            x[:, at] = 5.0 + torch.arange(many, device=DEV).to(dtype) / 64
            x[0, at] = 5.0
            for n in (64, 5) if rows < 70 else (64,):
                check(gpu_lib, x, None, n)


@pytest.mark.parametrize("V", [50, 2500, 9001, 33000, 100000])
@pytest.mark.parametrize("dtype", TYPES)
def test_masks(gpu_lib, V, dtype):
    x = logits(V, 12, V, dtype)
    lowest = torch.finfo(dtype).min
    x[0] = float("-inf")
    x[1, 1:] = float("-inf")
    x[2, :-1] = float("-inf")
    x[3, 3] = float("nan")
    x[4, V - 1] = float("inf")
    x[5] = lowest
    x[6, 2:] = lowest
    x[7] = float("-inf")
    x[7, 7] = lowest
    x[8, :] = float("nan")
    x[9, ::2] = float("-inf")
    x[10] = torch.finfo(dtype).max
    x[11, 4:] = float("-inf")
    t = torch.tensor([3, 0, V - 1, 3, 0, 7, 1, 7, 2, 2, V - 1, 4], dtype=torch.int32, device=DEV)
    for n in (0, 6, 64):
        check(gpu_lib, x, t, n)
        check(gpu_lib, x[:1], t[:1], n)
        check(gpu_lib, x[3:4], t[3:4], n)


def test_tokens_that_are_padding_or_do_not_exist(gpu_lib):
    x = logits(1, 8, 500, torch.float32)
    x[6], x[7] = float("nan"), float("-inf")
    t = torch.tensor([-1, 0, 499, 500, -(1 << 31), (1 << 31) - 1, -1, -5], dtype=torch.int32, device=DEV)
    check(gpu_lib, x, t, 3)
    logp = gpu_lib.token_scores(x, t)[0].cpu()
    assert logp[0] == 0 and logp[4] == 0 and logp[6] == 0 and logp[7] == 0 and bool(logp[3].isnan()) and bool(logp[5].isnan())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,V,lead,pitch", [(6, 1000, 1, 1003), (3, 9001, 3, 9007), (2, 40001, 5, 40010), (1100, 2101, 1, 2103), (4100, 77, 7, 99)])
def test_rows_at_odd_places(gpu_lib, dtype, rows, V, lead, pitch):
    store = logits(2, 1, lead + rows * pitch + 8, dtype)[0]
    x = store[lead:lead + rows * pitch].view(rows, pitch)[:, :V]
    check(gpu_lib, x, some_tokens(2, rows, V), 17)
    same = gpu_lib.token_scores(x.contiguous(), some_tokens(2, rows, V), n_top=17)
    for a, b in zip(gpu_lib.token_scores(x, some_tokens(2, rows, V), n_top=17), same):
        assert torch.equal(a, b)   # where a row begins in memory changes nothing


def test_only_what_is_asked_for(gpu_lib):
    x = logits(4, 5, 700, torch.float16)
    t = some_tokens(4, 5, 700)
    full = gpu_lib.token_scores(x, t, n_top=4)
    logp, entropy, tokens, values = gpu_lib.token_scores(x, None, n_top=4, entropy=False)
    assert logp is None and entropy is None and torch.equal(tokens, full[2]) and torch.equal(values, full[3])
    assert torch.equal(gpu_lib.token_scores(x, t, entropy=False)[0], full[0])
    logp, entropy, tokens, values = gpu_lib.token_scores(torch.empty((0, 30), device=DEV), torch.empty(0, dtype=torch.int32, device=DEV), n_top=3)
    assert logp.shape == (0,) and entropy.shape == (0,) and tokens.shape == (0, 3) and values.shape == (0, 3)


def test_a_workspace_for_the_largest_call_serves_the_others(gpu_lib):
    q = gpu_lib
    ws = torch.empty(q.token_scores_workspace(300, 100000, 64), dtype=torch.uint8, device=DEV)
    for rows, V, n in ((300, 5000, 3), (1, 100000, 64), (200, 40000, 10), (15, 99999, 64)):
        check(q, logits(rows, rows, V, torch.bfloat16), some_tokens(rows, rows, V), n, workspace=ws)
