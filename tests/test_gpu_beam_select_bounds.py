"""Selection where scores are so large next to the logits that many sums round to the same value, and the logit that belongs to
a value cannot be told from the value alone.  fp64 sums of two numbers are the same everywhere, so every comparison is exact."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# beams and vocabularies on both sides of the choices: rows in one launch (short ones, longer ones, rows read twice) and in two
SIZES = [(1, 1, 300, 4), (2, 3, 500, 7), (1, 20, 300, 40), (1, 4, 1000, 5), (2, 16, 2000, 16), (50, 25, 600, 9), (1, 4, 2500, 5), (1, 40, 600, 12), (2, 2, 20000, 30)]


def expected(v, logits, n):
    """v, logits [B, W, V] -> parent, token, value of the n best by value, hypothesis, logit, token."""
    B, W, V = v.shape
    w, k = np.divmod(np.arange(W * V), V)
    out = [np.lexsort((k, -logits[b].ravel(), w, -v[b].ravel()))[:n] for b in range(B)]
    return np.stack([w[o] for o in out]), np.stack([k[o] for o in out]), np.stack([v[b].ravel()[o] for b, o in enumerate(out)])


def check(q, score, logits, n, soft):
    B, W = score.shape
    x = logits.double().numpy().reshape(B, W, -1)
    if soft:   # (logits for which the logarithm vanishes next to its one term that does not)
        top = x.max(axis=2, keepdims=True)
        log_sum = np.log(np.exp(x - top).sum(axis=2, keepdims=True))
        assert not log_sum.any()
        v = score.double().numpy()[:, :, None] + (x - top)
    else:
        v = score.double().numpy()[:, :, None] + x
    par, tok, val, _ = q.beam_select(score.to(DEV), logits.to(DEV), n, log_softmax=soft)
    want = expected(v, x, n)
    np.testing.assert_array_equal(par.cpu().numpy(), want[0])
    np.testing.assert_array_equal(tok.cpu().numpy(), want[1])
    np.testing.assert_array_equal(val.cpu().numpy(), want[2].astype(np.float32))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score,logit", [(1.0, -1e-20), (2.0, -1e-17), (4.0, -3e-17), (16.0, -8e-16), (1.0, 1e-20), (-1.0, -1e-20), (2.0 ** 100, -1.0)])
@pytest.mark.parametrize("B,W,V,n", SIZES)
def test_logits_that_vanish_beside_the_score(gpu_lib, dtype, score, logit, B, W, V, n):
    check(gpu_lib, torch.full((B, W), score), torch.full((B * W, V), logit).to(dtype), n, False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("score", [2.0 ** 40, 2.0 ** 40 + 2.0 ** 17, -2.0 ** 40, 3.0 * 2.0 ** 36])
@pytest.mark.parametrize("B,W,V,n", SIZES)
def test_values_that_round_to_the_same(gpu_lib, dtype, score, B, W, V, n):
    """Logits of either sign, most of them less than half a step of the values; negative ones only where ties go first."""
    r = np.random.RandomState(W + V)
    logits = r.uniform(-1.5, 0.5, (B, W, V)) * 2.0 ** -13
    logits[:, ::2] = -np.abs(logits[:, ::2])
    check(gpu_lib, torch.full((B, W), score), torch.from_numpy(logits.reshape(B * W, V)).to(dtype), n, False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score,top", [(200.0, 100.0), (128.0, 128.0), (2.0 ** 30, 120.0)])
@pytest.mark.parametrize("B,W,V,n", SIZES)
def test_normalised_values_that_round_to_the_same(gpu_lib, dtype, score, top, B, W, V, n):
    """One logit of `top`, beside which the exponentials of the others vanish, and tiny ones, negative where ties go first."""
    r = np.random.RandomState(W + V)
    logits = r.choice([-1e-20, -2e-20, 1e-20], (B, W, V))
    logits[:, ::2] = -np.abs(logits[:, ::2])
    logits = torch.from_numpy(logits.reshape(B * W, V)).to(dtype)
    logits[torch.arange(B * W), torch.from_numpy(r.randint(0, V, B * W))] = top
    check(gpu_lib, torch.full((B, W), score), logits, n + W, True)
