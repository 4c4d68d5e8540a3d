"""The operators together, as the rescoring of N-best lists by a language model's output layer uses them: hidden states to 4-bit floats,
output layer, scores of the tokens that the hypotheses hold (padded to one length); on other streams, two at a time, captured and
replayed."""
import numpy as np
import pytest
import torch

from tests import plain_mx4 as plain
from tests.plain64 import HALF_STEP

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Rescorer:
    """A list of hypotheses of at most `length` tokens; the sums of their tokens' log probabilities order them."""

    def __init__(self, q, seed, lists, length, H, V, n_top=4, dtype=torch.bfloat16):
        g = torch.Generator().manual_seed(seed)
        self.q, self.n, self.dtype, self.shape = q, n_top, dtype, (lists, length)
        rows = lists * length
        w = (torch.randn((V, H), generator=g) * torch.exp(torch.randn((V, 1), generator=g)) / H ** 0.5).to(DEV)
        self.w_codes, self.w_scale = q.quantize_mx4(w)
        self.mat = q.pack_mx4(self.w_codes, self.w_scale, H)
        self.bias = (0.5 * torch.randn(V, generator=g)).to(DEV)
        self.ws = torch.empty(q.linear_mx4_workspace(self.mat, rows), dtype=torch.uint8, device=DEV)
        self.ws_scores = torch.empty(q.token_scores_workspace(rows, V, n_top), dtype=torch.uint8, device=DEV)
        self.state = torch.empty((rows, H), dtype=torch.bfloat16, device=DEV)
        self.token = torch.empty(rows, dtype=torch.int32, device=DEV)
        self.fill(seed)

    def fill(self, seed):
        """Other hypotheses, in place."""
        g = torch.Generator().manual_seed(1000 + seed)
        rows, (lists, length) = self.token.shape[0], self.shape
        self.state.copy_(torch.randn(self.state.shape, generator=g))
        token = torch.randint(0, self.mat.rows, (lists, length), generator=g, dtype=torch.int32)
        lengths = torch.randint(0, length + 1, (lists, 1), generator=g)   # some are empty
        token[torch.arange(length)[None, :] >= lengths] = -1
        self.token.copy_(token.view(rows))

    def run(self):
        q = self.q
        codes, scale = q.quantize_mx4(self.state)
        logits = q.linear_mx4(self.mat, codes, scale, bias=self.bias, dtype=self.dtype, workspace=self.ws)
        logp, entropy, tokens, values = q.token_scores(logits, self.token, n_top=self.n, workspace=self.ws_scores)
        return codes, scale, logits, logp, entropy, tokens, values, logp.view(self.shape).sum(1)


# one position (few tokens), a cut sum, small tiles, several ways of scoring
CASES = [(1, 1, 96, 1000), (3, 5, 200, 5003), (6, 14, 4100, 260), (10, 13, 640, 33000), (40, 30, 72, 2500)]


@pytest.mark.parametrize("lists,length,H,V", CASES)
def test_against_64_bits(gpu_lib, lists, length, H, V):
    r = Rescorer(gpu_lib, 1, lists, length, H, V)
    codes, scale, logits, logp, entropy, tokens, values, total = [o.cpu() for o in r.run()]
    want, want_scale = plain.quantize(r.state.double().cpu().numpy())
    assert np.array_equal(codes.numpy(), plain.join(want)) and np.array_equal(scale.numpy()[:, :want_scale.shape[1]], want_scale)
    w = plain.values(plain.split(r.w_codes.cpu().numpy()), r.w_scale.cpu().numpy()[:, :want_scale.shape[1]])
    a = plain.values(want, want_scale)
    y = a @ w.T + r.bias.double().cpu().numpy()
    bound = plain.sum_tolerance(H, np.abs(a) @ np.abs(w).T) + 2.0 ** -24 * np.abs(y)   # (the bias)
    assert (np.abs(logits.double().numpy() - y) <= bound + (np.abs(y) + bound) * HALF_STEP[r.dtype]).all()
    lp, ent, tok, val = plain.scores(logits.double().numpy(), r.token.cpu().numpy(), r.n)
    lse, bound = plain.scores_tolerance(V)
    assert (np.abs(logp.numpy() - lp) <= lse + np.abs(lp) * 2.0 ** -24).all()
    assert (np.abs(entropy.numpy() - ent) <= bound + ent * 2.0 ** -24).all()
    assert np.array_equal(tokens.numpy(), tok) and (np.abs(values.numpy() - val) <= lse + np.abs(val) * 2.0 ** -24).all()
    # a hypothesis' sum in fp32: padding adds nothing
    each = np.abs(lp).reshape(lists, length).sum(1)
    assert (np.abs(total.numpy() - lp.reshape(lists, length).sum(1)) <= length * (lse + each * 2.0 ** -23)).all()
    assert (total.numpy()[(r.token.cpu().view(lists, length) < 0).all(1).numpy()] == 0).all()


@pytest.mark.parametrize("lists,length,H,V", CASES)
def test_captured_and_replayed(gpu_lib, lists, length, H, V):
    r = Rescorer(gpu_lib, 2, lists, length, H, V)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        r.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = r.run()
    for seed in (3, 4, 5, 6):
        r.fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in out]
        for a, b in zip(got, r.run()):   # eager work between the replays, on the same workspaces
            assert torch.equal(a, b)


def test_two_graphs_that_share_workspaces(gpu_lib):
    """Their calls come one after the other."""
    r = Rescorer(gpu_lib, 3, 6, 14, 4100, 40000)
    big, small = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    r.run()
    torch.cuda.synchronize()
    with torch.cuda.graph(big):
        out = r.run()
    few = 20
    with torch.cuda.graph(small):
        codes, scale = r.q.quantize_mx4(r.state[:few])
        logits = r.q.linear_mx4(r.mat, codes, scale, bias=r.bias, workspace=r.ws)
        part = r.q.token_scores(logits, r.token[:few], n_top=r.n, workspace=r.ws_scores)
    for seed in (7, 8, 9):
        r.fill(seed)
        big.replay(), small.replay(), big.replay()
        torch.cuda.synchronize()
        got, got_part = [o.clone() for o in out], [o.clone() for o in part]
        for a, b in zip(got, r.run()):
            assert torch.equal(a, b)
        c, s = r.q.quantize_mx4(r.state[:few])
        for a, b in zip(got_part, r.q.token_scores(r.q.linear_mx4(r.mat, c, s, bias=r.bias), r.token[:few], n_top=r.n)):
            assert torch.equal(a, b)


def test_two_streams_at_a_time(gpu_lib):
    first, second = Rescorer(gpu_lib, 4, 10, 13, 640, 33000), Rescorer(gpu_lib, 5, 6, 14, 4100, 5003)
    want = [[o.clone() for o in r.run()] for r in (first, second)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(5):
        for i, r in enumerate((first, second)):
            with torch.cuda.stream(streams[i]):
                got[i].append(r.run())
    torch.cuda.synchronize()
    for i in range(2):
        for run in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(run, want[i]))


def test_equal_rows_score_alike_wherever_they_stand(gpu_lib):
    """Rows of one call whose logits are equal have equal scores, to the last bit."""
    q = gpu_lib
    for V in (300, 2500, 9001, 33000, 140000):
        x = torch.randn((1, V), generator=torch.Generator().manual_seed(V)).bfloat16().to(DEV).expand(37, V).contiguous()
        for out in q.token_scores(x, torch.full((37,), 5, dtype=torch.int32, device=DEV), n_top=7):
            assert bool((out == out[:1]).all())
