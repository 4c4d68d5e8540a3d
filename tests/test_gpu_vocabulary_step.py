"""The operators together, as a search over a large vocabulary uses them: norm and quantizer, output layer, selection, states
in the order of the new hypotheses; several steps, on another stream, and captured and replayed."""
import numpy as np
import pytest
import torch

from . import plain64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, W, H, V, END = 3, 4, 96, 5003, 2


class Search:
    """One step: x[token] + state -> norm -> 8-bit layer -> selection; the sum is the new state."""

    def __init__(self, q, seed):
        g = torch.Generator().manual_seed(seed)
        self.q, N = q, B * W
        self.embed = torch.randn((V, H), generator=g).to(DEV)
        self.norm = (1 + 0.1 * torch.randn(H, generator=g)).to(DEV)
        self.mat = q.pack_int8((torch.randn((V, H), generator=g)).to(DEV), q.LAYOUT_TILED)
        self.bias = (0.5 * torch.randn(V, generator=g)).to(DEV)
        self.state = torch.randn((N, H), generator=g).to(DEV)
        self.history = torch.zeros((N, 8), dtype=torch.int32, device=DEV)
        self.token = torch.randint(0, V, (B, W), generator=g).to(torch.int32).to(DEV)
        self.score = torch.zeros((B, W), device=DEV)
        self.score[:, 1:] = float("-inf")
        self.done = torch.zeros((B, W), dtype=torch.bool, device=DEV)
        self.sum = torch.empty_like(self.state)
        self.group = q.StateGroup([(self.sum, self.state), self.history], B, W)

    def step(self, t):
        q = self.q
        x = self.embed[self.token.reshape(-1).clamp(min=0).long()]
        codes, scale, total = q.rms_norm_quant(x, self.norm, 1e-5, residual=self.state, sum_out=self.sum)
        logits = q.linear_tokens(self.mat, codes, scale, bias=self.bias, dtype=torch.bfloat16)
        parent, token, score, done = q.beam_select(self.score, logits, finished=self.done, end_token=END)
        self.group.reorder(parent)
        self.history[:, t] = token.reshape(-1)
        self.token.copy_(token), self.score.copy_(score), self.done.copy_(done)
        return codes, scale, total, logits, parent, token, score, done


def test_steps_against_64_bits(gpu_lib):
    s = Search(gpu_lib, 1)
    w = gpu_lib.unpack_int4(s.mat).cpu().numpy()
    sw = s.mat.row_scale.cpu().numpy()
    history = torch.zeros((B * W, 8), dtype=torch.int32)
    for t in range(5):
        x = s.embed[s.token.reshape(-1).clamp(min=0).long()].cpu()
        state, score0, done0 = s.state.cpu(), s.score.cpu().numpy(), s.done.cpu().numpy()
        codes, scale, total, logits, parent, token, score, done = [o.cpu() for o in s.step(t)]
        want = plain64.rms_norm_quant(x, s.norm.cpu(), 1e-5, state)
        np.testing.assert_array_equal(codes.numpy()[:, :H], want[0])
        assert torch.equal(total, want[2])
        y, p = plain64.linear(want[0], scale.numpy(), w, sw, s.bias.cpu().numpy())
        assert (np.abs(logits.double().numpy() - y) <= 2.01 * 2.0 ** -24 * p + (2.0 ** -24 + 2.0 ** -8) * np.abs(y) * (1 + 2.0 ** -8)).all()
        v = plain64.candidates(score0, logits.float().numpy(), True, done0, END)
        pw, tw, vw = plain64.select(v, W)
        picked = np.array([[v[b, parent[b, j], token[b, j]] for j in range(W)] for b in range(B)])
        assert np.abs(picked - vw).max() < 1e-5 and np.abs(score.numpy() - vw).max() < 1e-4
        rows = (parent.long() + W * torch.arange(B)[:, None]).reshape(-1)
        assert torch.equal(s.state.cpu(), total[rows])
        history = history[rows]
        history[:, t] = token.reshape(-1)
        assert torch.equal(s.history.cpu(), history)


def snapshot(s):
    return [t.clone() for t in (s.state, s.history, s.token, s.score, s.done)]


def restore(s, snap):
    for t, v in zip((s.state, s.history, s.token, s.score, s.done), snap):
        t.copy_(v)


def test_another_stream_gives_the_same(gpu_lib):
    a, b = Search(gpu_lib, 2), Search(gpu_lib, 2)
    for t in range(4):
        a.step(t)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        for t in range(4):
            b.step(t)
    torch.cuda.current_stream().wait_stream(other)
    for x, y in zip(snapshot(a), snapshot(b)):
        assert torch.equal(x, y)


def test_captured_and_replayed(gpu_lib):
    """Every replay against the eager step from the same state, with eager work and synchronizations in between."""
    s = Search(gpu_lib, 3)
    start = snapshot(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.step(0)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    restore(s, start)
    with torch.cuda.graph(graph):
        out = s.step(0)
    restore(s, start)
    for _ in range(5):
        before = snapshot(s)
        graph.replay()
        torch.cuda.synchronize()
        after, got = snapshot(s), [o.clone() for o in out]
        restore(s, before)
        want = s.step(0)
        for x, y in zip(list(want) + snapshot(s), got + after):
            assert torch.equal(x, y)
        torch.cuda.synchronize()


def test_two_graphs_one_after_the_other_may_share_workspaces(gpu_lib):
    q = gpu_lib
    g = torch.Generator().manual_seed(4)
    K, N = 4096, 64
    m = q.pack_int8(torch.randn((N, K), generator=g).to(DEV), q.LAYOUT_TILED)
    xs = [torch.randn((r, K), generator=g).to(DEV) for r in (24, 40)]
    pairs = [q.quantize_tokens(x) for x in xs]
    want = [q.linear_tokens(m, c, s) for c, s in pairs]
    logits = [torch.randn((8, 9000), generator=g).to(DEV) for _ in range(2)]
    score = torch.zeros((2, 4), device=DEV)
    picks = [q.beam_select(score, l) for l in logits]
    ws = torch.empty(max(q.linear_tokens_workspace(m, 24), q.linear_tokens_workspace(m, 40), q.beam_select_workspace(2, 4, 9000, 4), 256),
                     dtype=torch.uint8, device=DEV)
    graphs, outs = [], []
    for (c, s), l in zip(pairs, logits):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append((q.linear_tokens(m, c, s, workspace=ws), q.beam_select(score, l, workspace=ws)))
        graphs.append(graph)
    for _ in range(3):
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for (y, p), w, pw in zip(outs, want, picks):
            assert torch.equal(y, w) and all(torch.equal(a, b) for a, b in zip(p[:3], pw[:3]))
        ws.fill_(255)
