"""Operators of a search step over a large vocabulary and of 8-bit layers with a range for each token, for timing.

``listed()`` names representative cases, ``draw(rng)`` gives one more of the same ranges, ``prepare(case, seed)`` makes
what a program holds before the call, ``run(state)`` is one call, ``work(case)`` what it cannot do without and
``exact(case, seed)`` its outputs from the definition in 64 bits.  With ``own`` false ``run`` computes the operators from
elementary torch operations, with ``own`` true it calls the library.

Kinds
  norm      sum with the residual, root-mean-square norm, 8-bit codes with a scale for each token
  quantize  8-bit codes with a scale for each token
  linear    8-bit codes x 8-bit weights, a scale for each token and each weight row
  select    the best extensions over beams and vocabulary, from logits
  reorder   the networks' states of the hypotheses that were selected
"""
from __future__ import annotations

import torch

own = False

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "fp16": 2, "bf16": 2}
EPS = 1e-5
# widths of the LSTM layers whose states a hypothesis carries: the networks of the benchmark (prediction network 768, two
# language models of 2 x 1024) and of the paper (prediction network and source language model 768, external 2 x 2048)
STATES = {"base": (768, 1024, 1024, 1024, 1024), "paper": (768, 768, 2048, 2048)}
END = 1   # the token that ends a hypothesis


def listed():
    return [
        # one token of a model of width 4096 as it is generated: pure latency
        dict(name="norm_one_token", kind="norm", rows=1, cols=4096, dtype="bf16", residual=True),
        # a prompt batch of 16 k tokens in front of an 8-bit layer
        dict(name="norm_prompt", kind="norm", rows=16384, cols=4096, dtype="bf16", residual=True),
        # the prediction network's output for one beam of 16, in front of an 8-bit layer
        dict(name="quantize_beam", kind="quantize", rows=16, cols=768, dtype="fp32"),
        # the encoder's frames (32 utterances x 500 frames, both directions of 640) with a range for each frame
        dict(name="quantize_frames", kind="quantize", rows=16000, cols=1280, dtype="fp32"),
        # output layer of a language model of 1024 cells over 32 k words, for one beam of 16
        dict(name="linear_vocab_beam", kind="linear", M=16, N=32000, K=1024, dtype="fp32", bias=True),
        # an odd layer for an odd batch
        dict(name="linear_odd", kind="linear", M=77, N=1000, K=1283, dtype="bf16", bias=True),
        # the input projection of the encoder's frames (4 x 640 gate rows)
        dict(name="linear_frames", kind="linear", M=16000, N=2560, K=1280, dtype="fp32", bias=False),
        # a large layer over a prompt batch
        dict(name="linear_prompt", kind="linear", M=8192, N=8192, K=8192, dtype="bf16", bias=False),
        # one utterance, four hypotheses, a vocabulary of word pieces
        dict(name="select_one", kind="select", B=1, W=4, V=1000, K=4, dtype="fp32", finished=False),
        # the benchmark's batch (64 utterances, beam 16) over 32 k words, some hypotheses through
        dict(name="select_batch", kind="select", B=64, W=16, V=32000, K=16, dtype="bf16", finished=True),
        # states of one beam of 16, and of the benchmark's batch with the paper's networks
        dict(name="reorder_beam", kind="reorder", B=1, W=16, net="base"),
        dict(name="reorder_batch", kind="reorder", B=64, W=16, net="paper"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "quantize", "linear", "linear", "linear", "select", "select", "reorder"])
    dtype = rng.choice(["fp32", "fp16", "bf16", "bf16"])
    if kind in ("norm", "quantize"):
        cols = _log(rng, 33, 16384)
        if rng.random() < 0.5:
            cols = max(64, cols // 64 * 64)
        case = dict(kind=kind, rows=_log(rng, 1, min(16384, (1 << 25) // cols)), cols=cols, dtype=dtype)
        return dict(case, residual=rng.random() < 0.7) if kind == "norm" else case
    if kind == "linear":
        K, N = _log(rng, 40, 8192), _log(rng, 16, 32000)
        if rng.random() < 0.6:
            K, N = max(64, K // 64 * 64), max(64, N // 64 * 64)
        M = _log(rng, 1, max(1, min(16384, (1 << 38) // (K * N), (1 << 28) // N)))
        return dict(kind=kind, M=M, N=N, K=K, dtype=dtype, bias=rng.random() < 0.5)
    if kind == "select":
        W, V = rng.choice([1, 2, 4, 5, 8, 10, 16, 16, 32]), _log(rng, 46, 131072)
        B = _log(rng, 1, max(1, min(64, (1 << 24) // (W * V))))
        return dict(kind=kind, B=B, W=W, V=V, K=rng.choice([W, W, min(64, 2 * W)]), dtype=dtype, finished=rng.random() < 0.5)
    return dict(kind=kind, B=_log(rng, 1, 64), W=rng.choice([1, 2, 4, 5, 8, 10, 16, 16, 32]), net=rng.choice(["base", "paper"]))


def _pitch(cols):
    return (cols + 15) // 16 * 16


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    randn = lambda *shape: torch.randn(shape, generator=g, device=DEV)
    rand = lambda *shape: torch.rand(shape, generator=g, device=DEV)
    s = dict(case=dict(case))
    kind = case["kind"]
    if kind in ("norm", "quantize"):
        t, rows, cols = TYPES[case["dtype"]], case["rows"], case["cols"]
        # tokens of different size, a few channels far larger than the others
        x = randn(rows, cols) * torch.exp(randn(rows, 1)) * (1.0 + 20.0 * (rand(cols) < 0.01))
        s["x"] = x.to(t)
        if kind == "norm":
            s["weight"] = (1.0 + 0.2 * randn(cols)).to(t)
            if case["residual"]:
                s["residual"] = randn(rows, cols).to(t)
                s["sum"] = torch.empty_like(s["x"])
    elif kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        w = randn(N, K)
        peak = w.abs().amax(1, keepdim=True)
        s["w"] = torch.round(w * (127.0 / peak)).to(torch.int8)
        s["w_scale"] = (peak[:, 0] / 127.0 / K ** 0.5).contiguous()
        s["a"] = torch.zeros((M, _pitch(K)), dtype=torch.int8, device=DEV)
        s["a"][:, :K] = torch.round(30.0 * randn(M, K)).clamp(-127, 127).to(torch.int8)
        s["a_scale"] = torch.exp(0.5 * randn(M)) / 30.0
        s["bias"] = 0.1 * randn(N) if case["bias"] else None
    elif kind == "select":
        B, W, V, K = case["B"], case["W"], case["V"], case["K"]
        s["logits"] = (3.0 * randn(B * W, V)).to(TYPES[case["dtype"]])
        s["logits"][:, 0] = float("-inf")   # a token that is never to be said
        s["score"] = torch.sort(-6.0 * rand(B, W), dim=1, descending=True).values.contiguous()
        s["finished"] = (rand(B, W) < 0.2).to(torch.uint8) if case["finished"] else None
    else:
        B, W = case["B"], case["W"]
        N = B * W
        s["parent"] = torch.randint(0, W, (B, W), generator=g, device=DEV, dtype=torch.int32)
        s["src"], s["dst"] = [], []
        for h in STATES[case["net"]]:
            s["src"] += [torch.randint(-7, 8, (N, h), generator=g, device=DEV, dtype=torch.int8), randn(N, h)]
        s["dst"] = [torch.empty_like(x) for x in s["src"]]
    if own:   # packed weights, workspaces and the block of state addresses, as a program keeps them
        from paper_2206_07882_amd import qrnnt as q
        s["q"] = q
        if kind == "linear":
            s["mat"] = q.pack_int8(s["w"], q.LAYOUT_TILED, s["w_scale"])
            s["ws"] = torch.empty(q.linear_tokens_workspace(s["mat"], M), dtype=torch.uint8, device=DEV)
        elif kind == "select":
            s["ws"] = torch.empty(q.beam_select_workspace(B, W, V, K), dtype=torch.uint8, device=DEV)
        elif kind == "reorder":
            s["group"] = q.StateGroup(list(zip(s["src"], s["dst"])), B, W)
    return s


def _codes(u):
    """8-bit codes of the rows of u as numbers, and the largest magnitude of each row.  In 64 bits: whether a value lies
    above or below the border of two codes goes by the value."""
    u = u.double()
    peak = u.abs().amax(1, keepdim=True)
    return torch.where(peak == 0, u, torch.round((u * 127.0) / peak)), peak


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        h = s["x"].float()
        if case["residual"]:
            s["sum"].copy_(h + s["residual"].float())
            h = s["sum"].float()
        codes, peak = _codes(h.double() * s["weight"].double())
        r = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
        out = dict(values=(codes * torch.where(peak == 0, 1.0, peak * r / 127.0)).float())
        return dict(out, sum=s["sum"]) if case["residual"] else out
    if kind == "quantize":
        codes, peak = _codes(s["x"])
        return dict(values=(codes * torch.where(peak == 0, 1.0, peak / 127.0)).float())
    if kind == "linear":
        y = torch.matmul(s["a"][:, :case["K"]].float(), s["w"].float().t())
        y = y * s["a_scale"][:, None] * s["w_scale"][None, :]
        if s["bias"] is not None:
            y = y + s["bias"]
        return y.to(TYPES[case["dtype"]])
    if kind == "select":   # in 64 bits: what is next to a border goes by the values, not by how their sums were rounded
        B, W, V, K = case["B"], case["W"], case["V"], case["K"]
        x = s["logits"].double()
        top = x.amax(1, keepdim=True)
        x = x - (top + torch.log(torch.exp(x - top).sum(1, keepdim=True)))
        x = (x.view(B, W, V) + s["score"].double()[:, :, None])
        if s["finished"] is not None:
            held = torch.full((V,), float("-inf"), dtype=torch.float64, device=x.device)
            held[END] = 0.0
            x = torch.where(s["finished"].bool()[:, :, None], s["score"].double()[:, :, None] + held, x)
        x, at = torch.sort(x.view(B, W * V), dim=1, descending=True, stable=True)
        x, at = x[:, :K], at[:, :K]
        none = x == float("-inf")
        parent = torch.where(none, -1, at // V).to(torch.int32)
        return dict(parent=parent, token=torch.where(none, -1, at % V).to(torch.int32), score=x.float())
    B, W = case["B"], case["W"]
    rows = (s["parent"].long() + W * torch.arange(B, device=DEV)[:, None]).view(-1)
    return [torch.index_select(x, 0, rows, out=y) for x, y in zip(s["src"], s["dst"])]


def run(s):
    if not own:
        return _plain(s)
    q, case = s["q"], s["case"]
    kind = case["kind"]
    if kind == "norm":
        codes, scale, total = q.rms_norm_quant(s["x"], s["weight"], EPS, residual=s.get("residual"), sum_out=s.get("sum"))
        out = dict(values=codes[:, :case["cols"]] * scale[:, None])
        return dict(out, sum=total) if case["residual"] else out
    if kind == "quantize":
        codes, scale = q.quantize_tokens(s["x"])
        return dict(values=codes[:, :case["cols"]] * scale[:, None])
    if kind == "linear":
        return q.linear_tokens(s["mat"], s["a"], s["a_scale"], bias=s["bias"], dtype=TYPES[case["dtype"]], workspace=s["ws"])
    if kind == "select":
        parent, token, score, _ = q.beam_select(s["score"], s["logits"], case["K"], finished=s["finished"], end_token=END,
                                                workspace=s["ws"])
        return dict(parent=parent, token=token, score=score)
    s["group"].reorder(s["parent"])
    return s["dst"]


def work(case):
    """Each input read once, each output written once (codes as bytes); a multiply-accumulate counts as two operations."""
    kind = case["kind"]
    if kind in ("norm", "quantize"):
        e, n = SIZE[case["dtype"]], case["rows"] * case["cols"]
        moved = n * (e + 1) + 4 * case["rows"]
        if kind == "norm":
            moved += case["cols"] * e + (2 * n * e if case["residual"] else 0)
        return dict(bytes=float(moved), flops=float((6 if kind == "norm" else 3) * n))
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return dict(bytes=float(M * K + N * K + 4 * (M + N) + (4 * N if case["bias"] else 0) + M * N * SIZE[case["dtype"]]),
                    flops=2.0 * M * N * K)
    if kind == "select":
        n = case["B"] * case["W"]
        return dict(bytes=float(n * case["V"] * SIZE[case["dtype"]] + 5 * n + 12 * case["B"] * case["K"]), flops=4.0 * n * case["V"])
    n = case["B"] * case["W"]
    return dict(bytes=float(2 * n * 5 * sum(STATES[case["net"]]) + 4 * n), flops=0.0)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("norm", "quantize"):
        x, total, size = s["x"].to(torch.float64), None, 1.0
        if kind == "norm":
            if case["residual"]:
                total = x + s["residual"].to(torch.float64)
                x = total.to(s["x"].dtype).to(torch.float64)   # the sum is kept, and normalised, in the type of its inputs
            size = x.pow(2).mean(dim=1).add(EPS).sqrt()[:, None]
            x = x * s["weight"].to(torch.float64)
        peak = x.abs().max(dim=1).values[:, None]
        peak = torch.where(peak > 0, peak, torch.ones_like(peak))
        # the root mean square divides values and range alike: the codes do not depend on it, their step does
        values = x.mul(127.0).div(peak).round() * (peak / 127.0 / size)
        return dict(values=values) if total is None else dict(values=values, sum=total)
    if kind == "linear":
        a = s["a"][:, :case["K"]].to(torch.float64) * s["a_scale"].to(torch.float64)[:, None]
        w = s["w"].to(torch.float64) * s["w_scale"].to(torch.float64)[:, None]
        y = a @ w.t().contiguous()
        return y if s["bias"] is None else y + s["bias"].to(torch.float64)
    if kind == "select":
        B, W, V = case["B"], case["W"], case["V"]
        lp = torch.log_softmax(s["logits"].to(torch.float64), dim=-1).reshape(B, W, V)
        lp[lp.isnan()] = float("-inf")
        if s["finished"] is not None:
            through = s["finished"] != 0
            lp[through] = float("-inf")
            lp[..., END] = torch.where(through, torch.zeros_like(lp[..., END]), lp[..., END])
        best = (lp + s["score"].to(torch.float64).unsqueeze(-1)).reshape(B, W * V).topk(case["K"], dim=1).values
        return dict(parent=None, token=None, score=best)
    out = []
    for x in s["src"]:
        rows = x.view(case["B"], case["W"], -1)
        picked = torch.gather(rows, 1, s["parent"].long()[:, :, None].expand(-1, -1, rows.shape[2]))
        out.append(picked.reshape(x.shape).to(torch.float64) if x.dtype == torch.float32 else None)
    return out
