"""Operators of 4-bit floating-point layers with a scale for each block of 32 (microscaled: E2M1 codes, E8M0 scales) and of
scoring given tokens from logits, for timing.

``listed()`` names representative cases, ``draw(rng)`` gives one more of the same ranges, ``prepare(case, seed)`` makes
what a program holds before the call, ``run(state)`` is one call, ``work(case)`` what it cannot do without and
``exact(case, seed)`` its outputs from the definition in 64 bits.  With ``own`` false ``run`` computes the operators from
elementary torch operations, with ``own`` true it calls the library.

Kinds
  quantize  4-bit codes with a scale for each block of 32 columns, and the values that they stand for (bfloat16 holds them all)
  linear    such codes x such weights
  scores    log probability of a given token for each row of logits, entropy, the best alternatives
"""
from __future__ import annotations

import torch

own = False

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "fp16": 2, "bf16": 2}
BLOCK = 32
VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)   # of the codes 0 to 7; 8 to 15 are their negatives


def listed():
    return [
        # hidden states of a language model of 1024 cells for one beam of 16: pure latency
        dict(name="quantize_beam", kind="quantize", rows=16, cols=1024, dtype="fp32"),
        # rows of an odd width
        dict(name="quantize_odd", kind="quantize", rows=333, cols=1283, dtype="fp16"),
        # the encoder's frames (32 utterances x 500 frames, both directions of 640)
        dict(name="quantize_frames", kind="quantize", rows=16000, cols=1280, dtype="bf16"),
        # output layer of a language model of 1024 cells over 32 k words, for one hypothesis and for one beam of 16
        dict(name="linear_vocab_one", kind="linear", M=1, N=32000, K=1024, dtype="fp32", bias=True),
        dict(name="linear_vocab_beam", kind="linear", M=16, N=32000, K=1024, dtype="bf16", bias=True),
        # an odd layer for an odd batch
        dict(name="linear_odd", kind="linear", M=77, N=1000, K=1283, dtype="bf16", bias=True),
        # the input projection of the encoder's frames (4 x 640 gate rows)
        dict(name="linear_frames", kind="linear", M=16000, N=2560, K=1280, dtype="fp32", bias=False),
        # a large layer over a prompt batch
        dict(name="linear_prompt", kind="linear", M=8192, N=8192, K=8192, dtype="bf16", bias=False),
        # the next token of one hypothesis over 32 k words
        dict(name="scores_one", kind="scores", rows=1, V=32000, n_top=5, dtype="fp32"),
        # a few positions over a very large vocabulary
        dict(name="scores_wide", kind="scores", rows=64, V=131072, n_top=20, dtype="fp32"),
        # the benchmark's batch (64 utterances, beam 16), as many alternatives as the beam has places
        dict(name="scores_batch", kind="scores", rows=1024, V=32000, n_top=16, dtype="bf16"),
        # rescoring of N-best lists: 16 k positions, no alternatives
        dict(name="scores_rescore", kind="scores", rows=16384, V=32000, n_top=0, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["quantize", "quantize", "linear", "linear", "linear", "scores", "scores", "scores"])
    dtype = rng.choice(["fp32", "fp16", "bf16", "bf16"])
    if kind == "quantize":
        cols = _log(rng, 1, 16384)
        if rng.random() < 0.5:
            cols = max(32, cols // 32 * 32)
        return dict(kind=kind, rows=_log(rng, 1, min(16384, (1 << 24) // cols)), cols=cols, dtype=dtype)
    if kind == "linear":
        K, N = _log(rng, 20, 8192), _log(rng, 16, 32000)
        if rng.random() < 0.6:
            K, N = max(64, K // 64 * 64), max(64, N // 64 * 64)
        M = _log(rng, 1, max(1, min(16384, (1 << 38) // (K * N), (1 << 28) // N)))
        return dict(kind=kind, M=M, N=N, K=K, dtype=dtype, bias=rng.random() < 0.5)
    V = _log(rng, 46, 262144)
    return dict(kind=kind, rows=_log(rng, 1, min(16384, (1 << 26) // V)), V=V, n_top=min(rng.choice([0, 0, 1, 5, 8, 16, 20, 64]), V - 1), dtype=dtype)


def _power(n):
    """2^n of whole numbers, in 64 bits and without an error."""
    return ((n.long() + 1023) << 52).view(torch.float64)


def _encode(x):
    """Codes (two to a byte, the even column in the low bits) and scales, with zeros and ones behind the columns.  In 64 bits:
    whether a value lies above or below the border of two codes goes by the value."""
    rows, cols = x.shape
    n = (cols + BLOCK - 1) // BLOCK
    v = torch.zeros((rows, n * BLOCK), dtype=torch.float64, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, n, BLOCK)
    peak = v.abs().amax(2)
    e = (torch.frexp(peak).exponent + (127 - 3)).clamp(min=0)   # floor(log2 peak) - 2
    e = torch.where(peak == 0, 127, e)
    u = v.abs() * _power(127 - e)[:, :, None]
    step = torch.where(u < 2, 0.5, torch.where(u < 4, 1.0, 2.0)).double()
    u = (torch.round(u / step) * step).clamp(max=6.0)
    at = torch.where(u < 2, u * 2, torch.where(u < 4, u + 2, u / 2 + 4)).to(torch.uint8)
    at = at + 8 * (v < 0).to(torch.uint8)
    at = at.view(rows, n * BLOCK)
    scale = torch.full((rows, (n + 7) // 8 * 8), 127, dtype=torch.uint8, device=x.device)
    scale[:, :n] = e.to(torch.uint8)
    return (at[:, 0::2] | (at[:, 1::2] << 4)).contiguous(), scale


def _decode(codes, scale, cols):
    """The values of codes and scales, in 32 bits."""
    table = torch.tensor(VALUES + tuple(-v for v in VALUES), device=codes.device)
    low, high = table[(codes & 15).int()], table[(codes >> 4).int()]
    v = torch.stack([low, high], dim=2).view(codes.shape[0], -1, BLOCK)
    step = _power(scale[:, :v.shape[1]].int() - 127).float()
    return (v * step[:, :, None]).view(codes.shape[0], -1)[:, :cols]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    randn = lambda *shape: torch.randn(shape, generator=g, device=DEV)
    rand = lambda *shape: torch.rand(shape, generator=g, device=DEV)
    # rows of different size, a few columns far larger than the others
    rows_of = lambda rows, cols: randn(rows, cols) * torch.exp(0.5 * randn(rows, 1)) * (1.0 + 20.0 * (rand(cols) < 0.01))
    s = dict(case=dict(case))
    kind = case["kind"]
    if kind == "quantize":
        s["x"] = rows_of(case["rows"], case["cols"]).to(TYPES[case["dtype"]])
    elif kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        s["w"], s["w_scale"] = _encode(randn(N, K) / K ** 0.5)
        s["a"], s["a_scale"] = _encode(rows_of(M, K))
        s["bias"] = 0.1 * randn(N) if case["bias"] else None
    else:
        rows, V = case["rows"], case["V"]
        s["logits"] = (3.0 * randn(rows, V)).to(TYPES[case["dtype"]])
        s["logits"][:, 0] = float("-inf")   # a token that is never to be said
        s["token"] = torch.randint(1, V, (rows,), generator=g, device=DEV, dtype=torch.int32)
    if own:   # packed weights and workspaces, as a program keeps them
        from paper_2206_07882_amd import qrnnt as q
        s["q"] = q
        if kind == "linear":
            s["mat"] = q.pack_mx4(s["w"], s["w_scale"], K)
            s["ws"] = torch.empty(q.linear_mx4_workspace(s["mat"], M), dtype=torch.uint8, device=DEV)
        elif kind == "scores":
            s["ws"] = torch.empty(q.token_scores_workspace(rows, V, case["n_top"]), dtype=torch.uint8, device=DEV)
    return s


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "quantize":
        codes, scale = _encode(s["x"])
        return dict(values=_decode(codes, scale, case["cols"]).to(torch.bfloat16))
    if kind == "linear":
        a, w = _decode(s["a"], s["a_scale"], case["K"]), _decode(s["w"], s["w_scale"], case["K"])
        y = torch.matmul(a, w.t())
        if s["bias"] is not None:
            y = y + s["bias"]
        return y.to(TYPES[case["dtype"]])
    x = s["logits"].float()
    V, n = case["V"], case["n_top"]
    top = x.amax(1, keepdim=True)
    d = x - top
    e = torch.exp(d)
    total = e.sum(1, dtype=torch.float64)
    log_sum = torch.log(total)
    token = s["token"].long()[:, None]
    logp = d.gather(1, token)[:, 0] - log_sum
    entropy = log_sum - torch.where(e > 0, e * d, 0.0).sum(1, dtype=torch.float64) / total
    out = dict(logp=logp.float(), entropy=entropy.float())
    if n:   # a logit and its column in one word that orders them: larger logits first, of equal ones the lowest column
        word = (x + 0.0).view(torch.int32).long()
        word = torch.where(word < 0, word ^ 0x7FFFFFFF, word)
        word = (word << 32) + ((1 << 32) - 1 - torch.arange(V, device=x.device))
        k = min(n, V)
        at = (1 << 32) - 1 - (torch.topk(word, k, dim=1).values & 0xFFFFFFFF)
        found = d.gather(1, at) - log_sum[:, None]
        none = found == float("-inf")
        tokens = torch.full((case["rows"], n), -1, dtype=torch.int32, device=x.device)
        values = torch.full((case["rows"], n), float("-inf"), device=x.device)
        tokens[:, :k] = torch.where(none, -1, at).to(torch.int32)
        values[:, :k] = found.float()
        out.update(tokens=tokens, values=values)
    return out


def run(s):
    if not own:
        return _plain(s)
    q, case = s["q"], s["case"]
    kind = case["kind"]
    if kind == "quantize":
        codes, scale = q.quantize_mx4(s["x"])
        return dict(values=q.dequantize_mx4(codes, scale, case["cols"], dtype=torch.bfloat16))
    if kind == "linear":
        return q.linear_mx4(s["mat"], s["a"], s["a_scale"], bias=s["bias"], dtype=TYPES[case["dtype"]], workspace=s["ws"])
    logp, entropy, tokens, values = q.token_scores(s["logits"], s["token"], n_top=case["n_top"], workspace=s["ws"])
    return dict(logp=logp, entropy=entropy, tokens=tokens, values=values) if case["n_top"] else dict(logp=logp, entropy=entropy)


def work(case):
    """Each input read once, each output written once (codes as half a byte and a 32nd; of the quantizer they are written and
    read again); a multiply-accumulate counts as two operations."""
    kind = case["kind"]
    if kind == "quantize":
        n, coded = case["rows"] * case["cols"], case["rows"] * ((case["cols"] + 31) // 32) * 17
        return dict(bytes=float(n * (SIZE[case["dtype"]] + 2) + 2 * coded), flops=float(4 * n))
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return dict(bytes=float((M + N) * ((K + 31) // 32) * 17 + (4 * N if case["bias"] else 0) + M * N * SIZE[case["dtype"]]),
                    flops=2.0 * M * N * K)
    n = case["rows"]
    return dict(bytes=float(n * case["V"] * SIZE[case["dtype"]] + 12 * n + 8 * n * case["n_top"]), flops=6.0 * n * case["V"])


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        x = s["x"].to(torch.float64)
        rows, cols = x.shape
        x = torch.nn.functional.pad(x, (0, -cols % BLOCK)).reshape(-1, BLOCK)
        peak = x.abs().max(dim=1, keepdim=True).values
        # the largest power of two that is not above the peak, a quarter of it
        unit = torch.exp2(torch.floor(torch.log2(peak)))
        unit = torch.where(unit > peak, unit / 2, torch.where(unit * 2 <= peak, unit * 2, unit)) / 4
        unit = torch.where(peak > 0, unit.clamp(min=2.0 ** -127), torch.ones_like(unit))
        u = x / unit
        grid = torch.tensor(VALUES, dtype=torch.float64, device=x.device)
        above = torch.searchsorted(grid, u.abs().contiguous()).clamp(max=7)   # first value that is not smaller
        below = (above - 1).clamp(min=0)
        up, down = grid[above] - u.abs(), u.abs() - grid[below]
        at = torch.where(up < down, above, torch.where(up > down, below, torch.where(above % 2 == 0, above, below)))
        values = torch.sign(u) * grid[at] * unit
        return dict(values=values.reshape(rows, -1)[:, :cols])
    if kind == "linear":
        def values(codes, scale):
            codes, scale = codes.to(torch.int64), scale.to(torch.int64)
            both = torch.stack((codes % 16, codes // 16), dim=-1).flatten(1)
            power, half = both % 8 // 2, both % 2
            size = torch.where(power == 0, 0.5 * half, (1.0 + 0.5 * half) * torch.exp2(power - 1.0)).to(torch.float64)
            size = torch.where(both >= 8, -size, size)
            unit = torch.exp2((scale - 127).to(torch.float64)).repeat_interleave(BLOCK, dim=1)
            return (size * unit[:, :size.shape[1]])[:, :case["K"]].contiguous()
        y = values(s["a"], s["a_scale"]) @ values(s["w"], s["w_scale"]).t().contiguous()
        return y if s["bias"] is None else y + s["bias"].to(torch.float64)
    out = dict(logp=[], entropy=[], values=[])
    rows_at_once = max(1, (1 << 27) // case["V"])
    for x, token in zip(s["logits"].split(rows_at_once), s["token"].split(rows_at_once)):
        lp = torch.log_softmax(x.to(torch.float64), dim=-1)
        out["logp"].append(lp[torch.arange(len(x), device=x.device), token.long()])
        out["entropy"].append(-torch.special.xlogy(lp.exp(), lp.exp()).sum(-1))
        best = lp.topk(min(case["n_top"], case["V"]), dim=-1).values
        out["values"].append(torch.nn.functional.pad(best, (0, case["n_top"] - best.shape[1]), value=float("-inf")))
    out = {k: torch.cat(v) for k, v in out.items()}
    if not case["n_top"]:
        del out["values"]
        return out
    return dict(logp=out["logp"], entropy=out["entropy"], tokens=None, values=out["values"])
