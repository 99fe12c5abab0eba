"""Operators for serving many tenants from one model: what a step of their requests needs around the shared products, and the
log-probabilities that scoring programs ask for.

Four kinds of case, each one call of the single-kernel entry points:

* norm:     bf16 rows plus what a layer adds to them, RMS norm, E4M3 codes with a scale per row or per block of 128
* adapters: low-rank adapters of many requests at once, from a pool, added to the output of a shared projection
* score:    hidden rows through the LM head to the log-probability of one given token per row and the entropy
* logprobs: logits to the log-probabilities of given tokens, the entropy and the top alternatives

With `own` false `run` computes the same in elementary torch operations.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
EPS = 1e-5


# ---------------------------------------------------------------------------------------------- the cases

def listed():
    return [
        # one answer's row in front of the QKV projection with a scale per row: the smallest call
        {"name": "norm-row-1", "kind": "norm", "rows": 1, "d": 4096, "block": 0, "both": False},
        # an ordinary ragged request at the 32B width, codes in blocks and the bf16 rows for adapters beside the product
        {"name": "norm-block-1931-32b", "kind": "norm", "rows": 1931, "d": 5120, "block": 128, "both": True},
        # a whole chunk of a long prompt
        {"name": "norm-block-16384", "kind": "norm", "rows": 16384, "d": 4096, "block": 128, "both": False},
        # 64 requests of one token each, every one with an adapter of its own, O projection
        {"name": "adapters-64x1", "kind": "adapters", "requests": 64, "rows": 1, "spread": 0, "adapters": 64, "rank": 16,
         "mixed": False, "k": 4096, "n": 4096, "dtype": "bf16"},
        # posts of a few users: ragged rows, ranks from 4 to 64, some requests without an adapter
        {"name": "adapters-posts-50x150", "kind": "adapters", "requests": 50, "rows": 150, "spread": 1, "adapters": 9, "rank": 16,
         "mixed": True, "k": 4096, "n": 4096, "dtype": "bf16"},
        # long prompts of two tenants, down projection, rank 64
        {"name": "adapters-down-2x8000", "kind": "adapters", "requests": 2, "rows": 8000, "spread": 1, "adapters": 2, "rank": 64,
         "mixed": False, "k": 14336, "n": 4096, "dtype": "bf16"},
        # the probability of one answer
        {"name": "score-1", "kind": "score", "rows": 1, "d": 4096, "vocab": 128256, "dtype": "bf16"},
        # a 150-token post scored token by token at the 32B width
        {"name": "score-150-32b", "kind": "score", "rows": 150, "d": 5120, "vocab": 152064, "dtype": "bf16"},
        # a prompt of 4001 tokens scored
        {"name": "score-4001", "kind": "score", "rows": 4001, "d": 4096, "vocab": 128256, "dtype": "bf16"},
        # one answer with its twenty best alternatives
        {"name": "logprobs-1-top20", "kind": "logprobs", "rows": 1, "vocab": 128256, "dtype": "f32", "given": 1, "top": 20, "masked": False},
        # a batch of bf16 logits, five alternatives each
        {"name": "logprobs-256-top5-bf16", "kind": "logprobs", "rows": 256, "vocab": 152064, "dtype": "bf16", "given": 1, "top": 5,
         "masked": False},
        # many answers held to a few labels by masked logits, three labels looked up
        {"name": "logprobs-1024-labels", "kind": "logprobs", "rows": 1024, "vocab": 128256, "dtype": "f32", "given": 3, "top": 3,
         "masked": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    pick = rng.random()
    if pick < 0.25:
        block = rng.choice([0, 128, 128])
        d = rng.choice([4096, 5120, 8192, 256, (8 * _log(rng, 8, 1024) if block == 0 else 128 * _log(rng, 1, 64))])
        return {"kind": "norm", "rows": _log(rng, 1, 16384 * 4096 // max(d, 4096)), "d": d, "block": block, "both": rng.random() < 0.5}
    if pick < 0.5:
        k, n = rng.choice([(4096, 4096), (14336, 4096), (4096, 6144), (5120, 5120), (256, 1024), (8 * _log(rng, 4, 600), 8 * _log(rng, 4, 600))])
        single = rng.random() < 0.4
        case = {"kind": "adapters", "requests": _log(rng, 1, 128), "rows": 1 if single else _log(rng, 2, 2000), "spread": rng.choice([0, 1, 2]),
                "adapters": _log(rng, 1, 64), "rank": rng.choice([8, 16, 16, 32, 64, 128, rng.randint(1, 128)]),
                "mixed": rng.random() < 0.5, "k": k, "n": n, "dtype": "f32" if rng.random() < 0.15 else "bf16"}
        cap = 40_000_000 if case["dtype"] == "f32" else 150_000_000       # (float32 is the checking path: short ones)
        while case["requests"] > 1 and case["requests"] * case["rows"] * (k + n) > cap:
            case["requests"] -= 1
        return case
    if pick < 0.75:
        d, v = rng.choice([(4096, 128256), (4096, 128256), (5120, 152064), (256, 1024), (64 * _log(rng, 1, 80), _log(rng, 100, 150000))])
        dtype = "f32" if d == 256 or rng.random() < 0.15 else "bf16"
        cap = (60 if dtype == "f32" else 4000) * 4096 * 128256
        return {"kind": "score", "rows": _log(rng, 1, max(2, min(8000, cap // (d * v)))), "d": d, "vocab": v, "dtype": dtype}
    return {"kind": "logprobs", "rows": _log(rng, 1, 800), "vocab": rng.choice([_log(rng, 100, 150000), 1024, 128256, 152064]),
            "dtype": rng.choice(["f32", "bf16"]), "given": rng.choice([0, 1, 1, 2, 5]), "top": rng.choice([0, 1, 5, 20, rng.randint(1, 64)]),
            "masked": rng.random() < 0.3}


# ---------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _norm_inputs(case, seed):
    """a residual stream with some channels far larger than the rest, what a layer adds to it, gains"""
    g, m, d = _gen(seed), case["rows"], case["d"]
    x = torch.randn(m, d, generator=g, device=DEV) * torch.where(torch.rand(d, generator=g, device=DEV) < 0.004, 40.0, 1.0)
    delta = torch.randn(m, d, generator=g, device=DEV) * 0.3
    gain = 1.0 + 0.2 * torch.randn(d, generator=g, device=DEV)
    return [t.to(torch.bfloat16) for t in (x, delta, gain)]


def _segments(case):
    """-> int64 [n, 3] of (first row, rows, adapter or -1), all rows, rank of each adapter: the same for every seed"""
    r = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    ranks = [r.choice([4, 8, 16, 16, 32, 64]) if case["mixed"] else case["rank"] for _ in range(case["adapters"])]
    segs, row = [], 0
    for i in range(case["requests"]):
        n = case["rows"]
        if case["spread"] and n > 1:
            n = min(3 * n, max(1, round(n * math.exp(r.gauss(0.0, 0.3 * case["spread"]) - 0.05 * case["spread"] ** 2))))
        segs.append((row, n, -1 if case["mixed"] and r.random() < 0.1 else i % case["adapters"]))
        row += n
    return np.array(segs, dtype=np.int64), row, ranks


def _adapter_inputs(case, seed):
    """normalised rows, the shared projection's output, the pool of adapters A [n, R, K], B [n, N, R], scales (of an adapter of lower
    rank than its slot the rest of the slot holds what was there before)"""
    segs, rows, ranks = _segments(case)
    g, dt = _gen(seed), torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    count, width = len(ranks), (max(ranks) + 7) // 8 * 8
    x = torch.randn(rows, case["k"], generator=g, device=DEV).to(dt)
    c = (torch.randn(rows, case["n"], generator=g, device=DEV) * 1.3).to(dt)
    a = (torch.randn(count, width, case["k"], generator=g, device=DEV) / math.sqrt(case["k"])).to(dt)
    b = (torch.randn(count, case["n"], width, generator=g, device=DEV) * 0.2).to(dt)
    return x, c, a, b, np.array(ranks, dtype=np.int32), np.array([4.0 / math.sqrt(r) for r in ranks], dtype=np.float32), segs


def _score_inputs(case, seed):
    """normalised rows that lean towards the token that follows, as a trained model's do; head; tokens"""
    g, m, d, v = _gen(seed), case["rows"], case["d"], case["vocab"]
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    w = (torch.randn(v, d, generator=g, device=DEV) * 0.02).to(dt)
    t = torch.randint(0, v, (m,), generator=g, device=DEV)
    lean = torch.rand(m, 1, generator=g, device=DEV) * 8.0
    x = torch.randn(m, d, generator=g, device=DEV) + lean * w[t].float() / (0.02 * math.sqrt(d))
    return x.to(dt), w, t.to(torch.int32)


def _logprob_inputs(case, seed):
    """logits with a few likely tokens; masked: all but a few labels at -infinity, and in every 50th row all of them"""
    g, m, v = _gen(seed), case["rows"], case["vocab"]
    z = torch.randn(m, v, generator=g, device=DEV) * 2.2
    top = torch.randint(0, v, (m, 24), generator=g, device=DEV)
    z.scatter_add_(1, top, torch.rand(m, 24, generator=g, device=DEV) * 10.0)
    t = torch.randint(0, v, (m, case["given"]), generator=g, device=DEV)
    t[::2] = top[::2, :case["given"]]
    if case["masked"]:
        labels = torch.randperm(v, generator=g, device=DEV)[:7]
        kept = torch.full_like(z, -math.inf)
        kept[:, labels] = z[:, labels]
        kept[49::50] = -math.inf
        z = kept
        if case["given"]:
            t[:, 0] = labels[torch.randint(0, 7, (m,), generator=g, device=DEV)]
    return z.to(torch.float32 if case["dtype"] == "f32" else torch.bfloat16), t.to(torch.int32)


def prepare(case, seed):
    st = {"kind": case["kind"]}
    if case["kind"] == "norm":
        st["x"], st["delta"], st["gain"] = _norm_inputs(case, seed)
        st["block"], st["both"] = case["block"], case["both"]
    elif case["kind"] == "adapters":
        st["x"], st["base"], st["a"], st["b"], st["ranks"], st["scales"], st["segs"] = _adapter_inputs(case, seed)
    elif case["kind"] == "score":
        st["x"], st["w"], st["tokens"] = _score_inputs(case, seed)
    else:
        st["logits"], st["tokens"] = _logprob_inputs(case, seed)
        st["top"] = case["top"]
    return st


# ---------------------------------------------------------------------------------------------- one pass

def run(st):
    if own:
        return _run_own(st)
    return {"norm": _norm_plain, "adapters": _adapters_plain, "score": _score_plain, "logprobs": _logprobs_plain}[st["kind"]](st)


def _run_own(st):
    from paper_2505_07203_amd import binding as B
    if st["kind"] == "norm":
        h, codes, scales, y = B.po_op_add_rmsnorm_quantize(st["x"], st["delta"], st["gain"], EPS, block=st["block"], normed=st["both"])
        return h, codes.view(torch.float8_e4m3fn), scales, y
    if st["kind"] == "adapters":
        return B.po_op_adapters(st["x"], st["a"], st["b"], st["ranks"], st["scales"], st["segs"], residual=st["base"])
    if st["kind"] == "score":
        return B.po_op_lm_head_logprobs(st["x"], st["w"], st["tokens"])
    return B.po_op_token_logprobs(st["logits"], st["tokens"], top=st["top"])


def _norm_plain(st):
    h = (st["x"].float() + st["delta"].float()).to(torch.bfloat16)
    f = h.float()
    y = f * torch.rsqrt((f * f).mean(1, keepdim=True) + EPS) * st["gain"].float()
    rows, d = y.shape
    g = y.view(rows, d // 128, 128) if st["block"] else y.view(rows, 1, d)
    amax = g.abs().amax(-1, keepdim=True)
    s = torch.where(amax > 0, amax, torch.ones_like(amax))
    codes = (g * (448.0 / s)).to(torch.float8_e4m3fn).view(rows, d)
    scales = torch.where(amax > 0, s / 448.0, s)[:, :, 0]
    return h, codes, scales.t().contiguous() if st["block"] else scales[:, 0], y.to(torch.bfloat16) if st["both"] else None


def _adapters_plain(st):
    count, width, k = st["a"].shape
    segs = torch.from_numpy(st["segs"]).to(DEV)
    ranks, scales = torch.from_numpy(st["ranks"]).to(DEV), torch.from_numpy(st["scales"]).to(DEV)
    rows_of = torch.repeat_interleave(segs[:, 2], segs[:, 1], output_size=len(st["x"]))           # the adapter of each row
    mine = (torch.arange(count, device=DEV)[None] == rows_of[:, None])[:, :, None] & (torch.arange(width, device=DEV)[None] < ranks[:, None])[None]
    t = (st["x"].float() @ st["a"].float().view(-1, k).t()).view(-1, count, width)
    t = torch.where(mine, t * scales[None, :, None], torch.zeros_like(t)).view(-1, count * width)
    b = st["b"].float().permute(0, 2, 1).reshape(count * width, -1)
    return (st["base"].float() + t @ b).to(st["base"].dtype)


def _score_plain(st):
    z = st["x"].float() @ st["w"].float().t()
    m = z.amax(1, keepdim=True)
    d = z - m
    e = torch.exp(d)
    s = e.sum(1)
    lp = d.gather(1, st["tokens"].long()[:, None])[:, 0] - torch.log(s)
    return lp, torch.log(s) - (d * e).sum(1) / s


def _logprobs_plain(st):
    z, t, top = st["logits"].float(), st["tokens"].long(), st["top"]
    m = z.amax(1, keepdim=True)
    some = m > -math.inf
    d = z - torch.where(some, m, torch.zeros_like(m))
    e = torch.exp(d)
    s = e.sum(1, keepdim=True)
    s = torch.where(some, s, torch.ones_like(s))
    lp = d - torch.log(s)
    ent = torch.log(s[:, 0]) - torch.where(e > 0, d * e, torch.zeros_like(e)).sum(1) / s[:, 0]
    best = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :top]
    top_lp = lp.gather(1, best)
    return lp.gather(1, t), ent, torch.where(top_lp > -math.inf, best, -1).to(torch.int32), top_lp


# ---------------------------------------------------------------------------------------------- work

def work(case):
    if case["kind"] == "norm":
        m, d = case["rows"], case["d"]
        return {"bytes": m * d * (9 if case["both"] else 7) + 2 * d + 4 * m * (d // 128 if case["block"] else 1), "flops": 8 * m * d}
    if case["kind"] == "adapters":
        segs, rows, ranks = _segments(case)
        e, k, n = 4 if case["dtype"] == "f32" else 2, case["k"], case["n"]
        used = set(int(s[2]) for s in segs if s[2] >= 0)
        with_one = sum(int(s[1]) for s in segs if s[2] >= 0)
        flops = sum(2 * int(s[1]) * ranks[int(s[2])] * (k + n) for s in segs if s[2] >= 0)
        return {"bytes": e * (with_one * k + 2 * rows * n + sum(ranks[i] * (k + n) for i in used)), "flops": flops}
    if case["kind"] == "score":
        e, m, d, v = 4 if case["dtype"] == "f32" else 2, case["rows"], case["d"], case["vocab"]
        return {"bytes": e * d * (m + v) + 12 * m, "flops": 2 * m * d * v}
    e, m, v = 4 if case["dtype"] == "f32" else 2, case["rows"], case["vocab"]
    return {"bytes": m * (e * v + 8 * case["given"] + 8 * case["top"] + 4), "flops": 6 * m * v}


# ---------------------------------------------------------------------------------------------- exact results

def exact(case, seed):
    return {"norm": _norm64, "adapters": _adapters64, "score": _score64, "logprobs": _logprobs64}[case["kind"]](case, seed)


def _norm64(case, seed):
    x, delta, gain = (t.double() for t in _norm_inputs(case, seed))
    h = (x + delta).float().to(torch.bfloat16).double()             # (the sum of two bf16 values, rounded as the stream is stored)
    y = h / torch.sqrt(h.square().sum(1, keepdim=True) / case["d"] + EPS) * gain
    blocks = y.unflatten(1, (-1, case["block"] or case["d"]))
    top = blocks.abs().max(-1, keepdim=True).values
    codes = (blocks * 448.0 / top).float().to(torch.float8_e4m3fn).double().flatten(1)
    scales = (top / 448.0).squeeze(-1)
    return h, codes, scales.t() if case["block"] else scales[:, 0], y if case["both"] else None


def _adapters64(case, seed):
    x, c, a, b, ranks, scales, segs = _adapter_inputs(case, seed)
    out = c.double()
    for row, n, which in segs.tolist():
        if which >= 0:
            r = int(ranks[which])
            t = x[row:row + n].double() @ a[which, :r].double().t()
            out[row:row + n] += float(scales[which]) * (t @ b[which, :, :r].double().t())
    return out


def _score64(case, seed):
    x, w, t = _score_inputs(case, seed)
    lps, ents = [], []
    wt = w.double().t().contiguous()
    for r0 in range(0, len(x), 1024):
        lp = torch.log_softmax(x[r0:r0 + 1024].double() @ wt, 1)
        lps.append(lp.gather(1, t[r0:r0 + 1024].long()[:, None])[:, 0])
        ents.append(-(lp.exp() * lp).sum(1))
    return torch.cat(lps), torch.cat(ents)


def _logprobs64(case, seed):
    z, t = _logprob_inputs(case, seed)
    t = t.long()
    lps, ents, ids, tops = [], [], [], []
    for r0 in range(0, len(z), 128):
        x = z[r0:r0 + 128].double()
        lp = torch.log_softmax(x, 1)
        lp[x.amax(1) == -math.inf] = -math.inf
        p = lp.exp()
        ents.append(-(p * lp.clamp(min=-1e4)).sum(1))
        lps.append(lp.gather(1, t[r0:r0 + 128]))
        order = torch.argsort(-x, dim=1, stable=True)[:, :case["top"]]
        v = lp.gather(1, order)
        order[v == -math.inf] = -1
        ids.append(order.to(torch.int32))
        tops.append(v)
    return tuple(torch.cat(v) for v in (lps, ents, ids, tops))
