"""Operators for a batch of short requests that share one cached profile: attention that reads the shared prefix once for
all of them, linear layers in FP8 with a scale for each block of 128, and drawing an answer from the logits.

Three kinds of case, each one call (a linear layer: two, quantisation and product) of the single-kernel entry points:

* attention: requests of q_len rows each with kv_len keys of their own behind a shared prefix of `prefix` keys
* linear:    bf16 activations, quantised in groups of 128, times E4M3 weights with a scale per 128 x 128 block
* sample:    one token per row of float32 logits from one given random number per row

With `own` false `run` computes the same in elementary torch operations.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
# heads, KV heads, head dimension of the model shapes in `paper_2505_07203_amd.inputs` and their smaller relatives
HEADS = {"tiny": (4, 2, 64), "8b": (32, 8, 128), "32b": (40, 8, 128), "hd64": (16, 4, 64)}
LOG2E = 1.4426950408889634


# ---------------------------------------------------------------------------------------------- the cases

def listed():
    return [
        # post recommendation: a user's 50 posts of 150 tokens behind their profile of 14 000 tokens, one layer
        {"name": "attention-posts-50x150-behind-14000", "kind": "attention", "shape": "8b", "dtype": "bf16", "form": "posts",
         "requests": 50, "rows": 150, "spread": 0, "prefix": 14000, "own": 0},
        # ragged posts behind a shorter profile, five query heads to a KV head, a prefix that ends inside a tile
        {"name": "attention-posts-ragged-32b", "kind": "attention", "shape": "32b", "dtype": "bf16", "form": "posts",
         "requests": 9, "rows": 211, "spread": 2, "prefix": 4001, "own": 0},
        # 64 requests answer one token each behind a shared profile, with histories of their own
        {"name": "attention-single-64-behind-14000", "kind": "attention", "shape": "8b", "dtype": "bf16", "form": "single",
         "requests": 64, "rows": 1, "spread": 2, "prefix": 14000, "own": 300},
        # the smallest serving call: two requests, one token each, a short shared prompt
        {"name": "attention-single-2-behind-500", "kind": "attention", "shape": "8b", "dtype": "bf16", "form": "single",
         "requests": 2, "rows": 1, "spread": 1, "prefix": 500, "own": 40},
        # the float32 path that checks the others
        {"name": "attention-f32-posts", "kind": "attention", "shape": "8b", "dtype": "f32", "form": "posts",
         "requests": 8, "rows": 100, "spread": 2, "prefix": 1999, "own": 0},
        # O projection of a single token, with the residual
        {"name": "linear-o-1", "kind": "linear", "shape": "8b", "rows": 1, "n": 4096, "k": 4096, "epilogue": "residual"},
        # down projection of one 150-token post
        {"name": "linear-down-150", "kind": "linear", "shape": "8b", "rows": 150, "n": 4096, "k": 14336, "epilogue": "residual"},
        # gate and up projections of an ordinary ragged request, SiLU and product in the epilogue
        {"name": "linear-gate-up-1931", "kind": "linear", "shape": "8b", "rows": 1931, "n": 28672, "k": 4096, "epilogue": "silu"},
        # QKV projection of a batch of posts at the 32B shape
        {"name": "linear-qkv-8192-32b", "kind": "linear", "shape": "32b", "rows": 8192, "n": 7168, "k": 5120, "epilogue": "store"},
        # one answer
        {"name": "sample-1", "kind": "sample", "rows": 1, "vocab": 128256, "params": "filtered"},
        # a batch of answers, every request with settings of its own
        {"name": "sample-64-mixed", "kind": "sample", "rows": 64, "vocab": 128256, "params": "mixed"},
        # a large batch without filters at the larger vocabulary
        {"name": "sample-256-free", "kind": "sample", "rows": 256, "vocab": 152064, "params": "free"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    pick = rng.random()
    if pick < 0.45:
        shape = rng.choice(["8b", "8b", "32b", "hd64", "tiny"])
        dtype = "f32" if shape == "tiny" or rng.random() < 0.15 else "bf16"
        case = {"kind": "attention", "shape": shape, "dtype": dtype, "spread": rng.choice([0, 1, 2]),
                "form": rng.choice(["posts", "posts", "single"])}
        case["prefix"] = rng.choice([0, _log(rng, 40, 16000), _log(rng, 40, 16000), _log(rng, 2000, 16000)])
        if case["form"] == "posts":
            case.update(requests=_log(rng, 1, 60), rows=_log(rng, 4, 500), own=0)
        else:
            case.update(requests=_log(rng, 1, 128), rows=1, own=_log(rng, 1, 3000))
        # (float32 runs at a tenth of the rate and is the checking path: short ones)
        cap = 6_000_000 if dtype == "f32" else 80_000_000
        mean = case["prefix"] + case["own"] + case["rows"]
        while case["requests"] > 1 and case["requests"] * case["rows"] * mean * HEADS[shape][0] > cap * 32:
            case["requests"] -= 1
        return case
    if pick < 0.8:
        d, f, qkv = rng.choice([(4096, 14336, 6144), (4096, 14336, 6144), (5120, 27648, 7168)])
        n, k, epilogue = rng.choice([(qkv, d, "store"), (d, d, "residual"), (2 * f, d, "silu"), (d, f, "residual")])
        return {"kind": "linear", "shape": "8b" if d == 4096 else "32b", "rows": _log(rng, 1, 6000 * 36700160 // max(n * k, 36700160)),
                "n": n, "k": k, "epilogue": epilogue}
    return {"kind": "sample", "rows": _log(rng, 1, 256), "vocab": rng.choice([_log(rng, 300, 150000), 1024, 128256, 152064]),
            "params": rng.choice(["filtered", "mixed", "mixed", "free"])}


# ---------------------------------------------------------------------------------------------- inputs

def _requests(case):
    """-> [(q_row, q_len, kv_row, kv_len)], rows of q, rows of the requests' own K / V

    posts: rows packed as the library packs requests, each from a multiple of 64 on, keys in the same rows;
    single: query rows one behind the other, each request's keys in a region of its own"""
    r = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    seqs, q_row, kv_row = [], 0, 0
    for _ in range(case["requests"]):
        base = case["rows"] if case["form"] == "posts" else case["own"]
        n = base
        if case["spread"]:
            n = max(1, round(base * math.exp(r.gauss(0.0, 0.35 * case["spread"]) - 0.06 * case["spread"] ** 2)))
            n = min(n, 4 * base)
        if case["form"] == "posts":
            seqs.append((kv_row, n, kv_row, n))
        else:
            seqs.append((q_row, 1, kv_row, n))
            q_row += 1
        kv_row += (n + 63) // 64 * 64
    return seqs, (kv_row if case["form"] == "posts" else q_row), kv_row


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 17)
    return g


def _attention_inputs(case, seed):
    """q, own K rows, own V, prefix K rows, prefix V; V transposed for bf16 (the cache's layout), rows for float32"""
    hq, hkv, hd = HEADS[case["shape"]]
    _, nq, nk = _requests(case)
    g, dt = _gen(seed), torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    n2, n2c = case["prefix"], (case["prefix"] + 63) // 64 * 64

    def normal(*shape):     # about the size a normalised activation gives through N(0, 0.02^2) weights
        return torch.randn(*shape, generator=g, device=DEV) * 1.3
    q = normal(nq, hq, hd)
    if case["dtype"] == "bf16":            # the full path hands queries over times log2(e) / sqrt(hd)
        q = q * float(np.float32(LOG2E / math.sqrt(hd)))
        v, v2 = normal(hkv * hd, nk), normal(hkv * hd, max(n2c, 64))
    else:
        v, v2 = normal(nk, hkv, hd), normal(max(n2, 1), hkv, hd)
    return q.to(dt), normal(nk, hkv, hd).to(dt), v.to(dt), normal(max(n2, 1), hkv, hd).to(dt), v2.to(dt)


def _linear_inputs(case, seed):
    """activations (some channels far larger than the rest, as trained models have them), weights, residual"""
    g, m, n, k = _gen(seed), case["rows"], case["n"], case["k"]
    x = torch.randn(m, k, generator=g, device=DEV)
    x *= torch.where(torch.rand(k, generator=g, device=DEV) < 0.004, 30.0, 1.0)
    w = torch.randn(n, k, generator=g, device=DEV) * 0.02
    r = torch.randn(m, n, generator=g, device=DEV).to(torch.bfloat16) if case["epilogue"] == "residual" else None
    return x.to(torch.bfloat16), w.to(torch.bfloat16), r


def _block_weights(w):
    """[N, K] -> E4M3 codes, float32 scales [ceil(N / 128), K / 128]"""
    n, k = w.shape
    p = torch.zeros((n + 127) // 128 * 128, k, device=w.device)
    p[:n] = w
    p = p.view(-1, 128, k // 128, 128)
    amax = p.abs().amax((1, 3))
    s = torch.where(amax > 0, amax, torch.ones_like(amax))
    c = (p * (448.0 / s)[:, None, :, None]).to(torch.float8_e4m3fn).view(-1, k)[:n]
    return c.view(torch.uint8).contiguous(), s / 448.0


def _weights(case, w):
    """codes and scales as the product reads them; gate and up rows interleaved in blocks of 32 for the SiLU epilogue"""
    if case["epilogue"] != "silu":
        return _block_weights(w)
    f = case["n"] // 2
    (cg, sg), (cu, su) = _block_weights(w[:f]), _block_weights(w[f:])
    codes = torch.stack((cg.view(f // 32, 32, -1), cu.view(f // 32, 32, -1)), 1).reshape(2 * f, -1)
    return codes.contiguous(), torch.stack((sg, su))


def _sample_inputs(case, seed):
    """logits with a few likely tokens, every other row on the bf16 grid (equal values), and each row's settings"""
    g, rows, v = _gen(seed), case["rows"], case["vocab"]
    z = torch.randn(rows, v, generator=g, device=DEV) * 2.2
    top = torch.randint(0, v, (rows, 24), generator=g, device=DEV)
    z.scatter_add_(1, top, torch.rand(rows, 24, generator=g, device=DEV) * 10.0)
    z[1::2] = z[1::2].to(torch.bfloat16).float()
    u = torch.rand(rows, generator=g, device=DEV)
    r = random.Random(int(seed) * 31 + 5)
    if case["params"] == "free":
        t, k, p, mp = [1.0] * rows, [0] * rows, [1.0] * rows, [0.0] * rows
    elif case["params"] == "filtered":
        t, k, p, mp = [0.8] * rows, [50] * rows, [0.95] * rows, [0.0] * rows
    else:
        t = [r.choice([0.0, 0.6, 0.8, 1.0, 1.3]) for _ in range(rows)]
        k = [r.choice([0, 0, 1, 20, 50, 1000]) for _ in range(rows)]
        p = [r.choice([1.0, 0.98, 0.9, 0.5]) for _ in range(rows)]
        mp = [r.choice([0.0, 0.0, 0.02, 0.1]) for _ in range(rows)]
    f = [torch.tensor(a, dtype=torch.float32, device=DEV) for a in (t, p, mp)]
    return z, u, f[0], torch.tensor(k, dtype=torch.int32, device=DEV), f[1], f[2]


def prepare(case, seed):
    if case["kind"] == "attention":
        q, k, v, k2, v2 = _attention_inputs(case, seed)
        return {"kind": "attention", "q": q, "k": k, "v": v, "k2": k2, "v2": v2, "n2": case["prefix"],
                "seqs": np.array(_requests(case)[0], dtype=np.int64), "o": torch.zeros_like(q)}
    if case["kind"] == "linear":
        x, w, r = _linear_inputs(case, seed)
        codes, scales = _weights(case, w)
        return {"kind": "linear", "x": x, "codes": codes, "scales": scales, "r": r, "silu": case["epilogue"] == "silu"}
    return {"kind": "sample", "in": _sample_inputs(case, seed)}


# ---------------------------------------------------------------------------------------------- one pass

def run(st):
    if own:
        return _run_own(st)
    if st["kind"] == "attention":
        return _attention_plain(st)
    if st["kind"] == "linear":
        return _linear_plain(st)
    return _sample_plain(*st["in"])


def _run_own(st):
    from paper_2505_07203_amd import binding as B
    if st["kind"] == "attention":
        bf16 = st["q"].dtype == torch.bfloat16
        return B.po_op_attention_shared(st["q"], st["k"], st["v"], st["seqs"], k2=st["k2"], v2=st["v2"], n2=st["n2"],
                                        out=st["o"], q_prescaled=bf16)
    if st["kind"] == "linear":
        codes, scales = B.po_op_quantize_blocks(st["x"])
        return B.po_op_linear_fp8_block(codes, scales, st["codes"], st["scales"], residual=st["r"], silu_mul=st["silu"])
    z, u, t, k, p, mp = st["in"]
    return B.po_op_sample(z, u, temperature=t, top_k=k, top_p=p, min_p=mp)


def _attention_plain(st):
    q, k, v, k2, v2, n2, out = st["q"], st["k"], st["v"], st["k2"], st["v2"], st["n2"], st["o"]
    hq, hd, hkv = q.shape[1], q.shape[2], k.shape[1]
    group, bf16 = hq // hkv, q.dtype == torch.bfloat16
    scale = math.log(2.0) if bf16 else hd ** -0.5
    rows_of = (lambda a, n0, n1: a[:, n0:n1].float().view(hkv, hd, n1 - n0).transpose(1, 2)) if bf16 else \
              (lambda a, n0, n1: a[n0:n1].transpose(0, 1))
    kp = k2[:n2].float().permute(1, 2, 0)                         # [Hkv, hd, n2]
    vp = rows_of(v2, 0, n2)                                       # [Hkv, n2, hd]
    for q0, nq, k0, nk in st["seqs"].tolist():
        kt = torch.cat((kp, k[k0:k0 + nk].float().permute(1, 2, 0)), 2).contiguous()
        vr = torch.cat((vp, rows_of(v, k0, k0 + nk)), 1).contiguous()
        qr = q[q0:q0 + nq].float().view(nq, hkv, group, hd).permute(1, 0, 2, 3).reshape(hkv, nq * group, hd)
        s = torch.matmul(qr, kt).view(hkv, nq, group, n2 + nk) * scale
        last = torch.arange(nq, device=q.device) + n2 + nk - nq
        hide = torch.arange(n2 + nk, device=q.device)[None] > last[:, None]
        s = s.masked_fill(hide[None, :, None], -math.inf)
        p = torch.exp(s - s.amax(-1, keepdim=True)).view(hkv, nq * group, n2 + nk)
        o = torch.matmul(p, vr) / p.sum(-1, keepdim=True)
        out[q0:q0 + nq] = o.view(hkv, nq, group, hd).permute(1, 0, 2, 3).reshape(nq, hq, hd).to(out.dtype)
    return out


def _linear_plain(st):
    x, codes, scales, n, k = st["x"], st["codes"], st["scales"], st["codes"].shape[0], st["codes"].shape[1]
    g = x.float().view(-1, k // 128, 128)
    amax = g.abs().amax(-1, keepdim=True)
    s = torch.where(amax > 0, amax, torch.ones_like(amax))
    a = ((g * (448.0 / s)).to(torch.float8_e4m3fn).float() * (s / 448.0)).view(-1, k)
    w = codes.view(torch.float8_e4m3fn).float()
    if st["silu"]:
        w = w.view(n // 64, 2, 32, k).transpose(0, 1).reshape(2, n // 2, k)
        w = w * scales.repeat_interleave(128, 1)[:, :n // 2].repeat_interleave(128, 2)
        gate, up = a @ w[0].t(), a @ w[1].t()
        return (gate * torch.sigmoid(gate) * up).to(torch.bfloat16)
    c = a @ (w * scales.repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)).t()
    return (c if st["r"] is None else c + st["r"].float()).to(torch.bfloat16)


def _sample_plain(z, u, t, k, p, mp):
    rows, v = z.shape
    z64 = z.double()
    d = z64 - z64.amax(1, keepdim=True)
    greedy = t <= 0
    w = torch.exp(d / torch.where(greedy, torch.ones_like(t), t).double()[:, None])
    order = torch.sort(z, dim=1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    at = torch.arange(v, device=z.device)[None]
    n_k = torch.where((k > 0) & ~greedy, k, torch.where(greedy, 1, v)).clamp(max=v).long()
    before = ws.cumsum(1)
    s_k = before.gather(1, (n_k - 1)[:, None])
    before = torch.cat((torch.zeros_like(before[:, :1]), before[:, :-1]), 1)
    keep = (at < n_k[:, None]) & ((p >= 1)[:, None] | (before < p.double()[:, None] * s_k)) & (ws >= mp.double()[:, None])
    keep[:, 0] = True
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, torch.zeros_like(ws)))
    c = kept.cumsum(1)
    token = (c <= u.double()[:, None] * c[:, -1:]).sum(1)
    lp = torch.log(kept.gather(1, token[:, None]) / c[:, -1:])[:, 0]
    return token.to(torch.int32), lp.float()


# ---------------------------------------------------------------------------------------------- work

def work(case):
    if case["kind"] == "attention":
        hq, hkv, hd = HEADS[case["shape"]]
        e = 4 if case["dtype"] == "f32" else 2
        seqs = _requests(case)[0]
        rows, keys = sum(s[1] for s in seqs), case["prefix"] + sum(s[3] for s in seqs)
        seen = sum(s[1] * (case["prefix"] + s[3]) - s[1] * (s[1] - 1) // 2 for s in seqs)
        return {"bytes": e * hd * (2 * rows * hq + 2 * keys * hkv), "flops": 4 * hq * hd * seen}
    if case["kind"] == "linear":
        m, n, k = case["rows"], case["n"], case["k"]
        out = {"store": n, "residual": 2 * n, "silu": n // 2}[case["epilogue"]]
        return {"bytes": 2 * m * k + n * k + 4 * (n // 128) * (k // 128) + 2 * m * out, "flops": 2 * m * n * k}
    return {"bytes": case["rows"] * (4 * case["vocab"] + 28), "flops": 10 * case["rows"] * case["vocab"]}


# ---------------------------------------------------------------------------------------------- exact results

def exact(case, seed):
    if case["kind"] == "attention":
        return _attention64(case, seed)
    if case["kind"] == "linear":
        return _linear64(case, seed)
    return _sample64(case, seed)


def _attention64(case, seed):
    q, k, v, k2, v2 = (a.double() for a in _attention_inputs(case, seed))
    hq, hkv, hd = HEADS[case["shape"]]
    n2 = case["prefix"]
    if case["dtype"] == "bf16":
        v, v2 = (a.t().reshape(-1, hkv, hd) for a in (v, v2))
    factor = math.log(2.0) if case["dtype"] == "bf16" else 1.0 / math.sqrt(hd)
    out = torch.zeros_like(q)
    seqs = _requests(case)[0]
    for h in range(hq):
        c = h * hkv // hq
        pk, pv = k2[:n2, c].contiguous(), v2[:n2, c].contiguous()
        for i in range(0, len(seqs), 16):                         # (the prefix in products of many rows)
            part = seqs[i:i + 16]
            idx = torch.cat([torch.arange(a, a + n, device=DEV) for a, n, _, _ in part])
            sp = factor * (q[idx, h] @ pk.t())
            at = 0
            for a, n, b, m in part:
                so = factor * (q[a:a + n, h] @ k[b:b + m, c].t())
                so += torch.triu(torch.full_like(so, -math.inf), m - n + 1)
                s = torch.cat((sp[at:at + n], so), 1)
                p = torch.softmax(s, 1)
                out[a:a + n, h] = p[:, :n2] @ pv + p[:, n2:] @ v[b:b + m, c]
                at += n
    return out


def _linear64(case, seed):
    x, w, r = _linear_inputs(case, seed)
    m, n, k = case["rows"], case["n"], case["k"]

    def stored(t, rows):
        """what the codes and float32 scales of blocks of rows x 128 stand for (rows divides the tensor here)"""
        b = t.double().view(t.shape[0] // rows, rows, k // 128, 128)
        top = b.abs().amax((1, 3), keepdim=True)
        top[top == 0] = 1.0
        return ((b * (448.0 / top)).to(torch.float8_e4m3fn).double() * (top / 448.0).float().double()).view(-1, k)
    a = stored(x, 1)
    if case["epilogue"] == "silu":
        g, up = (a @ stored(h, 128).t() for h in (w[:n // 2], w[n // 2:]))
        return g / (1.0 + torch.exp(-g)) * up
    c = a @ stored(w, 128).t()
    return c if r is None else c + r.double()


def _sample64(case, seed):
    z, u, t, k, p, mp = (a.cpu().numpy() for a in _sample_inputs(case, seed))
    tokens, lps = [], []
    for i in range(z.shape[0]):
        x = z[i].astype(np.float64)
        if t[i] <= 0:
            tokens.append(int(np.argmax(x)))
            lps.append(0.0)
            continue
        w = np.exp((x - x.max()) / np.float64(t[i]))
        kept = np.arange(len(x))
        if k[i] > 0 or p[i] < 1:
            kept = np.argsort(-x, kind="stable")
            if k[i] > 0:
                kept = kept[:k[i]]
            if p[i] < 1:
                total = np.cumsum(w[kept])
                kept = kept[:1 + int(np.searchsorted(total, np.float64(p[i]) * total[-1], side="left"))]
            kept = np.sort(kept)
        kept = kept[w[kept] >= np.float64(mp[i])]
        total = np.cumsum(w[kept])
        j = min(int(np.searchsorted(total, np.float64(u[i]) * total[-1], side="right")), len(kept) - 1)
        tokens.append(int(kept[j]))
        lps.append(math.log(w[kept[j]] / total[-1]))
    return torch.tensor(tokens, dtype=torch.int32, device=DEV), torch.tensor(lps, dtype=torch.float64, device=DEV)
