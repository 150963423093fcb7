"""Performance cases of the 4-bit operators and of the cache's eviction: a draft model's forward pass in 4 bits, with a bounded cache.

A case is one pass through an operator as a program that runs a decoder layer makes it. `op` names it:

  append   sp_cache_append     keys and values of new tokens go into a paged cache of 4-bit elements, rotated on the way; queries rotated
  attend   sp_attend           ragged queries over a paged cache of 4-bit elements
  weights  sp_attend_weights   the attention weight that every cached token has drawn, added up over query rows and the heads of a group
  evict    sp_cache_evict      the tokens of most weight of every kv head move to other pages, in their order
  linear   sp_mx4_quantise and sp_mx4_matmul: a projection of bf16 activations, microscaled to 4 bits, with 4-bit weights

4-bit elements are E2M1 codes, two to a byte (the lower element in the lower bits), with a power of two as scale for 32 elements of a row, held as its
exponent + 127 in a byte: the smallest power of two s >= 2^-64 with max |x| <= 6 s. No torch type stands for them, so what is stored in 4 bits is returned
as its bytes, codes and scales, whole numbers that have to be equal: scaling by powers of two is exact, and so is the choice of the nearest code.

Inputs are made on the GPU from the seed. Keys, values and queries are N(0, 1) with a magnitude of its own for every kv head; a hundredth of the cached
keys carries a query vector on top, as retrieved passages and attention sinks do. Block tables are random permutations of the pool's pages.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
GROUP = 32                      # elements that share a 4-bit scale
BLOCK = 32                      # tokens that share an 8-bit scale
TOP8 = 448.0                    # largest E4M3 value
FLOOR = -64                     # logarithm of the smallest scale
LUT = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
MAX_FLOPS = 5.0e11              # drawn cases stay below the largest listed ones
MAX_BYTES = 4.0e8
MAX_LOGITS = 1.0e9              # (row, key) pairs of a drawn attention


def listed():
    llama = dict(H=32, kv=8, d=64)          # 16-layer draft's heads
    qwen = dict(H=16, kv=8, d=128)          # 28-layer draft's heads
    group8 = dict(H=32, kv=4, d=128)        # eight query heads to a kv head

    def paged(name, op, heads, **kw):
        base = {"name": name, "op": op, **heads, "layout": "HND", "cache": "mx4", "n_lo": 1, "n_hi": 1, "window": 0, "lens_seed": 1}
        return {**base, **kw}

    def linear(name, rows, k, n):
        return {"name": name, "op": "linear", "rows": rows, "k": k, "n": n}

    return [
        # one lookahead token of one request: launch latency is all there is
        paged("append-1", "append", llama, B=1, ctx_lo=1000, ctx_hi=1000, page=256, rot=64, style="half"),
        # sixteen requests in the middle of their prompts: ragged chunks at odd places, half of each head rotated in pairs
        paged("append-16-chunks", "append", group8, B=16, n_lo=300, n_hi=4096, ctx_lo=1, ctx_hi=5000, page=512, rot=64, style="pairs", lens_seed=3),
        # one request's next token after an 8K prompt
        paged("attend-1-8k", "attend", llama, B=1, ctx_lo=8192, ctx_hi=8192, page=256),
        # continuous decoding: 48 requests with contexts as the ragged configuration has them
        paged("attend-48-ragged", "attend", llama, B=48, ctx_lo=2048, ctx_hi=65536, page=256, lens_seed=25),
        # a 2K chunk of a 32K prompt: the matrix-bound side
        paged("attend-2k-chunk-32k", "attend", qwen, B=1, n_lo=2048, n_hi=2048, ctx_lo=32768, ctx_hi=32768, page=512),
        # the step after attend-48-ragged: what its tokens looked at is added up
        paged("weights-48-ragged", "weights", llama, B=48, ctx_lo=2048, ctx_hi=65536, page=256, lens_seed=25),
        # the last 64 rows of a 32K prompt as the window that decides what stays, on the bf16 pages of the importance pass
        paged("weights-64-rows-32k", "weights", qwen, B=1, n_lo=64, n_hi=64, ctx_lo=32768, ctx_hi=32768, page=512, cache="bf16"),
        # one request in the middle of its answer: back to 1024 of 1280 tokens
        paged("evict-1", "evict", llama, B=1, ctx_lo=1280, ctx_hi=1280, page=256, budget_lo=1024, budget_hi=1024, sinks=4, recent=64),
        # sixteen prompts that have just been read shrink to 2K to 8K tokens each, token-major pages
        paged("evict-16-ragged", "evict", qwen, B=16, ctx_lo=4001, ctx_hi=65536, page=512, cache="bf16", layout="NHD", budget_lo=2048, budget_hi=8192,
              sinks=4, recent=32, lens_seed=7),
        # one row onto the vocabulary of the lookahead example: its weights are read once
        linear("linear-1", 1, 2048, 32000),
        # a decoding batch through a square projection
        linear("linear-48", 48, 4096, 4096),
        # a whole 8K prompt through an up projection: the matrix-bound side
        linear("linear-8k", 8192, 4096, 8192),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "weights", "weights", "evict", "evict", "linear", "linear", "linear"])
    if op == "linear":
        k, n = 32 * _log_uniform(rng, 2, 256), _log_uniform(rng, 16, 33000)
        rows = _log_uniform(rng, 1, 8192)
        return {"op": op, "rows": max(1, min(rows, int(MAX_FLOPS / (2.0 * n * k)))), "k": k, "n": n}
    H, kv, d = rng.choice([(32, 8, 64), (32, 8, 64), (16, 8, 128), (32, 4, 128), (4, 2, 64)])
    cache = "mx4" if op in ("append", "attend") else rng.choice(["mx4", "mx4", "e4m3", "bf16"])
    case = {"op": op, "H": H, "kv": kv, "d": d, "layout": rng.choice(["HND", "HND", "NHD"]), "page": rng.choice([32, 64, 256, 512, 4096]),
            "cache": cache, "window": 0, "lens_seed": rng.randrange(1000)}
    kind = "token" if op == "evict" else rng.choice(["token", "token", "rows", "mixed"] if op == "weights" else ["token", "token", "rows", "chunk", "mixed"])
    case["B"] = {"token": _log_uniform(rng, 1, 96), "rows": rng.randint(1, 16), "chunk": rng.randint(1, 4), "mixed": rng.randint(4, 24)}[kind]
    if kind == "token":
        case["n_lo"] = case["n_hi"] = 1
    elif kind == "rows":
        case["n_lo"] = case["n_hi"] = rng.choice([2, 5, 8, 16, 32, 64])
    elif kind == "chunk":
        case["n_lo"], case["n_hi"] = 100, _log_uniform(rng, 200, 4096)
    else:
        case["n_lo"], case["n_hi"] = 1, rng.choice([64, 300, 512])
    if op == "append":
        case["ctx_lo"], case["ctx_hi"] = rng.randint(0, 500), _log_uniform(rng, 501, 6000)
        case["rot"], case["style"] = rng.choice([d, d, d // 2, 0]), rng.choice(["half", "half", "pairs"])
        return case
    top = min(131072, int(MAX_LOGITS / (case["B"] * H * case["n_hi"])), int(MAX_BYTES / (case["B"] * kv * d * 2)))
    case["ctx_hi"] = _log_uniform(rng, min(max(500, case["n_hi"]), top), top)
    case["ctx_lo"] = rng.choice([1, max(1, case["ctx_hi"] // 8), case["ctx_hi"]])
    if op == "evict":
        case["budget_hi"] = _log_uniform(rng, 1, case["ctx_hi"])
        case["budget_lo"] = rng.choice([1, max(1, case["budget_hi"] // 4), case["budget_hi"]])
        case["sinks"], case["recent"] = rng.choice([0, 4, 4, 16]), rng.choice([0, 1, 32, 64, 200])
    else:
        case["window"] = rng.choice([0, 0, 0, 700])
    while work(case)["flops"] > MAX_FLOPS or work(case)["bytes"] > MAX_BYTES:
        case["ctx_hi"] = case["ctx_hi"] // 2
        case["ctx_lo"] = min(case["ctx_lo"], case["ctx_hi"])
        case["n_hi"] = max(case["n_lo"], min(case["n_hi"], case["ctx_hi"]))
        if op == "evict":
            case["budget_hi"] = min(case["budget_hi"], case["ctx_hi"])
            case["budget_lo"] = min(case["budget_lo"], case["budget_hi"])
    return case


def lengths(case):
    """New tokens, tokens of context and budgets of every request. The context of an append is what was there before it, that of
    an attention counts the new tokens too."""
    rng = random.Random(case["lens_seed"])
    new, ctx, budget = [], [], []
    for _ in range(case["B"]):
        lo = max(case["ctx_lo"], 1)
        n = _log_uniform(rng, case["n_lo"], case["n_hi"])
        c = _log_uniform(rng, lo, max(case["ctx_hi"], lo)) if case["ctx_hi"] > 0 else 0
        new.append(n)
        ctx.append(c if case["op"] == "append" else max(c, n))
        if case["op"] == "evict":
            budget.append(_log_uniform(rng, case["budget_lo"], case["budget_hi"]))
    return new, ctx, budget


def visible(n, ctx, window):
    """(row, key) pairs of n queries at the end of ctx tokens that see themselves and what came before."""
    if not window:
        return n * ctx - n * (n - 1) // 2
    return sum(min(window, ctx - n + r + 1) for r in range(n))


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _quantise4(x):
    """[..., n] in 32 bits -> codes [..., n / 2] and scales [..., n / 32], bytes both."""
    y = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    m, e = torch.frexp(y.abs().amax(dim=-1))                # max = m 2^e, m in [1/2, 1): 6 s = 3/4 2^(t + 3)
    t = torch.where(m > 0.75, e - 2, e - 3).clamp(min=FLOOR)
    t = torch.where(m == 0, FLOOR, t)
    z = y * torch.exp2(-t.float())[..., None]
    a = z.abs()
    code = (a > 0.25).to(torch.uint8)                       # nearest, halfway to the even code
    for edge, up in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= edge) if up else (a > edge)
    code += torch.signbit(z).to(torch.uint8) * 8
    code = code.view(*x.shape[:-1], x.shape[-1] // 2, 2)
    return code[..., 0] | (code[..., 1] << 4), (t + 127).to(torch.uint8)


def _values4(codes, scales, dtype=torch.float32):
    """What codes and scales stand for."""
    lut = torch.tensor(LUT + [-x for x in LUT], dtype=dtype, device=DEV)
    pairs = torch.stack([lut.repeat(16), lut.repeat_interleave(16)], dim=1)                 # of a byte
    x = pairs[codes.to(torch.int32)].reshape(*codes.shape[:-1], scales.shape[-1], GROUP)
    x *= torch.exp2(scales.to(dtype) - 127)[..., None]
    return x.reshape(*codes.shape[:-1], -1)


def _scale8(amax):
    """Smallest power of two s >= 2^-64 with amax <= 448 s."""
    m, e = torch.frexp(amax.clamp(min=TOP8 * 2.0 ** FLOOR) / TOP8)
    return torch.where(m > 0.5, torch.exp2(e.float()), torch.exp2(e.float() - 1))


def _pool(case, g, pages, extra=None):
    """One pool in its layout, and its scales: [pages][kv][page][d / 32] bytes, [pages][kv][page / 32] floats, or None."""
    kv, d, P = case["kv"], case["d"], case["page"]
    x = _randn(g, pages, kv, P, d) * torch.exp2(_randn(g, kv) * 0.5)[None, :, None, None]
    if extra is not None:
        x.view(-1)[extra[0]] += extra[1]
    scale = None
    if case["cache"] == "bf16":
        x = x.to(torch.bfloat16)
    elif case["cache"] == "mx4":
        x, scale = _quantise4(x)
    else:
        x = x.view(pages, kv, P // BLOCK, BLOCK, d)
        scale = _scale8(x.abs().amax(dim=(-1, -2)))
        x = (x / scale[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(pages, kv, P, d)
    return (x.transpose(1, 2).contiguous() if case["layout"] == "NHD" else x), scale


def _cache(case, g, total, q=None, spare=None):
    """Pools, scales and block table for `total[b]` tokens of each request; with `spare`, a second table of pages for so many."""
    kv, d, P = case["kv"], case["d"], case["page"]
    rows = [[-(-t // P) for t in total]] + ([] if spare is None else [[-(-t // P) for t in spare]])
    pages = sum(sum(r) for r in rows) + 3
    perm, at, tables = torch.randperm(pages, generator=g, device=DEV).to(torch.int32), 0, []
    for need in rows:
        table = torch.zeros(len(need), max(max(need), 1), dtype=torch.int32, device=DEV)
        for b, n in enumerate(need):
            table[b, :n] = perm[at:at + n]
            at += n
        tables.append(table)
    table, extra = tables[0], None
    if q is not None:                       # keys that carry a query: (flat index, value) pairs
        idx, val = [], []
        for b, (t, of) in enumerate(zip(total, q)):
            j = torch.randint(0, t, (max(1, t // 100),), generator=g, device=DEV).unique()
            h = torch.randint(0, kv, (j.numel(),), generator=g, device=DEV)
            r = torch.randint(0, of.shape[0], (j.numel(),), generator=g, device=DEV)
            base = (table[b].long()[j // P] * kv + h) * P + j % P
            idx.append((base[:, None] * d + torch.arange(d, device=DEV)).reshape(-1))
            val.append(of[r, h * (case["H"] // kv)].float().reshape(-1))
        extra = (torch.cat(idx), torch.cat(val))
    k, ks = _pool(case, g, pages, extra)
    v, vs = (None, None) if case["op"] == "weights" else _pool(case, g, pages)
    return {"k": k, "v": v, "ks": ks, "vs": vs, "table": table, "dst": tables[-1], "pages": pages}


def prepare(case, seed):
    g = _gen(seed)
    if case["op"] == "linear":
        rows, k, n = case["rows"], case["k"], case["n"]
        x = (_randn(g, rows, k) * torch.exp2(_randn(g, k) * 0.5)).to(torch.bfloat16)        # some channels are larger than others
        w, ws = _quantise4(_randn(g, n, k) * (torch.exp2(_randn(g, n) * 0.5) / math.sqrt(k))[:, None])
        return {"case": case, "x": x, "w": w, "ws": ws, "a": torch.empty(rows, k // 2, dtype=torch.uint8, device=DEV),
                "as": torch.empty(rows, k // GROUP, dtype=torch.uint8, device=DEV), "y": torch.empty(rows, n, dtype=torch.bfloat16, device=DEV)}
    new, ctx, budget = lengths(case)
    H, kv, d, T = case["H"], case["kv"], case["d"], sum(new)
    off = [0]
    for n in new:
        off.append(off[-1] + n)
    s = {"case": case, "off": off, "off_dev": torch.tensor(off, dtype=torch.int64, device=DEV),
         "lens": torch.tensor(ctx, dtype=torch.int32, device=DEV), "max_len": max(ctx), "max_n": max(new), "T": T}
    if case["op"] == "append":
        qkv = _randn(g, T, (H + 2 * kv) * d)
        qkv[:, H * d:] *= torch.exp2(_randn(g, 2 * kv) * 0.5).repeat_interleave(d)
        s["qkv"] = qkv.to(torch.bfloat16)
        s |= _cache(case, g, [c + n for c, n in zip(ctx, new)])
        n_pos = max(c + n for c, n in zip(ctx, new)) + 8
        half = case["rot"] // 2
        s["cos"] = s["sin"] = None
        if half:
            angle = torch.arange(n_pos, device=DEV, dtype=torch.float64)[:, None] * (
                500000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half))[None, :]
            s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["q_out"] = torch.empty(T, H, d, dtype=torch.bfloat16, device=DEV)
        return s
    if case["op"] == "evict":
        s |= _cache(case, g, ctx, spare=[min(c, m) for c, m in zip(ctx, budget)])
        s |= {"budget": torch.tensor(budget, dtype=torch.int32, device=DEV), "max_budget": max(budget)}
        # a few tokens draw most of the weight, and a tenth has drawn none yet
        w = torch.exp(_randn(g, case["B"], kv, s["max_len"]) * 2)
        s["weights"] = w * (torch.rand(w.shape, generator=g, device=DEV) < 0.9)
        s["new_lens"] = torch.empty(case["B"], dtype=torch.int32, device=DEV)
        s["kept"] = torch.full((case["B"], kv, s["max_budget"]), -1, dtype=torch.int32, device=DEV)
        s["new_weights"] = torch.zeros(case["B"], kv, s["max_budget"], device=DEV)
        return s
    s["q"] = _randn(g, T, H, d).to(torch.bfloat16)
    s |= _cache(case, g, ctx, [s["q"][a:b] for a, b in zip(off, off[1:])])
    if case["op"] == "attend":
        s |= {"out": torch.empty(T, H, d, dtype=torch.bfloat16, device=DEV), "lse": torch.empty(T, H, device=DEV)}
        return s
    # what the attention before has left: the logarithms of its denominators; and what the tokens had drawn until then
    x, have = _logits(s)
    s["lse"] = torch.logsumexp(x, dim=-1).permute(0, 2, 1, 3).reshape(x.shape[0], x.shape[2], H)[have].contiguous()
    s["old"] = torch.exp(_randn(g, case["B"], kv, s["max_len"]))
    s["weights"] = torch.zeros_like(s["old"])
    return s


# ---- the plain form --------------------------------------------------------------------------------------------------

def _heads_first(pool, case):
    return pool.transpose(1, 2) if case["layout"] == "NHD" else pool        # [pages][kv][page][bytes or elements]


def _padded(s):
    """Row b, column r: the packed index of request b's r-th new token, and whether it has one."""
    r = torch.arange(s["max_n"], device=DEV)
    n = s["off_dev"][1:] - s["off_dev"][:-1]
    have = r[None, :] < n[:, None]
    return torch.where(have, s["off_dev"][:-1, None] + r[None, :], 0), have


def _rotate(x, pos, s):
    """[T, heads, d] in 32 bits, rotated to the positions [T]."""
    rot, half = s["case"]["rot"], s["case"]["rot"] // 2
    if not rot:
        return x
    c, sn = s["cos"][pos][:, None, :], s["sin"][pos][:, None, :]
    y = x.clone()
    if s["case"]["style"] == "half":
        a, b = x[..., :half], x[..., half:rot]
        y[..., :half], y[..., half:rot] = a * c - b * sn, b * c + a * sn
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * sn, b * c + a * sn
    return y


def _plain_append(s):
    case = s["case"]
    H, kv, d, P, T = case["H"], case["kv"], case["d"], case["page"], s["T"]
    start = s["lens"].long()
    seq = torch.repeat_interleave(torch.arange(start.numel(), device=DEV), s["off_dev"][1:] - s["off_dev"][:-1], output_size=T)
    pos = torch.arange(T, device=DEV) - s["off_dev"][seq] + start[seq]
    page = s["table"].long()[seq, pos // P]
    x = s["qkv"].float()
    s["q_out"].copy_(_rotate(x[:, :H * d].reshape(T, H, d), pos, s))
    k = _rotate(x[:, H * d:(H + kv) * d].reshape(T, kv, d), pos, s)
    v = x[:, (H + kv) * d:].reshape(T, kv, d)
    for pool, scales, y in ((s["k"], s["ks"], k), (s["v"], s["vs"], v)):
        codes, scale = _quantise4(y)
        _heads_first(pool, case)[page, :, pos % P] = codes
        scales[page, :, pos % P] = scale
    return _appended(s)


def _appended(s):
    return {"k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"], "q": s["q_out"]}


def _gathered(s, name, dtype=torch.float32):
    """[B][kv][tokens][d] of one pool in 32 bits (or more), all pages of the block table."""
    case, table = s["case"], s["table"].long()
    x = _heads_first(s[name], case)[table]                                                      # [B][width][kv][P][..]
    if case["cache"] == "mx4":
        x = _values4(x, s[name + "s"][table], dtype)
    elif case["cache"] == "e4m3":
        x = x.contiguous().view(torch.float8_e4m3fn).to(dtype) * s[name + "s"][table].to(dtype).repeat_interleave(BLOCK, dim=3)[..., None]
    else:
        x = x.to(dtype)
    return x.transpose(1, 2).reshape(x.shape[0], case["kv"], -1, case["d"])


def _logits(s):
    """[B][kv][rows][G][keys] in 32 bits, minus infinity where a row sees no key, and which padded rows there are."""
    case = s["case"]
    H, kv, d = case["H"], case["kv"], case["d"]
    G, L = H // kv, s["max_len"]
    at, have = _padded(s)
    B, N = at.shape
    q = s["q"].float()[at].view(B, N, kv, G, d).permute(0, 2, 1, 3, 4).reshape(B, kv, N * G, d)
    x = torch.matmul(q, _gathered(s, "k")[:, :, :L].transpose(2, 3)).mul_(1 / math.sqrt(d)).view(B, kv, N, G, L)
    pos = (s["lens"].long() - (s["off_dev"][1:] - s["off_dev"][:-1]))[:, None] + torch.arange(N, device=DEV)     # [B][N]
    j = torch.arange(L, device=DEV)
    hide = (j > pos[..., None]) | ~have[..., None]
    if case["window"]:
        hide |= j <= pos[..., None] - case["window"]
    return x.masked_fill_(hide[:, None, :, None, :], -math.inf), have


def _plain_attend(s):
    case = s["case"]
    x, have = _logits(s)
    B, kv, N, G, L = x.shape
    m = x.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = x.sub_(m).exp_()
    l = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.view(B, kv, N * G, L), _gathered(s, "v")[:, :, :L]).view(B, kv, N, G, case["d"])
    o = torch.where(l > 0, o / l, torch.zeros_like(o)).permute(0, 2, 1, 3, 4).reshape(B, N, case["H"], case["d"])
    lse = (m + l.log()).squeeze(-1).permute(0, 2, 1, 3).reshape(B, N, case["H"])
    return {"out": o[have].to(torch.bfloat16), "lse": lse[have]}


def _plain_weights(s):
    x, have = _logits(s)
    B, kv, N, G, L = x.shape
    at, _ = _padded(s)
    lse = s["lse"][at].view(B, N, kv, G).permute(0, 2, 1, 3)[..., None]
    w = x.sub_(torch.where(lse == -math.inf, torch.zeros_like(lse), lse)).exp_().sum(dim=(2, 3))
    lens = s["lens"].long()[:, None, None]
    older = lens - (s["off_dev"][1:] - s["off_dev"][:-1])[:, None, None]                        # tokens that were there before
    j = torch.arange(L, device=DEV)
    w = torch.where(j < older, s["old"] + w, w)
    s["weights"].copy_(torch.where(j < lens, w, s["weights"]))
    return {"weights": s["weights"]}


def _plain_evict(s):
    case = s["case"]
    kv, P, L, width = case["kv"], case["page"], s["max_len"], s["max_budget"]
    B = case["B"]
    lens, budget = s["lens"].long(), s["budget"].long()
    first = budget.clamp(max=case["sinks"])
    last = (budget - first).clamp(max=case["recent"])
    n = torch.minimum(lens, budget)
    j = torch.arange(L, device=DEV)
    held = (j < first[:, None]) | (j >= (lens - last)[:, None])
    key = torch.where(held[:, None, :], math.inf, s["weights"])
    key = torch.where((j < lens[:, None])[:, None, :], key, -math.inf)
    order = key.sort(dim=-1, descending=True, stable=True).indices                              # equal weights: the earlier token
    keep = torch.zeros(B, kv, L, dtype=torch.bool, device=DEV)
    keep.scatter_(2, order, (j < n[:, None])[:, None, :].expand(B, kv, L))
    b, h, src = keep.nonzero(as_tuple=True)                                                     # in the tokens' order
    slot = (keep.cumsum(dim=2) - 1)[b, h, src]
    s["kept"][b, h, slot] = src.to(torch.int32)
    s["new_weights"][b, h, slot] = s["weights"][b, h, src]
    s["new_lens"].copy_(n)
    frm, to = s["table"].long()[b, src // P], s["dst"].long()[b, slot // P]
    for pool, scales in ((s["k"], s["ks"]), (s["v"], s["vs"])):
        view = _heads_first(pool, case)
        x = view[frm, h, src % P]
        if case["cache"] == "mx4":
            scales[to, h, slot % P] = scales[frm, h, src % P]
        elif case["cache"] == "e4m3":                                                           # a block takes the largest scale that comes into it
            mine = scales[frm, h, src % P // BLOCK]
            blocks = torch.zeros(B, kv, -(-width // BLOCK), device=DEV)
            line = (b * kv + h) * blocks.shape[2] + slot // BLOCK
            blocks.view(-1).scatter_reduce_(0, line, mine, "amax")
            new = blocks.view(-1)[line]
            scales[to, h, slot % P // BLOCK] = new
            x = (x.view(torch.float8_e4m3fn).float() * (mine / new)[:, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        view[to, h, slot % P] = x
    return _evicted(s)


def _evicted(s):
    """The cache, and what is known of it: 8-bit codes as the values that they stand for, beside their scales."""
    out = {"k": s["k"], "v": s["v"], "kept": s["kept"], "weights": s["new_weights"], "lens": s["new_lens"]}
    if s["case"]["cache"] == "e4m3":
        out |= {"k": s["k"].view(torch.float8_e4m3fn), "v": s["v"].view(torch.float8_e4m3fn)}
    return out if s["case"]["cache"] == "bf16" else out | {"ks": s["ks"], "vs": s["vs"]}


def _plain_linear(s):
    a = _values4(*_quantise4(s["x"].float()))
    s["y"].copy_(torch.matmul(a, _values4(s["w"], s["ws"]).t()))
    return {"y": s["y"]}


# ---- the framework's operators ---------------------------------------------------------------------------------------

def _plan(s):
    """What a program makes once for a model and its batch sizes: the cache's description, and a workspace where one is needed."""
    import paper_2603_02631_amd as sp
    case = s["case"]
    kv, d, P = case["kv"], case["d"], case["page"]
    head, token = (P * d, d) if case["layout"] == "HND" else (d, kv * d)
    kind = {"mx4": sp.SP_CACHE_MX4, "e4m3": sp.SP_CACHE_E4M3, "bf16": sp.SP_CACHE_BF16}[case["cache"]]
    desc = sp.CacheDesc(case["H"], kv, d, kind, s["pages"], P, kv * P * d, head, token)
    plan = {"desc": desc, "off": sp.host_offsets(s["off"])}
    if case["op"] == "attend":
        size = sp.sp_attend_workspace(desc, plan["off"], case["B"], s["max_len"])
        plan["ws"] = torch.empty(max(size, 256), dtype=torch.uint8, device=DEV)
    return plan


def _own_run(s):
    import paper_2603_02631_amd as sp
    case = s["case"]
    if case["op"] == "linear":
        rows, k, n = case["rows"], case["k"], case["n"]
        sp.sp_mx4_quantise(s["x"], rows, k, s["a"], s["as"])
        sp.sp_mx4_matmul(s["a"], s["as"], rows, s["w"], s["ws"], n, k, s["y"])
        return {"y": s["y"]}
    if "plan" not in s:
        s["plan"] = _plan(s)
    p = s["plan"]
    H, kv, d = case["H"], case["kv"], case["d"]
    if case["op"] == "append":
        q, k, v = s["qkv"].split([H * d, kv * d, kv * d], dim=1)
        sp.sp_cache_append(p["desc"], k, v, p["off"], s["off_dev"], s["lens"], s["table"], s["k"], s["v"], s["ks"], s["vs"],
                           q=q, q_out=s["q_out"], cos=s["cos"], sin=s["sin"], rot_dim=case["rot"],
                           rot_style=sp.SP_ROTATE_HALF if case["style"] == "half" else sp.SP_ROTATE_PAIRS)
        return _appended(s)
    if case["op"] == "attend":
        sp.sp_attend(p["desc"], s["q"], p["off"], s["off_dev"], s["lens"], s["max_len"], s["table"], s["k"], s["v"], s["ks"], s["vs"],
                     1 / math.sqrt(d), s["out"], s["lse"], p["ws"], causal=1, window=case["window"])
        return {"out": s["out"], "lse": s["lse"]}
    if case["op"] == "weights":
        sp.sp_attend_weights(p["desc"], s["q"], p["off"], s["off_dev"], s["lens"], s["max_len"], s["table"], s["k"], s["ks"], 1 / math.sqrt(d),
                             s["lse"], s["old"], s["weights"], causal=1, window=case["window"])
        return {"weights": s["weights"]}
    sp.sp_cache_evict(p["desc"], s["lens"], s["max_len"], s["budget"], s["max_budget"], case["sinks"], case["recent"], s["weights"],
                      s["table"], s["dst"], s["k"], s["v"], s["ks"], s["vs"], s["new_lens"], s["kept"], s["new_weights"])
    return _evicted(s)


def run(state):
    if own:
        return _own_run(state)
    return {"append": _plain_append, "attend": _plain_attend, "weights": _plain_weights, "evict": _plain_evict,
            "linear": _plain_linear}[state["case"]["op"]](state)


# ---- 64 bits ---------------------------------------------------------------------------------------------------------

def _nearest4(x):
    """What rows of 64-bit values become in 4 bits: the nearest multiple of the spacing at their place, group by group."""
    y = x.view(*x.shape[:-1], -1, GROUP)
    top = y.abs().amax(dim=-1, keepdim=True).clamp(min=2.0 ** -90)
    s = torch.exp2(torch.ceil(torch.log2(top / 6.0) - 1e-13).clamp(min=FLOOR))
    z = y / s
    step = torch.where(z.abs() < 2, 0.5, torch.where(z.abs() < 4, 1.0, 2.0))
    return (torch.round(z / step) * step * s).view(x.shape)


def _exact_append(s):
    """Rotated queries as products of complex numbers; bytes have no nearer value."""
    case = s["case"]
    H, d, rot = case["H"], case["d"], case["rot"]
    x = s["qkv"][:, :H * d].double().view(s["T"], H, d).clone()
    starts = s["lens"].tolist()
    for b, (lo, hi) in enumerate(zip(s["off"], s["off"][1:])):
        if rot:
            here = slice(starts[b], starts[b] + hi - lo)
            turn = torch.complex(s["cos"][here].double(), s["sin"][here].double())[:, None, :]
            part = x[lo:hi, :, :rot]
            if case["style"] == "half":
                z = torch.complex(part[..., :rot // 2].contiguous(), part[..., rot // 2:].contiguous()) * turn
                part.copy_(torch.cat([z.real, z.imag], dim=-1))
            else:
                z = torch.view_as_complex(part.reshape(*part.shape[:-1], rot // 2, 2).contiguous()) * turn
                part.copy_(torch.view_as_real(z).reshape(part.shape))
    return {"k": None, "v": None, "ks": None, "vs": None, "q": x}


def _each_head(s):
    """(request, head, its logits in 64 bits, the group's values or None) one by one."""
    case = s["case"]
    H, kv, d = case["H"], case["kv"], case["d"]
    lens = s["lens"].tolist()
    for b, (lo, hi) in enumerate(zip(s["off"], s["off"][1:])):
        one = {**s, "table": s["table"][b:b + 1, :-(-lens[b] // case["page"])]}
        k = _gathered(one, "k", torch.float64)[0, :, :lens[b]]
        v = None if s["v"] is None else _gathered(one, "v", torch.float64)[0, :, :lens[b]]
        pos = torch.arange(lens[b] - (hi - lo), lens[b], device=DEV)[:, None]
        j = torch.arange(lens[b], device=DEV)[None, :]
        seen = (j <= pos) & ((j > pos - case["window"]) if case["window"] else True)
        for h in range(H):
            g = h // (H // kv)
            x = (s["q"][lo:hi, h].double() @ k[g].T) / math.sqrt(d)
            yield b, h, torch.where(seen, x, torch.full_like(x, -math.inf)), None if v is None else v[g]


def _exact_attend(s):
    case = s["case"]
    out = torch.zeros(s["T"], case["H"], case["d"], dtype=torch.float64, device=DEV)
    lse = torch.full((s["T"], case["H"]), -math.inf, dtype=torch.float64, device=DEV)
    for b, h, x, v in _each_head(s):
        here = slice(s["off"][b], s["off"][b + 1])
        lse[here, h] = torch.logsumexp(x, dim=1)
        out[here, h] = torch.softmax(x, dim=1) @ v
    return {"out": out, "lse": lse}


def _exact_weights(s):
    case = s["case"]
    w = s["weights"].double()
    for b, n in enumerate(s["lens"].tolist()):
        before = n - (s["off"][b + 1] - s["off"][b])
        w[b, :, :n] = 0
        w[b, :, :before] = s["old"][b, :, :before].double()
    for b, h, x, _ in _each_head(s):
        z = s["lse"][s["off"][b]:s["off"][b + 1], h].double()
        w[b, h // (case["H"] // case["kv"]), :x.shape[1]] += torch.exp(x - z[:, None]).sum(dim=0)
    return {"weights": w}


def _exact_evict(s):
    """Line by line: the floats are what they were, 8-bit codes those of the block's scale. Bytes have no nearer value."""
    case = s["case"]
    P, kind = case["page"], case["cache"]
    width = torch.float64
    pools = {n: _heads_first(s[n].view(torch.float8_e4m3fn) if kind == "e4m3" else s[n], case) for n in ("k", "v")}
    out = {n: p.to(width) if kind != "mx4" else None for n, p in pools.items()}
    scales = {n: s[n].to(width) for n in ("ks", "vs")} if kind == "e4m3" else {}
    weights = s["new_weights"].double()
    for b, (n, m) in enumerate(zip(s["lens"].tolist(), s["budget"].tolist())):
        lo = min(case["sinks"], m)
        hi = n - min(case["recent"], m - lo)
        for h in range(case["kv"]):
            at = torch.arange(n, device=DEV)
            if n > m:
                w = s["weights"][b, h, lo:hi].double()
                rest = m - lo - (n - hi)
                order = torch.argsort(-w, stable=True)[:rest] + lo
                at = torch.cat([at[:lo], order.sort().values, at[hi:]])
            weights[b, h, :at.numel()] = s["weights"][b, h, at].double()
            if kind == "mx4":
                continue
            frm = s["table"][b].long()[at // P]
            for name in ("k", "v"):
                x = pools[name][frm, h, at % P].to(width)
                for i in range(0, at.numel() if kind == "e4m3" else 0, BLOCK):
                    mine = s[name + "s"][frm[i:i + BLOCK], h, at[i:i + BLOCK] % P // BLOCK].double()
                    new = mine.max()
                    scales[name + "s"][s["dst"][b, i // P].long(), h, i % P // BLOCK] = new
                    y = x[i:i + BLOCK] * (mine / new)[:, None]
                    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
                    x[i:i + BLOCK] = torch.round(y / step) * step
                slot = torch.arange(at.numel(), device=DEV)
                out[name][s["dst"][b].long()[slot // P], h, slot % P] = x
    if case["layout"] == "NHD" and kind != "mx4":
        out = {n: x.transpose(1, 2).contiguous() for n, x in out.items()}
    return {**out, **scales, "kept": None, "weights": weights, "lens": None}


def _exact_linear(s):
    w = _values4(s["w"], s["ws"], torch.float64)
    return {"y": _nearest4(s["x"].double()) @ w.T}


def exact(case, seed):
    """What run() returns, in 64 bits from the definition."""
    if case["op"] == "evict" and case["cache"] == "e4m3" and case["B"] * case["kv"] * case["budget_hi"] > 400000:
        return None                         # block by block it would take too long
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "weights": _exact_weights, "evict": _exact_evict,
            "linear": _exact_linear}[case["op"]](s)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    if case["op"] == "linear":
        rows, k, n = float(case["rows"]), case["k"], case["n"]
        return {"bytes": 2 * rows * k + n * k * 17 / 32 + 2 * rows * n, "flops": 2 * rows * n * k}
    new, ctx, budget = lengths(case)
    H, kv, d = case["H"], case["kv"], case["d"]
    T = sum(new)
    half = kv * {"mx4": d * 17 / 32, "e4m3": d + 4 / BLOCK, "bf16": 2.0 * d}[case["cache"]]     # a token's keys, or its values
    if case["op"] == "append":
        # projections in, rotated queries out, the table's rows, the cache's new tokens
        return {"bytes": T * ((2 * H + 2 * kv) * d * 2.0 + 4.0 * case["rot"] + 2 * half), "flops": 3.0 * T * (H + kv) * max(case["rot"], 1)}
    if case["op"] == "evict":
        # every weight, kept tokens in and out
        kept = sum(min(c, m) for c, m in zip(ctx, budget))
        return {"bytes": 4.0 * kv * sum(ctx) + kept * (4 * half + 8.0 * kv), "flops": 1.0 * kv * sum(ctx)}
    window = case["window"]
    seen = sum(min(c, window + n - 1) if window else c for n, c in zip(new, ctx))
    pairs = sum(visible(n, c, window) for n, c in zip(new, ctx))
    if case["op"] == "weights":
        # keys, queries and their denominators, old and new weights
        return {"bytes": seen * half + T * H * (2.0 * d + 4.0) + 8.0 * kv * sum(ctx), "flops": 2.0 * d * H * pairs}
    return {"bytes": seen * 2 * half + T * H * (4.0 * d + 4.0), "flops": 4.0 * d * H * pairs}
