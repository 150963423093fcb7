"""A draft model's lookahead pass, from prompt tokens to kept chunks, on the library's operators.

A decoder with random weights (the shapes of a configuration of ``synth``) reads a prompt in chunks and then picks lookahead
tokens one by one; per layer sp_cache_append rotates and stores keys and values in a paged cache and sp_attend attends over
it, and sp_logprobs picks the next token off the logits. The queries of the lookahead tokens and the very pages that the pass
has filled go to sp_score_paged, and its scores to sp_select. Norms and the MLP's activation are torch's, and so are the projections, unless they are
asked for in 4 bits: then sp_mx4_quantise brings weights (once) and activations to microscaled 4-bit elements and sp_mx4_matmul multiplies them.
With a budget the cache shrinks to it after the prompt: sp_attend_weights adds up what every cached token draws while the prompt is read, and
sp_cache_evict moves those that drew the most, with the first and the last ones, to other pages, on which the lookahead goes on.

    python examples/lookahead.py                          # the "tiny" configuration
    python examples/lookahead.py --workload llama1b-8k
    python examples/lookahead.py --cache e4m3             # 8-bit pages: the lookahead alone (the importance pass reads bf16 pages)
    python examples/lookahead.py --cache mx4 --projections mx4 --budget 256      # 4-bit pages and projections, at most 256 prompt tokens kept
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time
from dataclasses import dataclass

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2603_02631_amd as sp  # noqa: E402
import synth  # noqa: E402

DEV = "cuda:0"
PAGE = 512          # tokens of a page; sp_score_paged takes multiples of 512
VOCAB = 32000
CHUNK = 2048        # prompt tokens of one pass
SINKS, RECENT = 4, 32       # first and last tokens that an eviction keeps in any case


class Projection:
    """x @ w for w [in][out], in bf16 or with both in microscaled 4-bit elements."""

    def __init__(self, w, four: bool):
        self.w = None if four else w
        if four:
            self.K, self.N = w.shape
            self.codes, self.scales = quantised(w.t().contiguous())

    def __call__(self, x):
        if self.w is not None:
            return x @ self.w
        codes, scales = quantised(x)
        y = torch.empty(x.shape[0], self.N, dtype=torch.bfloat16, device=DEV)
        sp.sp_mx4_matmul(codes, scales, x.shape[0], self.codes, self.scales, self.N, self.K, y)
        return y


def quantised(x):
    n, k = x.shape
    codes, scales = torch.empty(n, k // 2, dtype=torch.uint8, device=DEV), torch.empty(n, k // sp.SP_MX4_GROUP, dtype=torch.uint8, device=DEV)
    sp.sp_mx4_quantise(x, n, k, codes, scales)
    return codes, scales


@dataclass
class Layer:
    qkv: Projection
    out: Projection
    up: Projection
    down: Projection


def rms(x):
    y = x.float()
    return (y * torch.rsqrt(y.square().mean(dim=-1, keepdim=True) + 1e-6)).to(torch.bfloat16)


class Draft:
    """Weights, paged cache, rotation tables and workspaces of one request."""

    def __init__(self, w, cache: str, prompt_len: int, seed: int = 0, projections: str = "bf16", budget: int = 0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        H, kv, d = w.n_q_heads, w.n_kv_heads, w.head_dim
        hidden = H * d
        self.w, self.prompt_len, self.total = w, prompt_len, prompt_len + w.n_q

        def weight(n, m, gain=1.0):
            return Projection((torch.randn(n, m, generator=g, device=DEV) * (gain / math.sqrt(n))).to(torch.bfloat16), projections == "mx4")

        self.embed = torch.randn(VOCAB, hidden, generator=g, device=DEV).to(torch.bfloat16)
        self.layers = [Layer(weight(hidden, (H + 2 * kv) * d, 2.0), weight(hidden, hidden), weight(hidden, 2 * hidden), weight(2 * hidden, hidden))
                       for _ in range(w.n_layers)]
        self.head = weight(hidden, VOCAB, 3.0)
        self.budget = budget if 0 < budget < prompt_len else 0
        width = -(-self.total // PAGE)
        pages = width + (-(-(self.budget + w.n_q) // PAGE) if self.budget else 0)       # with those that an eviction fills
        kind, dt, elems = {"bf16": (sp.SP_CACHE_BF16, torch.bfloat16, d), "e4m3": (sp.SP_CACHE_E4M3, torch.uint8, d), "mx4": (sp.SP_CACHE_MX4, torch.uint8, d // 2)}[cache]
        self.desc = sp.CacheDesc(H, kv, d, kind, pages, PAGE, kv * PAGE * d, PAGE * d, d)
        self.k, self.v = ([torch.zeros(pages, kv, PAGE, elems, dtype=dt, device=DEV) for _ in self.layers] for _ in range(2))

        def scales():
            if cache == "e4m3":
                return torch.zeros(pages, kv, PAGE // sp.SP_CACHE_BLOCK, device=DEV)
            return torch.zeros(pages, kv, PAGE, d // sp.SP_MX4_GROUP, dtype=torch.uint8, device=DEV) if cache == "mx4" else None

        self.ks, self.vs = ([scales() for _ in self.layers] for _ in range(2))
        order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)[None, :]
        self.table, self.spare = order[:, :width].contiguous(), order[:, width:].contiguous()
        self.gone = 0       # tokens that an eviction has dropped: a new one's position is that many behind its slot
        self.drawn = [torch.zeros(1, kv, prompt_len, device=DEV) for _ in self.layers] if self.budget else None
        half = d // 2
        angle = torch.arange(self.total, device=DEV, dtype=torch.float64)[:, None] * (
            500000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half))[None, :]
        self.cos, self.sin = angle.cos().float(), angle.sin().float()
        sizes = [sp.sp_attend_workspace(self.desc, [0, n], 1, self.total) for n in {1, min(CHUNK, prompt_len), prompt_len % CHUNK or 1}]
        self.ws = torch.empty(max(max(sizes), 256), dtype=torch.uint8, device=DEV)
        self.ws_lp = torch.empty(max(sp.sp_logprobs_workspace(1, VOCAB, 1), 256), dtype=torch.uint8, device=DEV)

    def forward(self, ids, start: int, queries=None):
        """Hidden states of `ids` behind `start` tokens of context; appends every layer's rotated queries to `queries`. While a prompt that will be
        cut is read, what its tokens draw is added up."""
        w, n = self.w, ids.numel()
        H, kv, d = w.n_q_heads, w.n_kv_heads, w.head_dim
        off = sp.host_offsets([0, n])
        off_dev = torch.tensor([0, n], dtype=torch.int64, device=DEV)
        start_dev = torch.tensor([start], dtype=torch.int32, device=DEV)
        lens = start_dev + n
        positions = torch.arange(start + self.gone, start + self.gone + n, dtype=torch.int32, device=DEV) if self.gone else None
        adding = self.drawn is not None and not self.gone
        x = self.embed[ids.long()]
        for i, layer in enumerate(self.layers):
            q, k, v = layer.qkv(rms(x)).split([H * d, kv * d, kv * d], dim=1)
            turned = torch.empty(n, H, d, dtype=torch.bfloat16, device=DEV)
            attended = torch.empty_like(turned)
            lse = torch.empty(n, H, device=DEV) if adding else None
            sp.sp_cache_append(self.desc, k, v, off, off_dev, start_dev, self.table, self.k[i], self.v[i], self.ks[i], self.vs[i],
                               q=q, q_out=turned, cos=self.cos, sin=self.sin, rot_dim=d, positions=positions)
            sp.sp_attend(self.desc, turned, off, off_dev, lens, start + n, self.table, self.k[i], self.v[i], self.ks[i], self.vs[i],
                         w.scale, attended, lse, self.ws)
            if adding:
                sp.sp_attend_weights(self.desc, turned, off, off_dev, lens, start + n, self.table, self.k[i], self.ks[i], w.scale, lse, self.drawn[i], self.drawn[i])
            if queries is not None:
                queries[i].append(turned)
            x = x + layer.out(attended.view(n, H * d))
            x = x + layer.down(torch.nn.functional.silu(layer.up(rms(x))))
        return rms(x)

    def shrink(self):
        """The prompt's cache to its budget, every layer and kv head by itself; returns which tokens were kept, [kv heads][budget] a layer."""
        lens, budget = (torch.tensor([n], dtype=torch.int32, device=DEV) for n in (self.prompt_len, self.budget))
        new_lens, kept = torch.empty_like(lens), []
        for i, drawn in enumerate(self.drawn):
            kept.append(torch.empty(1, self.w.n_kv_heads, self.budget, dtype=torch.int32, device=DEV))
            sp.sp_cache_evict(self.desc, lens, self.prompt_len, budget, self.budget, SINKS, RECENT, drawn, self.table, self.spare, self.k[i], self.v[i], self.ks[i],
                              self.vs[i], new_lens, kept[i])
        self.table, self.spare, self.gone = self.spare, self.table, self.prompt_len - self.budget
        return [t[0] for t in kept]

    def next_token(self, hidden):
        """Greedy next token of the last row, its log probability and the entropy of the choice."""
        logits = self.head(hidden[-1:])
        token, lp = torch.empty(1, 1, dtype=torch.int32, device=DEV), torch.empty(1, 1, device=DEV)
        entropy = torch.empty(1, device=DEV)
        sp.sp_logprobs(logits, 1, VOCAB, None, 1, None, entropy, token, lp, self.ws_lp)
        return token[0], lp[0], entropy, logits


def run(workload: str = "tiny", cache: str = "bf16", prompt_len: int = 0, seed: int = 0, projections: str = "bf16", budget: int = 0):
    """The whole pass; returns what it left behind."""
    w = synth.get_config(workload)
    L = prompt_len or w.L
    m = Draft(w, cache, L, seed, projections, budget)
    g = torch.Generator(device=DEV).manual_seed(seed + 1)
    ids = torch.randint(0, VOCAB, (L,), generator=g, device=DEV, dtype=torch.int32)
    for at in range(0, L, CHUNK):
        hidden = m.forward(ids[at:at + CHUNK], at)
    kept = m.shrink() if m.budget else None
    tokens, chosen, queries = [], [], [[] for _ in m.layers]
    for step in range(w.n_q):
        token, lp, entropy, logits = m.next_token(hidden)
        tokens.append(token)
        chosen.append((lp, entropy, logits))
        hidden = m.forward(token, L - m.gone + step, queries)
    out = {"model": m, "prompt": ids, "tokens": torch.cat(tokens), "chosen": chosen}
    # one layer's queries are [head][lookahead row][element] for the importance pass
    out["queries"] = torch.stack([torch.cat(q).transpose(0, 1) for q in queries]).contiguous()
    if kept is not None:
        out["kept"] = kept
    if cache != "bf16" or m.budget:         # the importance pass reads all of the prompt's keys, in bf16
        return out
    desc = sp.ScoreDesc(w.n_layers, w.n_q_heads, w.n_kv_heads, w.head_dim, w.n_q, w.scale, sp.SP_LAYER_MAX, w.head_dim, PAGE * w.head_dim)
    scores = torch.empty(L, device=DEV)
    ws = torch.empty(sp.sp_score_workspace(desc, L, 1), dtype=torch.uint8, device=DEV)
    sp.sp_score_paged(desc, out["queries"], m.k, m.table, PAGE, w.n_kv_heads * PAGE * w.head_dim, L, scores, ws)
    C = -(-L // w.chunk)
    keep = sp.sp_keep_count(C, w.keep_num, w.keep_den)
    sel, spans = torch.empty(keep, dtype=torch.int32, device=DEV), torch.empty(keep, 2, dtype=torch.int64, device=DEV)
    n_spans = torch.empty(1, dtype=torch.int32, device=DEV)
    ws2 = torch.empty(sp.sp_select_workspace(L, w.chunk), dtype=torch.uint8, device=DEV)
    sp.sp_select(scores, L, w.pool, w.chunk, keep, sel, spans, n_spans, None, ws2)
    out |= {"scores": scores, "chunks": sel, "spans": spans[:int(n_spans.item())]}
    return out


def main() -> int:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--workload", default="tiny")
    ap.add_argument("--cache", default="bf16", choices=("bf16", "e4m3", "mx4"))
    ap.add_argument("--projections", default="bf16", choices=("bf16", "mx4"))
    ap.add_argument("--budget", type=int, default=0, help="prompt tokens that the cache keeps, 0: all")
    ap.add_argument("--prompt-len", type=int, default=0)
    args = ap.parse_args()
    run(args.workload, args.cache, args.prompt_len, 0, args.projections, args.budget)       # first calls
    torch.cuda.synchronize()
    t = time.perf_counter()
    out = run(args.workload, args.cache, args.prompt_len, 0, args.projections, args.budget)
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t) * 1e3
    lp = torch.cat([c[0] for c in out["chosen"]]).tolist()
    print(f"{args.workload}: {out['prompt'].numel()} prompt tokens, lookahead {out['tokens'].tolist()}, log probabilities "
          f"{[round(x, 2) for x in lp]}, {ms:.1f} ms with the making of the weights")
    if "kept" in out:
        print(f"kept {out['kept'][0].shape[1]} of the prompt's tokens; of the first layer and kv head {out['kept'][0][0].tolist()[:20]} ...")
    if "chunks" in out:
        print(f"kept chunks {out['chunks'].tolist()}, spans {out['spans'].tolist()}")
    return 0


if __name__ == "__main__":
    sys.exit(main())
