"""A draft model's lookahead pass, from prompt tokens to kept chunks, on the library's operators.

A decoder with random weights (the shapes of a configuration of ``synth``) reads a prompt in chunks and then picks lookahead
tokens one by one; per layer sp_cache_append rotates and stores keys and values in a paged cache and sp_attend attends over
it, and sp_logprobs picks the next token off the logits. The queries of the lookahead tokens and the very pages that the pass
has filled go to sp_score_paged, and its scores to sp_select. Projections, norms and the MLP are torch's.

    python examples/lookahead.py                          # the "tiny" configuration
    python examples/lookahead.py --workload llama1b-8k
    python examples/lookahead.py --cache e4m3             # 8-bit pages: the lookahead alone (the importance pass reads bf16 pages)
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


@dataclass
class Layer:
    qkv: torch.Tensor
    out: torch.Tensor
    up: torch.Tensor
    down: torch.Tensor


def rms(x):
    y = x.float()
    return (y * torch.rsqrt(y.square().mean(dim=-1, keepdim=True) + 1e-6)).to(torch.bfloat16)


class Draft:
    """Weights, paged cache, rotation tables and workspaces of one request."""

    def __init__(self, w, cache: str, prompt_len: int, seed: int = 0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        H, kv, d = w.n_q_heads, w.n_kv_heads, w.head_dim
        hidden = H * d
        self.w, self.prompt_len, self.total = w, prompt_len, prompt_len + w.n_q

        def weight(n, m, gain=1.0):
            return (torch.randn(n, m, generator=g, device=DEV) * (gain / math.sqrt(n))).to(torch.bfloat16)

        self.embed = torch.randn(VOCAB, hidden, generator=g, device=DEV).to(torch.bfloat16)
        self.layers = [Layer(weight(hidden, (H + 2 * kv) * d, 2.0), weight(hidden, hidden), weight(hidden, 2 * hidden), weight(2 * hidden, hidden))
                       for _ in range(w.n_layers)]
        self.head = weight(hidden, VOCAB, 3.0)
        pages = -(-self.total // PAGE)
        e4m3 = cache == "e4m3"
        self.desc = sp.CacheDesc(H, kv, d, sp.SP_CACHE_E4M3 if e4m3 else sp.SP_CACHE_BF16, pages, PAGE, kv * PAGE * d, PAGE * d, d)
        shape, dt = (pages, kv, PAGE, d), torch.uint8 if e4m3 else torch.bfloat16
        self.k = [torch.zeros(shape, dtype=dt, device=DEV) for _ in self.layers]
        self.v = [torch.zeros(shape, dtype=dt, device=DEV) for _ in self.layers]
        scales = (pages, kv, PAGE // sp.SP_CACHE_BLOCK)
        self.ks = [torch.zeros(scales, device=DEV) if e4m3 else None for _ in self.layers]
        self.vs = [torch.zeros(scales, device=DEV) if e4m3 else None for _ in self.layers]
        self.table = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)[None, :].contiguous()
        half = d // 2
        angle = torch.arange(self.total, device=DEV, dtype=torch.float64)[:, None] * (
            500000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half))[None, :]
        self.cos, self.sin = angle.cos().float(), angle.sin().float()
        sizes = [sp.sp_attend_workspace(self.desc, [0, n], 1, self.total) for n in {1, min(CHUNK, prompt_len), prompt_len % CHUNK or 1}]
        self.ws = torch.empty(max(max(sizes), 256), dtype=torch.uint8, device=DEV)
        self.ws_lp = torch.empty(max(sp.sp_logprobs_workspace(1, VOCAB, 1), 256), dtype=torch.uint8, device=DEV)

    def forward(self, ids, start: int, queries=None):
        """Hidden states of `ids` behind `start` tokens of context; appends every layer's rotated queries to `queries`."""
        w, n = self.w, ids.numel()
        H, kv, d = w.n_q_heads, w.n_kv_heads, w.head_dim
        off = sp.host_offsets([0, n])
        off_dev = torch.tensor([0, n], dtype=torch.int64, device=DEV)
        start_dev = torch.tensor([start], dtype=torch.int32, device=DEV)
        lens = start_dev + n
        x = self.embed[ids.long()]
        for i, layer in enumerate(self.layers):
            q, k, v = (rms(x) @ layer.qkv).split([H * d, kv * d, kv * d], dim=1)
            turned = torch.empty(n, H, d, dtype=torch.bfloat16, device=DEV)
            attended = torch.empty_like(turned)
            sp.sp_cache_append(self.desc, k, v, off, off_dev, start_dev, self.table, self.k[i], self.v[i], self.ks[i], self.vs[i],
                               q=q, q_out=turned, cos=self.cos, sin=self.sin, rot_dim=d)
            sp.sp_attend(self.desc, turned, off, off_dev, lens, start + n, self.table, self.k[i], self.v[i], self.ks[i], self.vs[i],
                         w.scale, attended, None, self.ws)
            if queries is not None:
                queries[i].append(turned)
            x = x + attended.view(n, H * d) @ layer.out
            x = x + torch.nn.functional.silu(rms(x) @ layer.up) @ layer.down
        return rms(x)

    def next_token(self, hidden):
        """Greedy next token of the last row, its log probability and the entropy of the choice."""
        logits = hidden[-1:] @ self.head
        token, lp = torch.empty(1, 1, dtype=torch.int32, device=DEV), torch.empty(1, 1, device=DEV)
        entropy = torch.empty(1, device=DEV)
        sp.sp_logprobs(logits, 1, VOCAB, None, 1, None, entropy, token, lp, self.ws_lp)
        return token[0], lp[0], entropy, logits


def run(workload: str = "tiny", cache: str = "bf16", prompt_len: int = 0, seed: int = 0):
    """The whole pass; returns what it left behind."""
    w = synth.get_config(workload)
    L = prompt_len or w.L
    m = Draft(w, cache, L, seed)
    g = torch.Generator(device=DEV).manual_seed(seed + 1)
    ids = torch.randint(0, VOCAB, (L,), generator=g, device=DEV, dtype=torch.int32)
    for at in range(0, L, CHUNK):
        hidden = m.forward(ids[at:at + CHUNK], at)
    tokens, chosen, queries = [], [], [[] for _ in m.layers]
    for step in range(w.n_q):
        token, lp, entropy, logits = m.next_token(hidden)
        tokens.append(token)
        chosen.append((lp, entropy, logits))
        hidden = m.forward(token, L + step, queries)
    out = {"model": m, "prompt": ids, "tokens": torch.cat(tokens), "chosen": chosen}
    # one layer's queries are [head][lookahead row][element] for the importance pass
    out["queries"] = torch.stack([torch.cat(q).transpose(0, 1) for q in queries]).contiguous()
    if cache != "bf16":
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
    ap.add_argument("--cache", default="bf16", choices=("bf16", "e4m3"))
    ap.add_argument("--prompt-len", type=int, default=0)
    args = ap.parse_args()
    run(args.workload, args.cache, args.prompt_len)       # first calls
    torch.cuda.synchronize()
    t = time.perf_counter()
    out = run(args.workload, args.cache, args.prompt_len)
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t) * 1e3
    lp = torch.cat([c[0] for c in out["chosen"]]).tolist()
    print(f"{args.workload}: {out['prompt'].numel()} prompt tokens, lookahead {out['tokens'].tolist()}, log probabilities "
          f"{[round(x, 2) for x in lp]}, {ms:.1f} ms with the making of the weights")
    if "chunks" in out:
        print(f"kept chunks {out['chunks'].tolist()}, spans {out['spans'].tolist()}")
    return 0


if __name__ == "__main__":
    sys.exit(main())
