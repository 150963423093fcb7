"""The lookahead example: the operators together, as a program runs them. Its pages hold what the definition says, its attention
follows from them, the importance pass reads the same pages, and its tokens are the logits' largest."""
from __future__ import annotations

import os
import sys

import numpy as np
import pytest
import torch

import operator_util as ou
import paper_2603_02631_amd as sp

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def gathered(m, pool, n, scales=None):
    """[tokens][kv][d] in 64 bits of one layer's pool."""
    x = pool.view(torch.float8_e4m3fn).double() if scales is not None else pool.double()
    if scales is not None:
        x = x * scales.double().repeat_interleave(sp.SP_CACHE_BLOCK, dim=2)[..., None]
    x = x[m.table[0].long()].transpose(1, 2)
    return x.reshape(-1, x.shape[2], x.shape[3])[:n].cpu().numpy()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("L", [1024, 700])
def test_lookahead_pass(cache, L):
    import lookahead
    out = lookahead.run("tiny", cache, L)
    m, w = out["model"], out["model"].w
    torch.cuda.synchronize()
    for token, (lp, entropy, logits) in zip(out["tokens"].tolist(), out["chosen"]):
        x = logits[0].double().cpu().numpy()
        want_lp, want_h, ids, lps, _ = ou.logprobs(x, token, 1)
        assert token == ids[0]
        assert abs(lp.item() - lps[0]) < 1e-4 and abs(entropy.item() - want_h) < 1e-3
    # the last lookahead step's attention, recomputed from the pages and the queries it used
    total = L + w.n_q
    for layer in range(w.n_layers):
        k = gathered(m, m.k[layer], total, m.ks[layer])
        v = gathered(m, m.v[layer], total, m.vs[layer])
        assert np.isfinite(k).all() and np.isfinite(v).all()
        q = out["queries"][layer][:, -1].contiguous()                       # [H][d]
        got = torch.empty(1, w.n_q_heads, w.head_dim, dtype=torch.bfloat16, device="cuda:0")
        sp.sp_attend(m.desc, q, [0, 1], torch.tensor([0, 1], device="cuda:0"), torch.tensor([total], dtype=torch.int32, device="cuda:0"), total,
                     m.table, m.k[layer], m.v[layer], m.ks[layer], m.vs[layer], w.scale, got, None, m.ws)
        got = got[0].double().cpu().numpy()
        for h in range(w.n_q_heads):
            o, z, A, S = ou.attend(q[h].double().cpu().numpy(), k[:, h // w.group], v[:, h // w.group], w.scale, 0, total)
            dx = (w.head_dim + 4) * 2.0 ** -24 * S
            assert np.all(np.abs(got[h] - o) <= (2.0 ** -8 + 2 * dx + 2.0 ** -12) * A + 2.0 ** -8 * np.abs(o))
    if cache == "bf16":
        # the importance pass on the same keys laid out densely
        keys = [torch.from_numpy(np.ascontiguousarray(gathered(m, m.k[i], L).transpose(1, 0, 2))).to(torch.bfloat16).cuda() for i in range(w.n_layers)]
        desc = sp.ScoreDesc(w.n_layers, w.n_q_heads, w.n_kv_heads, w.head_dim, w.n_q, w.scale, sp.SP_LAYER_MAX, w.head_dim, L * w.head_dim)
        scores = torch.empty(L, device="cuda:0")
        sp.sp_score(desc, out["queries"], keys, L, scores, torch.empty(sp.sp_score_workspace(desc, L, 1), dtype=torch.uint8, device="cuda:0"))
        np.testing.assert_allclose(out["scores"].cpu().numpy(), scores.cpu().numpy(), rtol=1e-5)
        assert out["chunks"].numel() == sp.sp_keep_count(-(-L // w.chunk), w.keep_num, w.keep_den)
