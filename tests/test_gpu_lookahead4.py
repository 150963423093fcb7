"""The lookahead example on 4-bit pages, with 4-bit projections and with a budget for its cache: it runs, its attention follows from its pages, its projections
from their codes, and what an eviction keeps from what was drawn."""
from __future__ import annotations

import os
import sys

import numpy as np
import pytest
import torch

import mx4_util as mu
import operator_util as ou
import paper_2603_02631_amd as sp

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def gathered(m, cache, pool, scales, n):
    """[tokens][kv][d] in 64 bits of one layer's pool."""
    pages = m.table[0].long()
    x = pool[pages]
    if cache == "mx4":
        x = mu.values(mu.unpack(x.cpu().numpy()), scales[pages].cpu().numpy())
    elif cache == "e4m3":
        x = (x.view(torch.float8_e4m3fn).double() * scales[pages].double().repeat_interleave(sp.SP_CACHE_BLOCK, dim=2)[..., None]).cpu().numpy()
    else:
        x = x.double().cpu().numpy()
    return np.concatenate(list(x), axis=1).transpose(1, 0, 2)[:n]


@pytest.mark.parametrize("cache,projections,budget", [("mx4", "bf16", 0), ("mx4", "mx4", 0), ("mx4", "mx4", 200), ("bf16", "bf16", 600), ("e4m3", "mx4", 1), ("bf16", "mx4", 5000)])
@pytest.mark.parametrize("L", [1024, 700])
def test_lookahead_pass(cache, projections, budget, L):
    import lookahead
    out = lookahead.run("tiny", cache, L, 0, projections, budget)
    m, w = out["model"], out["model"].w
    torch.cuda.synchronize()
    for token, (lp, entropy, logits) in zip(out["tokens"].tolist(), out["chosen"]):
        x = logits[0].double().cpu().numpy()
        _, want_h, ids, lps, _ = ou.logprobs(x, token, 1)
        assert token == ids[0] and abs(lp.item() - lps[0]) < 1e-4 and abs(entropy.item() - want_h) < 1e-3
    # the last lookahead step's attention, recomputed from the pages and the queries it used
    total = (budget if 0 < budget < L else L) + w.n_q
    for layer in range(w.n_layers):
        k, v = (gathered(m, cache, p, s, total) for p, s in ((m.k[layer], m.ks[layer]), (m.v[layer], m.vs[layer])))
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
    if 0 < budget < L:
        for layer, kept in enumerate(out["kept"]):
            for h, tokens in enumerate(kept.cpu().numpy()):
                drawn = m.drawn[layer][0, h].cpu().numpy()
                first = min(lookahead.SINKS, budget)
                last = min(lookahead.RECENT, budget - first)
                middle = np.argsort(-drawn[first:L - last], kind="stable")[:budget - first - last] + first
                np.testing.assert_array_equal(tokens, np.sort(np.concatenate([np.arange(first), middle, np.arange(L - last, L)])))
                # rows draw one each, of all heads of the group, within the cache's own rounding of sums
                assert abs(drawn.sum(dtype=np.float64) - L * w.group) < 1e-3 * L * w.group
    else:
        assert "kept" not in out
    assert ("chunks" in out) == (cache == "bf16" and not 0 < budget < L)


def test_a_projection_is_the_product_of_its_codes():
    import lookahead
    g = torch.Generator(device="cuda:0").manual_seed(1)
    w, x = (torch.randn(*s, generator=g, device="cuda:0").bfloat16() for s in ((256, 100), (7, 256)))
    p = lookahead.Projection(w, True)
    got = p(x).double().cpu().numpy()
    a, b = (mu.values(*mu.quantise(t.double().cpu().numpy())) for t in (x, w.t()))
    want = a @ b.T
    assert np.all(np.abs(got - want) <= 256 * 2.0 ** -24 * (np.abs(a) @ np.abs(b).T) + 2.0 ** -8 * np.abs(want))
    assert torch.equal(lookahead.Projection(w, False)(x), x @ w)
