"""sp_attend_weights and sp_cache_evict against their definitions in 64 bits, for caches of all three types, and a run of the cache's operators together.

Weights. A logit is off by dx = (d + 4) 2^-24 S (S = scale sum |q||k|); scaling to units of log 2, the subtraction of the lse and the exponential add 2^-22 (|x| + |lse|) + 2^-22. So a row's part p of a weight is off by at most 2 p (dx + 2^-22 (|x| + |lse| + 1)), and the sum of n of them
(and what was there) by (n + 1) 2^-24 of itself more. Evicted tokens are moved exactly."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import mx4_util as mu
import operator_util as ou
import paper_2603_02631_amd as sp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = ["bf16", "e4m3", "mx4"]
TYPE = {"bf16": sp.SP_CACHE_BF16, "e4m3": sp.SP_CACHE_E4M3, "mx4": sp.SP_CACHE_MX4}


def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).to(DEV)


def cache(kind, kv, d, page, widths, layout="HND", pad=0, seed=0, spare=2, table_tokens=0):
    if kind == "mx4":
        return mu.Paged4(kv, d, page, widths, layout, pad, spare, seed, table_tokens)
    return ou.Paged(kv, d, page, widths, kind == "e4m3", layout, pad, spare, seed, table_tokens)


def desc_of(c, H, kind):
    return sp.CacheDesc(H, c.kv, c.d, TYPE[kind], c.n_pages, c.page, c.page_stride, c.stride_head, c.stride_token)


def filled(kind, H, kv, d, news, lens, page, layout="HND", pad=0, seed=1, max_len=0, spare=2):
    rng = np.random.default_rng([seed, d])
    c = cache(kind, kv, d, page, [max(1, -(-n // page)) for n in lens], layout, pad, seed, spare, max_len)
    held = [c.fill(b, rng.standard_normal((L, kv, d)), rng.standard_normal((L, kv, d))) for b, L in enumerate(lens)]
    off = np.concatenate([[0], np.cumsum(news)]).astype(np.int64)
    return c, held, off, ou.bf16_round(rng.standard_normal((max(int(off[-1]), 1), H, d)))


def seen_logits(H, held, off, q, lens, scale, causal, window):
    """For each request [n][H][L] logits in 64 bits, minus infinity where a row does not see a key."""
    out = []
    for b, L in enumerate(lens):
        n = int(off[b + 1] - off[b])
        rows = q[off[b]:off[b + 1]].astype(np.float64)
        kv = held[b][0].shape[1] if L else 1
        x = np.zeros((n, H, L))
        for h in range(H):
            if L:
                x[:, h] = rows[:, h] @ held[b][0][:, h // (H // kv)].T * scale
        for r in range(n):
            lo, hi = ou.seen(L, n, r, causal, window)
            x[r, :, :lo], x[r, :, hi:] = -np.inf, -np.inf
        out.append(x)
    return out


def check_weights(kind, H, kv, d, news, lens, page=64, causal=1, window=0, old=True, in_place=False, layout="HND", pad=0, max_len=None, extra=0, seed=1, dead=()):
    c, held, off, q = filled(kind, H, kv, d, news, lens, page, layout, pad, seed, max_len or 0)
    scale, B = d ** -0.5, len(lens)
    max_len = max(lens) if max_len is None else max_len
    x = seen_logits(H, held, off, q, lens, scale, causal, window)
    lse = np.full((max(int(off[-1]), 1), H), -np.inf, dtype=np.float32)
    for b in range(B):
        with np.errstate(divide="ignore", invalid="ignore"):
            if lens[b]:
                m = x[b].max(axis=-1, keepdims=True)
                m = np.where(np.isfinite(m), m, 0)
                lse[off[b]:off[b + 1]] = (m + np.log(np.exp(x[b] - m).sum(axis=-1, keepdims=True)))[..., 0]
    for t, h in dead:
        lse[t, h] = -np.inf
    rng = np.random.default_rng(seed)
    before = np.exp(rng.standard_normal((B, kv, max_len + extra))).astype(np.float32)
    weights = dev(before) if in_place else torch.full(before.shape, 7.5, device=DEV)
    old_dev = None if not old else weights if in_place else dev(before)
    sp.sp_attend_weights(desc_of(c, H, kind), dev(ou.bf16_bits(q)), off.tolist(), dev(off), dev(np.asarray(lens, dtype=np.int32)), max_len, dev(c.table),
                         dev(c.k), dev(c.ks) if kind != "bf16" else None, scale, dev(lse), old_dev, weights, causal=causal, window=window)
    torch.cuda.synchronize()
    got = weights.cpu().numpy().astype(np.float64)
    G = H // kv
    for b, L in enumerate(lens):
        n = int(off[b + 1] - off[b])
        np.testing.assert_array_equal(got[b, :, L:], before[b, :, L:] if in_place else 7.5)
        z = lse[off[b]:off[b + 1]].astype(np.float64)[..., None]
        with np.errstate(invalid="ignore"):
            p = np.where(np.isfinite(z) & np.isfinite(x[b]), np.exp(x[b] - z), 0.0)
            size = np.where(p > 0, np.abs(x[b]) + np.abs(z) + 1, 0.0)
        for h in range(kv):
            heads = slice(h * G, (h + 1) * G)
            kept = np.where(np.arange(L) < (L - n if causal else L), before[b, h, :L].astype(np.float64), 0.0) if old else np.zeros(L)
            want = kept + p[:, heads].sum(axis=(0, 1))
            if not L:
                continue
            k = np.abs(held[b][0][:, h])
            rows = np.abs(q[off[b]:off[b + 1], heads]).astype(np.float64).reshape(-1, d)
            dx = np.zeros(L)
            if rows.size:                       # the largest of all rows
                dx = (d + 4) * 2.0 ** -24 * scale * (rows @ k.T).max(axis=0)
            tol = (2 * p[:, heads] * (dx + 2.0 ** -22 * size[:, heads])).sum(axis=(0, 1)) + (n * G + 1) * 2.0 ** -24 * want
            bad = ~(np.abs(got[b, h, :L] - want) <= tol)
            assert not bad.any(), (b, h, np.flatnonzero(bad)[:5], got[b, h, :L][bad][:5], want[bad][:5], tol[bad][:5])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H,kv,d", [(4, 2, 64), (2, 2, 128), (16, 1, 64), (16, 1, 128), (6, 2, 128), (5, 5, 64)])
def test_weights_of_single_tokens(kind, H, kv, d):
    check_weights(kind, H, kv, d, [1, 1, 0, 1, 1, 1], [1, 33, 40, 64, 257, 1000], 32)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H,kv,d", [(4, 2, 64), (16, 2, 128), (3, 1, 128)])
@pytest.mark.parametrize("layout,page,pad", [("NHD", 96, 32), ("HND", 512, 0)])
def test_weights_of_rows(kind, H, kv, d, layout, page, pad):
    check_weights(kind, H, kv, d, [8, 3, 16, 64, 200, 0], [8, 700, 31, 300, 200, 5], page, layout=layout, pad=pad)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("causal,window", [(0, 0), (1, 1), (1, 7), (1, 100)])
@pytest.mark.parametrize("news", [[1, 2, 5], [80, 1, 150]])
def test_weights_with_masks(kind, causal, window, news):
    check_weights(kind, 4, 1, 64, news, [200, 45, 310], causal=causal, window=window)
    check_weights(kind, 4, 2, 128, news, [200, 45, 310], causal=causal, window=window)


@pytest.mark.parametrize("kind", KINDS)
def test_weights_of_rows_that_see_nothing_and_empty_contexts(kind):
    check_weights(kind, 4, 2, 64, [5, 3, 1, 100, 2], [2, 0, 0, 30, 2], 32)
    check_weights(kind, 4, 2, 128, [5, 40, 1], [2, 0, 30], 32, max_len=100, extra=13)
    check_weights(kind, 4, 2, 64, [2, 3], [0, 0], 32, max_len=0, extra=4)
    check_weights(kind, 4, 2, 64, [3, 50], [100, 300], dead=[(1, 2), (0, 0), (30, 3)])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("old,in_place", [(False, False), (True, True), (False, True)])
def test_weights_in_place_and_from_nothing(kind, old, in_place):
    check_weights(kind, 4, 2, 64, [1, 40, 0], [300, 500, 60], old=old, in_place=in_place, extra=9)
    check_weights(kind, 4, 2, 128, [2, 90, 0], [300, 500, 60], old=old, in_place=in_place)


@pytest.mark.parametrize("kind", KINDS)
def test_weights_of_long_contexts(kind):
    check_weights(kind, 8, 2, 64, [1], [20000])
    check_weights(kind, 8, 4, 128, [20, 1], [5000, 9000])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("causal,window", [(1, 0), (0, 0), (1, 100)])
def test_weights_of_rows_that_waves_share(kind, causal, window):
    """Enough rows for several fours of waves: four of them for one long line, two where the work of the device is twice the longest line's."""
    check_weights(kind, 16, 1, 64, [45, 3, 70], [300, 40, 500], causal=causal, window=window)
    check_weights(kind, 8, 1, 128, [101, 1, 64], [300, 40, 700], causal=causal, window=window)
    check_weights(kind, 64, 16, 128, [128, 130, 131, 127, 1], [1000, 1000, 900, 1000, 30], causal=causal, window=window)


@pytest.mark.parametrize("n", [1, 30])
@pytest.mark.parametrize("kind", KINDS)
def test_a_nan_in_an_lse_gets_out(kind, n):
    c, held, off, q = filled(kind, 4, 2, 64, [n, n], [100, 90], 32)
    lse = np.zeros((2 * n, 4), dtype=np.float32)
    lse[0, 1] = np.nan
    w = torch.zeros(2, 2, 100, device=DEV)
    sp.sp_attend_weights(desc_of(c, 4, kind), dev(ou.bf16_bits(q)), off.tolist(), dev(off), dev(np.array([100, 90], dtype=np.int32)), 100, dev(c.table), dev(c.k),
                         dev(c.ks) if kind != "bf16" else None, 0.125, dev(lse), None, w)
    got = w.cpu().numpy()
    assert np.isnan(got[0, 0, :101 - n]).all() and np.isfinite(got[0, 1]).all() and np.isfinite(got[1]).all()


@pytest.mark.parametrize("H,kv,d", [(3, 1, 64), (6, 2, 128), (5, 1, 64)])
@pytest.mark.parametrize("n", [1, 3, 15])
def test_weights_where_a_logit_is_minus_infinity(H, kv, d, n):
    """Such a key draws nothing from any row; rows that fill up a tile of them must not make NaN of it."""
    c, held, off, q = filled("bf16", H, kv, d, [n], [300], 64)
    q[..., 0] = -np.abs(q[..., 0]) - 1
    at = [0, 37, 128, 250]
    pool = c.k.copy()
    for j in at:
        for h in range(kv):
            pool[c.at(0, h, j)] = 0x7f80
    lse = np.zeros((n, H), dtype=np.float32)
    old, got = torch.rand(1, kv, 300, device=DEV), []
    for keys in (c.k, pool):
        w = torch.full((1, kv, 300), 7.5, device=DEV)
        sp.sp_attend_weights(desc_of(c, H, "bf16"), dev(ou.bf16_bits(q)), [0, n], dev(off), dev(np.array([300], dtype=np.int32)), 300, dev(c.table), dev(keys), None,
                             0.125, dev(lse), old, w, causal=0)
        got.append(w.cpu())
    want = got[0].clone()
    want[:, :, at] = old.cpu()[:, :, at]
    assert torch.equal(got[1], want)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("other", [1, 40])
def test_a_request_without_rows_keeps_its_weights_whatever_its_keys(kind, other):
    c, held, off, q = filled(kind, 4, 2, 64, [0, other, 0], [130, 90, 64], 32)
    if kind == "bf16":
        keys, scales = c.k.copy(), None
        for b, L in ((0, 130), (2, 64)):
            for j in range(L):
                for h in range(2):
                    keys[c.at(b, h, j):c.at(b, h, j) + 64] = 0x7fc0
    else:
        keys, scales = c.k, c.ks.copy()
        for b, L in ((0, 130), (2, 64)):
            scales[c.table[b, :-(-L // 32)]] = 255 if kind == "mx4" else np.nan
    before = torch.rand(3, 2, 130, device=DEV)
    w = before.clone()
    sp.sp_attend_weights(desc_of(c, 4, kind), dev(ou.bf16_bits(q)), off.tolist(), dev(off), dev(np.array([130, 90, 64], dtype=np.int32)), 130, dev(c.table), dev(keys),
                         None if scales is None else dev(scales), 0.125, dev(np.zeros((other, 4), dtype=np.float32)), w, w)
    assert torch.equal(w[0], before[0]) and torch.equal(w[2], before[2]) and bool(torch.isfinite(w).all()) and not torch.equal(w[1], before[1])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 40])
def test_weights_of_keys_behind_a_window_whose_pages_hold_anything(kind, n):
    """A window's caller may have given their pages away: nothing of them gets into the weights, which stay what they were."""
    c, held, off, q = filled(kind, 4, 2, 64, [n], [300], 32)
    keys, scales = c.k.copy(), None if kind == "bf16" else c.ks.copy()
    lse, before, got = dev(np.zeros((n, 4), dtype=np.float32)), torch.rand(1, 2, 300, device=DEV), []
    for spoilt in (False, True):
        if spoilt:
            for page in range(5):                       # tokens before 160; the first row sees tokens from 300 - n - 50 + 1 > 200 on
                if kind == "bf16":
                    for j in range(32 * page, 32 * page + 32):
                        for h in range(2):
                            keys[c.at(0, h, j):c.at(0, h, j) + 64] = 0x7fc0
                else:
                    scales[c.table[0, page]] = 255 if kind == "mx4" else np.nan
        w = before.clone()
        sp.sp_attend_weights(desc_of(c, 4, kind), dev(ou.bf16_bits(q)), [0, n], dev(off), dev(np.array([300], dtype=np.int32)), 300, dev(c.table), dev(keys),
                             None if scales is None else dev(scales), 0.125, lse, w, w, causal=1, window=50)
        got.append(w)
    assert torch.equal(got[0], got[1]) and torch.equal(got[1][..., :160], before[..., :160]) and not torch.equal(got[1], before)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 4, 40])
@pytest.mark.parametrize("where", ["query", "key"])
def test_a_nan_that_a_row_sees_gets_into_the_weights(kind, n, where):
    """With the lse of the attention itself: the row's is NaN then, and so is what it adds to. Nothing gets into the other request."""
    H, kv, d, lens = 4, 2, 64, [100, 90]
    c, held, off, q = filled(kind, H, kv, d, [n, n], lens, 32)
    bits = ou.bf16_bits(q)
    k, ks, vs = c.k.copy(), c.ks.copy(), c.vs.copy()
    if where == "query":
        bits[0, 3, 17] = 0x7FC0                         # a head of the second kv head
    elif kind == "bf16":
        k[c.at(0, 1, 20) + 5] = 0x7FC0
    elif kind == "e4m3":
        ks[c.table[0, 0], 1] = np.nan
    else:
        ks[c.table[0, 0], 1, 20, 1] = 255
    desc, qd, top = desc_of(c, H, kind), dev(bits), dev(np.asarray(lens, dtype=np.int32))
    args = (qd, off.tolist(), dev(off), top, 100, dev(c.table))
    scales = (dev(ks), dev(vs)) if kind != "bf16" else (None, None)
    kd, out, lse = dev(k), torch.empty(2 * n, H, d, dtype=torch.bfloat16, device=DEV), torch.empty(2 * n, H, device=DEV)
    ws = torch.empty(max(256, sp.sp_attend_workspace(desc, off.tolist(), 2, 100)), dtype=torch.uint8, device=DEV)
    sp.sp_attend(desc, *args, kd, dev(c.v), *scales, 0.125, out, lse, ws)
    assert torch.isnan(lse[0, 3]).item() and bool(torch.isfinite(lse[n:]).all())
    w = torch.full((2, kv, 100), 7.5, device=DEV)
    sp.sp_attend_weights(desc, *args, kd, scales[0], 0.125, lse, None, w)
    got = w.cpu().numpy()
    assert np.isnan(got[0, 1, :101 - n]).all() and np.isfinite(got[1]).all()
    if where == "key":                                  # with another lse the key's own weight still says so
        sp.sp_attend_weights(desc, *args, kd, scales[0], 0.125, torch.zeros_like(lse), None, w)
        got = w.cpu().numpy()
        assert np.isnan(got[0, 1, 20]) and np.isfinite(got[1]).all()


# ---- eviction --------------------------------------------------------------------------------------------------------

def choice(w, L, m, sinks, recent):
    """Tokens that stay, in their order."""
    if L <= m:
        return list(range(L))
    lo = min(sinks, m)
    r = min(recent, m - lo)
    rest = m - lo - r
    key = np.where(w == 0, 0.0, w)          # -0 as 0
    order = sorted(range(lo, L - r), key=lambda j: (-key[j], j))[:rest]
    return list(range(lo)) + sorted(order) + list(range(L - r, L))


def evict(kind, c, H, lens, budgets, sinks, recent, weights, dst, max_len=None, max_budget=None, with_weights=True):
    B = len(lens)
    max_len = max(lens) if max_len is None else max_len
    max_budget = max(max(budgets), 0) if max_budget is None else max_budget
    pools = [dev(c.k), dev(c.v)] + ([dev(c.ks), dev(c.vs)] if kind != "bf16" else [None, None])
    new_lens = torch.full((B,), -5, dtype=torch.int32, device=DEV)
    kept = torch.full((B, c.kv, max_budget), -7, dtype=torch.int32, device=DEV)
    new_w = torch.full((B, c.kv, max_budget), -7.0, device=DEV) if with_weights else None
    sp.sp_cache_evict(desc_of(c, H, kind), dev(np.asarray(lens, dtype=np.int32)), max_len, dev(np.asarray(budgets, dtype=np.int32)), max_budget, sinks, recent,
                      dev(weights), dev(c.table), dev(dst), *pools, new_lens, kept, new_w)
    torch.cuda.synchronize()
    return pools, new_lens.cpu().numpy(), kept.cpu().numpy(), None if new_w is None else new_w.cpu().numpy()


def check_evict(kind, kv, d, lens, budgets, sinks=4, recent=8, page=64, layout="HND", pad=0, seed=1, weights=None, max_len=None, max_budget=None,
                hidden=(), with_weights=True):
    rng = np.random.default_rng([seed, d, kv])
    B, H = len(lens), 2 * kv
    most = max_budget if max_budget is not None else max(max(budgets), 0)
    top = [min(L, max(m, 0), most) for L, m in zip(lens, budgets)]
    need = [max(1, -(-n // page)) for n in top]
    c, held, _, _ = filled(kind, H, kv, d, [0] * B, lens, page, layout, pad, seed, max_len or 0, spare=sum(need) + 2)
    used = set(c.table[c.table >= 0].tolist())
    free = [p for p in rng.permutation(c.n_pages).tolist() if p not in used]
    dst = np.full((B, max(need)), -1, dtype=np.int32)
    for b, n in enumerate(need):
        for i in range(n):
            dst[b, i] = free.pop()
    for b, i in hidden:
        dst[b, i] = -1
    S = max(max_len or 0, max(lens), 1)
    if weights is None:
        weights = np.exp(2 * rng.standard_normal((B, kv, S))) * (rng.random((B, kv, S)) < 0.8)
    weights = weights.astype(np.float32)
    pools, new_lens, kept, new_w = evict(kind, c, H, lens, budgets, sinks, recent, weights, dst, max_len, max_budget, with_weights)
    want = {"k": c.k.copy(), "v": c.v.copy(), "ks": c.ks.copy(), "vs": c.vs.copy()}
    table = c.table
    for b, L in enumerate(lens):
        m = min(max(budgets[b], 0), most)
        assert new_lens[b] == min(L, m)
        for h in range(kv):
            stay = choice(weights[b, h], L, m, sinks, recent)
            np.testing.assert_array_equal(kept[b, h, :len(stay)], stay)
            assert (kept[b, h, len(stay):] == -7).all()
            if with_weights:
                np.testing.assert_array_equal(new_w[b, h, :len(stay)], weights[b, h, stay])
                assert (new_w[b, h, len(stay):] == -7).all()
            for name, scales in (("k", "ks"), ("v", "vs")):
                pool = getattr(c, name)
                for i0 in range(0, len(stay), ou.BLOCK):
                    if dst[b, i0 // page] < 0:
                        continue
                    block = stay[i0:i0 + ou.BLOCK]
                    if kind == "e4m3":
                        old = np.array([getattr(c, scales)[c.scale_at(b, h, j)] for j in block])
                        new = old.max()
                        want[scales][int(dst[b, i0 // page]), h, i0 % page // ou.BLOCK] = new
                    for i, j in enumerate(block):
                        c.table = table
                        frm = c.at(b, h, j)
                        c.table = dst
                        to = c.at(b, h, i0 + i)
                        c.table = table
                        if kind == "mx4":
                            want[name][to // 2:to // 2 + d // 2] = pool[frm // 2:frm // 2 + d // 2]
                            want[scales][int(dst[b, i0 // page]), h, (i0 + i) % page] = getattr(c, scales)[int(table[b, j // page]), h, j % page]
                        elif kind == "e4m3":
                            want[name][to:to + d] = ou.e4m3_codes(ou.E4M3[pool[frm:frm + d]] * (old[i] / new))
                        else:
                            want[name][to:to + d] = pool[frm:frm + d]
    for name, got in zip(("k", "v", "ks", "vs"), pools):
        if got is not None:
            g = got.cpu().numpy()
            np.testing.assert_array_equal(g.view(np.uint16) if g.dtype == np.int16 else g, want[name], err_msg=name)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layout,page,pad", [("HND", 64, 0), ("NHD", 96, 32), ("HND", 32, 0)])
def test_evict(kind, d, layout, page, pad):
    check_evict(kind, 2, d, [300, 100, 1, 0, 65, 200], [100, 100, 5, 5, 64, 33], page=page, layout=layout, pad=pad)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("sinks,recent", [(0, 0), (4, 0), (0, 16), (50, 60), (1000, 1000), (1, 1)])
def test_evict_protects_the_first_and_last(kind, sinks, recent):
    check_evict(kind, 2, 64, [300, 90, 40], [70, 50, 1], sinks, recent)


@pytest.mark.parametrize("kind", KINDS)
def test_evict_budgets_of_nothing_and_of_more_than_there_is(kind):
    check_evict(kind, 1, 64, [100, 50, 0, 33], [0, -3, 10, 1000])
    check_evict(kind, 1, 64, [100, 50], [200, 60], max_budget=40)
    check_evict(kind, 1, 64, [100, 50], [0, 0])
    check_evict(kind, 1, 128, [500, 20], [90, 90], max_len=900, max_budget=128)


@pytest.mark.parametrize("seed", range(3))
def test_evict_ties_go_to_the_earlier_token(seed):
    rng = np.random.default_rng(seed)
    for values in ([1.0], [0.0, -0.0], [0.5, 0.5, 2.0], [1.0, np.nextafter(np.float32(1), np.float32(2)), 3.0], [np.inf, 1.0], [-1.0, -2.0, 0.0, 1e-42, -1e-42]):
        w = rng.choice(np.array(values, dtype=np.float32), (2, 2, 3000))
        check_evict("mx4", 2, 64, [3000, 1100], [700, 500], 4, 20, weights=w, seed=seed)


@pytest.mark.parametrize("L,m", [(20000, 5000), (20000, 19999), (6000, 40), (3000, 700)])
def test_evict_by_weights_that_are_near_each_other(L, m):
    """More contenders than are listed at a time share the first digits, with and without equal weights among them."""
    rng = np.random.default_rng(L + m)
    check_evict("mx4", 1, 64, [L], [m], 4, 32, page=4096, weights=1 + rng.random((1, 1, L)) * 0.2)
    check_evict("mx4", 1, 64, [L], [m], 4, 32, page=4096, weights=1 + rng.integers(0, 7, (1, 1, L)) * 2.0 ** -23)
    check_evict("mx4", 1, 64, [L], [m], 0, 0, page=4096, weights=rng.integers(0, 1 << 24, (1, 1, L)).astype(np.float64))


def test_evict_orders_nan_and_infinity():
    """A positive NaN above, a negative one below everything, infinities as numbers."""
    L, m = 40, 9
    w = np.arange(L, dtype=np.float32)[None, None] * -1.0
    bits = w.view(np.uint32)
    bits[0, 0, 30], bits[0, 0, 20], bits[0, 0, 0], bits[0, 0, 12] = 0x7FC00000, 0x7F800000, 0xFFFFFFFF, 0x7FFFFFFF
    bits[0, 0, 1], bits[0, 0, 2] = 0xFFC00000, 0xFF800000
    c, _, _, _ = filled("mx4", 2, 1, 64, [0], [L], 64, spare=3)
    dst = np.array([[p for p in range(c.n_pages) if p != c.table[0, 0]][:1]], dtype=np.int32)
    for m in (1, 2, 3, 6, 37, 38, 39):
        want = sorted([30, 12, 20, *range(3, 12), *range(13, 20), *range(21, 30), *range(31, 40), 2, 1, 0][:m] if m > 2 else [30, 12][:m] if m == 2 else [12])
        _, _, kept, _ = evict("mx4", c, 2, [L], [m], 0, 0, w, dst)
        np.testing.assert_array_equal(kept[0, 0], want)


@pytest.mark.parametrize("L,m", [(40, 100), (300, 120), (3000, 2999), (6000, 700), (9000, 8999)])
def test_evict_passes_weights_on_as_they_are(L, m):
    """Bit for bit, whatever the selection takes them for: the sign of zero, and what a NaN carries."""
    rng = np.random.default_rng(L)
    w = (rng.integers(-3, 4, (1, 1, L)) / np.float32(2)).astype(np.float32)
    bits = w.view(np.uint32)
    bits[w == 0] = rng.choice(np.array([0, 1 << 31], dtype=np.uint32), int((w == 0).sum()))
    at = rng.choice(L, 12, replace=False)
    bits[0, 0, at[:8]] = [0x7FC00001, 0x7FC12345, 0x7F800001, 0x7FBFFFFF, 0x7FFFFFFE, 0x7F800000, 0x00000001, 0x80000001]
    c, _, _, _ = filled("mx4", 2, 1, 64, [0], [L], 4096, spare=5)
    free = [p for p in range(c.n_pages) if p not in c.table[0].tolist()]
    dst = np.array([free[:-(-m // 4096)]], dtype=np.int32)
    _, new_lens, kept, new_w = evict("mx4", c, 2, [L], [m], 4, 8, w, dst)
    n = int(new_lens[0])
    assert n == min(L, m)
    np.testing.assert_array_equal(new_w[0, 0, :n].view(np.uint32), bits[0, 0, kept[0, 0, :n]])


def by_bits(bits, lo, hi, want):
    """The `want` largest of tokens lo .. hi - 1 as the order of weights has them: by their bits (NaN quiet, -0 as 0), negative ones reversed, ties to the earlier."""
    u = bits.astype(np.uint64)
    nan = (u & 0x7FFFFFFF) > 0x7F800000
    u = np.where(nan, u | 0x400000, np.where(u == 0x80000000, 0, u))
    key = np.where(u >> 31 == 1, 0xFFFFFFFF - u, u + 0x80000000).astype(np.int64)
    return sorted(sorted(range(lo, hi), key=lambda j: (-key[j], j))[:want])


@pytest.mark.parametrize("L,m,spread", [(6000, 5000, 900), (6000, 5990, 900), (9000, 4000, 6000), (9000, 8990, 6000), (3000, 2995, 400)])
def test_evict_where_the_last_to_stay_is_nan(L, m, spread):
    """Long lines of which many weights are the NaN below all numbers, whose bits are those of places without a token; with ties, and other NaNs among them."""
    rng = np.random.default_rng(L + m)
    w = rng.standard_normal((1, 1, L)).astype(np.float32)
    bits = w.view(np.uint32)
    at = rng.permutation(L)
    bits[0, 0, at[:spread]] = 0xFFFFFFFF
    bits[0, 0, at[spread:spread + 90]] = np.repeat(np.array([0xFFC00000, 0xFFFFFFFE, 0x7FC00000, 0x7FFFFFFF, 0xFF800000, 0x7F800000], dtype=np.uint32), 15)
    c, _, _, _ = filled("mx4", 2, 1, 64, [0], [L], 4096, spare=8)
    dst = np.array([[p for p in range(c.n_pages) if p not in c.table[0].tolist()][:-(-m // 4096)]], dtype=np.int32)
    for sinks, recent in ((0, 0), (4, 32)):
        _, _, kept, new_w = evict("mx4", c, 2, [L], [m], sinks, recent, w, dst)
        stay = [*range(sinks), *by_bits(bits[0, 0], sinks, L - recent, m - sinks - recent), *range(L - recent, L)]
        np.testing.assert_array_equal(kept[0, 0], stay)
        np.testing.assert_array_equal(new_w[0, 0].view(np.uint32), bits[0, 0, stay])


@pytest.mark.parametrize("scales", [[1.0, 2.0 ** -70, 2.0 ** 60, 2.0 ** -20], [0.0, 1.0, 0.0, 2.0], [0.0, 0.0, 0.0, 0.0], [np.nan, 1.0, 4.0, np.nan], [3.0, 0.7, 1.1, 2.9],
                                    [2.0 ** -126, 2.0 ** 126, 1.0, 2.0 ** 120]])
def test_evict_blocks_of_very_different_scales(scales):
    """Blocks of E4M3 codes of every kind under scales that are far apart, zero, NaN or no powers of two, whose tokens meet in one block: the largest scale, and
    E4M3 (code * (scale / s)), each step in float. Under a NaN all of a block is NaN."""
    kv, d, page, L, m = 1, 64, 32, 256, 70
    c, _, _, _ = filled("e4m3", 2, kv, d, [0], [L], page, spare=4)
    rng = np.random.default_rng(7)
    for pool in (c.k, c.v):
        for j in range(L):
            pool[c.at(0, 0, j):c.at(0, 0, j) + d] = rng.integers(0, 256, d)
    for i in range(L // page):
        c.ks[c.table[0, i], 0, 0], c.vs[c.table[0, i], 0, 0] = scales[i % 4], scales[(i + 1) % 4]
    dst = np.array([[p for p in range(c.n_pages) if p not in c.table[0].tolist()][:3]], dtype=np.int32)
    w = rng.random((1, kv, L)).astype(np.float32)
    pools, _, kept, _ = evict("e4m3", c, 2, [L], [m], 0, 0, w, dst)
    stay = kept[0, 0]
    for pool, of, got, new in ((c.k, c.ks, pools[0], pools[2]), (c.v, c.vs, pools[1], pools[3])):
        got, new = got.cpu().numpy(), new.cpu().numpy()
        for i0 in range(0, m, 32):
            block = stay[i0:i0 + 32]
            old = np.array([of[c.table[0, j // page], 0, 0] for j in block], dtype=np.float32)
            top = np.float32(np.nan) if np.isnan(old).any() else old.max()
            np.testing.assert_array_equal(new[dst[0, i0 // page], 0, 0], top)
            for i, j in enumerate(block):
                to = int(dst[0, i0 // page]) * c.page_stride + i * c.stride_token
                mine = got[to:to + d]
                if np.isnan(top):
                    continue
                with np.errstate(under="ignore"):
                    x = ou.E4M3[pool[c.at(0, 0, j):c.at(0, 0, j) + d]].astype(np.float32)
                    y = x if old[i] == top else x * np.float32(old[i] / top)
                want = ou.e4m3_codes(y.astype(np.float64))
                nan = np.isnan(y)
                np.testing.assert_array_equal(np.isnan(ou.E4M3[mine]), nan)
                np.testing.assert_array_equal(mine[~nan], want[~nan])


@pytest.mark.parametrize("L,m", [(40000, 9000), (70001, 70000), (65536, 64), (5000, 4097)])
def test_evict_from_long_contexts(L, m):
    check_evict("mx4", 1, 64, [L, 3], [m, 2], 4, 32, page=4096)


@pytest.mark.parametrize("kind", KINDS)
def test_evict_to_pages_that_are_not_there(kind):
    check_evict(kind, 2, 64, [400, 90], [200, 70], page=32, hidden=[(0, 1), (0, 6), (1, 0)], with_weights=False)


def test_evict_on_another_stream_and_in_a_graph():
    kind, kv, d, page, L, m = "bf16", 2, 64, 64, 500, 128
    c, _, _, _ = filled(kind, 4, kv, d, [0], [L], page, spare=4)
    used = set(c.table[0].tolist())
    dst = np.array([[p for p in range(c.n_pages) if p not in used][:2]], dtype=np.int32)
    desc, k, v = desc_of(c, 4, kind), dev(c.k), dev(c.v)
    lens, budget, table, to = (dev(np.asarray(x, dtype=np.int32)) for x in ([L], [m], c.table, dst))
    w, new_lens = torch.zeros(1, kv, L, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    kept, new_w = torch.zeros(1, kv, m, dtype=torch.int32, device=DEV), torch.zeros(1, kv, m, device=DEV)

    def call():
        sp.sp_cache_evict(desc, lens, L, budget, m, 4, 16, w, table, to, k, v, None, None, new_lens, kept, new_w)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(3):
        x = np.random.default_rng(seed).random((1, kv, L)).astype(np.float32)
        w.copy_(torch.from_numpy(x))
        graph.replay()
        torch.cuda.synchronize()
        for h in range(kv):
            np.testing.assert_array_equal(kept[0, h].cpu().numpy(), choice(x[0, h], L, m, 4, 16))
        first = kept.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(first, kept)


# ---- together --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
def test_a_cache_held_to_a_budget(kind, d):
    """Prompt, attention, weights, eviction, and decoding on what was kept: every step's results from the definition on what the pages hold."""
    H, kv, page, L, m, steps = 4, 2, 64, 300, 96, 6
    rng = np.random.default_rng(5)
    e = {"bf16": torch.bfloat16, "e4m3": torch.uint8, "mx4": torch.uint8}[kind]
    pages = 12
    row = d // 2 if kind == "mx4" else d
    desc = sp.CacheDesc(H, kv, d, TYPE[kind], pages, page, kv * page * d, page * d, d)
    k, v = (torch.zeros(pages, kv, page, row, dtype=e, device=DEV) for _ in range(2))
    shape = {"bf16": None, "e4m3": (pages, kv, page // 32), "mx4": (pages, kv, page, d // 32)}[kind]
    ks, vs = (None if shape is None else torch.zeros(shape, dtype=torch.uint8 if kind == "mx4" else torch.float32, device=DEV) for _ in range(2))
    table, spare = (torch.tensor([x], dtype=torch.int32, device=DEV) for x in ([3, 9, 0, 7, 5], [10, 2]))
    scale = d ** -0.5

    def held(tab, n):
        out = []
        for pool, s in ((k, ks), (v, vs)):
            x = pool[tab[0].long()]
            if kind == "mx4":
                x = mu.values(mu.unpack(x.cpu().numpy()), s[tab[0].long()].cpu().numpy())
            elif kind == "e4m3":
                x = (x.view(torch.float8_e4m3fn).double() * s[tab[0].long()].double().repeat_interleave(32, dim=2)[..., None]).cpu().numpy()
            else:
                x = x.double().cpu().numpy()
            out.append(np.concatenate(list(x), axis=1).transpose(1, 0, 2)[:n])
        return out

    def step(tab, start, n, positions=None):
        x = torch.from_numpy(rng.standard_normal((n, (H + 2 * kv) * d)).astype(np.float32)).to(torch.bfloat16).to(DEV)
        q, key, val = x.split([H * d, kv * d, kv * d], dim=1)
        off_dev = torch.tensor([0, n], device=DEV)
        lens = torch.tensor([start + n], dtype=torch.int32, device=DEV)
        sp.sp_cache_append(desc, key, val, [0, n], off_dev, torch.tensor([start], dtype=torch.int32, device=DEV), tab, k, v, ks, vs)
        q = q.contiguous().view(n, H, d)
        out, lse = torch.empty(n, H, d, dtype=torch.bfloat16, device=DEV), torch.empty(n, H, device=DEV)
        ws = torch.empty(max(256, sp.sp_attend_workspace(desc, [0, n], 1, start + n)), dtype=torch.uint8, device=DEV)
        sp.sp_attend(desc, q, [0, n], off_dev, lens, start + n, tab, k, v, ks, vs, scale, out, lse, ws)
        return q, off_dev, lens, out, lse

    def look(q, tab, n, out, lse):
        kk, vv = held(tab, n)
        rows = q.shape[0]
        x = np.stack([q[:, h].double().cpu().numpy() @ kk[:, h // (H // kv)].T * scale for h in range(H)], axis=1)
        x = np.where(np.arange(n) <= (n - rows + np.arange(rows))[:, None, None], x, -np.inf)
        p = np.exp(x - x.max(axis=-1, keepdims=True))
        z = p.sum(axis=-1, keepdims=True)
        p /= z
        o = np.stack([p[:, h] @ vv[:, h // (H // kv)] for h in range(H)], axis=1)
        np.testing.assert_allclose(lse.cpu().numpy(), (x.max(axis=-1, keepdims=True) + np.log(z))[..., 0], atol=2e-5)
        assert np.abs(out.double().cpu().numpy() - o).max() < 0.03
        return p

    def add(q, off_dev, lens, n, tab, lse, old, w, rows):
        sp.sp_attend_weights(desc, q, [0, rows], off_dev, lens, n, tab, k, ks, scale, lse, old, w)

    q, off_dev, lens, out, lse = step(table, 0, L)
    w = torch.zeros(1, kv, L + steps, device=DEV)
    add(q, off_dev, lens, L, table, lse, None, w, L)
    p = look(q, table, L, out, lse)
    total = p.reshape(L, kv, H // kv, L).sum(axis=(0, 2))
    np.testing.assert_allclose(w[0, :, :L].cpu().numpy(), total, rtol=1e-4)
    new_lens, kept = torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(1, kv, m, dtype=torch.int32, device=DEV)
    new_w = torch.zeros(1, kv, m, device=DEV)
    before = held(table, L)
    sp.sp_cache_evict(desc, lens, L, torch.tensor([m], dtype=torch.int32, device=DEV), m, 4, 16, w, table, spare, k, v, ks, vs, new_lens, kept, new_w)
    assert new_lens.item() == m
    after = held(spare, m)
    for h in range(kv):
        stay = kept[0, h].cpu().numpy()
        np.testing.assert_array_equal(stay, choice(w[0, h].cpu().numpy(), L, m, 4, 16))
        for x, y in zip(before, after):
            if kind == "e4m3":              # codes among the subnormals of a larger scale move by half a step of it at most
                assert np.abs(y[:, h] - x[stay, h]).max() <= 2.0 ** -10 * 2.0 ** -6
            else:
                np.testing.assert_array_equal(y[:, h], x[stay, h])
    w2 = torch.zeros(1, kv, m + steps, device=DEV)
    w2[:, :, :m] = new_w
    total = new_w[0].double().cpu().numpy()
    for i in range(steps):
        q, off_dev, lens, out, lse = step(spare, m + i, 1)
        add(q, off_dev, lens, m + i + 1, spare, lse, w2, w2, 1)
        p = look(q, spare, m + i + 1, out, lse)
        total = np.concatenate([total, np.zeros((kv, 1))], axis=1) + p.reshape(1, kv, H // kv, -1).sum(axis=(0, 2))
        np.testing.assert_allclose(w2[0, :, :m + i + 1].cpu().numpy(), total, rtol=1e-4)
