"""sp_attend against the definition in 64 bits on exactly the values that the cache holds.

Tolerances. Logits are sums of d exact products in fp32: off by at most (d + 4) 2^-24 S with S = scale sum |q||k|, and so is lse,
beside 2^-20 for the sum and its logarithm and 2^-22 |lse| for the last rounding. Probabilities are rounded to bf16 (eight
significant bits: 2^-8 of each at most) before the second product and the result is rounded to bf16 (2^-8 of it): with A = sum p |v| the
output is off by at most (2^-8 + 2 dx + 2^-12) A + 2^-8 |o|, where dx is the logits' error."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import operator_util as ou
import paper_2603_02631_amd as sp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).to(DEV)


def desc_of(c, H):
    return sp.CacheDesc(H, c.kv, c.d, sp.SP_CACHE_E4M3 if c.e4m3 else sp.SP_CACHE_BF16, c.n_pages, c.page, c.page_stride,
                        c.stride_head, c.stride_token)


def build(H, kv, d, news, lens, page, e4m3, layout, pad, seed, k_scale=1.0, spread=False, max_len=0):
    rng = np.random.default_rng([seed, d])
    widths = [max(1, -(-n // page)) for n in lens]
    c = ou.Paged(kv, d, page, widths, e4m3, layout, pad, seed=seed, table_tokens=max_len)
    held = []
    for b, L in enumerate(lens):
        k = rng.standard_normal((L, kv, d)) * k_scale
        v = rng.standard_normal((L, kv, d))
        if spread:                                      # blocks of very different size
            m = np.exp2(rng.integers(-6, 7, (L // 32 + 1, kv))).repeat(32, axis=0)[:L, :, None]
            k, v = k * m / 8, v * m[::-1]
        held.append(c.fill(b, k, v))
    off = np.concatenate([[0], np.cumsum(news)]).astype(np.int64)
    q = ou.bf16_round(rng.standard_normal((max(int(off[-1]), 1), H, d)))
    return c, held, off, q


def call(c, H, off, q, lens, max_len, scale, causal, window, stream=None, with_lse=True):
    T, d = int(off[-1]), c.d
    out = torch.full((max(T, 1), H, d), 0x7FC0, dtype=torch.int16, device=DEV)
    lse = torch.full((max(T, 1), H), float("nan"), device=DEV) if with_lse else None
    desc = desc_of(c, H)
    size = sp.sp_attend_workspace(desc, off.tolist(), len(lens), max_len)
    ws = torch.full((max(size, 256),), 0xFF, dtype=torch.uint8, device=DEV)      # NaN patterns: nothing may rely on its contents
    args = [dev(ou.bf16_bits(q)), off.tolist(), dev(off), dev(np.asarray(lens, dtype=np.int32)), max_len, dev(c.table), dev(c.k), dev(c.v),
            dev(c.ks) if c.e4m3 else None, dev(c.vs) if c.e4m3 else None]
    torch.cuda.synchronize()
    sp.sp_attend(desc, *args, scale, out, lse, ws, causal=causal, window=window, stream=stream)
    torch.cuda.synchronize()
    return ou.bits_to_f64(out.cpu().numpy().view(np.uint16)), None if lse is None else lse.cpu().numpy().astype(np.float64)


def verify(c, H, held, off, q, lens, scale, causal, window, out, lse, rows=None):
    G, d = H // c.kv, c.d
    for b, L in enumerate(lens):
        n = int(off[b + 1] - off[b])
        for r in range(n):
            t = int(off[b]) + r
            if rows is not None and t not in rows:
                continue
            lo, hi = ou.seen(L, n, r, causal, window)
            for h in range(H):
                k, v = held[b][0][:, h // G], held[b][1][:, h // G]
                o, z, A, S = ou.attend(q[t, h].astype(np.float64), k, v, scale, lo, hi)
                if hi <= lo:
                    assert np.all(out[t, h] == 0) and lse[t, h] == -np.inf, (b, r, h)
                    continue
                dx = (d + 4) * 2.0 ** -24 * S
                assert abs(lse[t, h] - z) <= dx + 2.0 ** -20 + 2.0 ** -22 * abs(z), (b, r, h, lse[t, h], z)
                tol = (2.0 ** -8 + 2 * dx + 2.0 ** -12) * A + 2.0 ** -8 * np.abs(o)
                bad = np.abs(out[t, h] - o) > tol
                assert not bad.any(), (b, r, h, np.flatnonzero(bad)[:4], out[t, h][bad][:4], o[bad][:4], tol[bad][:4])


def check(H, kv, d, news, lens, page, e4m3, layout="HND", pad=0, seed=1, causal=1, window=0, scale=None, max_len=None, rows=None, **kw):
    c, held, off, q = build(H, kv, d, news, lens, page, e4m3, layout, pad, seed, max_len=max_len or 0, **kw)
    scale = scale or d ** -0.5
    out, lse = call(c, H, off, q, lens, max(lens) if max_len is None else max_len, scale, causal, window)
    verify(c, H, held, off, q, lens, scale, causal, window, out, lse, rows)


SHAPES = [(4, 2, 64), (2, 2, 128), (8, 1, 64), (16, 1, 128), (6, 2, 128), (5, 5, 64)]


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("H,kv,d", SHAPES)
def test_single_tokens(e4m3, H, kv, d):
    check(H, kv, d, [1, 1, 1, 0, 1, 1, 1], [1, 2, 33, 40, 64, 257, 1000], 32, e4m3)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("H,kv,d", SHAPES[:4])
@pytest.mark.parametrize("layout,page,pad", [("NHD", 96, 16), ("HND", 512, 0)])
def test_a_few_rows(e4m3, H, kv, d, layout, page, pad):
    check(H, kv, d, [8, 3, 16, 1], [8, 700, 31, 300], page, e4m3, layout, pad)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("H,kv,d", SHAPES[:3])
def test_prompt_chunks(e4m3, H, kv, d):
    check(H, kv, d, [130, 1, 67, 300], [130, 90, 500, 333], 64, e4m3)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("causal,window", [(0, 0), (1, 1), (1, 7), (1, 100)])
@pytest.mark.parametrize("news", [[1, 2, 5], [80, 1, 150]])
def test_masks(e4m3, causal, window, news):
    check(4, 1, 64, news, [200, 45, 310], 64, e4m3, causal=causal, window=window)
    check(4, 2, 128, news, [200, 45, 310], 64, e4m3, causal=causal, window=window)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_see_nothing_and_empty_contexts(e4m3, d):
    """More queries than context: the first rows see no key; contexts of no token."""
    check(4, 2, d, [5, 3, 1, 100, 2], [2, 0, 0, 30, 2], 32, e4m3)
    check(4, 2, d, [2, 3], [0, 0], 32, e4m3, max_len=0)
    check(4, 2, d, [3, 70], [0, 1], 32, e4m3, causal=0)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("news", [[1, 8], [100, 70]])
@pytest.mark.parametrize("d", [64, 128])
def test_large_logits_and_blocks_of_different_size(e4m3, news, d):
    """Logits that grow by hundreds along the context, so that the running maximum moves often and most keys vanish."""
    check(4, 2, d, news, [600, 350], 64, e4m3, k_scale=12.0)
    check(4, 2, d, news, [600, 350], 64, e4m3, spread=True)
    check(4, 2, d, news, [600, 350], 64, e4m3, scale=1e-3)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("H,kv,d", [(4, 1, 64), (2, 1, 128)])
def test_long_contexts(e4m3, H, kv, d):
    """Contexts that are split among workgroups, at lengths around the splits' ends; one far shorter than max_len says."""
    check(H, kv, d, [1, 1, 8, 1], [5000, 4097, 8191, 1], 512, e4m3, max_len=10000 if d == 64 else None)
    check(H, kv, d, [300, 40], [3000, 9000], 512, e4m3, rows=set(range(0, 340, 13)))


def test_max_len_bounds_the_contexts():
    """Longer contexts count as max_len, negative ones as none."""
    c, held, off, q = build(4, 2, 64, [1, 1, 2], [100, 100, 100], 32, True, "HND", 0, 3)
    out, lse = call(c, 4, off, q, [100, -5, 2 ** 31 - 1], 64, 0.125, 1, 0)
    verify(c, 4, held, off, q, [64, 0, 64], 0.125, 1, 0, out, lse)


@pytest.mark.parametrize("news", [[1, 1], [90, 2]])
def test_scales_that_are_no_powers_of_two(news):
    """Another rounding to bf16 for each element: 2^-8 of every key and value."""
    c, held, off, q = build(4, 2, 64, news, [300, 200], 32, True, "HND", 0, 4)
    ok = ~np.isnan(c.ks)
    rng = np.random.default_rng(1)
    f = np.float32(1) + rng.random(c.ks.shape).astype(np.float32) * np.float32(0.9)
    for b, L in enumerate([300, 200]):
        for j in range(L):
            for h in range(2):
                at = c.scale_at(b, h, j)
                held[b][0][j, h] *= f[at]
                held[b][1][j, h] *= f[at]
    c.ks, c.vs = np.where(ok, c.ks * f, c.ks), np.where(ok, c.vs * f, c.vs)
    out, lse = call(c, 4, off, q, [300, 200], 300, 0.125, 1, 0)
    for b, L in enumerate([300, 200]):
        n = int(off[b + 1] - off[b])
        for r in range(0, n, 7):
            t = int(off[b]) + r
            for h in range(4):
                o, z, A, S = ou.attend(q[t, h].astype(np.float64), held[b][0][:, h // 2], held[b][1][:, h // 2], 0.125, 0, L - n + r + 1)
                dx = 2.0 ** -8 * S + 68 * 2.0 ** -24 * S
                assert abs(lse[t, h] - z) <= dx + 1e-5
                assert np.all(np.abs(out[t, h] - o) <= (2.0 ** -7 + 2 * dx + 2.0 ** -12) * A + 2.0 ** -8 * np.abs(o))


@pytest.mark.parametrize("news,lens", [([1, 1], [6000, 900]), ([100, 1], [700, 2000])])
def test_same_result_every_time_on_any_stream_and_in_graphs(news, lens):
    c, held, off, q = build(4, 2, 64, news, lens, 64, True, "HND", 0, 6)
    a = call(c, 4, off, q, lens, max(lens), 0.125, 1, 0)
    b = call(c, 4, off, q, lens, max(lens), 0.125, 1, 0, stream=torch.cuda.Stream())
    np.testing.assert_array_equal(a[0], b[0])
    np.testing.assert_array_equal(a[1], b[1])
    b = call(c, 4, off, q, lens, max(lens), 0.125, 1, 0, with_lse=False)
    np.testing.assert_array_equal(a[0], b[0])
    desc, T = desc_of(c, 4), int(off[-1])
    out, lse = torch.empty(T, 4, 64, dtype=torch.int16, device=DEV), torch.empty(T, 4, device=DEV)
    ws = torch.empty(max(256, sp.sp_attend_workspace(desc, off.tolist(), 2, max(lens))), dtype=torch.uint8, device=DEV)
    args = [dev(ou.bf16_bits(q)), sp.host_offsets(off.tolist()), dev(off), dev(np.asarray(lens, dtype=np.int32)), max(lens), dev(c.table),
            dev(c.k), dev(c.v), dev(c.ks), dev(c.vs)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sp.sp_attend(desc, *args, 0.125, out, lse, ws)
    for _ in range(3):
        out.zero_()
        lse.zero_()
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        np.testing.assert_array_equal(a[0], ou.bits_to_f64(out.cpu().numpy().view(np.uint16)))
        np.testing.assert_array_equal(a[1], lse.cpu().numpy().astype(np.float64))


@pytest.mark.parametrize("news", [1, 70])
def test_pages_beyond_32_bit_offsets(news):
    """Pages 2^31 elements apart."""
    d, P, L, stride = 64, 32, 64, 1 << 31
    rng = np.random.default_rng(2)
    pools, held = [], []
    scales = torch.zeros(2, 2, 1, 1, device=DEV)
    for i in range(2):
        pool = torch.zeros(stride + P * d, dtype=torch.uint8, device=DEV)
        x, y = rng.standard_normal((L, 1, d)), np.zeros((L, 1, d))
        for page, part in ((1, slice(0, 32)), (0, slice(32, 64))):
            s = ou.scale_of(np.abs(x[part]).max())
            codes = ou.e4m3_codes(x[part, 0] / s)
            pool[page * stride:page * stride + P * d] = torch.from_numpy(codes.reshape(-1)).to(DEV)
            scales[i, page, 0, 0] = s
            y[part, 0] = ou.E4M3[codes] * s
        pools.append(pool)
        held.append(y)
    desc = sp.CacheDesc(1, 1, d, sp.SP_CACHE_E4M3, 2, P, stride, P * d, d)
    q = ou.bf16_round(rng.standard_normal((news, 1, d)))
    out, lse = torch.empty(news, 1, d, dtype=torch.int16, device=DEV), torch.empty(news, 1, device=DEV)
    ws = torch.empty(max(256, sp.sp_attend_workspace(desc, [0, news], 1, L)), dtype=torch.uint8, device=DEV)
    sp.sp_attend(desc, dev(ou.bf16_bits(q)), [0, news], dev(np.array([0, news])), dev(np.array([L], dtype=np.int32)), L,
                 dev(np.array([[1, 0]], dtype=np.int32)), *pools, scales[0], scales[1], 0.125, out, lse, ws)
    torch.cuda.synchronize()

    class C:
        kv = 1
    C.d = d
    verify(C, 1, [held], np.array([0, news]), q, [L], 0.125, 1, 0, ou.bits_to_f64(out.cpu().numpy().view(np.uint16)),
           lse.cpu().numpy().astype(np.float64))


@pytest.mark.parametrize("e4m3", [True, False])
def test_more_requests_than_lanes(e4m3):
    """Work is shared out over more requests than a wave has lanes, empty ones and ones without queries among them."""
    rng = np.random.default_rng(9)
    news, lens = rng.integers(0, 4, 70), rng.integers(0, 200, 70)
    lens[[3, 66]] = 590, 600
    check(4, 1, 64, news.tolist(), lens.tolist(), 64, e4m3, max_len=600)
    check(3, 1, 128, news.tolist(), lens.tolist(), 64, e4m3, max_len=600)


@pytest.mark.parametrize("e4m3", [True, False])
def test_more_prompt_chunks_than_the_list_of_a_launch(e4m3):
    rng = np.random.default_rng(10)
    news = rng.integers(4, 8, 67)
    news[[5, 40]] = 1, 50
    check(16, 1, 64, news.tolist(), (news + rng.integers(0, 60, 67)).tolist(), 32, e4m3)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("H,kv,d,page,news,lens,window", [
    (16, 1, 64, 96, [1130], [2300], 0),         # 71 tiles of query rows
    (4, 2, 64, 32, [300, 150], [2200, 900], 0),
    (6, 2, 128, 96, [200, 1, 90], [1500, 1100, 95], 0),
    (4, 2, 128, 32, [300, 150], [2200, 900], 70)])
def test_long_chunks_shared_out_over_kv_heads(e4m3, H, kv, d, page, news, lens, window):
    check(H, kv, d, news, lens, page, e4m3, window=window, rows=set(range(0, sum(news), 17)) | {sum(news) - 1})


@pytest.mark.parametrize("news", [[1, 3], [90, 70]])
@pytest.mark.parametrize("d", [64, 128])
def test_scales_of_zero_where_a_block_is_zero(news, d):
    c, held, off, q = build(4, 2, d, news, [300, 200], 32, True, "HND", 0, 12)
    for b, L in enumerate([300, 200]):
        for j0 in range(0, L, 96):
            for h in range(2):
                for j in range(j0, min(L, j0 + 32)):
                    o = c.at(b, h, j)
                    c.k[o:o + d] = c.v[o:o + d] = 0
                    held[b][0][j, h] = held[b][1][j, h] = 0
                c.ks[c.scale_at(b, h, j0)] = c.vs[c.scale_at(b, h, j0)] = 0
    out, lse = call(c, 4, off, q, [300, 200], 300, 0.125, 1, 0)
    verify(c, 4, held, off, q, [300, 200], 0.125, 1, 0, out, lse)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("news,lens", [([1, 3], [300, 200]), ([90, 70], [300, 200]), ([2, 1], [3000, 2500]), ([90, 70], [3000, 2500])])
def test_a_nan_that_is_seen_gets_out(e4m3, news, lens):
    """A NaN key makes a row and its lse NaN, a NaN value one element; the other kv head and the other request stay as they are."""
    for which in ("k", "v"):
        c, held, off, q = build(4, 2, 64, news, lens, 64, e4m3, "HND", 0, 13)
        getattr(c, which)[c.at(0, 1, 57) + 5] = 0x7F if e4m3 else 0x7FC0
        out, lse = call(c, 4, off, q, lens, max(lens), 0.125, 1, 0)
        n = news[0]
        if which == "k":
            assert np.isnan(out[:n, 2:]).all() and np.isnan(lse[:n, 2:]).all()
        else:
            assert np.isnan(out[:n, 2:, 5]).all() and np.isfinite(lse[:n, 2:]).all()
            assert np.isfinite(np.delete(out[:n, 2:], 5, axis=2)).all()
        assert np.isfinite(out[:n, :2]).all() and np.isfinite(lse[:n, :2]).all()
        assert np.isfinite(out[n:]).all() and np.isfinite(lse[n:]).all()


@pytest.mark.parametrize("news", [[1, 3], [30, 8], [60, 64]])
def test_contexts_that_may_be_larger_than_a_cache(news):
    """A bound of 2^20 tokens a request: keys are read past the caches, work is shared out as for the longest lengths."""
    check(4, 4, 64, news, [700, 65], 512, True, max_len=1 << 20)
    check(2, 2, 128, news, [700, 65], 512, False, max_len=1 << 20)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("H,kv,d", [(8, 2, 128), (4, 2, 128), (8, 2, 64)])
@pytest.mark.parametrize("news,lens", [([1, 3], [300, 200]), ([8, 4], [300, 200]), ([90, 70], [300, 200]), ([2, 1], [3000, 2500]),
                                       ([8, 4], [3000, 2500]), ([90, 70], [3000, 2500])])
def test_a_nan_that_is_seen_gets_out_of_every_kernel(e4m3, H, kv, d, news, lens):
    """As above at both head sizes, with one to four query heads a kv head: few and many rows, whole and shared out, at the beginning of
    a context, in its middle, and at its last key, which only the last row sees."""
    G, n, L = H // kv, news[0], lens[0]
    for which in ("k", "v"):
        for key in (0, 57, L // 2, L - 1):
            c, held, off, q = build(H, kv, d, news, lens, 64, e4m3, "HND", 0, 13)
            getattr(c, which)[c.at(0, 1, key) + 5] = 0x7F if e4m3 else 0x7FC0
            out, lse = call(c, H, off, q, lens, max(lens), 0.125, 1, 0)
            rows = slice(n - 1, n) if key == L - 1 else slice(0, n)         # that see it
            if which == "k":
                assert np.isnan(out[rows, G:]).all() and np.isnan(lse[rows, G:]).all(), key
            else:
                assert np.isnan(out[rows, G:, 5]).all() and np.isfinite(lse[rows, G:]).all(), key
                assert np.isfinite(np.delete(out[rows, G:], 5, axis=2)).all(), key
            assert np.isfinite(out[:n, :G]).all() and np.isfinite(lse[:n, :G]).all(), key
            assert np.isfinite(out[n:]).all() and np.isfinite(lse[n:]).all(), key


@pytest.mark.parametrize("news", [[1, 3], [90, 70]])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("e4m3", [True, False])
def test_queries_of_zero_at_the_largest_scales(news, d, e4m3):
    """Logits of exactly zero however large scale and key scales are: the values' mean, and the logarithm of the number of keys."""
    lens = [300, 200]
    c, held, off, q = build(4, 2, d, news, lens, 32, e4m3, "HND", 0, 14)
    if e4m3:
        c.ks = np.where(np.isnan(c.ks), c.ks, np.float32(2.0 ** 100))
        for b in range(2):
            held[b] = [np.zeros_like(held[b][0]), held[b][1]]       # whatever the keys are
    q[:] = 0
    out, lse = call(c, 4, off, q, lens, 300, 2.3e38, 1, 0)
    verify(c, 4, held, off, q, lens, 1.0, 1, 0, out, lse)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("H,kv,d", [(8, 2, 64), (4, 2, 128)])
def test_masks_where_few_rows_are_shared_out(e4m3, H, kv, d):
    """Windows leave far fewer blocks than the bound on the lengths says; without a mask every row sees all. One context is shorter than its rows."""
    news, lens = [1, 8, 3, 5, 2], [3000, 9000, 5200, 2, 0]
    c, held, off, q = build(H, kv, d, news, lens, 64, e4m3, "HND", 0, 15, max_len=9000)
    assert sp.sp_attend_workspace(desc_of(c, H), off.tolist(), len(lens), 9000) > 0
    for causal, window in ((0, 0), (1, 0), (1, 1), (1, 31), (1, 100), (1, 2500), (1, 8999), (1, 9000), (1, 1 << 40)):
        out, lse = call(c, H, off, q, lens, 9000, 0.125, causal, window)
        verify(c, H, held, off, q, lens, 0.125, causal, window, out, lse)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("others", [1, 99])
def test_lines_of_more_parts_than_lanes(e4m3, d, others):
    """A context of 40000 tokens of one kv head is joined from more than 64 partial results: by four waves a row, or by one where there are many lines."""
    rng = np.random.default_rng(16)
    check(2, 1, d, [2] + [1] * others, [40000] + rng.integers(1, 80, others).tolist(), 512, e4m3)
