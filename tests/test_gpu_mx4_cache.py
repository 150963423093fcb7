"""A paged cache of 4-bit elements: sp_cache_append byte by byte against the definition, sp_attend against 64 bits on exactly the values that the
cache holds.

Tolerances of sp_attend as for the other caches: logits off by (d + 4) 2^-24 S with S = scale sum |q||k|; probabilities and results rounded to bf16, 2^-8 each."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import mx4_util as mu
import operator_util as ou
import paper_2603_02631_amd as sp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).to(DEV)


def desc_of(c, H):
    return sp.CacheDesc(H, c.kv, c.d, sp.SP_CACHE_MX4, c.n_pages, c.page, c.page_stride, c.stride_head, c.stride_token)


# ---- append ----------------------------------------------------------------------------------------------------------

def append_case(H, kv, d, news, starts, page, rot, style, layout="HND", pad=0, seed=0, positions=False, bad=False):
    rng = np.random.default_rng([seed, d, rot])
    widths = [max(1, -(-(s + n) // page)) for s, n in zip(starts, news)]
    c = mu.Paged4(kv, d, page, widths, layout, pad, seed=seed)
    T = sum(news)
    qkv = rng.standard_normal((T, (H + 2 * kv) * d)) * np.exp2(rng.integers(-3, 4, (T, 1)))
    qkv = ou.bf16_round(qkv)
    if bad:
        qkv[0, H * d + 3], qkv[T - 1, (H + kv) * d + 40] = np.inf, np.nan
    n_pos = 64 + max(s + n for s, n in zip(starts, news))
    angle = np.arange(n_pos)[:, None] * 10000.0 ** -(np.arange(max(rot // 2, 1)) / max(rot // 2, 1))
    cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    pos = rng.integers(0, n_pos, T).astype(np.int32) if positions else None
    if bad:
        c.table[0, 0] = -1
    off = np.concatenate([[0], np.cumsum(news)]).astype(np.int64)
    k, v, ks, vs = dev(c.k), dev(c.v), dev(c.ks), dev(c.vs)
    bits = ou.bf16_bits(np.nan_to_num(qkv, nan=0, posinf=0))
    bits = np.where(np.isnan(qkv), 0x7FC0, np.where(np.isinf(qkv), 0x7F80, bits)).astype(np.uint16)
    x = dev(bits)
    q_out = torch.zeros(T, H, d, dtype=torch.bfloat16, device=DEV)
    parts = x.split([H * d, kv * d, kv * d], dim=1)
    sp.sp_cache_append(desc_of(c, H), parts[1], parts[2], off.tolist(), dev(off), dev(np.asarray(starts, dtype=np.int32)), dev(c.table), k, v, ks, vs,
                       q=parts[0], q_out=q_out, cos=dev(cos) if rot else None, sin=dev(sin) if rot else None, rot_dim=rot,
                       rot_style=sp.SP_ROTATE_HALF if style == "half" else sp.SP_ROTATE_PAIRS, positions=None if pos is None else dev(pos))
    torch.cuda.synchronize()
    # the definition, token by token
    want_q = np.zeros((T, H, d))
    for b, (n, s) in enumerate(zip(news, starts)):
        for i in range(n):
            t, j = int(off[b]) + i, s + i
            p = int(pos[t]) if positions else j
            row = qkv[t].reshape(H + 2 * kv, d)
            for h in range(H):
                want_q[t, h] = ou.bf16_round(ou.rotate(row[h], p, cos, sin, rot, style))
            if c.table[b, j // page] < 0:
                continue
            for h in range(kv):
                y = ou.rotate(row[H + h], p, cos, sin, rot, style)
                c.put(c.k, c.ks, b, h, j, *mu.quantise(y))
                c.put(c.v, c.vs, b, h, j, *mu.quantise(row[H + kv + h]))
    for name, got, want in (("ks", ks, c.ks), ("vs", vs, c.vs), ("k", k, c.k), ("v", v, c.v)):
        np.testing.assert_array_equal(got.cpu().numpy(), want, err_msg=name)
    np.testing.assert_array_equal(q_out.double().cpu().numpy(), want_q)


@pytest.mark.parametrize("style", ["half", "pairs"])
@pytest.mark.parametrize("H,kv,d,rot", [(4, 2, 64, 64), (4, 2, 64, 32), (2, 1, 64, 48), (2, 2, 64, 0), (8, 2, 128, 128), (4, 1, 128, 64), (2, 2, 128, 80),
                                        (3, 3, 128, 16), (2, 1, 64, 16), (2, 1, 128, 112)])
def test_append(H, kv, d, rot, style):
    append_case(H, kv, d, [5, 0, 40, 1, 70], [0, 3, 17, 31, 60], 32, rot, style)


@pytest.mark.parametrize("layout,page,pad", [("NHD", 96, 0), ("NHD", 64, 32), ("HND", 256, 64)])
def test_append_layouts_and_positions(layout, page, pad):
    append_case(4, 2, 64, [1, 1, 1], [5, 0, 99], page, 64, "half", layout, pad)
    append_case(4, 2, 128, [33, 100], [40, 0], page, 64, "pairs", layout, pad, positions=True)


def test_append_what_is_not_finite_and_pages_that_are_not_there():
    append_case(2, 1, 64, [3, 4], [0, 30], 32, 0, "half", bad=True)
    append_case(2, 1, 128, [3, 4], [0, 30], 32, 0, "half", bad=True)


# ---- attend ----------------------------------------------------------------------------------------------------------

def build(H, kv, d, news, lens, page, layout="HND", pad=0, seed=1, k_scale=1.0, spread=False, max_len=0):
    rng = np.random.default_rng([seed, d])
    c = mu.Paged4(kv, d, page, [max(1, -(-n // page)) for n in lens], layout, pad, seed=seed, table_tokens=max_len)
    held = []
    for b, L in enumerate(lens):
        k, v = rng.standard_normal((L, kv, d)) * k_scale, rng.standard_normal((L, kv, d))
        if spread:                                      # tokens and groups of very different size
            m = np.exp2(rng.integers(-6, 7, (L, kv, d // 32))).repeat(32, axis=2)
            k, v = k * m / 8, v * m[::-1]
        held.append(c.fill(b, k, v))
    off = np.concatenate([[0], np.cumsum(news)]).astype(np.int64)
    q = rng.standard_normal((max(int(off[-1]), 1), H, d))
    if spread:
        q *= np.exp2(rng.integers(-12, 1, q.shape))
    return c, held, off, ou.bf16_round(q)


def call(c, H, off, q, lens, max_len, scale, causal=1, window=0, stream=None):
    T, d = int(off[-1]), c.d
    out = torch.full((max(T, 1), H, d), 0x7FC0, dtype=torch.int16, device=DEV)
    lse = torch.full((max(T, 1), H), float("nan"), device=DEV)
    desc = desc_of(c, H)
    ws = torch.full((max(sp.sp_attend_workspace(desc, off.tolist(), len(lens), max_len), 256),), 0xFF, dtype=torch.uint8, device=DEV)
    args = [dev(ou.bf16_bits(q)), off.tolist(), dev(off), dev(np.asarray(lens, dtype=np.int32)), max_len, dev(c.table), dev(c.k), dev(c.v), dev(c.ks), dev(c.vs)]
    torch.cuda.synchronize()
    sp.sp_attend(desc, *args, scale, out, lse, ws, causal=causal, window=window, stream=stream)
    torch.cuda.synchronize()
    return ou.bits_to_f64(out.cpu().numpy().view(np.uint16)), lse.cpu().numpy().astype(np.float64)


def logit_error(q, k, scale):
    """Largest error of a row's logits over keys k: sums of exact products in fp32."""
    return (q.size + 4) * 2.0 ** -24 * float((np.abs(k) @ np.abs(q)).max() * scale)


def verify(c, H, held, off, q, lens, scale, out, lse, causal=1, window=0, rows=None):
    G = H // c.kv
    for b, L in enumerate(lens):
        n = int(off[b + 1] - off[b])
        for r in range(n):
            t = int(off[b]) + r
            if rows is not None and t not in rows:
                continue
            lo, hi = ou.seen(L, n, r, causal, window)
            for h in range(H):
                k, v = held[b][0][:, h // G], held[b][1][:, h // G]
                o, z, A, _ = ou.attend(q[t, h].astype(np.float64), k, v, scale, lo, hi)
                if hi <= lo:
                    assert np.all(out[t, h] == 0) and lse[t, h] == -np.inf, (b, r, h)
                    continue
                dx = logit_error(q[t, h].astype(np.float64), k[lo:hi], scale)
                assert abs(lse[t, h] - z) <= dx + 2.0 ** -20 + 2.0 ** -22 * abs(z), (b, r, h, lse[t, h], z)
                bad = ~(np.abs(out[t, h] - o) <= (2.0 ** -8 + 2 * dx + 2.0 ** -12) * A + 2.0 ** -8 * np.abs(o))
                assert not bad.any(), (b, r, h, np.flatnonzero(bad)[:4], out[t, h][bad][:4], o[bad][:4])


def check(H, kv, d, news, lens, page, layout="HND", pad=0, seed=1, causal=1, window=0, scale=None, max_len=None, rows=None, **kw):
    c, held, off, q = build(H, kv, d, news, lens, page, layout, pad, seed, max_len=max_len or 0, **kw)
    scale = scale or d ** -0.5
    out, lse = call(c, H, off, q, lens, max(lens) if max_len is None else max_len, scale, causal, window)
    verify(c, H, held, off, q, lens, scale, out, lse, causal, window, rows)


SHAPES = [(4, 2, 64), (2, 2, 128), (8, 1, 64), (16, 1, 128), (6, 2, 128), (5, 5, 64)]


@pytest.mark.parametrize("H,kv,d", SHAPES)
def test_single_tokens(H, kv, d):
    check(H, kv, d, [1, 1, 1, 0, 1, 1, 1], [1, 2, 33, 40, 64, 257, 1000], 32)


@pytest.mark.parametrize("H,kv,d", SHAPES[:4])
@pytest.mark.parametrize("layout,page,pad", [("NHD", 96, 32), ("HND", 512, 0)])
def test_a_few_rows(H, kv, d, layout, page, pad):
    check(H, kv, d, [8, 3, 16, 1], [8, 700, 31, 300], page, layout, pad)


@pytest.mark.parametrize("H,kv,d", SHAPES[:3])
@pytest.mark.parametrize("layout,page", [("HND", 64), ("NHD", 32)])
def test_prompt_chunks(H, kv, d, layout, page):
    check(H, kv, d, [130, 1, 67, 300], [130, 90, 500, 333], page, layout)


@pytest.mark.parametrize("causal,window", [(0, 0), (1, 1), (1, 7), (1, 100)])
@pytest.mark.parametrize("news", [[1, 2, 5], [80, 1, 150]])
def test_masks(causal, window, news):
    check(4, 1, 64, news, [200, 45, 310], 64, causal=causal, window=window)
    check(4, 2, 128, news, [200, 45, 310], 64, causal=causal, window=window)


@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_see_nothing_and_empty_contexts(d):
    check(4, 2, d, [5, 3, 1, 100, 2], [2, 0, 0, 30, 2], 32)
    check(4, 2, d, [2, 3], [0, 0], 32, max_len=0)
    check(4, 2, d, [3, 70], [0, 1], 32, causal=0)


@pytest.mark.parametrize("news", [[1, 8], [100, 70]])
@pytest.mark.parametrize("d", [64, 128])
def test_large_logits_and_groups_of_different_size(news, d):
    check(4, 2, d, news, [600, 350], 64, k_scale=12.0)
    check(4, 2, d, news, [600, 350], 64, spread=True)
    check(4, 2, d, news, [600, 350], 64, scale=1e-3)


@pytest.mark.parametrize("news,lens,H,kv,d", [([1], [20000], 8, 2, 64), ([1, 1], [9000, 3], 4, 4, 128), ([8], [6000], 32, 8, 64), ([16], [5000], 4, 2, 128),
                                              ([1, 1, 1, 1], [5000, 4000, 100, 7000], 16, 8, 128), ([300], [4000], 4, 2, 64)])
def test_contexts_shared_out(news, lens, H, kv, d):
    """Long contexts among several workgroups, whose partial results are joined."""
    check(H, kv, d, news, lens, 64, rows=set(range(0, sum(news), max(1, sum(news) // 4))))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [2, 90])
def test_a_nan_gets_out_and_stays_in_its_request(d, n):
    """A group of a key (or value) that says NaN, seen by one request; slots past the contexts say NaN throughout."""
    lens = [200, 100]
    for what in ("ks", "vs"):
        c, held, off, q = build(4, 2, d, [n, n], lens, 64)
        getattr(c, what)[int(c.table[0, 1]), 1, 5, 1] = 255          # token 69 of request 0, kv head 1
        out, lse = call(c, 4, off, q, lens, 200, d ** -0.5)
        first = max(0, 69 - (200 - n))                               # the first row that sees it
        got = out[first:n, 2:]
        assert np.isnan(got).any(axis=-1).all() if what == "vs" else np.isnan(got).all()
        assert np.isfinite(out[n:]).all() and np.isfinite(out[:n, :2]).all()
    q[0, 1, 7] = np.nan
    bits = ou.bf16_bits(np.nan_to_num(q))
    c, held, off, _ = build(4, 2, d, [n, n], lens, 64)
    bits[0, 1, 7] = 0x7FC0
    out, lse = call(c, 4, off, (bits.astype(np.uint32) << 16).view(np.float32), lens, 200, d ** -0.5)
    assert np.isnan(out[0, 1]).all() and np.isnan(lse[0, 1]) and np.isfinite(out[n:]).all() and np.isfinite(out[:n, 2:]).all()


def test_a_far_pool():
    """Pages more than 2^32 bytes from the pool's beginning."""
    d, page, n_pages = 64, 512, (1 << 33) // (512 * 32) // 2 + 8
    kv = 2
    rng = np.random.default_rng(3)
    desc = sp.CacheDesc(4, kv, d, sp.SP_CACHE_MX4, n_pages, page, kv * page * d, page * d, d)
    k, v = (torch.zeros(n_pages, kv, page, d // 2, dtype=torch.uint8, device=DEV) for _ in range(2))
    ks, vs = (torch.full((n_pages, kv, page, d // 32), 127, dtype=torch.uint8, device=DEV) for _ in range(2))
    assert k.numel() > 1 << 32
    table = torch.tensor([[n_pages - 1, n_pages - 3]], dtype=torch.int32, device=DEV)
    L = 700
    x = ou.bf16_round(rng.standard_normal((2, L, kv, d)))
    off = np.array([0, L], dtype=np.int64)
    kd, vd = dev(ou.bf16_bits(x[0]).reshape(L, -1)), dev(ou.bf16_bits(x[1]).reshape(L, -1))
    sp.sp_cache_append(desc, kd, vd, [0, L], dev(off), torch.zeros(1, dtype=torch.int32, device=DEV), table, k, v, ks, vs)
    q = ou.bf16_round(rng.standard_normal((70, 4, d)))
    held = [[mu.values(*mu.quantise(y)) for y in x]]
    for n in (1, 70):
        out, lse = torch.empty(n, 4, d, dtype=torch.bfloat16, device=DEV), torch.empty(n, 4, device=DEV)
        ws = torch.empty(max(256, sp.sp_attend_workspace(desc, [0, n], 1, L)), dtype=torch.uint8, device=DEV)
        sp.sp_attend(desc, dev(ou.bf16_bits(q[:n])), [0, n], torch.tensor([0, n], device=DEV), torch.tensor([L], dtype=torch.int32, device=DEV), L, table,
                     k, v, ks, vs, d ** -0.5, out, lse, ws)
        torch.cuda.synchronize()

        class C:
            pass
        c = C()
        c.kv, c.d = kv, d
        verify(c, 4, held, np.array([0, n]), q, [L], d ** -0.5, out.double().cpu().numpy(), lse.double().cpu().numpy(), rows={0, n - 1})
