"""sp_cache_append against the definition written out in numpy: byte for byte (the operator rounds every product and sum
to fp32 on its own), and against the formula in 64 bits within the rounding of what the cache holds."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import operator_util as ou
import paper_2603_02631_amd as sp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BLOCK = ou.BLOCK


def dev(a):
    if a is None:
        return None
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view({2: np.int16}.get(a.itemsize, a.dtype) if a.dtype == np.uint16 else a.dtype)).to(DEV)


def table_of(rot, n_pos):
    half = max(rot // 2, 1)
    ang = np.arange(n_pos)[:, None] * (10000.0 ** (-np.arange(half) / half))[None, :]
    return np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)


def desc_of(c, H):
    return sp.CacheDesc(H, c.kv, c.d, sp.SP_CACHE_E4M3 if c.e4m3 else sp.SP_CACHE_BF16, c.n_pages, c.page, c.page_stride,
                        c.stride_head, c.stride_token)


class Reference:
    """The definition applied to a numpy cache, token by token."""

    def __init__(self, c):
        self.c = c

    def store(self, b, start, k, v):
        """k, v: float32 [n][kv][d], rotated already."""
        c, n = self.c, k.shape[0]
        cap = c.table.shape[1] * c.page
        for pool, scales, x in ((c.k, c.ks, k), (c.v, c.vs, v)):
            for j0 in range(start // BLOCK * BLOCK, start + n, BLOCK):
                if j0 >= cap or not 0 <= c.table[b, j0 // c.page] < c.n_pages:
                    continue
                js = [j for j in range(j0, j0 + BLOCK) if start <= j < start + n]
                if not js:
                    continue
                for h in range(c.kv):
                    if not c.e4m3:
                        for j in js:
                            o = c.at(b, h, j)
                            pool[o:o + c.d] = ou.bf16_bits(ou.bf16_round(x[j - start, h]))
                        continue
                    rows = np.stack([x[j - start, h] for j in js]).astype(np.float64)
                    fine = np.isfinite(rows)
                    s = ou.scale_of(np.abs(rows[fine]).max() if fine.any() else 0.0)
                    at = c.scale_at(b, h, j0)
                    if start > j0 and scales[at] >= s:
                        s = float(scales[at])
                    for j in range(j0, min(start, j0 + BLOCK)):
                        o = c.at(b, h, j)
                        old = ou.E4M3[pool[o:o + c.d]] * (float(scales[at]) / s)
                        pool[o:o + c.d] = ou.e4m3_codes(old)
                    scales[at] = s
                    for j, row, ok in zip(js, rows, fine):
                        o = c.at(b, h, j)
                        codes = ou.e4m3_codes(np.where(ok, row, 0.0) / s)
                        pool[o:o + c.d] = np.where(ok, codes, 0x7F)


def same_codes(got, want):
    """Codes are equal, a NaN code's sign aside."""
    nan = (want & 127) == 127
    np.testing.assert_array_equal((got & 127) == 127, nan)
    np.testing.assert_array_equal(got[~nan], want[~nan])


def run(c, H, off, start, qkv, cos, sin, rot, style, positions=None, with_q=True, stream=None, state=None):
    """Calls the library on the reference cache's present contents; returns (k, v, ks, vs, q_out) as numpy."""
    kv, d, T = c.kv, c.d, int(off[-1])
    s = {"k": dev(c.k), "v": dev(c.v), "ks": dev(c.ks) if c.e4m3 else None, "vs": dev(c.vs) if c.e4m3 else None}
    x = dev(ou.bf16_bits(qkv))
    q_out = torch.zeros(max(T, 1), H, d, dtype=torch.int16, device=DEV)
    sp.sp_cache_append(desc_of(c, H), x[:, H * d:(H + kv) * d], x[:, (H + kv) * d:], off, dev(np.asarray(off, dtype=np.int64)),
                       dev(np.asarray(start, dtype=np.int32)), dev(c.table), s["k"], s["v"], s["ks"], s["vs"],
                       q=x[:, :H * d] if with_q else None, q_out=q_out if with_q else None, cos=dev(cos), sin=dev(sin), rot_dim=rot,
                       rot_style=sp.SP_ROTATE_HALF if style == "half" else sp.SP_ROTATE_PAIRS,
                       positions=None if positions is None else dev(np.asarray(positions, dtype=np.int32)))
    torch.cuda.synchronize()
    as_u = (lambda t: t.cpu().numpy()) if c.e4m3 else (lambda t: t.cpu().numpy().view(np.uint16))
    return (as_u(s["k"]), as_u(s["v"]), None if s["ks"] is None else s["ks"].cpu().numpy(),
            None if s["vs"] is None else s["vs"].cpu().numpy(), q_out.cpu().numpy().view(np.uint16))


def check(c, H, news, starts, seed, rot, style, positions=None, with_q=True, scale=1.0, poison=None):
    rng = np.random.default_rng(seed)
    kv, d, T = c.kv, c.d, sum(news)
    off = np.concatenate([[0], np.cumsum(news)]).astype(np.int64).tolist()
    qkv = ou.bf16_round(rng.standard_normal((max(T, 1), (H + 2 * kv) * d)) * scale)
    if poison is not None:
        for t, e, val in poison:
            qkv[t, e] = val
    n_pos = max([s + n for s, n in zip(starts, news)] + [1]) + 5
    cos, sin = table_of(rot, n_pos)
    ref = Reference(c)
    got = None
    want_q = np.zeros((max(T, 1), H, d), dtype=np.uint16)
    rotated = {}
    for b, n in enumerate(news):
        ks = np.zeros((n, kv, d), dtype=np.float32)
        for i in range(n):
            t = off[b] + i
            p = int(np.clip(positions[t] if positions is not None else starts[b] + i, 0, n_pos - 1))
            for h in range(H):
                want_q[t, h] = ou.bf16_bits(ou.bf16_round(ou.rotate(qkv[t, h * d:(h + 1) * d], p, cos, sin, rot, style)))
            for h in range(kv):
                x = qkv[t, (H + h) * d:(H + h + 1) * d]
                ks[i, h] = ou.rotate(x, p, cos, sin, rot, style)
                if poison is None:
                    y = ou.rotate64(x, p, cos, sin, rot, style)
                    assert np.all(np.abs(ks[i, h] - y) <= 2.0 ** -22 * (np.abs(x).max() * 2))
        rotated[b] = (ks, qkv[off[b]:off[b + 1], (H + kv) * d:].reshape(n, kv, d))
    got = run(c, H, off, starts, qkv, cos if rot else None, sin if rot else None, rot, style, positions, with_q)
    for b in range(len(news)):
        ref.store(b, starts[b], *rotated[b])
    if c.e4m3:
        same_codes(got[0], c.k)
        same_codes(got[1], c.v)
        np.testing.assert_array_equal(got[2], c.ks)
        np.testing.assert_array_equal(got[3], c.vs)
    else:
        np.testing.assert_array_equal(got[0], c.k)
        np.testing.assert_array_equal(got[1], c.v)
    if with_q and T:
        np.testing.assert_array_equal(got[4], want_q)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("H,kv,d,rot,style,layout,page,pad", [
    (4, 2, 64, 64, "half", "HND", 32, 0), (4, 2, 64, 32, "pairs", "NHD", 64, 16), (8, 1, 128, 128, "half", "NHD", 32, 0),
    (6, 2, 128, 64, "half", "HND", 96, 32), (2, 2, 128, 48, "pairs", "HND", 64, 0), (3, 3, 64, 0, "half", "NHD", 32, 0),
    (16, 1, 64, 16, "half", "HND", 32, 0), (5, 1, 128, 128, "pairs", "HND", 128, 0)])
def test_append_matches_the_definition(e4m3, H, kv, d, rot, style, layout, page, pad):
    c = ou.Paged(kv, d, page, [4, 4, 4, 4, 4], e4m3, layout, pad, seed=H)
    # a prompt from the start, none, one token, a block's end, and one that crosses several blocks and pages
    check(c, H, [33, 0, 1, 31, 70], [0, 0, 0, 1, 5], 1, rot, style)
    # the same requests go on in the middle of a block: older codes keep or change their scale
    check(c, H, [1, 3, 1, 1, 7], [33, 0, 1, 32, 75], 2, rot, style, scale=4.0)
    check(c, H, [1, 1, 1, 1, 1], [34, 3, 2, 33, 82], 3, rot, style, scale=0.01)
    # rejected tokens are written over
    check(c, H, [2, 0, 1, 0, 3], [33, 0, 2, 0, 82], 4, rot, style)


def test_append_token_by_token_holds_what_one_call_holds():
    """Powers of two: the codes do not depend on how a block was filled, but for values that fell among the subnormals
    on the way (below 2^-6 of the scale then)."""
    rng = np.random.default_rng(8)
    kv, d, H, n = 2, 64, 2, 45
    qkv = ou.bf16_round(rng.standard_normal((n, (H + 2 * kv) * d)) * np.exp2(rng.integers(-3, 4, (n, 1))))
    whole, step = ou.Paged(kv, d, 32, [2], True, seed=1), ou.Paged(kv, d, 32, [2], True, seed=1)
    cos, sin = table_of(64, 64)
    k1, v1, ks1, vs1, q1 = run(whole, H, [0, n], [0], qkv, cos, sin, 64, "half")
    for i in range(n):
        r = run(step, H, [0, 1], [i], qkv[i:i + 1], cos, sin, 64, "half")
        step.k, step.v, step.ks, step.vs = r[:4]
    np.testing.assert_array_equal(ks1, step.ks)
    np.testing.assert_array_equal(vs1, step.vs)
    for a, b in ((k1, step.k), (v1, step.v)):
        fine = (a & 127) >= 16              # E4M3 codes of at least 2^-5: never among the subnormals' neighbours by rounding
        np.testing.assert_array_equal(a[fine], b[fine])
        assert np.all(np.abs(np.nan_to_num(ou.E4M3[a]) - np.nan_to_num(ou.E4M3[b])) <= 2.0 ** -9)


@pytest.mark.parametrize("e4m3", [True, False])
def test_append_places_that_hold_no_page_and_positions(e4m3):
    c = ou.Paged(2, 64, 32, [2, 2, 1], e4m3, seed=3)
    c.table[1, 1] = -1                      # no page: not stored
    c.table[2, 1] = c.n_pages               # nor here
    positions = np.arange(200)[::-1].copy() % 50
    positions[:2] = [-7, 10 ** 6]           # clamped into the table
    check(c, 4, [40, 50, 40], [20, 10, 30], 5, 64, "half", positions=positions)      # 20 + 40 and 30 + 40 pass the table's 64 slots


def test_append_without_queries_and_empty_calls():
    c = ou.Paged(2, 128, 64, [2], True, seed=4)
    check(c, 2, [50], [3], 6, 128, "half", with_q=False)
    check(c, 2, [0], [53], 7, 128, "half")


@pytest.mark.parametrize("d", [64, 128])
def test_append_extreme_values(d):
    """Zeros, the largest bf16 values, the smallest, and values that are not finite: they are stored as NaN codes and do not
    count for the scale."""
    c = ou.Paged(1, d, 32, [3], True, seed=5)
    H = 1
    big = float(np.array(0x7F7F0000, dtype=np.uint32).view(np.float32))
    tiny = float(np.array(0x00010000, dtype=np.uint32).view(np.float32))
    poison = [(3, e, 0.0) for e in range(3 * d)] + [(40, H * d + 5, big), (41, 2 * H * d + 1, -big), (5, 2 * d + 3, np.inf),
                                                    (6, 2 * d + 9, np.nan), (7, d + 7, np.nan), (50, 2 * d + 2, tiny)]
    check(c, H, [64], [0], 9, 0, "half", poison=poison)
    z = ou.Paged(1, d, 32, [2], True, seed=6)
    check(z, H, [33], [0], 10, d, "half", scale=0.0)
    check(z, H, [1], [33], 11, d, "half", scale=1e-30)
    check(z, H, [1], [34], 12, d, "half", scale=1e30)


def test_append_exact_thresholds_of_the_scale():
    """A largest value of exactly 448 s keeps s, the next larger bf16 takes 2 s."""
    for amax, want in ((448.0, 1.0), (450.0, 2.0), (896.0, 2.0), (3.5, 2.0 ** -7), (3.515625, 2.0 ** -6)):
        c = ou.Paged(1, 64, 32, [1], True, seed=7)
        qkv = np.zeros((1, 3 * 64), dtype=np.float32)
        qkv[0, 64] = qkv[0, 128] = amax
        got = run(c, 1, [0, 1], [0], qkv, None, None, 0, "half")
        page = c.table[0, 0]
        assert got[2][page, 0, 0] == want and got[3][page, 0, 0] == want


def test_append_beyond_32_bit_offsets_and_on_another_stream():
    """Pages 2^31 elements apart; the call is enqueued on a stream of its own."""
    kv, d, P, n = 1, 64, 32, 40
    stride = 1 << 31
    pool_k = torch.zeros(stride + P * d, dtype=torch.uint8, device=DEV)
    pool_v = torch.zeros(stride + P * d, dtype=torch.uint8, device=DEV)
    desc = sp.CacheDesc(1, kv, d, sp.SP_CACHE_E4M3, 2, P, stride, P * d, d)
    rng = np.random.default_rng(3)
    qkv = ou.bf16_round(rng.standard_normal((n, 3 * d)))
    scales = torch.zeros(2, 2, 1, 1, device=DEV)
    table, off, start = dev(np.array([[1, 0]], dtype=np.int32)), dev(np.array([0, n])), dev(np.array([0], dtype=np.int32))
    x = dev(ou.bf16_bits(qkv))
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    sp.sp_cache_append(desc, x[:, d:2 * d], x[:, 2 * d:], [0, n], off, start, table, pool_k, pool_v, scales[0], scales[1], stream=st)
    st.synchronize()
    for pool, col, s in ((pool_k, 1, scales[0]), (pool_v, 2, scales[1])):
        hi, lo = pool[stride:stride + P * d].cpu().numpy().reshape(P, d), pool[:P * d].cpu().numpy().reshape(P, d)
        ref = qkv[:, col * d:(col + 1) * d].astype(np.float64)
        for page, rows, part in ((1, hi, ref[:32]), (0, lo, ref[32:])):
            s1 = ou.scale_of(np.abs(part).max())
            assert float(s[page, 0, 0]) == s1
            np.testing.assert_array_equal(rows[:len(part)], ou.e4m3_codes(part / s1))


def test_append_in_place_queries_and_graph_replays():
    """q_out may be q; a recorded call gives on every replay what the eager call gives."""
    kv, d, H, P, B = 2, 64, 4, 64, 3
    rng = np.random.default_rng(4)
    desc = sp.CacheDesc(H, kv, d, sp.SP_CACHE_E4M3, 4, P, kv * P * d, P * d, d)
    bits = lambda *s: dev(ou.bf16_bits(ou.bf16_round(rng.standard_normal(s))))
    q, k, v = bits(B, H * d), bits(B, kv * d), bits(B, kv * d)
    cos, sin = (dev(t) for t in table_of(64, 64))
    off, table = dev(np.arange(B + 1)), dev(np.array([[0], [3], [1]], dtype=np.int32))
    pools = [torch.zeros(4 * kv * P * d, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.zeros(4, kv, P // 32, device=DEV) for _ in range(2)]
    start = torch.tensor([0, 5, 31], dtype=torch.int32, device=DEV)
    work = q.clone()

    def call(q_in, q_out):
        sp.sp_cache_append(desc, k, v, list(range(B + 1)), off, start, table, *pools, *scales, q=q_in, q_out=q_out, cos=cos, sin=sin,
                           rot_dim=64)

    out = torch.zeros_like(q)
    call(q, out)
    eager = [t.clone() for t in pools + scales]
    call(work, work)
    torch.cuda.synchronize()
    assert torch.equal(work, out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(q, out)
    for step in range(3):
        for t in pools + scales + [out]:
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, work)
        # everything lies on zeroed pools; where nothing was there before, a single token sets its block's scale
        if step == 0:
            first = [t.clone() for t in pools + scales]
        for t, u in zip(pools + scales, first):
            assert torch.equal(t, u)
    assert torch.equal(pools[0], eager[0]) and torch.equal(scales[1], eager[3])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale", [7.0, 14.0, 3.0, 0.4375, 1.7])
def test_append_behind_tokens_whose_scale_is_no_power_of_two(d, scale):
    """Pages that something else has filled: codes are those of x / s, half-way cases among them (175 / 7 = 25 lies between 24 and 26), which x times
    the rounded 1 / s misses."""
    c = ou.Paged(1, d, 32, [1], True, seed=11)
    page, rng = c.table[0, 0], np.random.default_rng(15)
    c.ks[page, 0, 0] = c.vs[page, 0, 0] = scale
    for j in range(3):
        c.k[c.at(0, 0, j):c.at(0, 0, j) + d] = rng.integers(0, 120, d)
        c.v[c.at(0, 0, j):c.at(0, 0, j) + d] = rng.integers(0, 120, d)
    n = 20
    half = rng.integers(8, 16, (n, 3 * d)) * 2 + 1                  # of codes 16 .. 30, two apart
    qkv = ou.bf16_round((half * np.float32(scale) * np.exp2(rng.integers(-6, 3, half.shape))).astype(np.float32) * rng.choice([-1, 1], half.shape))
    qkv = np.clip(qkv, -128 * scale, 128 * scale).astype(np.float32)
    qkv = ou.bf16_round(qkv)
    got = run(c, 1, [0, n], [3], qkv, None, None, 0, "half")
    Reference(c).store(0, 3, qkv[:, None, d:2 * d], qkv[:, None, 2 * d:])
    assert c.ks[page, 0, 0] == np.float32(scale)
    same_codes(got[0], c.k)
    same_codes(got[1], c.v)
    np.testing.assert_array_equal(got[2], c.ks)
    np.testing.assert_array_equal(got[3], c.vs)
