"""sp_mx4_quantise and sp_mx4_matmul against their definitions in 64 bits.

Quantisation is exact: scaling by a power of two is, and the nearest code is one of sixteen. Products of two elements and two powers of two are exact; a sum
of K of them in fp32 is off by at most K 2^-24 sum |a||w| (each addition by half a step of what has been added up), and a bf16 result by 2^-8 of itself."""
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


def rows_of(rows, K, bf16, seed):
    """Groups of very different size, ties between codes, zeros of both signs, the largest and smallest numbers."""
    rng = np.random.default_rng([seed, rows, K])
    x = rng.standard_normal((rows, K)) * np.exp2(rng.integers(-70, 60, (rows, K // 32)).repeat(32, axis=1))
    flat = x.reshape(-1, 32)
    for i in range(flat.shape[0]):
        kind = i % 9
        if kind == 1:
            flat[i] = 0.0
        elif kind == 2:
            flat[i] = -0.0
        elif kind == 3:                             # halfway between codes, with a 6 that fixes the scale
            flat[i] = np.resize([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, 0.0], 32) * 2.0 ** (i % 50 - 20)
        elif kind == 4:                             # all equal: the scale's own boundary
            flat[i] = [6.0, 6.03125, 3.0, 1.5][i // 9 % 4] * 2.0 ** (i % 40 - 20)
        elif kind == 5:
            flat[i, i % 32] = 3.3e38 if i % 2 else -1e-38
        elif kind == 6:
            flat[i] = 2.0 ** -66 * np.arange(32) / 8
    x = flat.reshape(rows, K).astype(np.float32)
    return ou.bf16_round(x) if bf16 else x


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("rows,K,pad", [(1, 32, 0), (1, 64, 0), (3, 96, 8), (7, 4128, 0), (130, 352, 40), (300, 2048, 0)])
def test_quantise(bf16, rows, K, pad):
    x = rows_of(rows, K, bf16, 1)
    wide = np.zeros((rows, K + pad), dtype=np.float32)
    wide[:, :K] = x
    src = dev(ou.bf16_bits(wide)) if bf16 else dev(wide)
    codes = torch.full((rows * K // 2 + 16,), 0xAA, dtype=torch.uint8, device=DEV)
    scales = torch.full((rows * K // 32 + 16,), 0xAA, dtype=torch.uint8, device=DEV)
    sp.sp_mx4_quantise(src, rows, K, codes, scales, dtype=sp.SP_LOGITS_BF16 if bf16 else sp.SP_LOGITS_F32)
    want, s = mu.quantise(x)
    got, gs = codes.cpu().numpy(), scales.cpu().numpy()
    np.testing.assert_array_equal(gs[:-16].reshape(s.shape), s)
    np.testing.assert_array_equal(mu.unpack(got[:-16].reshape(rows, K // 2)), want)
    assert (got[-16:] == 0xAA).all() and (gs[-16:] == 0xAA).all()


@pytest.mark.parametrize("bf16", [True, False])
def test_quantise_what_is_not_finite(bf16):
    x = rows_of(6, 128, bf16, 2)
    x[0, 5], x[1, 40], x[2, 127], x[3, :] = np.inf, -np.inf, np.nan, np.nan
    src = dev(ou.bf16_bits(x)) if bf16 else dev(x)
    if bf16:
        src[2, 127] = 0x7FC0
        src[3, :] = -0x3F
    codes, scales = torch.zeros(6, 64, dtype=torch.uint8, device=DEV), torch.zeros(6, 4, dtype=torch.uint8, device=DEV)
    sp.sp_mx4_quantise(src, 6, 128, codes, scales, dtype=sp.SP_LOGITS_BF16 if bf16 else sp.SP_LOGITS_F32)
    want, s = mu.quantise(x)
    assert (s == 255).sum() == 7
    np.testing.assert_array_equal(scales.cpu().numpy(), s)
    np.testing.assert_array_equal(codes.cpu().numpy(), mu.pack(want))


def operands(M, N, K, seed, spread=4):
    rng = np.random.default_rng([seed, M, N, K])
    out = []
    for n in (M, N):
        codes = rng.integers(0, 16, (n, K)).astype(np.uint8)
        scales = rng.integers(127 - spread, 127 + spread + 1, (n, K // 32)).astype(np.uint8)
        out += [codes, scales]
    return out


def product(a, sa, w, sw, bf16, pad=0):
    M, N, K = a.shape[0], w.shape[0], a.shape[1]
    fill = 0x7FC1 if bf16 else float("nan")
    out = torch.full((M, N + pad), fill, dtype=torch.int16 if bf16 else torch.float32, device=DEV)
    sp.sp_mx4_matmul(dev(mu.pack(a)), dev(sa), M, dev(mu.pack(w)), dev(sw), N, K, out, out_stride=N + pad)
    torch.cuda.synchronize()
    got = out.cpu().numpy()
    got = ou.bits_to_f64(got.view(np.uint16)) if bf16 else got.astype(np.float64)
    if pad:
        assert np.isnan(got[:, N:]).all()
    return got[:, :N]


def verify(got, a, sa, w, sw, bf16):
    K = a.shape[1]
    x, y = mu.values(a, sa), mu.values(w, sw)
    want, size = x @ y.T, np.abs(x) @ np.abs(y).T
    tol = K * 2.0 ** -24 * size + (2.0 ** -8 * np.abs(want) if bf16 else 0)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4])


SIZES = [(1, 1, 32), (1, 33, 64), (2, 16, 96), (16, 16, 128), (17, 31, 160), (5, 1000, 2048), (1, 4096, 4096), (31, 257, 544), (48, 130, 4128), (64, 64, 512),
         (65, 300, 256), (128, 128, 1024), (130, 515, 288), (257, 256, 2048), (300, 77, 32), (513, 641, 352), (1, 5, 8192), (1025, 31, 768), (1030, 2100, 352),
         (3090, 4110, 544), (3090, 4110, 640), (3090, 4110, 128), (1030, 2100, 384), (1030, 2100, 256)]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(bf16, M, N, K):
    ops = operands(M, N, K, 3)
    verify(product(*ops, bf16), *ops, bf16)


@pytest.mark.parametrize("M,N,K,pad", [(3, 17, 64, 5), (40, 96, 160, 1), (200, 130, 256, 3), (129, 254, 96, 2)])
def test_product_into_part_of_rows(M, N, K, pad):
    """Rows at odd places, what lies behind them stays."""
    ops = operands(M, N, K, 4)
    for bf16 in (True, False):
        verify(product(*ops, bf16, pad), *ops, bf16)


@pytest.mark.parametrize("M,N", [(1, 40), (20, 70), (300, 300)])
def test_far_scales_and_nan_rows(M, N):
    """Scales up to 2^100 apart: nothing is lost where the result holds it; a group that says NaN makes its row (or column) NaN and no other."""
    a, sa, w, sw = operands(M, N, 256, 5, spread=25)
    verify(product(a, sa, w, sw, False), a, sa, w, sw, False)
    sa[M // 2, 3] = 255
    sw[N // 3, 7] = 255
    got = product(a, sa, w, sw, False)
    nan = np.zeros((M, N), dtype=bool)
    nan[M // 2], nan[:, N // 3] = True, True
    np.testing.assert_array_equal(np.isnan(got), nan)


@pytest.mark.parametrize("M,N,K", [(1030, 2100, 288), (1030, 2100, 480), (3090, 4110, 96), (3090, 4110, 352)])
def test_what_lies_behind_a_row_adds_nothing_to_tiles(M, N, K):
    """A last step that is not full, with scales far apart, rows of zeros and rows that say NaN in their last group."""
    a, sa, w, sw = operands(M, N, K, 8, spread=25)
    a[::7], w[::5] = 0, 8                                                   # zeros of both signs
    sa[11, -1] = 255
    sw[N - 3, -1] = 255
    got = product(a, sa, w, sw, False)
    nan = np.zeros((M, N), dtype=bool)
    nan[11], nan[:, N - 3] = True, True
    np.testing.assert_array_equal(np.isnan(got), nan)
    zero = np.zeros((M, N), dtype=bool)
    zero[::7], zero[:, ::5] = True, True
    assert (got[zero & ~nan] == 0).all()
    sa[11, -1], sw[N - 3, -1] = 127, 127
    keep = ~nan
    x, y = mu.values(a, sa), mu.values(w, sw)
    want, size = x @ y.T, np.abs(x) @ np.abs(y).T
    assert (np.abs(got - want)[keep] <= (K * 2.0 ** -24 * size)[keep]).all()


@pytest.mark.parametrize("M,N", [(5, 20), (24, 40), (40, 72), (1030, 1100), (3090, 4110)])
@pytest.mark.parametrize("small", [18, 20, 22, 23])
def test_products_far_below_another_one_are_not_dropped(M, N, small):
    """One product of 1, in another group of 32 for every row, and products of 2^-small everywhere else of its row: whatever order they are added in, every
    partial sum is a multiple of 2^-23 below 2, which fp32 holds, so the result is exact."""
    K = 512
    a, w = np.full((M, K), 2, dtype=np.uint8), np.full((N, K), 2, dtype=np.uint8)
    sa, sw = np.full((M, K // 32), 127 - small, dtype=np.uint8), np.full((N, K // 32), 127, dtype=np.uint8)
    for m in range(M):
        g = m % (K // 32)
        sa[m, g] = 127
        a[m, 32 * g:32 * g + 32] = 0
        a[m, 32 * g + 7 * m % 32] = 2 if m % 3 else 10
    want = np.where(np.arange(M) % 3, 1.0, -1.0) + (K - 32) * 2.0 ** -small
    np.testing.assert_array_equal(product(a, sa, w, sw, False), np.broadcast_to(want[:, None], (M, N)))


@pytest.mark.parametrize("M,N", [(3, 20), (20, 20), (40, 70), (700, 1000)])
def test_rows_longer_than_tiles_take(M, N):
    """K just above 2^22: more tiles than few rows have, and still the kernel of few rows; a few elements of a row are not zero, the last ones among them."""
    K = (1 << 22) + 32
    rng = np.random.default_rng(M)
    at = np.unique(np.concatenate([rng.integers(0, K // 2, 60), [0, (1 << 21) - 1, 1 << 21, K // 2 - 1]]))         # bytes
    dense = []
    for n in (M, N):
        codes = torch.zeros(n, K // 2, dtype=torch.uint8, device=DEV)
        some = rng.integers(0, 256, (n, at.size)).astype(np.uint8)
        codes[:, torch.from_numpy(at).to(DEV)] = torch.from_numpy(some).to(DEV)
        dense.append((codes, torch.full((n, K // 32), 127, dtype=torch.uint8, device=DEV), mu.VALUES[mu.unpack(some)]))
    out = torch.empty(M, N, device=DEV)
    sp.sp_mx4_matmul(dense[0][0], dense[0][1], M, dense[1][0], dense[1][1], N, K, out)
    np.testing.assert_array_equal(out.cpu().numpy(), dense[0][2] @ dense[1][2].T)                                # quarters below 2^14: exact


def test_extreme_scale_bytes():
    a, sa, w, sw = operands(5, 20, 64, 6)
    a[:], w[:] = 2, 2
    sa[:, 0], sw[:, 0], sa[:, 1], sw[:, 1] = 254, 2, 0, 254                 # 2^127 2^-125, 2^-127 2^127
    np.testing.assert_array_equal(product(a, sa, w, sw, False), np.full((5, 20), 32 * 4.0 + 32 * 1.0))


@pytest.mark.parametrize("M", [1, 24, 300])
def test_another_stream_and_a_graph(M):
    """Quantisation and product behind each other, as a layer runs them, captured and replayed on new activations."""
    N, K = 200, 512
    _, _, w, sw = operands(M, N, K, 7)
    x = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
    codes, scales = torch.empty(M, K // 2, dtype=torch.uint8, device=DEV), torch.empty(M, K // 32, dtype=torch.uint8, device=DEV)
    wd, swd, out = dev(mu.pack(w)), dev(sw), torch.empty(M, N, device=DEV)

    def layer():
        sp.sp_mx4_quantise(x, M, K, codes, scales)
        sp.sp_mx4_matmul(codes, scales, M, wd, swd, N, K, out)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        layer()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for seed in range(3):
        rng = np.random.default_rng(seed)
        y = ou.bf16_round(rng.standard_normal((M, K)))
        x.copy_(torch.from_numpy(y))
        graph.replay()
        torch.cuda.synchronize()
        a, sa = mu.quantise(y)
        got = out.cpu().numpy().astype(np.float64)
        verify(got, a, sa, w, sw, False)
        layer()
        torch.cuda.synchronize()
        np.testing.assert_array_equal(out.cpu().numpy().astype(np.float64), got)


def test_nothing_to_do():
    sp.sp_mx4_quantise(None, 0, 64, None, None, dtype=sp.SP_LOGITS_BF16)
    z = torch.zeros(0, 5, device=DEV)
    sp.sp_mx4_matmul(None, None, 0, None, None, 5, 64, z)
