"""sp_logprobs against the definition in 64 bits.

Tolerances. The logits are exact inputs. A row's sum of V positive terms in fp32, added up in any order of at most V / 64
terms by one thread and a tree above, is off by at most (V / 64 + 20) 2^-24 of itself, each exponential by 2^-21 of itself (its argument is
rounded once, |x - m| <= 104 where it counts: 104 * 2^-24 < 2^-17, scaled by how much of the sum sits there), and
x - m is rounded once: 2^-24 |x - m|."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import operator_util as ou
import paper_2603_02631_amd as sp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def to_dev(x, bf16):
    t = torch.from_numpy(ou.bf16_bits(x).view(np.int16) if bf16 else np.ascontiguousarray(x, dtype=np.float32)).to(DEV)
    return t


def call(t, rows, vocab, targets, n_top, stream=None):
    lp = torch.full((rows,), 7.0, device=DEV)
    ent = torch.full((rows,), 7.0, device=DEV)
    ids = torch.full((rows, n_top), -5, dtype=torch.int32, device=DEV)
    tlp = torch.full((rows, n_top), 7.0, device=DEV)
    size = sp.sp_logprobs_workspace(rows, vocab, n_top)
    ws = torch.full((max(size, 256),), 0xFF, dtype=torch.uint8, device=DEV)
    tg = torch.from_numpy(np.asarray(targets, dtype=np.int32)).to(DEV)
    torch.cuda.synchronize()
    sp.sp_logprobs(t, rows, vocab, tg, n_top, lp, ent, ids, tlp, ws, stream=stream)
    torch.cuda.synchronize()
    return [a.cpu().numpy() for a in (lp, ent, ids, tlp)]


def close(got, want, tol):
    if np.isinf(want):
        return got == want
    return abs(got - want) <= tol


def check(x, targets, n_top, bf16, vocab=None, stream=None):
    rows, vocab = x.shape[0], vocab or x.shape[1]
    got = call(to_dev(x, bf16), rows, vocab, targets, n_top, stream)
    rel = (vocab / 64 + 20) * 2.0 ** -24 + 2.0 ** -17
    for r in range(rows):
        lp, h, ids, lps, mean = ou.logprobs(x[r, :vocab], int(targets[r]), n_top)
        assert got[2][r].tolist() == ids, (r, got[2][r], ids)
        big = np.abs(x[r, :vocab][np.isfinite(x[r, :vocab])]).max(initial=0)
        assert close(got[0][r], lp, rel + 2.0 ** -22 * (abs(lp) + big)), (r, got[0][r], lp)
        assert close(got[1][r], h, 2 * rel * (1 + mean) + 2.0 ** -22 * h), (r, got[1][r], h)
        for a, b in zip(got[3][r], lps):
            assert close(a, b, rel + 2.0 ** -22 * (abs(b) + big)), (r, a, b)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("rows,vocab,n_top", [(1, 1, 1), (1, 1, 0), (2, 7, 7), (3, 63, 5), (1, 64, 32), (5, 1000, 32), (2, 4097, 20),
                                              (1, 50021, 1), (300, 321, 3), (2, 131072, 8), (9, 20001, 32), (70, 12289, 5)])
def test_logprobs_match_the_definition(bf16, rows, vocab, n_top):
    rng = np.random.default_rng([rows, vocab])
    x = ou.bf16_round(rng.standard_normal((rows, vocab)) * 3) if bf16 else (rng.standard_normal((rows, vocab)) * 3).astype(np.float32)
    targets = rng.integers(0, vocab, rows)
    targets[0] = vocab - 1
    check(x, targets, n_top, bf16)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("rows,vocab,pad", [(3, 1001, 1), (2, 517, 3), (4, 4099, 8), (1, 33333, 2)])
def test_logprobs_of_a_padded_vocabulary_and_odd_strides(bf16, rows, vocab, pad):
    """The padding holds NaN and the largest values: it is never read as a logit."""
    rng = np.random.default_rng(vocab)
    x = ou.bf16_round(rng.standard_normal((rows, vocab + pad)) * 2)
    x[:, vocab:] = 3e38
    x[:, -1] = np.nan
    check(x, rng.integers(0, vocab, rows), 6, bf16, vocab=vocab)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("vocab", [130, 9000])
def test_logprobs_forbidden_tokens_ties_and_empty_rows(bf16, rows, vocab):
    rng = np.random.default_rng(2)
    base = ou.bf16_round(rng.standard_normal((rows, vocab)))
    targets = rng.integers(0, vocab, rows)
    few = np.full((rows, vocab), -np.inf, dtype=np.float32)             # three tokens are allowed, the rest are forbidden
    for r in range(rows):
        few[r, rng.choice(vocab, 3, replace=False)] = ou.bf16_round(rng.standard_normal(3))
    check(few, targets, 8, bf16)
    check(np.full((rows, vocab), -np.inf, dtype=np.float32), targets, 8, bf16)          # none is
    check(np.full((rows, vocab), 1.5, dtype=np.float32), targets, 32, bf16)             # all alike: uniform, lowest ids first
    lowest = np.full((rows, vocab), float(np.array(0xFF7F0000, dtype=np.uint32).view(np.float32)), dtype=np.float32)
    lowest[:, vocab // 2:vocab // 2 + 2] = base[:, :2]                  # forbidden by the type's lowest value
    check(lowest, targets, 5, bf16)
    two = np.zeros((rows, vocab), dtype=np.float32)                     # many ties at two values, zeros of both signs
    two[:, rng.choice(vocab, vocab // 2, replace=False)] = -0.0
    two[:, rng.choice(vocab, 20, replace=False)] = 2.0
    check(two, targets, 32, bf16)


@pytest.mark.parametrize("bf16", [True, False])
def test_logprobs_orders_that_are_hard_to_select_from(bf16):
    """Ascending and descending rows, and all large logits next to each other or one stride apart."""
    for vocab in (6000, 40000):
        up = ou.bf16_round(np.linspace(-9, 9, vocab))
        rows = [up, up[::-1].copy()]
        for step in (1, 8, 64, 256, 1024, 2048):
            x = np.full(vocab, -3.0)
            n = min(600, vocab // step)
            x[3 % step:3 % step + n * step:step][:n] = np.arange(n)[:x[3 % step:3 % step + n * step:step].size] % 97
            rows.append(ou.bf16_round(x))
        check(np.stack(rows).astype(np.float32), np.arange(len(rows)), 32, bf16)


def test_logprobs_range_targets_and_absent_outputs():
    rng = np.random.default_rng(5)
    x = (rng.standard_normal((4, 2000)) * 2).astype(np.float32)
    x[1] += 3e4                                          # a large common offset
    x[2, 77] = 80.0                                      # one token holds nearly everything
    x[3, 5] = -3e38
    check(x, np.array([-1, 2000, 77, 5]), 4, False)      # targets outside the vocabulary give 0
    t = to_dev(x, False)
    ent = torch.empty(4, device=DEV)
    sp.sp_logprobs(t, 4, 2000, None, 0, None, ent, None, None, torch.empty(256 + sp.sp_logprobs_workspace(4, 2000, 0),
                                                                           dtype=torch.uint8, device=DEV))
    full = call(t, 4, 2000, [0] * 4, 3)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(ent.cpu().numpy(), full[1])


def test_logprobs_same_result_every_time_on_any_stream_and_in_graphs():
    rng = np.random.default_rng(6)
    x = ou.bf16_round(rng.standard_normal((3, 60000)) * 2)
    t = to_dev(x, True)
    want = call(t, 3, 60000, [1, 2, 3], 16)
    other = call(t, 3, 60000, [1, 2, 3], 16, stream=torch.cuda.Stream())
    for a, b in zip(want, other):
        np.testing.assert_array_equal(a, b)
    outs = [torch.empty(3, device=DEV), torch.empty(3, device=DEV), torch.empty(3, 16, dtype=torch.int32, device=DEV),
            torch.empty(3, 16, device=DEV)]
    ws = torch.empty(max(256, sp.sp_logprobs_workspace(3, 60000, 16)), dtype=torch.uint8, device=DEV)
    tg = torch.tensor([1, 2, 3], dtype=torch.int32, device=DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sp.sp_logprobs(t, 3, 60000, tg, 16, *outs, ws)
    for _ in range(3):
        for o in outs:
            o.zero_()
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, outs):
            np.testing.assert_array_equal(a, b.cpu().numpy())


def test_logprobs_rows_beyond_32_bit_offsets():
    vocab, stride, rows = 1000, 1 << 30, 3               # the last row begins 2^31 elements in
    buf = torch.zeros((rows - 1) * stride + vocab, dtype=torch.float32, device=DEV)
    rng = np.random.default_rng(7)
    x = rng.standard_normal((rows, vocab)).astype(np.float32)
    for r in range(rows):
        buf[r * stride:r * stride + vocab] = torch.from_numpy(x[r]).to(DEV)
    t = buf.as_strided((rows, vocab), (stride, 1))
    got = call(t, rows, vocab, [4, 5, 6], 3)
    for r in range(rows):
        lp, h, ids, lps, mean = ou.logprobs(x[r], 4 + r, 3)
        assert got[2][r].tolist() == ids and abs(got[0][r] - lp) < 2e-5 and abs(got[1][r] - h) < 2e-5 * (1 + mean)


@pytest.mark.parametrize("bf16,width", [(True, 8), (False, 4)])
@pytest.mark.parametrize("rows", [1, 520])
def test_logprobs_with_the_best_thousands_in_a_few_places(bf16, width, rows):
    """All large logits in the chunks of 16 bytes that eight neighbouring threads of 512 read: thousands of them exceed what a bound on
    threads' maxima can exclude. 520 equal rows take one workgroup each."""
    vocab = 120000
    rng = np.random.default_rng(9)
    x = ou.bf16_round(rng.standard_normal(vocab))
    i = np.arange(vocab)
    here = (i // width) % 512 < 8
    x[here] = ou.bf16_round(20 + rng.standard_normal(int(here.sum())) * 3)
    got = call(to_dev(np.repeat(x[None], rows, axis=0), bf16), rows, vocab, [77] * rows, 32)
    lp, h, ids, lps, mean = ou.logprobs(x, 77, 32)
    assert got[2][0].tolist() == ids
    assert abs(got[0][0] - lp) <= 1e-3 and abs(got[1][0] - h) <= 1e-3
    np.testing.assert_allclose(got[3][0], lps, atol=1e-4)
    for a in got:
        assert (a == a[:1]).all()


def test_more_logits_than_a_cache_holds():
    """Rows of bf16 that are read past the caches; three of them against the definition."""
    rows, vocab, n_top = 1100, 130001, 4
    torch.manual_seed(3)
    t = (torch.randn(rows, vocab, device=DEV) * 3).to(torch.bfloat16)
    targets = np.arange(rows) * 7
    got = call(t, rows, vocab, targets, n_top)
    rel = (vocab / 64 + 20) * 2.0 ** -24 + 2.0 ** -17
    for r in (0, 517, 1099):
        x = t[r].float().cpu().numpy()
        lp, h, ids, lps, mean = ou.logprobs(x, int(targets[r]), n_top)
        assert got[2][r].tolist() == ids
        big = np.abs(x).max()
        assert close(got[0][r], lp, rel + 2.0 ** -22 * (abs(lp) + big))
        assert close(got[1][r], h, 2 * rel * (1 + mean) + 2.0 ** -22 * h)
        assert all(close(a, b, rel + 2.0 ** -22 * (abs(b) + big)) for a, b in zip(got[3][r], lps))
