"""4-bit caches, attention weights and eviction as programs call them: captured and replayed, on another stream than the current one, two calls at once,
far into large pools, call after call. What they compute is tested elsewhere; here one way of calling is held against another, or against
definitions on a few places."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import mx4_util as mu
import operator_util as ou
import paper_2603_02631_amd as sp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Step:
    """A layer's cache work for a ragged batch: append, attend, weights, evict, on inputs that stay at their addresses."""

    def __init__(self, kind, news, ctx, m, H=8, kv=2, d=64, page=64, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.kind, self.news, self.H, self.kv, self.d, self.m = kind, news, H, kv, d, m
        B, T = len(news), sum(news)
        self.lens_host = [c + n for c, n in zip(ctx, news)]
        self.top = max(self.lens_host)
        width, to = -(-self.top // page), -(-m // page)
        pages = B * (width + to)
        order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
        self.table, self.dst = order[:B * width].view(B, width).contiguous(), order[B * width:].view(B, to).contiguous()
        self.desc = sp.CacheDesc(H, kv, d, sp.SP_CACHE_MX4 if kind == "mx4" else sp.SP_CACHE_BF16, pages, page, kv * page * d, page * d, d)
        self.off_host = sp.host_offsets(np.concatenate([[0], np.cumsum(news)]).tolist())
        self.off = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int64, device=DEV)
        self.start, self.lens = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (ctx, self.lens_host))
        shape = (pages, kv, page, d // 2 if kind == "mx4" else d)
        if kind == "mx4":
            self.k, self.v = (torch.randint(0, 256, shape, dtype=torch.uint8, device=DEV, generator=g) for _ in range(2))
            self.ks, self.vs = (torch.randint(120, 130, (pages, kv, page, d // 32), dtype=torch.uint8, device=DEV, generator=g) for _ in range(2))
        else:
            self.k, self.v = (torch.randn(shape, device=DEV, generator=g).bfloat16() for _ in range(2))
            self.ks = self.vs = None
        self.x = torch.randn(T, (H + 2 * kv) * d, device=DEV, generator=g).bfloat16()
        self.q = torch.empty(T, H, d, dtype=torch.bfloat16, device=DEV)
        self.out, self.lse = torch.empty_like(self.q), torch.empty(T, H, device=DEV)
        angle = torch.rand(self.top, d // 2, device=DEV, generator=g)
        self.cos, self.sin = angle.cos(), angle.sin()
        self.old = torch.rand(B, kv, self.top, device=DEV, generator=g)
        self.w = torch.empty_like(self.old)
        self.ws = torch.empty(max(256, sp.sp_attend_workspace(self.desc, self.off_host, B, self.top)), dtype=torch.uint8, device=DEV)
        self.budget = torch.full((B,), m, dtype=torch.int32, device=DEV)
        self.new_lens = torch.empty(B, dtype=torch.int32, device=DEV)
        self.kept, self.new_w = torch.zeros(B, kv, m, dtype=torch.int32, device=DEV), torch.zeros(B, kv, m, device=DEV)

    def call(self, stream=None):
        H, kv, d = self.H, self.kv, self.d
        q, k, v = self.x.split([H * d, kv * d, kv * d], dim=1)
        sp.sp_cache_append(self.desc, k, v, self.off_host, self.off, self.start, self.table, self.k, self.v, self.ks, self.vs, q=q, q_out=self.q, cos=self.cos,
                           sin=self.sin, rot_dim=d, stream=stream)
        sp.sp_attend(self.desc, self.q, self.off_host, self.off, self.lens, self.top, self.table, self.k, self.v, self.ks, self.vs, d ** -0.5, self.out, self.lse,
                     self.ws, stream=stream)
        sp.sp_attend_weights(self.desc, self.q, self.off_host, self.off, self.lens, self.top, self.table, self.k, self.ks, d ** -0.5, self.lse, self.old, self.w,
                             stream=stream)
        sp.sp_cache_evict(self.desc, self.lens, self.top, self.budget, self.m, 4, 16, self.w, self.table, self.dst, self.k, self.v, self.ks, self.vs, self.new_lens,
                          self.kept, self.new_w, stream=stream)

    def state(self):
        torch.cuda.synchronize()
        parts = [self.k, self.v, self.q, self.out, self.lse, self.new_lens, self.kept, self.new_w]
        rows = [self.w[b, :, :n] for b, n in enumerate(self.lens_host)]
        return [t.clone() for t in (*parts, *rows, *([self.ks, self.vs] if self.ks is not None else []))]


def same(a, b):
    for x, y in zip(a, b):
        assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


NEWS = [([1, 1, 1, 1], [900, 64, 3, 2000]), ([1, 70, 8, 300], [500, 10, 0, 40])]


@pytest.mark.parametrize("kind", ["mx4", "bf16"])
@pytest.mark.parametrize("news,ctx", NEWS)
def test_a_step_gives_the_same_every_time_and_allocates_nothing(kind, news, ctx):
    s = Step(kind, news, ctx, 128)
    s.call()
    want = s.state()
    before = torch.cuda.memory_allocated()
    for _ in range(3):
        s.out.fill_(7)
        s.kept.zero_()
        s.call()
        assert torch.cuda.memory_allocated() == before
        same(s.state(), want)


@pytest.mark.parametrize("kind", ["mx4", "bf16"])
@pytest.mark.parametrize("news,ctx", NEWS)
def test_a_captured_step_replayed_on_new_inputs(kind, news, ctx):
    s = Step(kind, news, ctx, 128)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        s.call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.call()
    for seed in range(3):
        s.x.copy_(torch.randn(s.x.shape, generator=torch.Generator(device=DEV).manual_seed(50 + seed), device=DEV))
        graph.replay()
        got = s.state()
        s.call()
        same(s.state(), got)
        assert not torch.isnan(s.out).any() and not torch.isnan(s.w[0, :, :s.lens_host[0]]).any()


def test_lengths_that_change_between_replays():
    """max_len is what the graph was captured with; the lengths on the device are what counts."""
    s = Step("mx4", [1, 1, 1, 1], [900, 64, 3, 2000], 128)
    s.call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.call()
    for ctx in ([10, 1, 0, 31], [2000, 130, 127, 5]):
        s.start.copy_(torch.tensor(ctx, dtype=torch.int32))
        s.lens.copy_(torch.tensor(ctx, dtype=torch.int32) + 1)
        s.lens_host = [c + 1 for c in ctx]
        graph.replay()
        got = s.state()
        assert s.new_lens.tolist() == [min(n, 128) for n in s.lens_host]
        s.call()
        same(s.state(), got)


@pytest.mark.parametrize("kind", ["mx4", "bf16"])
def test_two_steps_at_once_on_two_streams(kind):
    """Each with its own workspace and caches, neither on the current stream."""
    a, b = Step(kind, *NEWS[0], 128, seed=1), Step(kind, *NEWS[1], 96, H=16, kv=4, seed=2)
    want = []
    for s in (a, b):
        s.call()
        want.append(s.state())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for s in (a, b):
            s.out.fill_(7)
            s.kept.zero_()
        torch.cuda.synchronize()
        for s, stream in zip((a, b), streams):
            s.call(stream.cuda_stream)
        torch.cuda.synchronize()
        same(a.state(), want[0])
        same(b.state(), want[1])


def test_two_products_at_once():
    g = torch.Generator(device=DEV).manual_seed(3)
    M, N, K = 700, 1000, 1024
    w, sw = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device=DEV, generator=g), torch.randint(110, 130, (N, K // 32), dtype=torch.uint8, device=DEV, generator=g)
    streams, jobs = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for rows in (M, 5):
        x = torch.randn(rows, K, device=DEV, generator=g).bfloat16()
        jobs.append((rows, x, torch.empty(rows, K // 2, dtype=torch.uint8, device=DEV), torch.empty(rows, K // 32, dtype=torch.uint8, device=DEV), torch.empty(rows, N, device=DEV)))

    def go(job, stream=None):
        rows, x, codes, scales, out = job
        sp.sp_mx4_quantise(x, rows, K, codes, scales, stream=stream)
        sp.sp_mx4_matmul(codes, scales, rows, w, sw, N, K, out, stream=stream)

    want = []
    for job in jobs:
        go(job)
        torch.cuda.synchronize()
        want.append(job[-1].clone())
    for _ in range(5):
        for job in jobs:
            job[-1].fill_(7)
        torch.cuda.synchronize()
        for job, stream in zip(jobs, streams):
            go(job, stream.cuda_stream)
        torch.cuda.synchronize()
        for job, y in zip(jobs, want):
            assert torch.equal(job[-1], y)


def test_weights_and_eviction_far_into_a_pool():
    """Pages, and their destinations, more than 2^32 bytes from the pool's beginning."""
    d, kv, page, H = 128, 2, 512, 4
    n_pages = (1 << 32) // (page * kv * d * 2) + 20
    desc = sp.CacheDesc(H, kv, d, sp.SP_CACHE_BF16, n_pages, page, kv * page * d, page * d, d)
    pool = torch.zeros(n_pages, kv, page, d, dtype=torch.bfloat16, device=DEV)
    assert pool.nbytes > 1 << 32
    table, dst = (torch.tensor([x], dtype=torch.int32, device=DEV) for x in ([n_pages - 1, n_pages - 3], [n_pages - 2, n_pages - 5]))
    L, m = 700, 600
    rng = np.random.default_rng(4)
    keys = ou.bf16_round(rng.standard_normal((L, kv, d)))
    for at, n in ((0, 512), (512, 188)):
        page_at = int(table[0, at // 512])
        pool[page_at, :, :n] = torch.from_numpy(keys[at:at + n].transpose(1, 0, 2).copy()).bfloat16().to(DEV)
    for n in (1, 40):
        q = ou.bf16_round(rng.standard_normal((n, H, d)))
        w = torch.zeros(1, kv, L, device=DEV)
        qd = torch.from_numpy(q).bfloat16().to(DEV)
        sp.sp_attend_weights(desc, qd, [0, n], torch.tensor([0, n], device=DEV), torch.tensor([L], dtype=torch.int32, device=DEV), L, table, pool, None, d ** -0.5,
                             torch.zeros(n, H, device=DEV), None, w, causal=0)
        x = np.einsum("nhd,lhd->hnl", q.astype(np.float64), keys[:, [0, 0, 1, 1]].astype(np.float64)) * d ** -0.5
        want = np.exp(x).sum(axis=1).reshape(kv, 2, L).sum(axis=1)
        # a logit is off by (d + 4) 2^-24 sum |q||k| scale < 132 * 128 * 25 * 2^-24 / 11 < 2^-8.7; a weight by twice that of itself, and 2^-18 for what follows
        np.testing.assert_allclose(w[0].cpu().numpy(), want, rtol=2.0 ** -7.5)
    new_lens, kept = torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(1, kv, m, dtype=torch.int32, device=DEV)
    sp.sp_cache_evict(desc, torch.tensor([L], dtype=torch.int32, device=DEV), L, torch.tensor([m], dtype=torch.int32, device=DEV), m, 4, 16, w, table, dst, pool, pool, None,
                      None, new_lens, kept)
    assert new_lens.tolist() == [m]
    for h in range(kv):
        tokens = kept[0, h].cpu().numpy()
        assert (np.diff(tokens) > 0).all()
        moved = torch.cat([pool[int(dst[0, 0]), h], pool[int(dst[0, 1]), h, :m - 512]]).float().cpu().numpy()
        np.testing.assert_array_equal(moved, keys[tokens, h])


@pytest.mark.parametrize("B,kv,most", [(40, 8, 2000), (20, 4, 2000), (6, 8, 2000)])
@pytest.mark.parametrize("n", [1, 2])
def test_weights_of_many_contexts(B, kv, most, n):
    """As many pairs of blocks as make a wave take eight, four, two of them; contexts that end before, at and behind a pair's end."""
    H, d, page = 2 * kv, 64, 64
    g = torch.Generator(device=DEV).manual_seed(B)
    lens = [0, 1, 63, 64, 65, most, *np.random.default_rng(B).integers(1, most, B).tolist()][:B]
    width = -(-most // page)
    pool = torch.randn(B * width, kv, page, d, generator=g, device=DEV).bfloat16()
    table = torch.randperm(B * width, generator=g, device=DEV).to(torch.int32).view(B, width)
    q = torch.randn(B * n, H, d, generator=g, device=DEV).bfloat16()
    lse, old = torch.rand(B * n, H, generator=g, device=DEV) + 2, torch.rand(B, kv, most, generator=g, device=DEV)
    w = torch.full_like(old, 7.5)
    off = list(range(0, B * n + 1, n))
    desc = sp.CacheDesc(H, kv, d, sp.SP_CACHE_BF16, B * width, page, kv * page * d, page * d, d)
    sp.sp_attend_weights(desc, q, off, torch.tensor(off, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), most, table, pool, None, d ** -0.5, lse, old, w)
    for b, L in enumerate(lens):
        assert bool((w[b, :, L:] == 7.5).all())
        if not L:
            continue
        k = pool[table[b].long()].transpose(1, 2).reshape(-1, kv, d)[:L].double()
        rows = q[b * n:(b + 1) * n].double().view(n, kv, 2, d)
        for h in range(kv):
            x = rows[:, h].reshape(-1, d) @ k[:, h].t().contiguous() * d ** -0.5
            S = rows[:, h].reshape(-1, d).abs() @ k[:, h].t().contiguous().abs() * d ** -0.5
            z = lse[b * n:(b + 1) * n, 2 * h:2 * h + 2].double().reshape(-1, 1)
            sees = torch.arange(L, device=DEV)[None, :] <= L - n + torch.arange(n, device=DEV).repeat_interleave(2)[:, None]
            p = torch.where(sees, torch.exp(x - z), 0.0)
            before = torch.where(torch.arange(L, device=DEV) < L - n, old[b, h, :L].double(), 0.0)
            want = before + p.sum(dim=0)
            # as for the other contexts: a logit is off by (d + 4) 2^-24 S, what follows adds 2^-22 (|x| + |lse| + 1), the sum half a step for each of its terms
            tol = (2 * p * ((d + 4) * 2.0 ** -24 * S + 2.0 ** -22 * (x.abs() + z.abs() + 1))).sum(dim=0) + (2 * n + 1) * 2.0 ** -24 * want
            assert bool(((w[b, h, :L].double() - want).abs() <= tol).all()), (b, h)


def test_a_projection_whose_codes_pass_two_gigabytes():
    """The last rows of a weight matrix of 2^31 bytes and more of codes, for few rows and for many."""
    K, N = 1 << 14, (1 << 18) + 40
    w = torch.zeros(N, K // 2, dtype=torch.uint8, device=DEV)
    sw = torch.full((N, K // 32), 127, dtype=torch.uint8, device=DEV)
    rng = np.random.default_rng(2)
    code = rng.integers(0, 16, (40, K)).astype(np.uint8)
    w[N - 40:] = torch.from_numpy(mu.pack(code)).to(DEV)
    for M in (2, 60):
        a = rng.integers(0, 16, (M, K)).astype(np.uint8)
        out = torch.empty(M, N, device=DEV)
        sp.sp_mx4_matmul(torch.from_numpy(mu.pack(a)).to(DEV), torch.full((M, K // 32), 127, dtype=torch.uint8, device=DEV), M, w, sw, N, K, out)
        want = mu.VALUES[a] @ mu.VALUES[code].T                 # quarters below 2^20: exact in any order
        np.testing.assert_array_equal(out[:, N - 40:].cpu().numpy(), want)
        assert not out[:, :N - 40].any()
