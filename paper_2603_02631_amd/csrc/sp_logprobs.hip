// sp_logprobs: log probabilities of given tokens, entropy and the likeliest tokens of rows of logits (paper: Algorithm 1
// ForwardWithAttn, the end of a draft model's forward pass, where the next lookahead token is picked).
//
// With m = max x, s = sum exp(x - m), u = sum (x - m) exp(x - m):
//   lse = m + log s,  lp_t = (x_t - m) - log s,  H = log s - u / s,
// in one pass: every thread keeps (m, s, u) of its own chunks of 16 bytes (every kThreads-th one) and moves m when a chunk exceeds
// it; the threads' parts are joined at the end.
//
// The likeliest k tokens come out of the same pass. A thread's m and the first chunk that reached it are all that is kept. The k-th best of 64
// groups' maxima is a bound that k elements reach, so the k best elements of the row do, and they lie in the chunks of threads
// whose maximum reaches it: usually k threads of 512. Only those threads' chunks are read a second time. Values are compared together with
// the chunk, lower first, so that rows full of equal logits (forbidden tokens) leave no more to do than others.
// What reached the bound is ranked by counting. Should it not fit the list (hundreds of the best in one thread's chunks),
// the k best are found one by one in the same chunks.
//
// A row belongs to one workgroup; few rows are split among several (a segment of the vocabulary each), whose parts a second launch joins.
// Bound by HBM for many rows: 4096 of 128000 of bf16 190 us, 5.5 TB/s of the 6.3 that a streaming read reaches (each logit costs an exponential and seven more operations,
// at 16 bits a logit about what its bytes take); by latency and two launches for few: one row of 131072 or 64 of 50021 12 us.
#include "sp_common.hpp"

namespace {

constexpr int kTop = SP_LOGPROBS_MAX_TOP;
constexpr int kList = 1024;                 // elements that reach the bound
constexpr int kMaxSplits = 32;
constexpr int64_t kMinSplit = 4096;         // logits of a segment
constexpr float kFar = 1e4f;                // exp(-kFar) is 0
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

struct Args {
    const uint8_t *logits;
    int64_t vocab, row_stride;
    const int32_t *targets;
    float *logprob, *entropy;
    int32_t *top_ids;
    float *top_logprobs;
    int32_t n_top, splits;
    float *part;            // [row][split][4]: m, s, u
    uint64_t *part_keys;    // [row][split][n_top], best first
};

__device__ __forceinline__ float neg_inf() { return -__builtin_huge_valf(); }
__device__ __forceinline__ float exp_(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
__device__ __forceinline__ float log_(float x) { return __builtin_amdgcn_logf(x) * kLn2; }

// Order of logits as unsigned integers, zeros of both signs alike; 0 stands for no logit.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t u = x == 0.f ? 0u : __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }

// Larger key: larger logit, lower token among equals.
__device__ __forceinline__ uint64_t key_of(float x, int64_t i) { return (uint64_t)order_of(x) << 32 | (0xffffffffu - (uint32_t)i); }

// Sums of a part of a row about its maximum (kLowest where it has no finite logit).
struct Sums {
    float m, s, u;

    __device__ __forceinline__ void move(float to)          // to >= m
    {
        const float d = fmaxf(m - to, -kFar), f = exp_(d);
        u = f * (u + d * s);
        s *= f;
        m = to;
    }
};

__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
    return x;
}

__device__ __forceinline__ float wave_sum(float x)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// Joins a wave's lanes; all of them get the result.
__device__ __forceinline__ void join_lanes(Sums &t)
{
    t.move(wave_max(t.m));
    t.s = wave_sum(t.s);
    t.u = wave_sum(t.u);
}

// A row in chunks of 16 bytes that begin at multiples of 16 bytes: the first and the last may hold less than E logits of it.
template <bool BF16>
struct Row {
    static constexpr int E = BF16 ? 8 : 4;
    const uint8_t *base;        // of chunk 0
    int64_t skip, vocab;        // elements of chunk 0 before the row
    uint32_t chunks;

    __device__ __forceinline__ Row(const Args &a, int64_t r)
    {
        const uint8_t *row = a.logits + r * a.row_stride * (BF16 ? 2 : 4);
        const int64_t odd = (int64_t)(reinterpret_cast<uintptr_t>(row) & 15);
        base = row - odd;
        skip = odd / (BF16 ? 2 : 4);
        vocab = a.vocab;
        chunks = (uint32_t)((vocab + skip + E - 1) / E);
    }

    __device__ __forceinline__ int64_t index(uint32_t c, int e) const { return (int64_t)c * E + e - skip; }

    __device__ __forceinline__ bool whole(uint32_t c) const { return index(c, 0) >= 0 && index(c, E) <= vocab; }

    // Logits of a chunk; -inf in the places that are not the row's, which are not read. ONCE: they pass the caches by.
    template <bool ONCE = false>
    __device__ __forceinline__ void load(uint32_t c, float (&x)[E]) const
    {
        if (whole(c)) {
            const u32x4 *p = reinterpret_cast<const u32x4 *>(base + (int64_t)c * 16);
            u32x4 w;
            if constexpr (ONCE) w = __builtin_nontemporal_load(p);
            else w = *p;
#pragma unroll
            for (int e = 0; e < E; ++e)
                x[e] = BF16 ? __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16) : __uint_as_float(w[e % 4]);
            return;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            x[e] = neg_inf();
            if (index(c, e) >= 0 && index(c, e) < vocab) {
                if (BF16) x[e] = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t *>(base + (int64_t)c * 16 + 2 * e) << 16);
                else x[e] = *reinterpret_cast<const float *>(base + (int64_t)c * 16 + 4 * e);
            }
        }
    }

    __device__ __forceinline__ float at(int64_t i) const
    {
        const uint8_t *p = base + (i + skip) * (BF16 ? 2 : 4);
        return BF16 ? __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t *>(p) << 16) : *reinterpret_cast<const float *>(p);
    }
};

// The k-th largest of 64 lanes' values, 0 if fewer than k lanes hold one, and the last chunk that counts among lanes that hold it:
// exactly k of the lanes (or all, if fewer hold a value) are at or before (value, chunk).
__device__ __forceinline__ void bound_of(uint32_t v, uint32_t chunk, int k, uint32_t *value, uint32_t *last)
{
    uint32_t t = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t c = t | 1u << bit;
        if (__popcll(__ballot(v >= c)) >= k) t = c;
    }
    *value = t;
    *last = 0xffffffffu;
    const bool same = v == t;
    const int want = k - __popcll(__ballot(v > t));
    if (t != 0 && __popcll(__ballot(same)) > want) {
        uint32_t lo = 0;                                    // the want-th smallest chunk among them
        for (int bit = 29; bit >= 0; --bit)
            if (__popcll(__ballot(same && chunk < lo + (1u << bit))) < want) lo += 1u << bit;
        *last = lo;
    }
}

template <int kThreads>
struct Shared {
    static constexpr int kWaves = kThreads / 64;
    uint32_t order[kThreads], chunk[kThreads];
    float sums[kWaves][3];
    uint64_t list[kList];
    uint64_t best[kWaves];
    uint16_t column[kThreads];
    uint32_t bound, last, columns, found;
};

template <bool BF16, int kThreads, bool ONCE>
__global__ __launch_bounds__(kThreads) void sp_logprobs_kernel(Args a)
{
    __shared__ Shared<kThreads> sh;
    constexpr int kWaves = kThreads / 64, E = Row<BF16>::E;
    const int64_t r = blockIdx.y;
    const int split = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Row<BF16> row(a, r);
    const uint32_t each = (row.chunks + a.splits - 1) / a.splits;
    const uint32_t from = min(row.chunks, split * each), to = min(row.chunks, from + each);

    Sums t{kLowest, 0.f, 0.f};
    float best = neg_inf();
    uint32_t best_chunk = from + tid;
    constexpr int kUnroll = 2;
    for (uint32_t c0 = from + tid; c0 < to; c0 += kThreads * kUnroll) {
        float x[kUnroll][E];
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            const uint32_t c = c0 + i * kThreads;
            if (c < to) row.template load<ONCE>(c, x[i]);
            else
#pragma unroll
                for (int e = 0; e < E; ++e) x[i][e] = neg_inf();
        }
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            float top = x[i][0];
#pragma unroll
            for (int e = 1; e < E; ++e) top = fmaxf(top, x[i][e]);
            if (top > best) {
                best = top;
                best_chunk = c0 + i * kThreads;
                t.move(top);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float d = fmaxf(x[i][e] - t.m, -kFar), p = exp_(d);
                t.s += p;
                t.u += d * p;
            }
        }
    }

    if (a.n_top > 0) {
        sh.order[tid] = from + tid < to ? order_of(best) : 0u;
        sh.chunk[tid] = best_chunk;
    }
    join_lanes(t);
    if (lane == 0) {
        sh.sums[wave][0] = t.m;
        sh.sums[wave][1] = t.s;
        sh.sums[wave][2] = t.u;
    }
    if (tid == 0) sh.columns = sh.found = 0;
    __syncthreads();
    t = lane < kWaves ? Sums{sh.sums[lane][0], sh.sums[lane][1], sh.sums[lane][2]} : Sums{kLowest, 0.f, 0.f};
    join_lanes(t);
    const float log_s = t.s > 0.f ? log_(t.s) : 0.f;
    if (tid == 0) {
        if (a.splits > 1) {
            float *p = a.part + (r * a.splits + split) * 4;
            p[0] = t.m;
            p[1] = t.s;
            p[2] = t.u;
        } else {
            if (a.logprob) {
                const int64_t i = a.targets[r];
                float lp = 0.f;
                if (i >= 0 && i < a.vocab) {
                    const float x = row.at(i);
                    lp = x == neg_inf() ? x : (x - t.m) - log_s;
                }
                a.logprob[r] = lp;
            }
            if (a.entropy) a.entropy[r] = t.s > 0.f ? log_s - t.u / t.s : 0.f;
        }
    }
    const int k = a.n_top;
    if (k == 0) return;

    if (wave == 0) {                        // lane l: the best of threads l, l + 64, ...
        uint32_t v = 0, c = 0xffffffffu;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t v2 = sh.order[lane + 64 * w], c2 = sh.chunk[lane + 64 * w];
            if (v2 > v || (v2 == v && c2 < c)) {
                v = v2;
                c = c2;
            }
        }
        uint32_t bound, last;
        bound_of(v, c, k, &bound, &last);
        if (lane == 0) {
            sh.bound = bound;
            sh.last = last;
        }
    }
    __syncthreads();
    const uint32_t bound = sh.bound, last = sh.last, mine = sh.order[tid];
    if (mine != 0 && (mine > bound || (mine == bound && sh.chunk[tid] <= last))) sh.column[atomicAdd(&sh.columns, 1u)] = (uint16_t)tid;
    __syncthreads();
    const uint32_t depth = (to - from + kThreads - 1) / kThreads, items = sh.columns * depth;
    for (uint32_t n = tid; n < items; n += kThreads) {
        const uint32_t c = from + sh.column[n / depth] + n % depth * kThreads;
        if (c >= to) continue;
        float x[E];
        row.load(c, x);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint32_t o = order_of(x[e]);
            const int64_t i = row.index(c, e);
            if (i >= 0 && i < a.vocab && (o > bound || (o == bound && c <= last))) {
                const uint32_t at = atomicAdd(&sh.found, 1u);
                if (at < kList) sh.list[at] = key_of(x[e], i);
            }
        }
    }
    __syncthreads();
    const uint32_t found = sh.found;
    const auto report = [&](int rank, uint64_t key) {
        if (a.splits > 1) {
            a.part_keys[(r * a.splits + split) * k + rank] = key;
            return;
        }
        const float x = value_of((uint32_t)(key >> 32));
        a.top_ids[r * k + rank] = (int32_t)(0xffffffffu - (uint32_t)key);
        a.top_logprobs[r * k + rank] = x == neg_inf() ? x : (x - t.m) - log_s;
    };
    if (found <= kList) {
        for (uint32_t i = tid; i < found; i += kThreads) {
            const uint64_t key = sh.list[i];
            int rank = 0;
            for (uint32_t j = 0; j < found; ++j) rank += sh.list[j] > key;
            if (rank < k) report(rank, key);
        }
        for (int i = tid; i < k; i += kThreads)             // a segment with fewer than k logits
            if (i >= (int)found) report(i, 0);
        return;
    }
    uint64_t above = ~0ull;
    for (int i = 0; i < k; ++i) {
        uint64_t top = 0;
        for (uint32_t n = tid; n < items; n += kThreads) {
            const uint32_t c = from + sh.column[n / depth] + n % depth * kThreads;
            if (c >= to) continue;
            float x[E];
            row.load(c, x);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int64_t j = row.index(c, e);
                const uint64_t key = j >= 0 && j < a.vocab ? key_of(x[e], j) : 0;
                if (key < above && key > top) top = key;
            }
        }
#pragma unroll
        for (int o = 32; o; o >>= 1) {
            const uint64_t y = __shfl_xor((unsigned long long)top, o);
            top = y > top ? y : top;
        }
        __syncthreads();
        if (lane == 0) sh.best[wave] = top;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) top = sh.best[w] > top ? sh.best[w] : top;
        if (tid == 0) report(i, top);
        above = top;
    }
}

// Joins the segments of a row, whose best keys are sorted. The first keys of all segments, 64 at most and at least k of them, give a bound
// that k keys reach; what reaches it is ranked by counting.
constexpr int kJoinThreads = 512;

template <bool BF16>
__global__ __launch_bounds__(kJoinThreads) void sp_logprobs_join_kernel(Args a)
{
    __shared__ uint64_t keys[kMaxSplits * kTop], list[kMaxSplits * kTop];
    __shared__ float sums[3];
    __shared__ uint32_t bound, found;
    const int64_t r = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, k = a.n_top;
    for (int i = tid; i < a.splits * k; i += kJoinThreads) keys[i] = a.part_keys[r * a.splits * k + i];
    if (wave == 0) {
        Sums t{kLowest, 0.f, 0.f};
        if (lane < a.splits) {
            const float *p = a.part + (r * a.splits + lane) * 4;
            t = Sums{p[0], p[1], p[2]};
        }
        join_lanes(t);
        if (lane == 0) {
            sums[0] = t.m;
            sums[1] = t.s;
            sums[2] = t.u;
            found = 0;
        }
    }
    __syncthreads();
    if (wave == 1 && k > 0) {
        const int each = 64 / a.splits, s = lane / each, j = lane % each;
        uint32_t value, last;
        bound_of(s < a.splits && j < k ? (uint32_t)(keys[s * k + j] >> 32) : 0u, 0, k, &value, &last);
        if (lane == 0) bound = value;
    }
    __syncthreads();
    const Sums t{sums[0], sums[1], sums[2]};
    const float log_s = t.s > 0.f ? log_(t.s) : 0.f;
    if (tid == 0) {
        if (a.logprob) {
            const int64_t i = a.targets[r];
            float lp = 0.f;
            if (i >= 0 && i < a.vocab) {
                const float x = Row<BF16>(a, r).at(i);
                lp = x == neg_inf() ? x : (x - t.m) - log_s;
            }
            a.logprob[r] = lp;
        }
        if (a.entropy) a.entropy[r] = t.s > 0.f ? log_s - t.u / t.s : 0.f;
    }
    if (k == 0) return;
    for (int i = tid; i < a.splits * k; i += kJoinThreads)
        if (keys[i] != 0 && (uint32_t)(keys[i] >> 32) >= bound) list[atomicAdd(&found, 1u)] = keys[i];
    __syncthreads();
    const int n = (int)found;
    for (int i = tid; i < n; i += kJoinThreads) {
        const uint64_t key = list[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += list[j] > key;
        if (rank < k) {
            const float x = value_of((uint32_t)(key >> 32));
            a.top_ids[r * k + rank] = (int32_t)(0xffffffffu - (uint32_t)key);
            a.top_logprobs[r * k + rank] = x == neg_inf() ? x : (x - t.m) - log_s;
        }
    }
}

// Rows of up to so many chunks of 16 bytes go to workgroups of 256 threads, longer ones to 512: 4096 rows of 1000 fp32 logits take 15 us with 256
// threads and 26 with 512, 300 rows of 128000 bf16 ones 48 and 33.
constexpr int64_t kShort = 2048;

// Long rows are read past the caches where they are fp32 (1000 rows of 50000 40.4 us without, 37.8 with), and of bf16 where they are more bytes than the
// last cache holds: 4096 rows of 128000 195 and 190, but 600 42.7 and 43.1, 300 called again and again 32.5 and 37.6.
constexpr int64_t kOnce = int64_t(1) << 28;

// Segments of a row: as many as keep the device busy (two workgroups of 512 threads on each of 256 compute units; one row of 131072 of bf16 20 us whole, 12.3 in
// 32 segments), unless the row is read in less time than the second launch takes: whole and split, 8 rows of 32000 of bf16 8.7 and 10.5 us, 64 of 50021 11.8 and 12.6,
// but one of 50000 of fp32 13.9 and 10.2.
constexpr int64_t kWholeBytes = 7168 * 16, kTarget = 512;

int splits_of(int64_t n_rows, int64_t vocab, int bytes)
{
    const int64_t want = n_rows > 0 && vocab * bytes > kWholeBytes ? kTarget / n_rows : 1, most = vocab / kMinSplit;
    const int64_t s = want < most ? want : most;
    return (int)(s < 1 ? 1 : (s > kMaxSplits ? kMaxSplits : s));
}

size_t keys_at(int64_t n_rows, int splits) { return sp::align_up((size_t)n_rows * splits * 4 * sizeof(float), 256); }

size_t workspace_need(int64_t n_rows, int splits, int n_top)
{
    if (splits <= 1) return 0;
    return keys_at(n_rows, splits) + sp::align_up((size_t)n_rows * splits * n_top * sizeof(uint64_t), 256);
}

sp_status check_sizes(int64_t n_rows, int64_t vocab, int32_t n_top)
{
    if (n_rows < 0 || n_rows >= (int64_t(1) << 31))
        return sp::fail(SP_ERR_INVALID_ARG, "n_rows = %lld outside 0..2^31-1", (long long)n_rows);
    if (vocab < 1 || vocab >= (int64_t(1) << 31))
        return sp::fail(SP_ERR_INVALID_ARG, "vocab = %lld outside 1..2^31-1", (long long)vocab);
    if (n_top < 0 || n_top > SP_LOGPROBS_MAX_TOP || n_top > vocab)
        return sp::fail(SP_ERR_INVALID_ARG, "n_top = %d outside 0..min(%d, vocab)", n_top, SP_LOGPROBS_MAX_TOP);
    return SP_OK;
}

template <bool BF16>
sp_status run(const Args &a, int64_t n_rows, hipStream_t st)
{
    // rows go to the second grid dimension, 65535 at a time
    for (int64_t r0 = 0; r0 < n_rows; r0 += 65535) {
        const int64_t n = n_rows - r0 < 65535 ? n_rows - r0 : 65535;
        Args b = a;
        b.logits += r0 * a.row_stride * (BF16 ? 2 : 4);
        if (b.targets) b.targets += r0;
        if (b.logprob) b.logprob += r0;
        if (b.entropy) b.entropy += r0;
        if (b.n_top) {
            b.top_ids += r0 * a.n_top;
            b.top_logprobs += r0 * a.n_top;
        }
        const dim3 grid((unsigned)a.splits, (unsigned)n);
        if (a.vocab <= kShort * (BF16 ? 8 : 4)) hipLaunchKernelGGL((sp_logprobs_kernel<BF16, 256, false>), grid, dim3(256), 0, st, b);
        else if (!BF16 || n_rows * a.vocab * 2 > kOnce) hipLaunchKernelGGL((sp_logprobs_kernel<BF16, 512, true>), grid, dim3(512), 0, st, b);
        else hipLaunchKernelGGL((sp_logprobs_kernel<BF16, 512, false>), grid, dim3(512), 0, st, b);
        SP_HIP_CHECK(hipGetLastError());
    }
    if (a.splits > 1) {
        hipLaunchKernelGGL((sp_logprobs_join_kernel<BF16>), dim3((unsigned)n_rows), dim3(kJoinThreads), 0, st, a);
        SP_HIP_CHECK(hipGetLastError());
    }
    return SP_OK;
}

}  // namespace

extern "C" sp_status sp_logprobs_workspace(int64_t n_rows, int64_t vocab, int32_t n_top, size_t *bytes)
{
    if (!bytes) return sp::fail(SP_ERR_INVALID_ARG, "bytes is null");
    if (sp_status rc = check_sizes(n_rows, vocab, n_top)) return rc;
    // for both types, and for fewer rows, which may be split more often: no row is split in more than kTarget / 2 of them
    *bytes = 0;
    for (int64_t n = 1; n <= n_rows && n <= kTarget / 2; ++n) {
        const size_t need = workspace_need(n, splits_of(n, vocab, 4), n_top);
        *bytes = need > *bytes ? need : *bytes;
    }
    return SP_OK;
}

extern "C" sp_status sp_logprobs(const void *logits_dev, int32_t dtype, int64_t n_rows, int64_t vocab, int64_t row_stride,
                                 const int32_t *targets_dev, int32_t n_top, float *logprob_dev, float *entropy_dev,
                                 int32_t *top_ids_dev, float *top_logprobs_dev, void *ws_dev, size_t ws_bytes,
                                 void *hip_stream)
{
    if (sp_status rc = check_sizes(n_rows, vocab, n_top)) return rc;
    if (dtype != SP_LOGITS_F32 && dtype != SP_LOGITS_BF16)
        return sp::fail(SP_ERR_INVALID_ARG, "dtype = %d is neither SP_LOGITS_F32 nor SP_LOGITS_BF16", dtype);
    if (row_stride < vocab || row_stride > (int64_t(1) << 40))
        return sp::fail(SP_ERR_INVALID_ARG, "row_stride = %lld outside vocab..2^40", (long long)row_stride);
    if (!targets_dev != !logprob_dev)
        return sp::fail(SP_ERR_INVALID_ARG, "targets_dev and logprob_dev come together or not at all");
    if (n_rows == 0) return SP_OK;
    if (!logits_dev) return sp::fail(SP_ERR_INVALID_ARG, "logits_dev is null");
    if ((uintptr_t)logits_dev % (dtype == SP_LOGITS_F32 ? 4 : 2) != 0)
        return sp::fail(SP_ERR_INVALID_ARG, "logits_dev is not aligned to its elements");
    if (n_top > 0 && (!top_ids_dev || !top_logprobs_dev))
        return sp::fail(SP_ERR_INVALID_ARG, "top_ids_dev or top_logprobs_dev is null with n_top = %d", n_top);
    const int splits = splits_of(n_rows, vocab, dtype == SP_LOGITS_F32 ? 4 : 2);
    const size_t need = workspace_need(n_rows, splits, n_top);
    if (need > 0) {
        if (!ws_dev) return sp::fail(SP_ERR_WORKSPACE, "ws_dev is null (%zu bytes needed)", need);
        if ((uintptr_t)ws_dev % 256 != 0) return sp::fail(SP_ERR_WORKSPACE, "ws_dev is not 256-byte aligned");
        if (ws_bytes < need) return sp::fail(SP_ERR_WORKSPACE, "workspace too small: %zu < %zu", ws_bytes, need);
    }
    Args a{static_cast<const uint8_t *>(logits_dev), vocab, row_stride, targets_dev, logprob_dev, entropy_dev, top_ids_dev,
           top_logprobs_dev, n_top, splits, static_cast<float *>(ws_dev), nullptr};
    a.part_keys = reinterpret_cast<uint64_t *>(static_cast<uint8_t *>(ws_dev) + keys_at(n_rows, a.splits));
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return dtype == SP_LOGITS_BF16 ? run<true>(a, n_rows, st) : run<false>(a, n_rows, st);
}
