// sp_cache_evict: the tokens of a paged cache that have drawn the most attention move to other pages, of each kv head by itself, the rest is left behind.
//
// Two launches. sp_evict_select_kernel, a workgroup for each (request, kv head): the weight of the last token that stays, as an exact selection by digits
// of the weights' ordered bits, then a walk over the tokens in order that lists those that stay: all above it, and of those equal to it the first ones. sp_evict_move_kernel: 32 destination slots of a kv head a workgroup, keys and values.
// Out of place: every slot can be moved at once, and pages that requests share stay as they are.
#include "sp_cache.hpp"

namespace {

constexpr int kThreads = 1024;          // of the selection
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 2048;
static_assert(kBins == 2 * kThreads, "two counters a thread");
constexpr int kMoveThreads = 256;
constexpr int kBlock = sp::kCacheBlock;
constexpr int64_t kMaxLen = int64_t(1) << 30;
constexpr int64_t kMaxKept = int64_t(1) << 29;      // a launch's threads fit 32 bits

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;

struct EvictArgs {
    sp::CacheView c;                    // the block table of the source
    const int32_t *dst;
    int64_t dst_stride;
    const int32_t *lens, *budget;
    const float *weights;
    int64_t weights_stride, sinks, recent;
    int32_t max_len, max_budget, B;
    uint8_t *k_pool, *v_pool;
    void *k_scale, *v_scale;
    int32_t *new_lens, *kept;
    float *new_weights;
};

// What request b keeps: n of len tokens, the first `lo` and those from `hi` on among them.
struct Share {
    int len, n, lo, hi;

    __device__ __forceinline__ Share(const EvictArgs &a, int b)
    {
        len = min(max(a.lens[b], 0), a.max_len);
        const int m = min(max(a.budget[b], 0), a.max_budget);
        n = min(len, m);
        lo = (int)min(a.sinks, (int64_t)m);
        hi = len - (int)min(a.recent, (int64_t)(m - lo));
    }
};

// Bits that order as the weights do; -0 as 0.
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __float_as_uint(x);
    if (u == 0x80000000u) return u;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// A wave's stretch of a line's contenders, in order: R weights a lane, 64 neighbours a register. Lines of up to R * 1024 contenders are read once (HELD); longer
// ones R registers at a time in every pass.
template <int R, bool HELD>
struct Stretch {
    const float *w;
    int first, last, lane;
    float x[R];

    __device__ __forceinline__ void load(int at)
    {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            x[r] = 0.f;
            if (at + 64 * r + lane < last) x[r] = w[at + 64 * r + lane];
        }
    }

    // f(token, its weight, whether there is one) in the tokens' order, all lanes together
    template <class F>
    __device__ __forceinline__ void each(F f)
    {
        if constexpr (HELD) {
            int at = __builtin_amdgcn_readfirstlane(first), l = lane;
            asm volatile("" : "+v"(l), "+s"(at));           // nothing of a pass is kept for the next: there are no registers for it
#pragma unroll
            for (int r = 0; r < R; ++r) {
                asm volatile("" : "+v"(x[r]));
                if (at + 64 * r < last) f(at + 64 * r + l, x[r], at + 64 * r + l < last);
            }
        } else
            for (int at = first; at < last; at += 64 * R) {
                load(at);
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (at + 64 * r < last) f(at + 64 * r + lane, x[r], at + 64 * r + lane < last);
            }
    }
};

// Digits of 11, 11 and 10 bits, the most significant first: the first one tells weights apart by two bits of their mantissa, so that lanes seldom meet at a
// counter (with digits of eight bits, most of them at one: 75 us for 16 requests of up to 65536 tokens over 8 kv heads).
template <int R, bool HELD>
__global__ __launch_bounds__(kThreads) void sp_evict_select_kernel(EvictArgs a)
{
    __shared__ uint32_t bins[kBins];
    __shared__ uint32_t wave_sum[kWaves];
    __shared__ int wave_above[kWaves], wave_equal[kWaves];
    __shared__ uint32_t found_digit, found_count;
    __shared__ int found_above;
    const int b = blockIdx.x / a.c.n_kv_heads, kvh = blockIdx.x % a.c.n_kv_heads;
    const Share s(a, b);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int64_t line = (int64_t)b * a.c.n_kv_heads + kvh;
    const float *w = a.weights + line * a.weights_stride;
    int32_t *kept = a.kept + line * a.max_budget;
    float *out = a.new_weights ? a.new_weights + line * a.max_budget : nullptr;
    if (kvh == 0 && tid == 0) a.new_lens[b] = s.n;
    if (s.len == s.n) {                                     // all of them
        for (int i = tid; i < s.n; i += kThreads) {
            kept[i] = i;
            if (out) out[i] = w[i];
        }
        return;
    }
    // tokens [lo, hi) contend for `want` places
    const int want = s.n - s.lo - (s.len - s.hi);
    for (int i = tid; i < s.lo; i += kThreads) {
        kept[i] = i;
        if (out) out[i] = w[i];
    }
    for (int i = tid; i < s.len - s.hi; i += kThreads) {
        const int at = s.lo + want + i;
        kept[at] = s.hi + i;
        if (out) out[at] = w[s.hi + i];
    }
    if (want <= 0) return;
    const int count = s.hi - s.lo, each = ((count + kWaves - 1) / kWaves + 63) / 64 * 64;
    Stretch<R, HELD> mine{w, s.lo + min(wave * each, count), s.lo + min((wave + 1) * each, count), lane};
    if constexpr (HELD) mine.load(mine.first);

    uint32_t prefix = 0, mask = 0;      // digits of the least weight that stays, as far as they are known
    int above = 0;                      // contenders whose digits are larger
#pragma unroll 1
    for (int digit = 0; digit < 3; ++digit) {
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, n_bins = digit == 2 ? 1024 : kBins;
        for (int i = tid; i < kBins; i += kThreads) bins[i] = 0;
        __syncthreads();
        mine.each([&](int, float y, bool in) {
            const uint32_t x = ordered(y), d = x >> shift & (n_bins - 1);
            const bool counts = in && (x & mask) == prefix;
            const uint64_t who = __ballot(counts);
            if (who == 0) return;
            // counts: their order changes nothing. Lanes that all meet at one counter add once
            const int leader = __ffsll((unsigned long long)who) - 1;
            const uint32_t common = (uint32_t)__builtin_amdgcn_readlane((int)d, leader);
            if (__ballot(counts && d != common) == 0) {
                if (lane == leader) atomicAdd(&bins[common], (uint32_t)__popcll(who));
            } else if (counts) atomicAdd(&bins[d], 1u);
        });
        __syncthreads();
        // two counters a thread, the largest digits first
        const uint32_t n0 = bins[kBins - 1 - 2 * tid], n1 = bins[kBins - 2 - 2 * tid], sum = n0 + n1;
        uint32_t upto = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t y = (uint32_t)__shfl_up((int)upto, o);
            if (lane >= o) upto += y;
        }
        if (lane == 63) wave_sum[wave] = upto;
        __syncthreads();
        uint32_t before = above + upto - sum;
#pragma unroll
        for (int v = 0; v < kWaves; ++v)
            if (v < wave) before += wave_sum[v];
        if (before < (uint32_t)want && before + sum >= (uint32_t)want) {
            const bool second = before + n0 < (uint32_t)want;
            found_digit = kBins - 1 - 2 * tid - second;
            found_above = (int)(before + (second ? n0 : 0));
            found_count = second ? n1 : n0;
        }
        __syncthreads();
        prefix |= found_digit << shift;
        mask |= (uint32_t)(n_bins - 1) << shift;
        above = found_above;
        if (above + found_count == (uint32_t)want) break;   // all that share the digits stay
    }
    const int ties = want - above;      // of those that share the known digits the first so many stay

    int more = 0, equal = 0;
    mine.each([&](int, float y, bool in) {
        const uint32_t x = ordered(y) & mask;
        more += __popcll(__ballot(in && x > prefix));
        equal += __popcll(__ballot(in && x == prefix));
    });
    if (lane == 0) {
        wave_above[wave] = more;
        wave_equal[wave] = equal;
    }
    __syncthreads();
    int rank = 0, tied = 0;             // contenders above, and equal ones, before this wave's
#pragma unroll
    for (int v = 0; v < kWaves; ++v)
        if (v < wave) {
            rank += wave_above[v];
            tied += wave_equal[v];
        }
    const uint64_t below = (uint64_t(1) << lane) - 1;
    mine.each([&](int token, float y, bool in) {
        const uint32_t x = ordered(y) & mask;
        const uint64_t up = __ballot(in && x > prefix), eq = __ballot(in && x == prefix);
        const int e = tied + __popcll(eq & below);
        if (in && (x > prefix || (x == prefix && e < ties))) {
            const int at = s.lo + rank + __popcll(up & below) + min(e, ties);
            kept[at] = token;
            if (out) out[at] = y;
        }
        rank += __popcll(up);
        tied += __popcll(eq);
    });
}

// Four codes times a ratio, rounded to codes again; 448 is the largest that comes out, NaN stays NaN.
__device__ __forceinline__ uint32_t rescale4(uint32_t c, float ratio)
{
    const f32x2 x = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), y = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * ratio, x[1] * ratio, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] * ratio, y[1] * ratio, r, true);
    return (uint32_t)r;
}

template <int D, int KIND>
__global__ __launch_bounds__(kMoveThreads) void sp_evict_move_kernel(EvictArgs a)
{
    constexpr int kRow = (int)sp::cache_bytes(KIND, D), kPieces = kRow / 16;        // bytes of a token's head, and 16-byte pieces
    constexpr int kGroups = D / SP_MX4_GROUP;
    __shared__ int64_t from[kBlock], from_scale[kBlock];    // of the slots' tokens: bytes into a pool, and places among the scales
    __shared__ float scale[2][kBlock], ratio[2][kBlock];    // E4M3: keys, values
    const int b = blockIdx.y / a.c.n_kv_heads, kvh = blockIdx.y % a.c.n_kv_heads;
    const Share s(a, b);
    const int slot0 = blockIdx.x * kBlock, count = min(s.n - slot0, kBlock);
    if (count <= 0) return;
    const int64_t page_blocks = a.c.page_tokens / kBlock;
    if (slot0 >= a.dst_stride * a.c.page_tokens) return;
    const int64_t to_page = a.dst[b * a.dst_stride + slot0 / a.c.page_tokens];
    if (to_page < 0 || to_page >= a.c.n_pages) return;
    const int64_t in_page = slot0 % a.c.page_tokens;
    const int64_t to = sp::cache_bytes(KIND, to_page * a.c.page_stride + kvh * a.c.stride_head + in_page * a.c.stride_token);
    const int64_t to_scale = (to_page * a.c.n_kv_heads + kvh) * page_blocks + in_page / kBlock;     // of blocks
    const int64_t token_bytes = sp::cache_bytes(KIND, a.c.stride_token);
    const int tid = threadIdx.x;
    if (tid < count) {
        const int64_t j = a.kept[((int64_t)b * a.c.n_kv_heads + kvh) * a.max_budget + slot0 + tid];
        int64_t page = a.c.table[b * a.c.table_stride + j / a.c.page_tokens];
        page = page < 0 ? 0 : page >= a.c.n_pages ? a.c.n_pages - 1 : page;          // never outside the pools
        const int64_t at = j % a.c.page_tokens, blk = (page * a.c.n_kv_heads + kvh) * page_blocks + at / kBlock;
        from[tid] = sp::cache_bytes(KIND, page * a.c.page_stride + kvh * a.c.stride_head + at * a.c.stride_token);
        from_scale[tid] = KIND == SP_CACHE_MX4 ? (blk * kBlock + at % kBlock) * kGroups : blk;
        if constexpr (KIND == SP_CACHE_E4M3) {
            scale[0][tid] = static_cast<const float *>(a.k_scale)[blk];
            scale[1][tid] = static_cast<const float *>(a.v_scale)[blk];
        }
    }
    __syncthreads();
    if constexpr (KIND == SP_CACHE_E4M3) {
        if (tid < 2 * kBlock) {                             // a half wave for the keys' scales, one for the values'
            const int of = tid / kBlock, i = tid % kBlock;
            const float mine = i < count ? scale[of][i] : scale[of][0];
            float top = mine;
#pragma unroll
            for (int o = 16; o; o >>= 1) top = __builtin_elementwise_maximum(top, __shfl_xor(top, o));
            ratio[of][i] = mine == top ? 1.f : mine / top;
            if (i == 0) static_cast<float *>(of ? a.v_scale : a.k_scale)[to_scale] = top;
        }
        __syncthreads();
    }
    for (int x = tid; x < 2 * count * kPieces; x += kMoveThreads) {
        const int of = x >= count * kPieces, y = x - of * count * kPieces, i = y / kPieces, piece = y % kPieces;
        uint8_t *pool = of ? a.v_pool : a.k_pool;
        u32x4 w = *reinterpret_cast<const u32x4 *>(pool + from[i] + 16 * piece);
        if constexpr (KIND == SP_CACHE_E4M3) {
            const float f = ratio[of][i];
            if (f != 1.f)
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = rescale4(w[e], f);
        }
        *reinterpret_cast<u32x4 *>(pool + to + i * token_bytes + 16 * piece) = w;
    }
    if constexpr (KIND == SP_CACHE_MX4) {
        if (tid < 2 * kBlock && tid % kBlock < count) {
            const int of = tid / kBlock, i = tid % kBlock;
            uint8_t *scales = static_cast<uint8_t *>(of ? a.v_scale : a.k_scale);
            const uint8_t *src = scales + from_scale[i];
            uint8_t *dst = scales + (to_scale * kBlock + i) * kGroups;
            if constexpr (kGroups == 2) *reinterpret_cast<uint16_t *>(dst) = *reinterpret_cast<const uint16_t *>(src);
            else *reinterpret_cast<uint32_t *>(dst) = *reinterpret_cast<const uint32_t *>(src);
        }
    }
}

void select(const EvictArgs &a, dim3 grid, hipStream_t st)
{
    if (a.max_len <= 4 * kThreads) hipLaunchKernelGGL((sp_evict_select_kernel<4, true>), grid, dim3(kThreads), 0, st, a);
    else if (a.max_len <= 16 * kThreads) hipLaunchKernelGGL((sp_evict_select_kernel<16, true>), grid, dim3(kThreads), 0, st, a);
    else if (a.max_len <= 64 * kThreads) hipLaunchKernelGGL((sp_evict_select_kernel<64, true>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((sp_evict_select_kernel<16, false>), grid, dim3(kThreads), 0, st, a);
}

template <int D>
void move(const EvictArgs &a, int kind, dim3 grid, hipStream_t st)
{
    if (kind == SP_CACHE_MX4) hipLaunchKernelGGL((sp_evict_move_kernel<D, SP_CACHE_MX4>), grid, dim3(kMoveThreads), 0, st, a);
    else if (kind == SP_CACHE_E4M3) hipLaunchKernelGGL((sp_evict_move_kernel<D, SP_CACHE_E4M3>), grid, dim3(kMoveThreads), 0, st, a);
    else hipLaunchKernelGGL((sp_evict_move_kernel<D, SP_CACHE_BF16>), grid, dim3(kMoveThreads), 0, st, a);
}

}  // namespace

extern "C" sp_status sp_cache_evict(const sp_cache_desc *desc, int32_t B, const int32_t *lens_dev, int64_t max_len, const int32_t *budget_dev,
                                    int64_t max_budget, int64_t sinks, int64_t recent, const float *weights_dev, int64_t weights_stride,
                                    const int32_t *block_table_dev, int64_t table_stride, const int32_t *dst_table_dev, int64_t dst_stride,
                                    void *k_pool_dev, void *v_pool_dev, void *k_scale_dev, void *v_scale_dev, int32_t *new_lens_dev,
                                    int32_t *kept_dev, float *new_weights_dev, void *hip_stream)
{
    if (sp_status rc = sp::check_cache(desc)) return rc;
    if (B < 0 || B > 4096) return sp::fail(SP_ERR_INVALID_ARG, "B = %d outside 0..4096", B);
    if (max_len < 0 || max_len > kMaxLen) return sp::fail(SP_ERR_INVALID_ARG, "max_len = %lld outside 0..2^30", (long long)max_len);
    if (max_budget < 0 || max_budget > kMaxLen)
        return sp::fail(SP_ERR_INVALID_ARG, "max_budget = %lld outside 0..2^30", (long long)max_budget);
    if (sinks < 0 || recent < 0) return sp::fail(SP_ERR_INVALID_ARG, "sinks = %lld or recent = %lld is negative", (long long)sinks, (long long)recent);
    for (const int64_t stride : {table_stride, dst_stride})
        if (stride < 1 || stride > (int64_t(1) << 31))
            return sp::fail(SP_ERR_INVALID_ARG, "a block table's stride of %lld is outside 1..2^31", (long long)stride);
    if (max_len > table_stride * desc->page_tokens)
        return sp::fail(SP_ERR_INVALID_ARG, "max_len = %lld exceeds the block table's %lld tokens", (long long)max_len,
                        (long long)(table_stride * desc->page_tokens));
    if (weights_stride < max_len || weights_stride > (int64_t(1) << 40))
        return sp::fail(SP_ERR_INVALID_ARG, "weights_stride = %lld is less than max_len = %lld or above 2^40", (long long)weights_stride, (long long)max_len);
    if ((int64_t)B * desc->n_kv_heads > 65535)
        return sp::fail(SP_ERR_UNSUPPORTED, "%d requests of %d kv heads are more than a launch holds", B, desc->n_kv_heads);
    if (B == 0) return SP_OK;
    if (!lens_dev || !budget_dev || !block_table_dev || !dst_table_dev || !new_lens_dev)
        return sp::fail(SP_ERR_INVALID_ARG, "lens_dev, budget_dev, block_table_dev, dst_table_dev or new_lens_dev is null");
    if (lens_dev == new_lens_dev || budget_dev == new_lens_dev)
        return sp::fail(SP_ERR_INVALID_ARG, "new_lens_dev must be neither lens_dev nor budget_dev");
    const int64_t most = max_len < max_budget ? max_len : max_budget;       // tokens that a request keeps at most
    if (max_len > 0 && !weights_dev) return sp::fail(SP_ERR_INVALID_ARG, "weights_dev is null");
    if (most > 0 && !kept_dev) return sp::fail(SP_ERR_INVALID_ARG, "kept_dev is null");
    if (most >= kMaxKept) return sp::fail(SP_ERR_UNSUPPORTED, "%lld kept tokens are more than a launch holds", (long long)most);
    if (sp_status rc = sp::check_pools(*desc, k_pool_dev, v_pool_dev, k_scale_dev, v_scale_dev)) return rc;
    if (new_weights_dev && new_weights_dev == weights_dev) return sp::fail(SP_ERR_INVALID_ARG, "new_weights_dev must not be weights_dev");

    const EvictArgs a{sp::view_of(*desc, block_table_dev, table_stride), dst_table_dev, dst_stride, lens_dev, budget_dev, weights_dev, weights_stride,
                      sinks, recent, (int32_t)max_len, (int32_t)max_budget, B, static_cast<uint8_t *>(k_pool_dev), static_cast<uint8_t *>(v_pool_dev),
                      k_scale_dev, v_scale_dev, new_lens_dev, kept_dev, new_weights_dev};
    const unsigned lines = (unsigned)(B * desc->n_kv_heads);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    select(a, dim3(lines), st);
    SP_HIP_CHECK(hipGetLastError());
    if (most == 0) return SP_OK;
    const dim3 grid((unsigned)sp::ceil_div(most, kBlock), lines);
    if (desc->head_dim == 64) move<64>(a, desc->cache_type, grid, st);
    else move<128>(a, desc->cache_type, grid, st);
    SP_HIP_CHECK(hipGetLastError());
    return SP_OK;
}
