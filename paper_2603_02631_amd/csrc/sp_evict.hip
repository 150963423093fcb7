// sp_cache_evict: the tokens of a paged cache that have drawn the most attention move to other pages, of each kv head by itself, the rest is left
// behind.
//
// Two launches. sp_evict_select_kernel, a workgroup for each (request, kv head): the weight of the last token that stays, as an exact selection by
// digits of the weights' ordered bits, then a walk over the tokens in order that lists those that stay: all above it, and of those equal to it the
// first ones. sp_evict_move_kernel: 32 destination slots of a kv head a workgroup, keys and values.
// Out of place: every slot can be moved at once, and pages that requests share stay as they are.
#include "sp_cache.hpp"

namespace {

constexpr int kBins = 2048;             // counters of the selection
constexpr int kMoveThreads = 256;
constexpr int kBlock = sp::kCacheBlock;
constexpr int64_t kMaxLen = int64_t(1) << 30;
constexpr int64_t kMaxKept = (int64_t(1) << 29) - kBlock;      // a launch's threads fit 32 bits

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;

struct EvictArgs {
    sp::CacheView c;                    // the block table of the source
    const int32_t *dst;
    int64_t dst_stride;
    const int32_t *lens, *budget;
    const float *weights;
    int64_t weights_stride, sinks, recent;
    int32_t max_len, max_budget;
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

// Bits that order as the weights do (0 added: -0 counts as 0).
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// A wave's stretch of a line's contenders, in order: R times 64 neighbours at a time, as their ordered bits. Stretches that have no more are read
// once (HELD). Places without a token hold 0, which is below every weight (but for one NaN) and behind all tokens. R is small: code that is long
// and passed once waits for its own instructions (with lines of 65536 weights held in registers, R = 64, a call for a line of 1280 took 23 us, with
// R = 8 12).
template <int R, bool HELD>
struct Stretch {
    const float *w;
    int first, last, lane;
    float x[R];

    __device__ __forceinline__ void load(int at)
    {
        const float *src = w + at + lane;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            x[r] = __uint_as_float(0xffffffffu);
            if (at + 64 * (r + 1) <= last) x[r] = src[64 * r];
            else if (at + 64 * r + lane < last) x[r] = src[64 * r];
        }
    }

    // f(the first of 64 tokens, this lane's bits, and its weight as it is) in the tokens' order, all lanes together
    template <class F>
    __device__ __forceinline__ void each(F f)
    {
        if constexpr (!HELD) load(first);
        for (int at = first; at < last; at += 64 * R) {
            uint32_t bits[R];
            float weight[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                weight[r] = x[r];
                bits[r] = ordered(x[r]);
            }
            if constexpr (!HELD)
                if (at + 64 * R < last) load(at + 64 * R);
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (at + 64 * r < last) f(at + 64 * r, bits[r], weight[r]);
        }
    }
};

// Lanes below this one that are in a mask.
__device__ __forceinline__ int rank_in(uint64_t mask) { return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0)); }

// One digit of the selection: of the counters of all values of a digit, the largest first, the one at which `want` contenders are reached.
struct Found {
    uint32_t digit, count;
    int above;                          // contenders with larger digits, those before this digit's among them
};

template <int THREADS>
__device__ __forceinline__ Found find_digit(const uint32_t *bins, int above, int want)
{
    constexpr int kWaves = THREADS / 64, kEach = kBins / THREADS;       // counters of a thread
    __shared__ uint32_t wave_sum[kWaves];
    __shared__ Found found;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    uint32_t n[kEach], sum = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        n[i] = bins[kBins - 1 - (kEach * tid + i)];
        sum += n[i];
    }
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
    if (before < (uint32_t)want && before + sum >= (uint32_t)want)
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (before < (uint32_t)want && before + n[i] >= (uint32_t)want) found = {(uint32_t)(kBins - 1 - (kEach * tid + i)), n[i], (int)before};
            before += n[i];
        }
    __syncthreads();
    return found;
}

// Bound by the chain of passes, not by bytes: 1280 contenders take 7.5 us, up to 65536 of each of 128 lines 30 us, a line's 256 KB read three times
// from L2 by one workgroup. Digits of 11, 11 and 10 bits, the most significant first: that one tells weights apart by two bits of their mantissa.
// Contenders that share it are listed in LDS where they fit, and the other digits are found among them; so a line is read three times: to count, to
// list, and to write down what stays. Where more share it than the list takes, the line is read for each digit, and weights that fall on one counter
// wait for one another: a call for one context of 65536 (131072) tokens that keeps 8192 takes 49 (77) us where weights are spread, 105 (192) where all
// lie between 1 and 1.2, 202 (383) where all are equal; a kv head's line is one workgroup's all the while.
template <int THREADS, int R, bool HELD>
__global__ __launch_bounds__(THREADS) void sp_evict_select_kernel(EvictArgs a)
{
    constexpr int kWaves = THREADS / 64, kList = 4096;
    __shared__ uint32_t bins[kBins];
    __shared__ uint32_t list[kList];
    __shared__ uint16_t list_wave[kList];
    __shared__ int listed, wave_above[kWaves], wave_equal[kWaves];
    const int b = blockIdx.x / a.c.n_kv_heads, kvh = blockIdx.x % a.c.n_kv_heads;
    const Share s(a, b);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int64_t line = (int64_t)b * a.c.n_kv_heads + kvh;
    const float *w = a.weights + line * a.weights_stride;
    int32_t *kept = a.kept + line * a.max_budget;
    float *out = a.new_weights ? a.new_weights + line * a.max_budget : nullptr;
    if (kvh == 0 && tid == 0) a.new_lens[b] = s.n;
    if (s.len == s.n) {                                     // all of them
        for (int i = tid; i < s.n; i += THREADS) {
            kept[i] = i;
            if (out) out[i] = w[i];
        }
        return;
    }
    // tokens [lo, hi) contend for `want` places
    const int want = s.n - s.lo - (s.len - s.hi), count = s.hi - s.lo, each = ((count + kWaves - 1) / kWaves + 63) / 64 * 64;
    Stretch<R, HELD> mine{w, s.lo + min(wave * each, count), s.lo + min((wave + 1) * each, count), lane};
    if (HELD && want > 0) mine.load(mine.first);
    for (int i = tid; i < s.lo; i += THREADS) {
        kept[i] = i;
        if (out) out[i] = w[i];
    }
    for (int i = tid; i < s.len - s.hi; i += THREADS) {
        const int at = s.lo + want + i;
        kept[at] = s.hi + i;
        if (out) out[at] = w[s.hi + i];
    }
    if (want <= 0) return;

    const auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < kBins / THREADS; ++i) bins[tid + i * THREADS] = 0;
        __syncthreads();
    };
    clear();
    mine.each([&](int, uint32_t x, float) { atomicAdd(&bins[x >> 21], 1u); });         // counts: their order changes nothing
    if (tid == 0) listed = 0;
    if (tid < kWaves) wave_equal[tid] = 0;
    __syncthreads();
    Found f = find_digit<THREADS>(bins, 0, want);
    const uint32_t top = f.digit;
    uint32_t least = top << 21;         // the least bits that stay, as far as their digits are known
    // Whether all that share the known digits stay: then what stays is above `below`, and there are no ties to look at. (`least` is not 0 then:
    // something is left behind.)
    bool all = f.above + f.count == (uint32_t)want;
    uint32_t below = all ? least - 1 : 0;
    int more = 0;                       // of this wave, certain to stay
    if (all) {
        mine.each([&](int, uint32_t x, float) { more += __popcll(__ballot(x > below)); });
        if (lane == 0) wave_above[wave] = more;
    } else if (f.count <= kList) {
        mine.each([&](int, uint32_t x, float) {
            more += __popcll(__ballot(x >> 21 > top));
            if (x >> 21 == top) {
                const int at = atomicAdd(&listed, 1);       // in any order: they are only counted
                list[at] = x;
                list_wave[at] = (uint16_t)wave;
            }
        });
        if (lane == 0) wave_above[wave] = more;
        clear();                                            // and the list is there
        for (int i = tid; i < (int)f.count; i += THREADS) atomicAdd(&bins[list[i] >> 10 & 2047], 1u);
        __syncthreads();
        f = find_digit<THREADS>(bins, f.above, want);
        least |= f.digit << 10;
        clear();
        for (int i = tid; i < listed; i += THREADS)
            if (list[i] >> 10 == least >> 10) atomicAdd(&bins[list[i] & 1023], 1u);
        __syncthreads();
        f = find_digit<THREADS>(bins, f.above, want);
        least |= f.digit;
        all = f.above + f.count == (uint32_t)want;
        below = all ? least - 1 : least;
        for (int i = tid; i < listed; i += THREADS) {
            if (list[i] > below) atomicAdd(&wave_above[list_wave[i]], 1);
            else if (list[i] == least) atomicAdd(&wave_equal[list_wave[i]], 1);
        }
    } else {
#pragma unroll 1
        for (int digit = 0; digit < 2; ++digit) {
            const int known = digit == 0 ? 21 : 10, shift = digit == 0 ? 10 : 0, values = digit == 0 ? 2047 : 1023;
            const uint32_t same = least >> known;
            clear();
            mine.each([&](int, uint32_t x, float) {
                if (x >> known == same) atomicAdd(&bins[x >> shift & values], 1u);
            });
            __syncthreads();
            f = find_digit<THREADS>(bins, f.above, want);
            least |= f.digit << shift;
        }
        all = f.above + f.count == (uint32_t)want;
        below = all ? least - 1 : least;
        int equal = 0;
        mine.each([&](int, uint32_t x, float) {
            more += __popcll(__ballot(x > below));
            equal += __popcll(__ballot(x == least));        // looked at where not all of them stay
        });
        if (lane == 0) {
            wave_above[wave] = more;
            wave_equal[wave] = equal;
        }
    }
    __syncthreads();
    int rank = s.lo, tied = 0;          // where this wave's go, without ties, and ties before them
#pragma unroll
    for (int v = 0; v < kWaves; ++v)
        if (v < wave) {
            rank += wave_above[v];
            tied += wave_equal[v];
        }
    if (all) {
        mine.each([&](int token, uint32_t x, float weight) {
            const uint64_t up = __ballot(x > below);
            if (x > below) {
                const uint32_t at = rank + rank_in(up);
                kept[at] = token + lane;
                if (out) out[at] = weight;
            }
            rank += __popcll(up);
        });
        return;
    }
    const int ties = want - f.above;    // of the equal ones the first so many stay
    mine.each([&](int token, uint32_t x, float weight) {
        const uint64_t up = __ballot(x > least), eq = __ballot(x == least);
        const int e = min(tied + rank_in(eq), ties);
        if (x > least || (x == least && e < ties)) {
            const uint32_t at = rank + rank_in(up) + e;
            kept[at] = token + lane;
            if (out) out[at] = weight;
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

// A slot's source is looked up by one thread, its bytes are moved by whole 16-byte pieces, neighbouring threads those of one token. Bound by HBM
// for many tokens: 16 requests that keep 2048 to 8192 tokens of 8 heads of 128 in bf16, 544 MB read and written, take 107 us, 5.1 TB/s (a large
// copy 4.8 to 5.2).
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

template <int THREADS, int R, bool HELD>
void select(const EvictArgs &a, dim3 grid, hipStream_t st)
{
    hipLaunchKernelGGL((sp_evict_select_kernel<THREADS, R, HELD>), grid, dim3(THREADS), 0, st, a);
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
    if (most > kMaxKept) return sp::fail(SP_ERR_UNSUPPORTED, "%lld kept tokens are more than a launch holds", (long long)most);
    if (sp_status rc = sp::check_pools(*desc, k_pool_dev, v_pool_dev, k_scale_dev, v_scale_dev)) return rc;
    if (new_weights_dev && new_weights_dev == weights_dev) return sp::fail(SP_ERR_INVALID_ARG, "new_weights_dev must not be weights_dev");

    const EvictArgs a{sp::view_of(*desc, block_table_dev, table_stride), dst_table_dev, dst_stride, lens_dev, budget_dev, weights_dev, weights_stride,
                      sinks, recent, (int32_t)max_len, (int32_t)max_budget, static_cast<uint8_t *>(k_pool_dev), static_cast<uint8_t *>(v_pool_dev),
                      k_scale_dev, v_scale_dev, new_lens_dev, kept_dev, new_weights_dev};
    const unsigned lines = (unsigned)(B * desc->n_kv_heads);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    // A line of 4000 contenders takes 512 and 1024 threads 11.5 and 12.4 us, moving included, one of 65536 (read in pieces) 65 and 47
    if (max_len <= 4096) select<512, 8, true>(a, dim3(lines), st);
    else select<1024, 8, false>(a, dim3(lines), st);
    SP_HIP_CHECK(hipGetLastError());
    if (most == 0) return SP_OK;
    const dim3 grid((unsigned)sp::ceil_div(most, kBlock), lines);
    if (desc->head_dim == 64) move<64>(a, desc->cache_type, grid, st);
    else move<128>(a, desc->cache_type, grid, st);
    SP_HIP_CHECK(hipGetLastError());
    return SP_OK;
}
