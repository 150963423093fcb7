// sp_cache_append: keys and values of new tokens into a paged cache, rotated on the way, with the queries beside them
// (paper: Algorithm 1 ForwardWithAttn, what a decoder layer does before its attention).
//
// Rotation of the pair (x, y) of index i at position p by the angle whose cosine and sine the table holds:
//   (x c - y s, y c + x s), each product and sum rounded to fp32 (no contraction: the bytes that land in the cache do
//   not depend on how a compiler fuses them).
// E4M3: with m the largest magnitude of the block's new tokens, the scale is the smallest power of two s >= 2^-64 with
//   m <= 448 s. Powers of two, because a block fills up over many calls: when a later token is larger, the older codes
//   are brought to the larger scale by shifting exponents, exactly but for what falls among the subnormals (below
//   2^-14 of the block's largest value), so a cache filled token by token holds what one filled at once does.
// MX4: each 32 elements of a token's head have a scale of their own (sp_mx4.hpp). Its largest magnitude lies in up to D / 16 neighbouring threads,
// in which of
//   them the rotation's pairing decides; they meet by shuffles of the wave, and no other token is looked at.
//
// One workgroup owns 32 cache slots (the tokens of one scale) of one kv head: keys, values and the queries of the head's group. A thread owns two
// vectors of eight elements of a token that the rotation pairs up, so that a pair never leaves its thread and the token's cosines and sines are
// loaded once for the key and all query heads.
// Bound by HBM for long inputs: 16 ragged chunks of 300 to 4096 tokens (32 query heads of 128 over 4, E4M3) 106 us, 4.9 TB/s read and written of
// the 5.2 that a large copy reaches (MX4 104 us, 4.8 TB/s of 504 MB, most of it inputs and queries; a single token 4.5 us in the kernel); a prompt
// of 8192 tokens (32 heads of 64 over 8, bf16), one round of workgroups, 26 us, 4.0. By a chain of four dependent loads (offsets, block table,
// inputs, old codes) and the call itself for single tokens: 13 us. With the kv heads of the same tokens far apart in the grid the chunks took 114.
#include "sp_cache.hpp"
#include "sp_mx4.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kBlock = sp::kCacheBlock;
constexpr float kFloorExp = -64;        // log2 of the smallest scale
constexpr int64_t kMaxGroups = int64_t(1) << 24;    // a launch's threads fit 32 bits

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;

struct AppendArgs {
    sp::CacheView c;
    const uint16_t *k, *v, *q;
    uint16_t *q_out;
    int64_t k_stride, v_stride, q_stride;
    const int64_t *off;
    const int32_t *start, *positions;
    const float *cos, *sin;
    int64_t n_pos;
    uint8_t *k_pool, *v_pool;
    void *k_scale, *v_scale;
    int32_t B, rot;
    bool single;        // no request brings more than one token: item x belongs to request x
};

__device__ __forceinline__ void unpack(u32x4 w, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

// Two floats to a pair of bf16, rounded to nearest.
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}

__device__ __forceinline__ u32x4 pack(const float (&x)[8])
{
    return u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
}

// The two vectors of thread v of a token: where they begin in a head, and whether they are rotated.
struct Lanes {
    int lo, hi;
    bool turned;
};

template <bool PAIRS>
__device__ __forceinline__ Lanes lanes_of(int v, int rot)
{
    if (PAIRS) return {16 * v, 16 * v + 8, 16 * v < rot};
    if (16 * v < rot) return {8 * v, 8 * v + rot / 2, true};
    return {16 * v, 16 * v + 8, false};
}

template <bool PAIRS>
__device__ __forceinline__ void rotate(float (&lo)[8], float (&hi)[8], const float (&c)[8], const float (&s)[8])
{
#pragma clang fp contract(off)
    if (PAIRS) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = lo[2 * i], y = lo[2 * i + 1], z = hi[2 * i], w = hi[2 * i + 1];
            lo[2 * i] = x * c[i] - y * s[i];
            lo[2 * i + 1] = y * c[i] + x * s[i];
            hi[2 * i] = z * c[4 + i] - w * s[4 + i];
            hi[2 * i + 1] = w * c[4 + i] + z * s[4 + i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = lo[i], y = hi[i];
            lo[i] = x * c[i] - y * s[i];
            hi[i] = y * c[i] + x * s[i];
        }
    }
}

__device__ __forceinline__ uint32_t magnitude(float x)
{
    const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;        // what is not finite does not count
}

// Exponent of the smallest power of two s >= 2^-64 with m <= 448 s; 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_exponent(uint32_t m)
{
    const int e = (int)(m >> 23) - 135 + ((m & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < (int)kFloorExp ? (int)kFloorExp : e;
}

__device__ __forceinline__ float exp2_of(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d)
{
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
    return (uint32_t)r;
}

__device__ __forceinline__ u32x2 quantise(const float (&x)[8], float inv)
{
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        y[i] = (__float_as_uint(x[i]) & 0x7f800000u) == 0x7f800000u ? __uint_as_float(0x7fc00000u) : x[i] * inv;
    return u32x2{codes4(y[0], y[1], y[2], y[3]), codes4(y[4], y[5], y[6], y[7])};
}

// Codes times a power of two of at most one, rounded to codes again.
__device__ __forceinline__ u32x2 rescale(u32x2 c, float ratio)
{
    u32x2 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        typedef __attribute__((ext_vector_type(2))) float f32x2;
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], true);
        r[i] = codes4(a.x * ratio, a.y * ratio, b.x * ratio, b.y * ratio);
    }
    return r;
}

// Which request item x (a block of slots) belongs to, and which of its blocks that is. Request b's items begin at
// off[b] / 32 + 2 b: enough, since n tokens from any slot touch at most n / 32 + 2 blocks (rounded down).
__device__ __forceinline__ int find_request(const AppendArgs &a, int x, int64_t *first)
{
    if (a.single) {
        *first = x;
        return x;
    }
    int lo = 0, hi = a.B;           // the last request that begins at or before x
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.off[mid] / kBlock + 2 * (int64_t)mid <= x) lo = mid; else hi = mid;
    }
    *first = a.off[lo] / kBlock + 2 * (int64_t)lo;
    return lo;
}

template <int D, int KIND, bool PAIRS>
__global__ __launch_bounds__(kThreads) void sp_cache_append_kernel(AppendArgs a)
{
    constexpr bool E4M3 = KIND == SP_CACHE_E4M3, MX4 = KIND == SP_CACHE_MX4;
    constexpr int kVecs = D / 16;                       // threads of a token
    constexpr int kParts = kThreads / (kBlock * kVecs); // 2 at head_dim 64: half the threads take keys, half values
    __shared__ uint32_t wave_max[2][kThreads / 64];

    // the kv heads of the same tokens side by side: their parts of a token's row are neighbours in memory
    const uint32_t x = blockIdx.x / (uint32_t)a.c.n_kv_heads;
    int64_t first;
    const int b = find_request(a, (int)x, &first);
    const int64_t t0 = a.off[b], n = a.off[b + 1] - t0;
    const int64_t start = a.start[b] > 0 ? a.start[b] : 0, end = start + n;
    const int64_t slot0 = (start / kBlock + ((int64_t)x - first)) * kBlock;
    if (n == 0 || slot0 >= end) return;

    const int kvh = blockIdx.x % (uint32_t)a.c.n_kv_heads, tid = threadIdx.x;
    const int part = kParts == 2 ? tid / (kThreads / 2) : 0, slot = tid / kVecs % kBlock, vec = tid % kVecs;
    const int64_t at = slot0 + slot;
    const bool fresh = at >= start && at < end, older = at < start;
    const int64_t t = fresh ? t0 + (at - start) : t0;
    const Lanes ln = lanes_of<PAIRS>(vec, a.rot);

    float c[8], s[8];
    if (fresh && ln.turned) {
        int64_t p = a.positions ? a.positions[t] : at;
        p = p < 0 ? 0 : (p >= a.n_pos ? a.n_pos - 1 : p);
        const f32x4 *cp = reinterpret_cast<const f32x4 *>(a.cos + p * (a.rot / 2) + 8 * vec);
        const f32x4 *sp = reinterpret_cast<const f32x4 *>(a.sin + p * (a.rot / 2) + 8 * vec);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            c[i] = cp[i / 4][i % 4];
            s[i] = sp[i / 4][i % 4];
        }
    }

    // the block's page: -1 where nothing is stored
    int64_t page = -1;
    if (slot0 < a.c.table_stride * a.c.page_tokens) page = a.c.table[b * a.c.table_stride + slot0 / a.c.page_tokens];
    const bool stored = page >= 0 && page < a.c.n_pages;
    const int64_t in_page = slot0 % a.c.page_tokens;
    const int64_t elem = page * a.c.page_stride + kvh * a.c.stride_head + (in_page + slot) * a.c.stride_token;
    const int64_t scale_at = (page * a.c.n_kv_heads + kvh) * (a.c.page_tokens / kBlock) + in_page / kBlock;

    if (stored) {
        constexpr int kItems = 2 / kParts;              // keys and values of a thread
        float lo[kItems][8], hi[kItems][8];
        uint32_t m[kItems];
        float old[kItems];
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const bool val = kItems == 2 ? i == 1 : part == 1;
            m[i] = 0;
            old[i] = 0.f;
            if (fresh) {
                const uint16_t *src = val ? a.v + t * a.v_stride : a.k + t * a.k_stride;
                unpack(*reinterpret_cast<const u32x4 *>(src + kvh * D + ln.lo), lo[i]);
                unpack(*reinterpret_cast<const u32x4 *>(src + kvh * D + ln.hi), hi[i]);
                if (!val && ln.turned) rotate<PAIRS>(lo[i], hi[i], c, s);
            }
            if (E4M3) {
                if (start > slot0) old[i] = static_cast<const float *>(val ? a.v_scale : a.k_scale)[scale_at];
                if (fresh)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t x = magnitude(lo[i][e]), y = magnitude(hi[i][e]);
                        m[i] = max(m[i], max(x, y));
                    }
#pragma unroll
                for (int o = 32; o; o >>= 1) m[i] = max(m[i], (uint32_t)__shfl_xor((int)m[i], o));
                if ((tid & 63) == 0) wave_max[i][tid >> 6] = m[i];
            }
        }
        if (E4M3) __syncthreads();                      // maxima are there, old scales have been read
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const bool val = kItems == 2 ? i == 1 : part == 1;
            if constexpr (MX4) {
                // A group's largest magnitude: of the octets of a token's neighbouring threads that lie in it.
                constexpr int kGroups = D / sp::kMx4Group;
                uint32_t tops[2] = {0, 0};
                if (fresh)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        tops[0] = max(tops[0], sp::mx4_magnitude(lo[i][e]));
                        tops[1] = max(tops[1], sp::mx4_magnitude(hi[i][e]));
                    }
                const int glo = ln.lo / sp::kMx4Group, ghi = ln.hi / sp::kMx4Group;
                int blo = 0, bhi = 0;
                uint32_t bytes = 0;
#pragma unroll
                for (int n = 0; n < kGroups; ++n) {
                    uint32_t top = max(glo == n ? tops[0] : 0u, ghi == n ? tops[1] : 0u);
#pragma unroll
                    for (int o = 1; o < kVecs; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
                    const int byte = sp::mx4_scale(top);
                    if (glo == n) blo = byte;
                    if (ghi == n) bhi = byte;
                    bytes |= (uint32_t)byte << (8 * n);
                }
                if (fresh) {
                    uint8_t *dst = (val ? a.v_pool : a.k_pool) + elem / 2;
                    *reinterpret_cast<uint32_t *>(dst + ln.lo / 2) = sp::mx4_codes(lo[i], blo);
                    *reinterpret_cast<uint32_t *>(dst + ln.hi / 2) = sp::mx4_codes(hi[i], bhi);
                    if (vec == 0) {
                        uint8_t *to = static_cast<uint8_t *>(val ? a.v_scale : a.k_scale) + (scale_at * kBlock + slot) * kGroups;
                        if constexpr (kGroups == 2) *reinterpret_cast<uint16_t *>(to) = (uint16_t)bytes;
                        else *reinterpret_cast<uint32_t *>(to) = bytes;
                    }
                }
                continue;
            }
            if (!E4M3) {
                if (fresh) {
                    uint16_t *dst = reinterpret_cast<uint16_t *>(val ? a.v_pool : a.k_pool) + elem;
                    *reinterpret_cast<u32x4 *>(dst + ln.lo) = pack(lo[i]);
                    *reinterpret_cast<u32x4 *>(dst + ln.hi) = pack(hi[i]);
                }
                continue;
            }
            constexpr int kWaves = kThreads / 64 / kParts;
            uint32_t all = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) all = max(all, wave_max[i][part * kWaves + w]);
            const int e = scale_exponent(all);
            float scale = exp2_of(e), inv = exp2_of(-e);
            if (old[i] > scale) {
                scale = old[i];
                inv = 1.f / scale;
                if (fresh && (__float_as_uint(scale) & 0x7fffffu) != 0) {    // not of this call's making: only a quotient is x / s there
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        lo[i][e] /= scale;
                        hi[i][e] /= scale;
                    }
                    inv = 1.f;
                }
            }
            uint8_t *dst = (val ? a.v_pool : a.k_pool) + elem;
            if (fresh) {
                *reinterpret_cast<u32x2 *>(dst + ln.lo) = quantise(lo[i], inv);
                *reinterpret_cast<u32x2 *>(dst + ln.hi) = quantise(hi[i], inv);
            } else if (older && old[i] != scale) {
                const float ratio = old[i] * inv;
                u32x2 *lp = reinterpret_cast<u32x2 *>(dst + ln.lo), *hp = reinterpret_cast<u32x2 *>(dst + ln.hi);
                *lp = rescale(*lp, ratio);
                *hp = rescale(*hp, ratio);
            }
            if (slot == 0 && vec == 0) static_cast<float *>(val ? a.v_scale : a.k_scale)[scale_at] = scale;
        }
    }

    if (a.q && fresh)
        for (int g = part; g < a.c.group; g += kParts) {
            const int h = kvh * a.c.group + g;
            const uint16_t *src = a.q + t * a.q_stride + (int64_t)h * D;
            uint16_t *dst = a.q_out + (t * a.c.n_q_heads + h) * D;
            float lo[8], hi[8];
            unpack(*reinterpret_cast<const u32x4 *>(src + ln.lo), lo);
            unpack(*reinterpret_cast<const u32x4 *>(src + ln.hi), hi);
            if (ln.turned) rotate<PAIRS>(lo, hi, c, s);
            *reinterpret_cast<u32x4 *>(dst + ln.lo) = pack(lo);
            *reinterpret_cast<u32x4 *>(dst + ln.hi) = pack(hi);
        }
}

template <int D, int KIND>
void launch(const AppendArgs &a, bool pairs, dim3 grid, hipStream_t st)
{
    if (pairs)
        hipLaunchKernelGGL((sp_cache_append_kernel<D, KIND, true>), grid, dim3(kThreads), 0, st, a);
    else
        hipLaunchKernelGGL((sp_cache_append_kernel<D, KIND, false>), grid, dim3(kThreads), 0, st, a);
}

template <int D>
void launch_kind(const AppendArgs &a, int kind, bool pairs, dim3 grid, hipStream_t st)
{
    if (kind == SP_CACHE_MX4) launch<D, SP_CACHE_MX4>(a, pairs, grid, st);
    else if (kind == SP_CACHE_E4M3) launch<D, SP_CACHE_E4M3>(a, pairs, grid, st);
    else launch<D, SP_CACHE_BF16>(a, pairs, grid, st);
}

bool bad_stride(int64_t stride, int64_t width) { return stride < width || stride % 8 != 0 || stride > (int64_t(1) << 40); }

}  // namespace

extern "C" sp_status sp_cache_append(const sp_cache_desc *desc, const void *k_dev, int64_t k_stride, const void *v_dev,
                                     int64_t v_stride, const void *q_dev, int64_t q_stride, void *q_out_dev,
                                     const int64_t *offsets_host, const int64_t *offsets_dev, int32_t B,
                                     const int32_t *start_dev, const int32_t *positions_dev,
                                     const int32_t *block_table_dev, int64_t table_stride, const float *cos_dev,
                                     const float *sin_dev, int64_t n_pos, int32_t rot_dim, int32_t rot_style,
                                     void *k_pool_dev, void *v_pool_dev, void *k_scale_dev, void *v_scale_dev,
                                     void *hip_stream)
{
    if (sp_status rc = sp::check_cache(desc)) return rc;
    int64_t total, longest;
    if (sp_status rc = sp::check_ragged(offsets_host, B, &total, &longest)) return rc;
    const int64_t kw = (int64_t)desc->n_kv_heads * desc->head_dim, qw = (int64_t)desc->n_q_heads * desc->head_dim;
    if (rot_dim < 0 || rot_dim > desc->head_dim || rot_dim % 16 != 0)
        return sp::fail(SP_ERR_INVALID_ARG, "rot_dim = %d is not a multiple of 16 in 0..head_dim", rot_dim);
    if (rot_style != SP_ROTATE_HALF && rot_style != SP_ROTATE_PAIRS)
        return sp::fail(SP_ERR_INVALID_ARG, "rot_style = %d is neither SP_ROTATE_HALF nor SP_ROTATE_PAIRS", rot_style);
    if (table_stride < 1 || table_stride > (int64_t(1) << 31))
        return sp::fail(SP_ERR_INVALID_ARG, "table_stride = %lld outside 1..2^31", (long long)table_stride);
    if (total == 0) return SP_OK;
    if (!k_dev || !v_dev) return sp::fail(SP_ERR_INVALID_ARG, "k_dev or v_dev is null");
    if (!q_dev != !q_out_dev) return sp::fail(SP_ERR_INVALID_ARG, "q_dev and q_out_dev come together or not at all");
    if (!offsets_dev || !start_dev || !block_table_dev)
        return sp::fail(SP_ERR_INVALID_ARG, "offsets_dev, start_dev or block_table_dev is null");
    if (rot_dim > 0) {
        if (!cos_dev || !sin_dev) return sp::fail(SP_ERR_INVALID_ARG, "cos_dev or sin_dev is null with rot_dim = %d", rot_dim);
        if (n_pos < 1 || n_pos > (int64_t(1) << 40))
            return sp::fail(SP_ERR_INVALID_ARG, "n_pos = %lld outside 1..2^40", (long long)n_pos);
        if ((uintptr_t)cos_dev % 16 != 0 || (uintptr_t)sin_dev % 16 != 0)
            return sp::fail(SP_ERR_INVALID_ARG, "cos_dev and sin_dev must be 16-byte aligned");
    }
    if (bad_stride(k_stride, kw) || bad_stride(v_stride, kw) || (q_dev && bad_stride(q_stride, qw)))
        return sp::fail(SP_ERR_INVALID_ARG, "a token stride is less than its row, above 2^40 or no multiple of 8 elements");
    if ((uintptr_t)k_dev % 16 != 0 || (uintptr_t)v_dev % 16 != 0 || (uintptr_t)q_dev % 16 != 0 || (uintptr_t)q_out_dev % 16 != 0)
        return sp::fail(SP_ERR_INVALID_ARG, "keys, values and queries must be 16-byte aligned");
    if (sp_status rc = sp::check_pools(*desc, k_pool_dev, v_pool_dev, k_scale_dev, v_scale_dev)) return rc;

    const bool single = longest <= 1;
    const int64_t groups = (single ? B : total / kBlock + 2 * (int64_t)B) * desc->n_kv_heads;
    if (groups >= kMaxGroups)
        return sp::fail(SP_ERR_UNSUPPORTED, "%lld new tokens of %d kv heads are more than a launch holds", (long long)total, desc->n_kv_heads);

    AppendArgs a{sp::view_of(*desc, block_table_dev, table_stride),
                 static_cast<const uint16_t *>(k_dev), static_cast<const uint16_t *>(v_dev),
                 static_cast<const uint16_t *>(q_dev), static_cast<uint16_t *>(q_out_dev),
                 k_stride, v_stride, q_stride, offsets_dev, start_dev, positions_dev, cos_dev, sin_dev, n_pos,
                 static_cast<uint8_t *>(k_pool_dev), static_cast<uint8_t *>(v_pool_dev), k_scale_dev, v_scale_dev,
                 B, rot_dim, single};
    const dim3 grid((unsigned)groups);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool pairs = rot_style == SP_ROTATE_PAIRS;
    if (desc->head_dim == 64) launch_kind<64>(a, desc->cache_type, pairs, grid, st);
    else launch_kind<128>(a, desc->cache_type, pairs, grid, st);
    SP_HIP_CHECK(hipGetLastError());
    return SP_OK;
}
