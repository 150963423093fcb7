// What kernels that read a paged cache share: the arguments that describe a call's queries, contexts and keys, addresses along a block table, and
// blocks of 32 tokens as the matrix instructions take them. Used by sp_attend and sp_attend_weights.
#pragma once

#include "sp_cache.hpp"
#include "sp_mx4.hpp"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

constexpr int kBlock = sp::kCacheBlock;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kMostScale = 2.3e38f;      // of a call: times log2(e) it is finite

// A block's key scale goes into its logits' factor, its value scale into the exponent (and out of the sum again): no operation for an element. The
// factor stays above zero, so that masked logits stay minus infinity, and finite, so that a product of zero stays a logit of zero; the value scale
// above 2^-64, so that exponents keep their range.
constexpr float kLeastScale = 5.42101086e-20f, kLeastFactor = 1.17549435e-38f, kMostFactor = 3.40282347e38f;

struct ContextArgs {
    sp::CacheView c;
    const uint16_t *q;
    const int64_t *off;
    const int32_t *lens;
    const uint8_t *k_pool, *v_pool;
    const void *k_scale, *v_scale;      // floats of E4M3 caches, bytes of MX4 ones
    int32_t max_len, window;            // a window is shorter than max_len, or 0
    int32_t B, causal;
    float scale;
    int32_t page_blocks, page_shift;    // blocks of 32 tokens in a page; their logarithm, or -1
};

__device__ __forceinline__ float neg_inf() { return -__builtin_huge_valf(); }
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_(float x) { return __builtin_amdgcn_logf(x); }
// NaN if one of them is. One operation, as are two that are nested; fmaxf would take one more for each operand that may be a signalling NaN: this
// file is compiled with NaNs honoured, since a row that sees one has to become NaN.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float factor_of(float scale, float key_scale)
{
    return __builtin_elementwise_minimum(larger(scale * key_scale, kLeastFactor), kMostFactor);
}
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}

// A value that is the same in all lanes, as a scalar.
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// What a request's rows see: row r (token r / G) keys [first(r), last(r)), all rows together [lo, hi). Key indices fit 32 bits:
// contexts are limited to 2^30 tokens, queries to 2^26.
struct Range {
    int len, n, lo, hi;
};

__device__ __forceinline__ Range range_of(const ContextArgs &a, int b)
{
    Range g;
    g.n = (int)(a.off[b + 1] - a.off[b]);
    g.len = a.lens[b];
    g.len = g.len < 0 ? 0 : (g.len > a.max_len ? a.max_len : g.len);
    g.lo = 0;
    g.hi = g.len;
    if (a.causal && a.window > 0) {
        const int64_t f = (int64_t)g.len - g.n - a.window + 1;
        g.lo = f > 0 ? (int)f : 0;
    }
    return g;
}

__device__ __forceinline__ uint32_t page_of_block(const ContextArgs &a, uint32_t blk)
{
    return a.page_shift >= 0 ? blk >> a.page_shift : blk / (uint32_t)a.page_blocks;
}

// An entry of request b's row of the block table.
__device__ __forceinline__ int page_entry(const ContextArgs &a, int b, uint32_t i)
{
    int page = a.c.table[b * a.c.table_stride + i];
    page = page < 0 ? 0 : page;                                     // never outside the pools
    return page >= (int)a.c.n_pages ? (int)a.c.n_pages - 1 : page;
}

// Two E4M3 codes of a word (the lower or the upper two) as bf16, exactly.
template <bool UPPER>
__device__ __forceinline__ uint32_t widen2(uint32_t w)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.f, UPPER));
}

__device__ __forceinline__ bf16x8 widen8(uint32_t c0, uint32_t c1)
{
    return __builtin_bit_cast(bf16x8, u32x4{widen2<false>(c0), widen2<true>(c0), widen2<false>(c1), widen2<true>(c1)});
}

// Four codes each of two keys: element i's pair of them as bf16.
__device__ __forceinline__ void widen_pairs(uint32_t x, uint32_t y, uint32_t (&pair)[4])
{
    const uint32_t lo = __builtin_amdgcn_perm(y, x, 0x05010400u), hi = __builtin_amdgcn_perm(y, x, 0x07030602u);
    pair[0] = widen2<false>(lo);
    pair[1] = widen2<true>(lo);
    pair[2] = widen2<false>(hi);
    pair[3] = widen2<true>(hi);
}

// A scalar address that moves, and loads at a lane's 32-bit offset from it: a load takes both as they are. What the compiler does not know to stay
// the same in a loop (asm) it does not add up beforehand, which would cost two vector operations for each load.
struct Moving {
    uint64_t p;

    Moving() = default;

    __device__ __forceinline__ explicit Moving(const uint8_t *at) : p(reinterpret_cast<uint64_t>(at)) { asm("" : "+s"(p)); }

    __device__ __forceinline__ void advance(int64_t bytes)
    {
        p += (uint64_t)bytes;
        asm("" : "+s"(p));
    }

    template <class T, bool STREAM = false>
    __device__ __forceinline__ T load(uint32_t lane) const
    {
        typedef const __attribute__((address_space(1))) uint8_t *Bytes;
        const auto *x = reinterpret_cast<const __attribute__((address_space(1))) T *>(reinterpret_cast<Bytes>(p) + lane);
        if constexpr (STREAM) return __builtin_nontemporal_load(x);
        else return *x;
    }
};

__device__ __forceinline__ uint32_t opaque(uint32_t lane)
{
    asm volatile("" : "+v"(lane));
    return lane;
}

// A request's cache of one kv head, and where a block of it lies: bytes from k and v, floats from ks and vs.
struct Line {
    const uint8_t *k, *v;
    const float *ks, *vs;
    const uint8_t *ks4, *vs4;       // of an MX4 cache: the D bytes of a block are at its place among scales times D
    int64_t page_bytes;
    uint32_t row_bytes, page_scales;

    const int32_t *table;

    __device__ __forceinline__ Line(const ContextArgs &a, int b, int kvh, int kind, int d)
    {
        table = a.c.table + b * a.c.table_stride;
        k = a.k_pool + sp::cache_bytes(kind, kvh * a.c.stride_head);
        v = a.v_pool + sp::cache_bytes(kind, kvh * a.c.stride_head);
        ks = static_cast<const float *>(a.k_scale) + (int64_t)kvh * a.page_blocks;
        vs = static_cast<const float *>(a.v_scale) + (int64_t)kvh * a.page_blocks;
        ks4 = static_cast<const uint8_t *>(a.k_scale) + (int64_t)kvh * a.page_blocks * d;
        vs4 = static_cast<const uint8_t *>(a.v_scale) + (int64_t)kvh * a.page_blocks * d;
        page_bytes = sp::cache_bytes(kind, a.c.page_stride);
        row_bytes = (uint32_t)sp::cache_bytes(kind, a.c.stride_token);
        page_scales = (uint32_t)a.c.n_kv_heads * (uint32_t)a.page_blocks;
    }
};

struct Place {
    int64_t off, scale;
};

// Block blk of request b as the block table has it: requested here, looked at in place(), as scalars, so that loads take a scalar base.
struct Entry {
    int page;
    uint32_t in_page;

    __device__ __forceinline__ Entry(const ContextArgs &a, const Line &l, int blk)
    {
        const uint32_t i = page_of_block(a, (uint32_t)blk);
        page = l.table[i];
        in_page = (uint32_t)blk - i * (uint32_t)a.page_blocks;
    }

    __device__ __forceinline__ Place place(const ContextArgs &a, const Line &l) const
    {
        const int p = min(max(__builtin_amdgcn_readfirstlane(page), 0), (int)a.c.n_pages - 1);      // never outside the pools
        return {p * l.page_bytes + (int64_t)((uint64_t)in_page * (kBlock * l.row_bytes)), (int64_t)((uint64_t)(uint32_t)p * l.page_scales) + in_page};
    }
};

// One block of 32 tokens as a wave loads it, straight into the registers that the matrix instructions take it from. Lane l = 16 g + c. Keys: row c
// of 16-key tile t, the contraction's elements in an order that makes a lane's share of a row contiguous (queries are loaded in the same order).
// Values: elements [c D/16, (c+1) D/16) of the eight keys 4g + j and 16 + 4g + j, j < 4: the keys whose logits the lane holds after the first
// product.
// Loads that take whole lines of 128 bytes pass the caches by: values, unless their rows have 64 bytes, and keys whose rows do. 32 requests of
// bf16, head_dim 128, 172 us without and 160 with; 48 of E4M3, head_dim 64, 157 and 143 (200 of up to 4000 tokens 52 and 49, but 56 with values
// too). The latter only for contexts that no cache would hold until the next call: 64 of up to 2000 tokens, called again and again, take 15.7 us
// without and 18.7 with.
template <int D, int KIND, bool STREAM>
struct Block {
    static constexpr bool E4M3 = KIND == SP_CACHE_E4M3;
    // Key i (of eight) of lane group g, as the first product leaves them.
    __device__ __forceinline__ static int key_of(int g, int i) { return 4 * g + (i & 3) + (i >> 2) * 16; }
    static constexpr int kLoads = E4M3 ? D / 64 : D / 32;           // 16-byte loads of a key's row share; dwords of a value's
    u32x4 k[2][kLoads];
    uint32_t v[8][kLoads];
    float ks, vs;

    __device__ __forceinline__ void load_keys(const Line &l, const Place &at, uint32_t lane)
    {
        lane = opaque(lane);
        Moving p(l.k + at.off);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) k[t][i] = p.load<u32x4, STREAM && kLoads == 1>(lane + 64 * i);
            p.advance(16 * (int64_t)l.row_bytes);
        }
        ks = 1.f;
        if (E4M3) ks = l.ks[at.scale];
    }

    __device__ __forceinline__ void load_values(const Line &l, const Place &at, uint32_t lane)
    {
        lane = opaque(lane);
        Moving p(l.v + at.off);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (kLoads == 1) v[j][0] = p.load<uint32_t>(lane);
            else if constexpr (kLoads == 2) {
                const u32x2 w = p.load<u32x2, true>(lane);
                v[j][0] = w[0];
                v[j][1] = w[1];
            } else {
                const u32x4 w = p.load<u32x4, true>(lane);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[j][i] = w[i];
            }
            p.advance((j == 3 ? 13 : 1) * (int64_t)l.row_bytes);
        }
        vs = 1.f;
        if (E4M3) vs = l.vs[at.scale];
    }

    // Elements of step s of tile t's rows.
    __device__ __forceinline__ bf16x8 key(int t, int s) const
    {
        if (E4M3) return widen8(k[t][s / 2][2 * (s % 2)], k[t][s / 2][2 * (s % 2) + 1]);
        return __builtin_bit_cast(bf16x8, k[t][s]);
    }

    // Element c D/16 + i of the lane's eight keys.
    __device__ __forceinline__ void values(bf16x8 (&f)[D / 16]) const
    {
        u32x4 r[D / 16];
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
#pragma unroll
            for (int p = 0; p < 4; ++p) {                           // keys 2p and 2p + 1
                if (E4M3) {
                    uint32_t pair[4];
                    widen_pairs(v[2 * p][i], v[2 * p + 1][i], pair);
#pragma unroll
                    for (int e = 0; e < 4; ++e) r[4 * i + e][p] = pair[e];
                } else {
                    r[2 * i][p] = __builtin_amdgcn_perm(v[2 * p + 1][i], v[2 * p][i], 0x05040100u);
                    r[2 * i + 1][p] = __builtin_amdgcn_perm(v[2 * p + 1][i], v[2 * p][i], 0x07060302u);
                }
            }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) f[i] = __builtin_bit_cast(bf16x8, r[i]);
    }

    // Values of tokens outside [lo, hi) may be NaN: they become zero.
    __device__ __forceinline__ void clear_values(int g, int first, int lo, int hi)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int key = first + key_of(g, j);
            if (key < lo || key >= hi)
#pragma unroll
                for (int i = 0; i < kLoads; ++i) v[j][i] = 0;
        }
    }
};

// A scale byte of a word on its way to a float's exponent, where the conversions take it from: they look at nothing else. `turn` is what
// turn_of() makes of the byte's number.
__device__ __forceinline__ uint32_t turn_of(int byte) { return (8 * byte + 9) & 31; }
__device__ __forceinline__ float exponent_of(uint32_t w, uint32_t turn) { return __uint_as_float(__builtin_amdgcn_alignbit(w, w, turn)); }

// Two 4-bit codes (byte BYTE of w) as bf16, times the scale: exact.
template <int BYTE>
__device__ __forceinline__ uint32_t widen4(uint32_t w, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, BYTE));
}

// The same for an MX4 cache, widened to bf16 with its scales. Row c of tile t is key 2c + t, so that the keys whose logits a lane holds after the
// first product are 8g .. 8g + 7, and the scales of a lane's two keys lie side by side; of a key's row a lane has elements [g D/4, (g + 1) D/4), of
// one group. Values: elements [c D/16, (c+1) D/16) of keys 8g .. 8g + 7, each key's under its scale and then paired by keys. (The scaled matrix
// instruction would take keys as they are with queries as sums of two E4M3 numbers, but it drops products below some 2^-13 of an instruction's
// largest: logits off by 2^-11 of theirs.) 48 contexts of 2048 to 65536 tokens (32 query heads of 64 over 8, 439 MB) take 91 us, 4.8 TB/s (E4M3,
// twice the bytes: 138). Not bound by operations (copies without the conversions, 60 of 137 vector operations fewer, take as long) nor by what is
// under way (keys two blocks ahead 96, both 103 and more): what is left is how memory serves pieces of 1 KB, and 64 bytes of scales. Not kept
// either: all values in one load instead of eight (4 us, without getting them to their lanes), all keys in one load (2 us), five workgroups a unit
// (registers for 96: 108 us), loads past the caches (the same).
template <int D, bool STREAM>
struct Block<D, SP_CACHE_MX4, STREAM> {
    static constexpr int kBytes = D / 32;                           // of a token's scales, and of a lane's part of a token's values
    static constexpr int kWords = kBytes / 2;                       // dwords of two tokens' scales
    uint32_t k[2][2 * kWords];
    uint32_t ks[kWords];
    u32x4 v[2];                     // a word for each key (as vectors: single ones of 16 bits would be cut to them and widened again with every use)
    u32x4 vs[kWords];

    __device__ __forceinline__ static int key_of(int g, int i) { return 8 * g + i; }

    __device__ __forceinline__ void load_keys(const Line &l, const Place &at, uint32_t lane, uint32_t scale_lane)
    {
        lane = opaque(lane);
        Moving p(l.k + at.off);
        const Moving s(l.ks4 + at.scale * D);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if constexpr (D == 64) {
                const u32x2 w = p.load<u32x2>(lane);
                k[t][0] = w[0];
                k[t][1] = w[1];
            } else {
                const u32x4 w = p.load<u32x4>(lane);
#pragma unroll
                for (int i = 0; i < 2 * kWords; ++i) k[t][i] = w[i];
            }
            p.advance(l.row_bytes);
        }
        if constexpr (D == 64) ks[0] = s.load<uint32_t>(opaque(scale_lane));
        else {
            const u32x2 w = s.load<u32x2>(opaque(scale_lane));
#pragma unroll
            for (int i = 0; i < kWords; ++i) ks[i] = w[i];
        }
    }

    __device__ __forceinline__ void load_values(const Line &l, const Place &at, uint32_t lane, uint32_t scale_lane)
    {
        lane = opaque(lane);
        Moving p(l.v + at.off);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (D == 64) v[j / 4][j % 4] = p.load<uint16_t>(lane);
            else v[j / 4][j % 4] = p.load<uint32_t>(lane);
            p.advance(l.row_bytes);
        }
        const Moving s(l.vs4 + at.scale * D);
        scale_lane = opaque(scale_lane);
#pragma unroll
        for (int i = 0; i < kWords; ++i) vs[i] = s.load<u32x4>(scale_lane + 16 * i);
    }

    // Elements of step s of tile t's rows, of lane group g.
    __device__ __forceinline__ bf16x8 key(int t, int s, int g) const
    {
        const float scale = D == 64 ? exponent_of(ks[0], turn_of(2 * t + g / 2)) : exponent_of(ks[t % kWords], turn_of(g));
        const uint32_t w = k[t][s];
        return __builtin_bit_cast(bf16x8, u32x4{widen4<0>(w, scale), widen4<1>(w, scale), widen4<2>(w, scale), widen4<3>(w, scale)});
    }

    __device__ __forceinline__ void values(bf16x8 (&f)[D / 16], int c) const
    {
        u32x4 r[D / 16];
        const int group = c * (D / 16) / sp::kMx4Group;
        const uint32_t turn[2] = {turn_of(group), turn_of(group + 2)};
#pragma unroll
        for (int p = 0; p < 4; ++p) {                               // keys 2p and 2p + 1
            float s[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                s[i] = D == 64 ? exponent_of(vs[0][p], turn[i]) : exponent_of(vs[p / 2 % kWords][2 * (p & 1) + i], turn[0]);
#pragma unroll
            for (int e = 0; e < D / 32; ++e) {                      // a byte: elements 2e and 2e + 1
                const uint32_t a = v[p / 2][2 * p % 4], b = v[p / 2][2 * p % 4 + 1];
                const uint32_t x = e == 0 ? widen4<0>(a, s[0]) : e == 1 ? widen4<1>(a, s[0]) : e == 2 ? widen4<2>(a, s[0]) : widen4<3>(a, s[0]);
                const uint32_t y = e == 0 ? widen4<0>(b, s[1]) : e == 1 ? widen4<1>(b, s[1]) : e == 2 ? widen4<2>(b, s[1]) : widen4<3>(b, s[1]);
                r[2 * e][p] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                r[2 * e + 1][p] = __builtin_amdgcn_perm(y, x, 0x07060302u);
            }
        }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) f[i] = __builtin_bit_cast(bf16x8, r[i]);
    }

    // Scales of tokens outside [lo, hi) may say NaN: they become the smallest.
    __device__ __forceinline__ void clear_values(int g, int first, int lo, int hi)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int key = first + key_of(g, j);
            if (key < lo || key >= hi) {
                if constexpr (D == 64) vs[0][j / 2] &= j & 1 ? 0x0000ffffu : 0xffff0000u;
                else vs[j / 4 % kWords][j & 3] = 0;
            }
        }
    }
};

constexpr int64_t kMaxLen = int64_t(1) << 30, kMaxTokens = int64_t(1) << 26;     // key indices and rows fit 32 bits

// Arguments that sp_attend and sp_attend_weights share, beside the cache's description and the offsets.
inline sp_status check_masks(const sp_cache_desc *desc, int64_t max_len, int64_t table_stride, float scale, int32_t causal, int64_t window)
{
    if (!(scale > 0.f) || scale > kMostScale) return sp::fail(SP_ERR_INVALID_ARG, "scale = %g must be > 0 and at most 2.3e38", (double)scale);
    if (causal != 0 && causal != 1) return sp::fail(SP_ERR_INVALID_ARG, "causal = %d is neither 0 nor 1", causal);
    if (window < 0 || (window > 0 && !causal))
        return sp::fail(SP_ERR_INVALID_ARG, "window = %lld must be 0, or positive with causal = 1", (long long)window);
    if (table_stride < 1 || table_stride > (int64_t(1) << 31))
        return sp::fail(SP_ERR_INVALID_ARG, "table_stride = %lld outside 1..2^31", (long long)table_stride);
    if (max_len > table_stride * desc->page_tokens)
        return sp::fail(SP_ERR_INVALID_ARG, "max_len = %lld exceeds the block table's %lld tokens", (long long)max_len,
                        (long long)(table_stride * desc->page_tokens));
    return SP_OK;
}

inline ContextArgs context_args(const sp_cache_desc &d, const void *q, const int64_t *off, const int32_t *lens, int64_t max_len, const int32_t *table,
                                int64_t table_stride, const void *k_pool, const void *v_pool, const void *k_scale, const void *v_scale,
                                float scale, int32_t causal, int64_t window, int32_t B)
{
    ContextArgs a{sp::view_of(d, table, table_stride), static_cast<const uint16_t *>(q), off, lens, static_cast<const uint8_t *>(k_pool),
                  static_cast<const uint8_t *>(v_pool), k_scale, v_scale, (int32_t)max_len,
                  window < max_len ? (int32_t)window : 0, B, causal, scale, (int32_t)(d.page_tokens / kBlock), -1};   // a longer window takes no key from a row
    for (int s = 0; s < 24; ++s)
        if (a.page_blocks == 1 << s) a.page_shift = s;
    return a;
}

}  // namespace
