// sp_attend: attention of ragged queries over a paged cache (paper: Algorithm 1 ForwardWithAttn, a decoder layer's
// attention over the cache that the importance pass reads afterwards).
//
//   out = sum_j p_j v_j,  p_j = exp(x_j - m) / l,  x_j = scale <q, k_j>,  m = max_j x_j,  l = sum_j exp(x_j - m),
//   lse = m + log l,
// in one pass over the keys: a reference m and a sum l that run along, and the partial output, scaled whenever m moves.
//
// Query rows of one request that share a kv head (n_b tokens of G heads) are taken together, so that a key is read once for
// all of them. Requests of up to kFewRows rows go to sp_attend_few_kernel, which is bound by the cache's bytes and splits
// a context among workgroups; others to sp_attend_many_kernel, tiles of 256 rows, which is bound by its operations and splits contexts only
// where there are too few tiles. The join kernels put splits together.
#include "sp_cache.hpp"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kFewRows = 64;        // query rows of a kv head that sp_attend_few_kernel takes at most
constexpr int kManyList = 64;
constexpr int kBlock = sp::kCacheBlock;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct AttendArgs {
    sp::CacheView c;
    const uint16_t *q;
    const int64_t *off;
    const int32_t *lens;
    const uint8_t *k_pool, *v_pool;
    const float *k_scale, *v_scale;
    uint16_t *out;
    float *lse;
    int64_t max_len, window;
    int32_t B, causal;
    float scale;
    int32_t page_blocks, page_shift;    // blocks of 32 tokens in a page; their logarithm, or -1
    // splits of sp_attend_few_kernel: `splits` of `split_blocks` blocks; `few_rows` rows a request and kv head in the workspace
    int32_t splits, split_blocks, few_rows;
    f32x2 *part_ml;                     // [split][request][kv head][few_rows]: reference (in units of log 2), sum
    float *part_o;                      // [...][head_dim]
    // tiles of sp_attend_many_kernel, and its splits of `many_keys` keys
    int32_t tiles, many_splits;
    int64_t many_keys;
    f32x2 *many_ml;                     // [split][tile][kv head][kManyRows]
    float *many_o;
    // the requests with many rows and their first tiles, if there are at most kManyList of them (else many_count is 0)
    int32_t many_count, many_b[kManyList], many_tile[kManyList];
};

__device__ __forceinline__ float neg_inf() { return -__builtin_huge_valf(); }
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_(float x) { return __builtin_amdgcn_logf(x); }
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}

// ---- a few rows: single tokens, lookahead rows -----------------------------------------------------------------------

// What a request's rows see: row r (token r / G) keys [first(r), last(r)), all rows together [lo, hi).
struct Range {
    int64_t len, n;
    int64_t lo, hi;
};

__device__ __forceinline__ Range range_of(const AttendArgs &a, int b)
{
    Range g;
    g.n = a.off[b + 1] - a.off[b];
    g.len = a.lens[b];
    g.len = g.len < 0 ? 0 : (g.len > a.max_len ? a.max_len : g.len);
    g.lo = 0;
    g.hi = g.len;
    if (a.causal && a.window > 0) {
        const int64_t f = g.len - g.n - a.window + 1;
        g.lo = f > 0 ? f : 0;
    }
    return g;
}

__device__ __forceinline__ uint32_t page_of_block(const AttendArgs &a, uint32_t blk)
{
    return a.page_shift >= 0 ? blk >> a.page_shift : blk / (uint32_t)a.page_blocks;
}

__device__ __forceinline__ int page_at(const AttendArgs &a, int b, uint32_t blk)
{
    int page = a.c.table[b * a.c.table_stride + page_of_block(a, blk)];
    page = page < 0 ? 0 : page;                                     // never outside the pools
    return page >= (int)a.c.n_pages ? (int)a.c.n_pages - 1 : page;
}

// Eight E4M3 codes as eight bf16, exactly: the upper halves of their float images.
__device__ __forceinline__ bf16x8 widen8(uint32_t c0, uint32_t c1)
{
    u32x4 r;
    const uint32_t w[2] = {c0, c1};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
        r[2 * i] = __builtin_amdgcn_perm(__float_as_uint(lo.y), __float_as_uint(lo.x), 0x07060302u);
        r[2 * i + 1] = __builtin_amdgcn_perm(__float_as_uint(hi.y), __float_as_uint(hi.x), 0x07060302u);
    }
    return __builtin_bit_cast(bf16x8, r);
}

// One block of 32 tokens as a wave loads it, straight into the registers that the matrix instructions take it from.
// Lane l = 16 g + c. Keys: row c of 16-key tile t, the contraction's elements in an order that makes a lane's share of a row contiguous
// (queries are loaded in the same order). Values: elements [c D/16, (c+1) D/16) of the eight keys 4g + j and 16 + 4g + j, j < 4: the
// keys whose logits the lane holds after the first product.
template <int D, bool E4M3>
struct Block {
    static constexpr int kLoads = E4M3 ? D / 64 : D / 32;           // 16-byte loads of a key's row share; dwords of a value's
    u32x4 k[2][kLoads];
    uint32_t v[8][kLoads];
    float ks, vs;

    __device__ __forceinline__ void load(const AttendArgs &a, int kvh, int page, uint32_t blk, uint32_t k_lane, uint32_t v_lane)
    {
        constexpr int ES = E4M3 ? 1 : 2;
        const uint32_t in_page = blk - page_of_block(a, blk) * (uint32_t)a.page_blocks;
        const int64_t base = (page * a.c.page_stride + kvh * a.c.stride_head + (int64_t)(in_page * kBlock) * a.c.stride_token) * ES;
        const int64_t row = a.c.stride_token * ES;
        const uint8_t *kp = a.k_pool + base, *vp = a.v_pool + base;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                k[t][i] = *reinterpret_cast<const u32x4 *>(kp + t * 16 * row + i * 64 + k_lane);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint8_t *p = vp + ((j & 3) + (j >> 2) * 16) * row + v_lane;
            if constexpr (kLoads == 1) v[j][0] = *reinterpret_cast<const uint32_t *>(p);
            else if constexpr (kLoads == 2) {
                const u32x2 w = *reinterpret_cast<const u32x2 *>(p);
                v[j][0] = w[0];
                v[j][1] = w[1];
            } else {
                const u32x4 w = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[j][i] = w[i];
            }
        }
        ks = vs = 1.f;
        if (E4M3) {
            const int64_t at = ((int64_t)page * a.c.n_kv_heads + kvh) * a.page_blocks + in_page;
            ks = a.k_scale[at];
            vs = a.v_scale[at];
        }
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
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const f32x2 x = h ? __builtin_amdgcn_cvt_pk_f32_fp8((int)v[2 * p][i], true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)v[2 * p][i], false);
                        const f32x2 y = h ? __builtin_amdgcn_cvt_pk_f32_fp8((int)v[2 * p + 1][i], true)
                                          : __builtin_amdgcn_cvt_pk_f32_fp8((int)v[2 * p + 1][i], false);
                        r[4 * i + 2 * h][p] = __builtin_amdgcn_perm(__float_as_uint(y.x), __float_as_uint(x.x), 0x07060302u);
                        r[4 * i + 2 * h + 1][p] = __builtin_amdgcn_perm(__float_as_uint(y.y), __float_as_uint(x.y), 0x07060302u);
                    }
                } else {
                    r[2 * i][p] = __builtin_amdgcn_perm(v[2 * p + 1][i], v[2 * p][i], 0x05040100u);
                    r[2 * i + 1][p] = __builtin_amdgcn_perm(v[2 * p + 1][i], v[2 * p][i], 0x07060302u);
                }
            }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) f[i] = __builtin_bit_cast(bf16x8, r[i]);
    }

    // Values of tokens outside [lo, hi) may be NaN: they become zero.
    __device__ __forceinline__ void clear_values(int g, int64_t first, int64_t lo, int64_t hi)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t key = first + 4 * g + (j & 3) + (j >> 2) * 16;
            if (key < lo || key >= hi)
#pragma unroll
                for (int i = 0; i < kLoads; ++i) v[j][i] = 0;
        }
    }
};

// Maximum over the four lanes that hold a query row's logits.
__device__ __forceinline__ float row_max(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}

__device__ __forceinline__ float row_sum(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// Running softmax of MT tiles of 16 query rows. The transposed logits put a row into a lane column (c = l % 16), so the
// probabilities are the second product's operand without crossing lanes. The reference m is moved only when a
// logit passes it by kSlack (the sums have room for 2^kSlack), which spares most blocks the exchange between lanes.
template <int D, int MT>
struct Rows {
    static constexpr float kSlack = 8.f;
    float m[MT], l[MT];             // l: this lane's keys only
    f32x4 o[MT][D / 16];            // row c, elements (4g + j) D/16 + i of tile i

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            m[t] = neg_inf();
            l[t] = 0.f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }

    // x: logits of this lane's eight keys in units of log 2. Returns their probabilities' bits times vs.
    __device__ __forceinline__ bf16x8 weigh(int t, const float (&x)[8], float vs)
    {
        float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        if (__any(top > m[t] + kSlack)) {
            const float mx = fmaxf(m[t], row_max(top));
            const float f = m[t] == neg_inf() ? 0.f : exp2_(m[t] - mx);
            l[t] *= f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[t][i] *= f;
            m[t] = mx;
        }
        const float ref = m[t] == neg_inf() ? 0.f : m[t];
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = exp2_(x[i] - ref);
        l[t] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = pack2(p[2 * i] * vs, p[2 * i + 1] * vs);
        return __builtin_bit_cast(bf16x8, r);
    }
};

// Bound by the bytes of the cache. Four waves take every fourth block of 32 tokens of the workgroup's split; a wave holds its rows'
// statistics and output by itself and loads a block ahead, the four meet in LDS at the end.
template <int D, bool E4M3, int MT>
__global__ __launch_bounds__(kThreads) void sp_attend_few_kernel(AttendArgs a)
{
    constexpr int kSteps = D / 32, kTiles = D / 16;
    __shared__ float merge_o[2][16 * MT][D];
    __shared__ f32x2 merge_ml[2][16 * MT];
    const int b = blockIdx.z, kvh = blockIdx.y, split = blockIdx.x, G = a.c.group;
    const Range rg = range_of(a, b);
    if (rg.n == 0 || rg.n * G > kFewRows) return;
    const int rows = (int)rg.n * G;
    const int64_t blk_lo = rg.lo / kBlock, blk_hi = (rg.hi + kBlock - 1) / kBlock;
    const int64_t from = blk_lo + (int64_t)split * a.split_blocks;
    const int64_t to = from + a.split_blocks < blk_hi ? from + a.split_blocks : blk_hi;
    if (from >= to && split > 0) return;

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
    const float scale2 = a.scale * kLog2e;
    bf16x8 q[MT][kSteps];
    int64_t first[MT], last[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int r = 16 * t + c, token = r / G, head = kvh * G + r % G;
        first[t] = rg.lo;
        last[t] = rg.hi;
        if (a.causal) {
            const int64_t p = rg.len - rg.n + token;
            last[t] = p + 1;
            first[t] = a.window > 0 && p - a.window + 1 > 0 ? p - a.window + 1 : 0;
        }
        const uint16_t *src = a.q + ((a.off[b] + token) * a.c.n_q_heads + head) * D;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int e = E4M3 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
            u32x4 w = {0, 0, 0, 0};
            if (r < rows) w = *reinterpret_cast<const u32x4 *>(src + e);
            q[t][s] = __builtin_bit_cast(bf16x8, w);
        }
    }
    // every row sees the keys of [all_lo, all_hi)
    const int64_t all_lo = a.causal && a.window > 0 && rg.len - a.window > 0 ? rg.len - a.window : 0;
    const int64_t all_hi = a.causal ? rg.len - rg.n + 1 : rg.hi;

    Rows<D, MT> acc;
    acc.clear();
    const uint32_t row_bytes = (uint32_t)a.c.stride_token * (E4M3 ? 1 : 2);
    const uint32_t k_lane = c * row_bytes + 16 * g, v_lane = 4 * g * row_bytes + c * (D / 16) * (E4M3 ? 1 : 2);
    Block<D, E4M3> cur, nxt;
    int64_t blk = from + wave;
    if (blk < to) {
        cur.load(a, kvh, page_at(a, b, (uint32_t)blk), (uint32_t)blk, k_lane, v_lane);
        int page = page_at(a, b, (uint32_t)(blk + kWaves < to ? blk + kWaves : blk));
        for (; blk < to; blk += kWaves) {
            const int64_t ahead = blk + kWaves < to ? blk + kWaves : blk, later = ahead + kWaves < to ? ahead + kWaves : ahead;
            nxt.load(a, kvh, page, (uint32_t)ahead, k_lane, v_lane);
            page = page_at(a, b, (uint32_t)later);

            bf16x8 kf[2][kSteps], vf[kTiles];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int s = 0; s < kSteps; ++s) kf[t][s] = cur.key(t, s);
            const int64_t key0 = blk * kBlock;
            const bool whole = key0 >= all_lo && key0 + kBlock <= all_hi;
            if (!whole) cur.clear_values(g, key0, rg.lo, rg.hi);
            cur.values(vf);
            const float sc = scale2 * cur.ks;
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[0][s], q[t][s], s0, 0, 0, 0);
                    s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[1][s], q[t][s], s1, 0, 0, 0);
                }
                float x[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[j] = s0[j] * sc;
                    x[4 + j] = s1[j] * sc;
                }
                if (!whole)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int64_t key = key0 + 4 * g + (j & 3) + (j >> 2) * 16;
                        if (key < first[t] || key >= last[t]) x[j] = neg_inf();
                    }
                const bf16x8 p = acc.weigh(t, x, cur.vs);
#pragma unroll
                for (int i = 0; i < kTiles; ++i) acc.o[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i], p, acc.o[t][i], 0, 0, 0);
            }
            cur = nxt;
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) acc.l[t] = row_sum(acc.l[t]);

    // waves 2 and 3 hand theirs to 0 and 1, then 1 to 0
#pragma unroll
    for (int half = 2; half >= 1; half >>= 1) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                if (g == 0) merge_ml[wave - half][16 * t + c] = f32x2{acc.m[t], acc.l[t]};
#pragma unroll
                for (int i = 0; i < kTiles; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) merge_o[wave - half][16 * t + c][(4 * g + j) * kTiles + i] = acc.o[t][i][j];
            }
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const f32x2 o = merge_ml[wave][16 * t + c];
                const float mx = fmaxf(acc.m[t], o[0]);
                const float f = acc.m[t] == neg_inf() ? 0.f : exp2_(acc.m[t] - mx), f2 = o[0] == neg_inf() ? 0.f : exp2_(o[0] - mx);
                acc.m[t] = mx;
                acc.l[t] = acc.l[t] * f + o[1] * f2;
#pragma unroll
                for (int i = 0; i < kTiles; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc.o[t][i][j] = acc.o[t][i][j] * f + merge_o[wave][16 * t + c][(4 * g + j) * kTiles + i] * f2;
            }
        __syncthreads();
    }
    if (wave != 0) return;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int r = 16 * t + c;
        if (r >= rows) continue;
        if (a.splits > 1) {
            const int64_t at = (((int64_t)split * a.B + b) * a.c.n_kv_heads + kvh) * a.few_rows + r;
            if (g == 0) a.part_ml[at] = f32x2{acc.m[t], acc.l[t]};
            float *dst = a.part_o + at * D + 4 * g * kTiles;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < kTiles; i += 4)
                    *reinterpret_cast<f32x4 *>(dst + j * kTiles + i) = f32x4{acc.o[t][i][j], acc.o[t][i + 1][j], acc.o[t][i + 2][j], acc.o[t][i + 3][j]};
        } else {
            const float inv = acc.l[t] > 0.f ? 1.f / acc.l[t] : 0.f;
            const int64_t row = (a.off[b] + r / G) * a.c.n_q_heads + kvh * G + r % G;
            uint32_t *dst = reinterpret_cast<uint32_t *>(a.out + row * D + 4 * g * kTiles);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < kTiles; i += 2) dst[(j * kTiles + i) / 2] = pack2(acc.o[t][i][j] * inv, acc.o[t][i + 1][j] * inv);
            if (a.lse && g == 0) a.lse[row] = acc.l[t] > 0.f ? (acc.m[t] + log2_(acc.l[t])) * kLn2 : neg_inf();
        }
    }
}

// Joins `count` splits of one row, the first at index `at` of the workspace's rows and `step` rows apart: their weights exp2(m_s - m)
// first, then the weighted sum, the splits shared out among the waves.
template <int D>
__device__ __forceinline__ void join_row(const AttendArgs &a, const f32x2 *ml, const float *po, int64_t at, int64_t step, int count, int64_t row)
{
    __shared__ float part[kWaves][D];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    float m = neg_inf();
    for (int s = lane; s < count; s += 64) m = fmaxf(m, ml[at + s * step][0]);
#pragma unroll
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    float l = 0.f;
    for (int s = lane; s < count; s += 64) {
        const f32x2 x = ml[at + s * step];
        if (x[0] != neg_inf()) l += x[1] * exp2_(x[0] - m);
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) l += __shfl_xor(l, o);
    float acc[D / 64] = {};
    for (int s = wave; s < count; s += kWaves) {
        const float ms = ml[at + s * step][0], f = ms == neg_inf() ? 0.f : exp2_(ms - m);
#pragma unroll
        for (int i = 0; i < D / 64; ++i) acc[i] += po[(at + s * step) * D + lane + 64 * i] * f;
    }
#pragma unroll
    for (int i = 0; i < D / 64; ++i) part[wave][lane + 64 * i] = acc[i];
    __syncthreads();
    if (tid < D) {
        const float o = ((part[0][tid] + part[1][tid]) + (part[2][tid] + part[3][tid])) * (l > 0.f ? 1.f / l : 0.f);
        a.out[row * D + tid] = __builtin_bit_cast(uint16_t, (__bf16)o);
    }
    if (a.lse && tid == 0) a.lse[row] = l > 0.f ? (m + log2_(l)) * kLn2 : neg_inf();
}

template <int D>
__global__ __launch_bounds__(kThreads) void sp_attend_join_kernel(AttendArgs a)
{
    const int b = blockIdx.z, kvh = blockIdx.y, r = blockIdx.x, G = a.c.group;
    const Range rg = range_of(a, b);
    if (rg.n * G > kFewRows || r >= rg.n * G) return;
    const int64_t blocks = (rg.hi + kBlock - 1) / kBlock - rg.lo / kBlock;
    int count = (int)((blocks + a.split_blocks - 1) / a.split_blocks);
    count = count < 1 ? 1 : (count > a.splits ? a.splits : count);          // split 0 always writes
    const int64_t at = ((int64_t)b * a.c.n_kv_heads + kvh) * a.few_rows + r, step = (int64_t)a.B * a.c.n_kv_heads * a.few_rows;
    join_row<D>(a, a.part_ml, a.part_o, at, step, count, (a.off[b] + r / G) * a.c.n_q_heads + kvh * G + r % G);
}

// ---- many rows: prompt chunks -----------------------------------------------------------------------------------------

constexpr int kManyThreads = 512;
constexpr int kManyRows = 256;      // query rows of a workgroup, 32 for each of its waves

typedef __attribute__((ext_vector_type(16))) float f32x16;

// Tile x of 256 rows: its request, first row, and the keys that its rows see together. Without a list, request b's tiles begin at
// off[b] G / 256 + b: enough, since n rows need at most n / 256 + 1 tiles (rounded down).
struct Tile {
    Range rg;
    int b, row0, rows;              // rows of this tile
    int64_t lo, hi;
};

__device__ __forceinline__ bool tile_of(const AttendArgs &a, int x, Tile *t)
{
    const int G = a.c.group;
    int lo = 0, hi = a.many_count ? a.many_count : a.B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        const int64_t begin = a.many_count ? a.many_tile[mid] : a.off[mid] * G / kManyRows + mid;
        if (begin <= x) lo = mid; else hi = mid;
    }
    t->b = a.many_count ? a.many_b[lo] : lo;
    t->rg = range_of(a, t->b);
    const int64_t row0 = (x - (a.many_count ? a.many_tile[lo] : a.off[lo] * G / kManyRows + lo)) * kManyRows, rows = t->rg.n * G - row0;
    if (t->rg.n * G <= kFewRows || rows <= 0) return false;
    t->row0 = (int)row0;
    t->rows = (int)(rows < kManyRows ? rows : kManyRows);
    t->lo = 0;
    t->hi = t->rg.len;
    if (a.causal) {
        const int64_t p0 = t->rg.len - t->rg.n + t->row0 / G, p1 = t->rg.len - t->rg.n + (t->row0 + t->rows - 1) / G;
        t->hi = p1 + 1 > 0 ? p1 + 1 : 0;
        if (a.window > 0 && p0 - a.window + 1 > 0) t->lo = p0 - a.window + 1;
    }
    return true;
}

// Bound by the matrix units at head_dim 128 and by the exponentials and their surroundings at 64. Eight waves of 32 rows share tiles
// of kKeys keys, which they bring to LDS as bf16: keys as they are, values transposed, so that both products take 16-byte operands from
// LDS. The transposed logits put a row into a lane column; the order of keys in a row of transposed values is the one in which a
// lane holds its probabilities, so these are the second product's operand as they are. Tiles are double-buffered, one barrier a
// tile; the next tile's loads are under way during the products.
// A block's key scale goes into its logits' factor, its value scale into the exponent (and out of the sum again): no operation for an element.
template <int D, bool E4M3>
struct Stage {
    static constexpr int kKeys = 8192 / D, kBlocks = kKeys / kBlock;
    static constexpr int ES = E4M3 ? 1 : 2;
    static constexpr int kKeyLoads = E4M3 ? 1 : 2;              // 16-byte loads of a thread
    static constexpr int kKeyLanes = D * ES / 16;               // threads of a key's row
    static constexpr int kValueLanes = D / 4;                   // threads of four keys' values, four elements each
    u32x4 k[kKeyLoads];
    uint32_t v[4][ES];
    float scale;                                                // thread i < 2 kBlocks: key or value scale of a block
    int key_row, key_col, value_key, value_octet, value_half, value_col;

    __device__ __forceinline__ Stage()
    {
        const int tid = threadIdx.x, part = tid / kValueLanes;
        key_row = tid / kKeyLanes;
        key_col = tid % kKeyLanes;
        value_col = tid % kValueLanes;
        value_octet = part >> 1;
        value_half = part & 1;
        // an octet holds keys 4h + j and 8 + 4h + j (j < 4) of 16: what lanes of half h of a wave hold after the first product
        value_key = 32 * (value_octet >> 2) + 16 * ((value_octet >> 1) & 1) + 4 * (value_octet & 1) + 8 * value_half;
    }

    // Pages of the blocks that this wave loads from, for the tile that begins at block blk.
    struct Pages {
        int key[kKeyLoads], value, scale;
    };

    __device__ __forceinline__ int block_of_keys(int i) const
    {
        return __builtin_amdgcn_readfirstlane((key_row + i * (kManyThreads / kKeyLanes)) / kBlock);
    }

    __device__ __forceinline__ Pages pages(const AttendArgs &a, int b, uint32_t blk, uint32_t last) const
    {
        Pages p;
#pragma unroll
        for (int i = 0; i < kKeyLoads; ++i) p.key[i] = page_at(a, b, min(blk + block_of_keys(i), last));
        p.value = page_at(a, b, min(blk + __builtin_amdgcn_readfirstlane(value_octet >> 2), last));
        p.scale = 0;
        if (E4M3 && threadIdx.x < 2 * kBlocks) p.scale = page_at(a, b, min(blk + threadIdx.x % kBlocks, last));
        return p;
    }

    // Blocks behind the last one are read as the last one: they are masked.
    __device__ __forceinline__ void load(const AttendArgs &a, int kvh, const Pages &p, uint32_t blk, uint32_t last)
    {
        const int64_t row = a.c.stride_token * ES;
#pragma unroll
        for (int i = 0; i < kKeyLoads; ++i) {
            const uint32_t at = min(blk + block_of_keys(i), last), in_page = at - page_of_block(a, at) * (uint32_t)a.page_blocks;
            const uint8_t *base = a.k_pool + (p.key[i] * a.c.page_stride + kvh * a.c.stride_head + (int64_t)(in_page * kBlock) * a.c.stride_token) * ES;
            const uint32_t r = (key_row + i * (kManyThreads / kKeyLanes)) % kBlock;
            k[i] = *reinterpret_cast<const u32x4 *>(base + r * (uint32_t)row + key_col * 16);
        }
        const uint32_t at = min(blk + __builtin_amdgcn_readfirstlane(value_octet >> 2), last), in_page = at - page_of_block(a, at) * (uint32_t)a.page_blocks;
        const uint8_t *base = a.v_pool + (p.value * a.c.page_stride + kvh * a.c.stride_head + (int64_t)(in_page * kBlock) * a.c.stride_token) * ES;
        const uint32_t lane = (value_key % kBlock) * (uint32_t)row + value_col * 4 * ES;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (E4M3) v[j][0] = *reinterpret_cast<const uint32_t *>(base + j * row + lane);
            else {
                const u32x2 w = *reinterpret_cast<const u32x2 *>(base + j * row + lane);
                v[j][0] = w[0];
                v[j][1] = w[1];
            }
        }
        if (E4M3 && threadIdx.x < 2 * kBlocks) {
            const uint32_t sb = min(blk + threadIdx.x % kBlocks, last), in = sb - page_of_block(a, sb) * (uint32_t)a.page_blocks;
            scale = (threadIdx.x < kBlocks ? a.k_scale : a.v_scale)[((int64_t)p.scale * a.c.n_kv_heads + kvh) * a.page_blocks + in];
        }
    }

    // 16-byte pieces: piece c of key row r, and octet o of element d's values, where their readers find them without bank conflicts.
    static __device__ __forceinline__ int key_slot(int r, int c) { return r * (D / 8) + (c ^ (D == 128 ? r & 15 : r & 7)); }
    static __device__ __forceinline__ int value_slot(int d, int o) { return d * (kKeys / 8) + (o ^ ((d ^ (d >> 2)) & 7)); }

    // Values of keys outside [lo, hi) become zero; `first` is the tile's first key.
    __device__ __forceinline__ void store(u32x4 *keys, u32x4 *values, float *scales, int64_t first, int64_t lo, int64_t hi)
    {
#pragma unroll
        for (int i = 0; i < kKeyLoads; ++i) {
            const int r = key_row + i * (kManyThreads / kKeyLanes);
            if constexpr (E4M3) {
                keys[key_slot(r, 2 * key_col)] = __builtin_bit_cast(u32x4, widen8(k[i][0], k[i][1]));
                keys[key_slot(r, 2 * key_col + 1)] = __builtin_bit_cast(u32x4, widen8(k[i][2], k[i][3]));
            } else
                keys[key_slot(r, key_col)] = k[i];
        }
        if (first < lo || first + kKeys > hi)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t key = first + value_key + j;
                if (key < lo || key >= hi)
#pragma unroll
                    for (int i = 0; i < ES; ++i) v[j][i] = 0;
            }
        u32x2 r[4];                                             // element 4 value_col + i of four keys
#pragma unroll
        for (int p = 0; p < 2; ++p)
            if constexpr (E4M3) {
                const f32x2 x0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[2 * p][0], false), x1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[2 * p][0], true);
                const f32x2 y0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[2 * p + 1][0], false), y1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[2 * p + 1][0], true);
                r[0][p] = __builtin_amdgcn_perm(__float_as_uint(y0.x), __float_as_uint(x0.x), 0x07060302u);
                r[1][p] = __builtin_amdgcn_perm(__float_as_uint(y0.y), __float_as_uint(x0.y), 0x07060302u);
                r[2][p] = __builtin_amdgcn_perm(__float_as_uint(y1.x), __float_as_uint(x1.x), 0x07060302u);
                r[3][p] = __builtin_amdgcn_perm(__float_as_uint(y1.y), __float_as_uint(x1.y), 0x07060302u);
            } else
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    r[2 * i][p] = __builtin_amdgcn_perm(v[2 * p + 1][i], v[2 * p][i], 0x05040100u);
                    r[2 * i + 1][p] = __builtin_amdgcn_perm(v[2 * p + 1][i], v[2 * p][i], 0x07060302u);
                }
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<u32x2 *>(values)[2 * value_slot(4 * value_col + i, value_octet) + value_half] = r[i];
        if (E4M3 && threadIdx.x < 2 * kBlocks) scales[threadIdx.x] = scale;
    }
};

template <int D, bool E4M3>
__global__ __launch_bounds__(kManyThreads) void sp_attend_many_kernel(AttendArgs a)
{
    using S = Stage<D, E4M3>;
    constexpr int kKeys = S::kKeys, kBlocks = S::kBlocks, kSteps = D / 16, kOut = D / 32;
    constexpr float kSlack = 8.f;
    __shared__ u32x4 keys[2][1024], values[2][1024];            // 16 KB each
    __shared__ float scales[2][2 * kBlocks];
    // neighbouring workgroups take different kv heads: with eight of them, each die's L2 holds one head's cache
    const int kvh = blockIdx.x % a.c.n_kv_heads, rest = blockIdx.x / a.c.n_kv_heads;
    const int x = a.tiles - 1 - rest % a.tiles, split = rest / a.tiles;     // later tiles of a prompt see more: they go first
    Tile t;
    if (!tile_of(a, x, &t)) return;
    const int64_t tile0 = t.lo / kKeys * kKeys;                 // first key of the first tile of keys
    const int64_t from = tile0 + (int64_t)split * a.many_keys;
    const int64_t to = from + a.many_keys < t.hi ? from + a.many_keys : t.hi;
    if (from >= to && split > 0) return;

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, h = lane >> 5, c = lane & 31;
    const int G = a.c.group, r = 32 * wave + c;                 // this lane's row of the tile
    const int token = (t.row0 + r) / G, head = kvh * G + (t.row0 + r) % G;
    const int64_t row = (a.off[t.b] + token) * a.c.n_q_heads + head;
    int64_t first = 0, last = t.rg.len;
    // keys that every row of this wave sees: [all_lo, all_hi); that some row sees: up to any_hi
    int64_t all_lo = 0, all_hi = t.rg.len, any_hi = t.rg.len, any_lo = 0;
    if (a.causal) {
        const int64_t p = t.rg.len - t.rg.n;
        last = p + token + 1;
        first = a.window > 0 && last - a.window > 0 ? last - a.window : 0;
        const int64_t low = p + (t.row0 + 32 * wave) / G + 1, high = p + (t.row0 + 32 * wave + 31) / G + 1;
        all_hi = low;
        any_hi = high;
        if (a.window > 0) {
            all_lo = high - a.window;
            any_lo = low - a.window;
        }
    }
    const bool busy = 32 * wave < t.rows;

    bf16x8 q[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        u32x4 w = {0, 0, 0, 0};
        if (r < t.rows) w = *reinterpret_cast<const u32x4 *>(a.q + row * D + 16 * s + 8 * h);
        q[s] = __builtin_bit_cast(bf16x8, w);
    }
    float m = neg_inf(), l = 0.f;
    f32x16 o[kOut];
#pragma unroll
    for (int i = 0; i < kOut; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    const float scale2 = a.scale * kLog2e;

    if (from < to) {
        S st;
        const uint32_t last_blk = (uint32_t)((t.hi - 1) / kBlock);
        uint32_t blk = (uint32_t)(from / kBlock);
        typename S::Pages pg = st.pages(a, t.b, blk, last_blk);
        st.load(a, kvh, pg, blk, last_blk);
        pg = st.pages(a, t.b, blk + kBlocks, last_blk);
        st.store(keys[0], values[0], scales[0], from, t.lo, t.hi);
        __syncthreads();
        int buf = 0;
        for (int64_t key0 = from; key0 < to; key0 += kKeys, buf ^= 1, blk += kBlocks) {
            const bool more = key0 + kKeys < to;
            if (more) {
                st.load(a, kvh, pg, blk + kBlocks, last_blk);
                pg = st.pages(a, t.b, blk + 2 * kBlocks, last_blk);
            }
            if (busy && key0 < any_hi && key0 + kKeys > any_lo) {
                const bool whole = key0 >= all_lo && key0 + kKeys <= all_hi;
#pragma unroll
                for (int u = 0; u < kBlocks; ++u) {
                    // blocks that no row of the tile sees: their scales may be anything
                    if (!whole && (key0 + 32 * u >= t.hi || key0 + 32 * u + 32 <= t.lo)) continue;
                    f32x16 x;
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
                    for (int s = 0; s < kSteps; ++s)
                        x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, keys[buf][S::key_slot(32 * u + c, 2 * s + h)]), q[s], x, 0, 0, 0);
                    if (!whole)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int64_t key = key0 + 32 * u + 8 * (e >> 2) + 4 * h + (e & 3);
                            if (key < first || key >= last) x[e] = neg_inf();
                        }
                    float sc = scale2, vexp = 0.f, vinv = 1.f;
                    if (E4M3) {
                        const float vs = scales[buf][kBlocks + u];
                        sc *= scales[buf][u];
                        vexp = log2_(vs);
                        vinv = 1.f / vs;
                    }
                    float top = x[0];
#pragma unroll
                    for (int e = 1; e < 16; ++e) top = fmaxf(top, x[e]);
                    top *= sc;
                    if (__any(top > m + kSlack)) {
                        const float mx = fmaxf(m, fmaxf(top, __shfl_xor(top, 32)));
                        const float f = m == neg_inf() ? 0.f : exp2_(m - mx);
                        l *= f;
#pragma unroll
                        for (int i = 0; i < kOut; ++i) o[i] *= f;
                        m = mx;
                    }
                    const float ref = (m == neg_inf() ? 0.f : m) - vexp;
                    float sum = 0.f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        x[e] = exp2_(x[e] * sc - ref);
                        sum += x[e];
                    }
                    l += sum * vinv;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const u32x4 w = {pack2(x[8 * k], x[8 * k + 1]), pack2(x[8 * k + 2], x[8 * k + 3]), pack2(x[8 * k + 4], x[8 * k + 5]),
                                         pack2(x[8 * k + 6], x[8 * k + 7])};
                        const bf16x8 p = __builtin_bit_cast(bf16x8, w);
#pragma unroll
                        for (int i = 0; i < kOut; ++i)
                            o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, values[buf][S::value_slot(32 * i + c, 4 * u + 2 * k + h)]),
                                                                          p, o[i], 0, 0, 0);
                    }
                }
            }
            if (more) st.store(keys[buf ^ 1], values[buf ^ 1], scales[buf ^ 1], key0 + kKeys, t.lo, t.hi);
            __syncthreads();
        }
    }
    l += __shfl_xor(l, 32);
    if (r >= t.rows) return;
    if (a.many_splits > 1) {
        const int64_t at = (((int64_t)split * a.tiles + x) * a.c.n_kv_heads + kvh) * kManyRows + r;
        if (h == 0) a.many_ml[at] = f32x2{m, l};
#pragma unroll
        for (int i = 0; i < kOut; ++i)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<f32x4 *>(a.many_o + at * D + 32 * i + 2 * e + 4 * h) = f32x4{o[i][e], o[i][e + 1], o[i][e + 2], o[i][e + 3]};
        return;
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int i = 0; i < kOut; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<u32x2 *>(a.out + row * D + 32 * i + 2 * e + 4 * h) =
                u32x2{pack2(o[i][e] * inv, o[i][e + 1] * inv), pack2(o[i][e + 2] * inv, o[i][e + 3] * inv)};
    if (a.lse && h == 0) a.lse[row] = l > 0.f ? (m + log2_(l)) * kLn2 : neg_inf();
}

template <int D, bool E4M3>
__global__ __launch_bounds__(kThreads) void sp_attend_many_join_kernel(AttendArgs a)
{
    constexpr int kKeys = Stage<D, E4M3>::kKeys;
    const int x = blockIdx.x / kManyRows, r = blockIdx.x % kManyRows, kvh = blockIdx.y, G = a.c.group;
    Tile t;
    if (!tile_of(a, x, &t) || r >= t.rows) return;
    const int64_t span = t.hi - t.lo / kKeys * kKeys;
    int count = (int)((span + a.many_keys - 1) / a.many_keys);
    count = count < 1 ? 1 : (count > a.many_splits ? a.many_splits : count);
    const int64_t at = ((int64_t)x * a.c.n_kv_heads + kvh) * kManyRows + r, step = (int64_t)a.tiles * a.c.n_kv_heads * kManyRows;
    join_row<D>(a, a.many_ml, a.many_o, at, step, count, (a.off[t.b] + (t.row0 + r) / G) * a.c.n_q_heads + kvh * G + (t.row0 + r) % G);
}

// How a call is laid out: which kernels run, and the splits of each.
struct Plan {
    int64_t total, most_few;            // rows in all; rows of a kv head of the largest request that has few
    bool few, many;
    int32_t few_rows, splits, split_blocks;
    int32_t tiles, many_splits, many_count, many_b[kManyList], many_tile[kManyList];
    int64_t many_keys;
    size_t part_o, many_ml, many_o, bytes;      // where the workspace's parts begin (part_ml at 0)
};

constexpr int64_t kFewTarget = 1024;    // workgroups that keep the device busy: four on each of 256 compute units
constexpr int64_t kMinSplit = 8;        // blocks of a split: two for each wave
constexpr int64_t kManyTarget = 256;    // one workgroup of eight waves on each compute unit
constexpr int64_t kManyMinKeys = 1024;  // keys of a split that are worth writing 256 rows of partial results

// Splits of `span` units for `lines` lines of work: about `target` workgroups in all, `least` units each, at most `most` splits.
void split_of(int64_t span, int64_t lines, int64_t target, int64_t least, int64_t most, int64_t *splits, int64_t *each)
{
    *each = sp::ceil_div(span * lines, target);
    if (*each < least) *each = least;
    if (sp::ceil_div(span, *each) > most) *each = sp::ceil_div(span, most);
    *splits = sp::ceil_div(span, *each);
}

sp_status make_plan(const sp_cache_desc *d, const int64_t *off, int32_t B, int64_t max_len, int64_t window, Plan *p)
{
    if (sp_status rc = sp::check_cache(d)) return rc;
    int64_t longest;
    if (sp_status rc = sp::check_ragged(off, B, &p->total, &longest)) return rc;
    if (max_len < 0 || max_len >= (int64_t(1) << 31))
        return sp::fail(SP_ERR_INVALID_ARG, "max_len = %lld outside 0..2^31-1", (long long)max_len);
    const int64_t G = d->n_q_heads / d->n_kv_heads, kv = d->n_kv_heads;
    int64_t used = 0, requests = 0;     // tiles and requests with many rows
    p->most_few = 0;
    p->few = p->many = false;
    for (int32_t b = 0; b < B; ++b) {
        const int64_t rows = (off[b + 1] - off[b]) * G;
        if (rows > kFewRows) {
            p->many = true;
            if (requests < kManyList) {
                p->many_b[requests] = b;
                p->many_tile[requests] = (int32_t)used;
            }
            ++requests;
            used += sp::ceil_div(rows, kManyRows);
        } else if (rows > 0) {
            p->few = true;
            p->most_few = rows > p->most_few ? rows : p->most_few;
        }
    }
    p->few_rows = p->most_few <= 16 ? 16 : (p->most_few <= 32 ? 32 : 64);
    const int64_t tile = 8192 / d->head_dim, tiles = requests <= kManyList ? used : p->total * G / kManyRows + B;
    if (tiles * kv >= (int64_t(1) << 31))
        return sp::fail(SP_ERR_UNSUPPORTED, "%lld query rows are more than a launch holds", (long long)(p->total * d->n_q_heads));
    p->tiles = (int32_t)tiles;
    p->many_count = requests <= kManyList ? (int32_t)requests : 0;

    // The workspace is sized without a window, which shortens what rows see and never takes more splits than the whole contexts would.
    int64_t splits, each, many_splits, many_each;
    split_of(sp::ceil_div(max_len, kBlock) + 1, B * kv, kFewTarget, kMinSplit, INT64_MAX, &splits, &each);
    split_of(sp::ceil_div(max_len, tile) + 1, tiles * kv > 0 ? tiles * kv : 1, kManyTarget, kManyMinKeys / tile, INT64_MAX, &many_splits, &many_each);
    const size_t few = p->few && splits > 1 ? (size_t)splits * B * kv * p->few_rows : 0;
    const size_t many = p->many && many_splits > 1 ? (size_t)many_splits * tiles * kv * kManyRows : 0;
    p->part_o = sp::align_up(few * sizeof(f32x2), 256);
    p->many_ml = p->part_o + sp::align_up(few * d->head_dim * sizeof(float), 256);
    p->many_o = p->many_ml + sp::align_up(many * sizeof(f32x2), 256);
    p->bytes = p->many_o + sp::align_up(many * d->head_dim * sizeof(float), 256);
    const int64_t few_seen = window + kFewRows, many_seen = window + kManyRows;     // of a long context
    if (window > 0 && window < max_len && few_seen < max_len)
        split_of(sp::ceil_div(few_seen, kBlock) + 1, B * kv, kFewTarget, kMinSplit, splits, &splits, &each);
    if (window > 0 && window < max_len && many_seen < max_len)
        split_of(sp::ceil_div(many_seen, tile) + 1, tiles * kv > 0 ? tiles * kv : 1, kManyTarget, kManyMinKeys / tile, many_splits, &many_splits, &many_each);
    p->splits = (int32_t)splits;
    p->split_blocks = (int32_t)each;
    p->many_splits = (int32_t)many_splits;
    p->many_keys = many_each * tile;
    return SP_OK;
}

template <int D, bool E4M3>
sp_status run(const AttendArgs &a, const Plan &p, hipStream_t st)
{
    if (p.few) {
        const dim3 grid((unsigned)p.splits, (unsigned)a.c.n_kv_heads, (unsigned)a.B);
        if (p.few_rows == 16) hipLaunchKernelGGL((sp_attend_few_kernel<D, E4M3, 1>), grid, dim3(kThreads), 0, st, a);
        else if (p.few_rows == 32) hipLaunchKernelGGL((sp_attend_few_kernel<D, E4M3, 2>), grid, dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL((sp_attend_few_kernel<D, E4M3, 4>), grid, dim3(kThreads), 0, st, a);
        SP_HIP_CHECK(hipGetLastError());
        if (p.splits > 1) {
            const dim3 rows((unsigned)p.most_few, (unsigned)a.c.n_kv_heads, (unsigned)a.B);
            hipLaunchKernelGGL((sp_attend_join_kernel<D>), rows, dim3(kThreads), 0, st, a);
            SP_HIP_CHECK(hipGetLastError());
        }
    }
    if (p.many) {
        const dim3 grid((unsigned)((int64_t)p.tiles * a.c.n_kv_heads * p.many_splits));
        hipLaunchKernelGGL((sp_attend_many_kernel<D, E4M3>), grid, dim3(kManyThreads), 0, st, a);
        SP_HIP_CHECK(hipGetLastError());
        if (p.many_splits > 1) {
            const dim3 rows((unsigned)((int64_t)p.tiles * kManyRows), (unsigned)a.c.n_kv_heads);
            hipLaunchKernelGGL((sp_attend_many_join_kernel<D, E4M3>), rows, dim3(kThreads), 0, st, a);
            SP_HIP_CHECK(hipGetLastError());
        }
    }
    return SP_OK;
}

}  // namespace

extern "C" sp_status sp_attend_workspace(const sp_cache_desc *desc, const int64_t *offsets_host, int32_t B, int64_t max_len,
                                         size_t *bytes)
{
    if (!bytes) return sp::fail(SP_ERR_INVALID_ARG, "bytes is null");
    Plan p;
    if (sp_status rc = make_plan(desc, offsets_host, B, max_len, 0, &p)) return rc;
    *bytes = p.bytes;
    return SP_OK;
}

extern "C" sp_status sp_attend(const sp_cache_desc *desc, const void *q_dev, const int64_t *offsets_host,
                               const int64_t *offsets_dev, int32_t B, const int32_t *lens_dev, int64_t max_len,
                               const int32_t *block_table_dev, int64_t table_stride, const void *k_pool_dev,
                               const void *v_pool_dev, const float *k_scale_dev, const float *v_scale_dev, float scale,
                               int32_t causal, int64_t window, void *out_dev, float *lse_dev, void *ws_dev,
                               size_t ws_bytes, void *hip_stream)
{
    Plan p;
    if (sp_status rc = make_plan(desc, offsets_host, B, max_len, window, &p)) return rc;
    if (!(scale > 0.f) || scale > 3.0e38f) return sp::fail(SP_ERR_INVALID_ARG, "scale must be finite and > 0");
    if (causal != 0 && causal != 1) return sp::fail(SP_ERR_INVALID_ARG, "causal = %d is neither 0 nor 1", causal);
    if (window < 0 || (window > 0 && !causal))
        return sp::fail(SP_ERR_INVALID_ARG, "window = %lld must be 0, or positive with causal = 1", (long long)window);
    if (table_stride < 1 || table_stride > (int64_t(1) << 31))
        return sp::fail(SP_ERR_INVALID_ARG, "table_stride = %lld outside 1..2^31", (long long)table_stride);
    if (max_len > table_stride * desc->page_tokens)
        return sp::fail(SP_ERR_INVALID_ARG, "max_len = %lld exceeds the block table's %lld tokens", (long long)max_len,
                        (long long)(table_stride * desc->page_tokens));
    if (p.total == 0) return SP_OK;
    if (!q_dev || !out_dev || !offsets_dev || !lens_dev || !block_table_dev)
        return sp::fail(SP_ERR_INVALID_ARG, "only lse_dev, and ws_dev where no workspace is needed, may be null");
    if ((uintptr_t)q_dev % 16 != 0 || (uintptr_t)out_dev % 16 != 0)
        return sp::fail(SP_ERR_INVALID_ARG, "q_dev and out_dev must be 16-byte aligned");
    if (sp_status rc = sp::check_pools(*desc, k_pool_dev, v_pool_dev, k_scale_dev, v_scale_dev)) return rc;
    if (p.bytes > 0) {
        if (!ws_dev) return sp::fail(SP_ERR_WORKSPACE, "ws_dev is null (%zu bytes needed)", p.bytes);
        if ((uintptr_t)ws_dev % 256 != 0) return sp::fail(SP_ERR_WORKSPACE, "ws_dev is not 256-byte aligned");
        if (ws_bytes < p.bytes) return sp::fail(SP_ERR_WORKSPACE, "workspace too small: %zu < %zu", ws_bytes, p.bytes);
    }

    AttendArgs a{sp::view_of(*desc, block_table_dev, table_stride), static_cast<const uint16_t *>(q_dev), offsets_dev,
                 lens_dev, static_cast<const uint8_t *>(k_pool_dev), static_cast<const uint8_t *>(v_pool_dev),
                 k_scale_dev, v_scale_dev, static_cast<uint16_t *>(out_dev), lse_dev, max_len, window, B, causal, scale};
    a.page_blocks = (int32_t)(desc->page_tokens / kBlock);
    a.page_shift = -1;
    for (int s = 0; s < 24; ++s)
        if (a.page_blocks == 1 << s) a.page_shift = s;
    a.splits = p.splits;
    a.split_blocks = p.split_blocks;
    a.few_rows = p.few_rows;
    a.tiles = p.tiles;
    a.many_splits = p.many_splits;
    a.many_keys = p.many_keys;
    a.many_count = p.many_count;
    for (int i = 0; i < p.many_count; ++i) {
        a.many_b[i] = p.many_b[i];
        a.many_tile[i] = p.many_tile[i];
    }
    uint8_t *ws = static_cast<uint8_t *>(ws_dev);
    a.part_ml = reinterpret_cast<f32x2 *>(ws);
    a.part_o = reinterpret_cast<float *>(ws + p.part_o);
    a.many_ml = reinterpret_cast<f32x2 *>(ws + p.many_ml);
    a.many_o = reinterpret_cast<float *>(ws + p.many_o);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool e4m3 = sp::cache_is_e4m3(*desc);
    if (desc->head_dim == 64) return e4m3 ? run<64, true>(a, p, st) : run<64, false>(a, p, st);
    return e4m3 ? run<128, true>(a, p, st) : run<128, false>(a, p, st);
}
