// sp_attend_weights: how much attention each token of a paged cache has drawn (what an eviction goes by; the paper's importance
// of a token is the attention that it draws, Appendix A.1.1, there over all layers at once and here for one layer's cache).
//
//   w[b, h, j] = old + sum_{r, g} exp(scale <q[r, g], k[b, h, j]> - lse[r, g])
// over the rows r that see key j and the query heads g of kv head h; lse is what sp_attend wrote. A key's weight is the sum over the rows of a kv
// head, so a wave that holds a block of keys goes through the rows and no sum crosses workgroups: nothing is added atomically, the order is fixed
// by the lengths. The products are Q K^T with a key in a lane column: a lane adds up its rows, and the lanes of a column meet once at the end. Keys
// are bf16 or become it, exactly; logits, exponentials and sums are fp32.
#include "sp_context.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
// Rows of a kv head that sp_weights_few_kernel takes at most: what a wave's tile holds. 12 rows of 16 contexts of 16000 tokens (8 heads of 64, MX4)
// take 23 us there and 33 in the other kernel, of 4 (8 of 128, bf16) 32 and 30.
constexpr int kFewRows = 16;
constexpr int kManyRows = 32;           // rows of a tile of sp_weights_many_kernel
constexpr int64_t kUnits = 256;         // compute units
constexpr int many_blocks(int d) { return 128 / d; }    // blocks of 32 keys of a wave there: as many as leave four waves a SIMD their registers

typedef __attribute__((ext_vector_type(16))) float f32x16;

struct WeightArgs : ContextArgs {
    const float *lse, *old;
    float *weights;
    int64_t stride;                     // entries of a line of weights
    int32_t per;                        // pairs of blocks of 32 tokens that a wave of sp_weights_few_kernel takes
};

// Keys [first, last) that a row sees; rows that a tile does not have see none.
struct Seen {
    int first, last;

    __device__ __forceinline__ Seen(const ContextArgs &a, const Range &rg, int token, bool there)
    {
        last = !there ? 0 : a.causal ? rg.len - rg.n + token + 1 : rg.len;
        first = a.causal && a.window > 0 && last > a.window ? last - a.window : 0;
    }

    __device__ __forceinline__ bool sees(int key) const { return key >= first && key < last; }
};

// What is taken from a row's logits, in units of log 2: its lse, or infinity for a row that adds nothing.
__device__ __forceinline__ float reference(float lse) { return lse == neg_inf() ? __builtin_huge_valf() : lse * kLog2e; }

// Stores a key's weight: what was there counts for keys before `older`.
__device__ __forceinline__ void store_weight(const WeightArgs &a, int64_t at, int key, int older, float sum)
{
    a.weights[at + key] = a.old && key < older ? a.old[at + key] + sum : sum;
}

__device__ __forceinline__ int older_of(const ContextArgs &a, const Range &rg) { return a.causal ? rg.len - rg.n : rg.len; }

// Lanes of group g (16 of them) take x of tile g: lanes of group 0 of every one of four tiles hold what counts.
__device__ __forceinline__ float gather4(float x0, float x1, float x2, float x3)
{
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x0), __float_as_uint(x2), false, false);     // [x0 lower | x2 lower]
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x1), __float_as_uint(x3), false, false);
    return __uint_as_float(__builtin_amdgcn_permlane16_swap(p[0], q[0], false, false)[0]);
}

// Lower half of a wave: x of tile 0, upper half: x of tile 1; their lower halves hold what counts.
__device__ __forceinline__ float gather2(float x0, float x1)
{
    return __uint_as_float(__builtin_amdgcn_permlane32_swap(__float_as_uint(x0), __float_as_uint(x1), false, false)[0]);
}

// Requests of up to 16 rows a kv head (none too: their weights are what they were). A wave has its rows in registers and takes pairs of blocks of
// 32 tokens, one of its workgroup's in turn, a pair ahead. After the products lane 16 g + c holds rows 4g .. 4g + 3 of a column's key. With at most
// four rows (LIVE = 1) only lanes of group 0 hold any, so four tiles of 16 keys are gathered into all lanes before the exponentials, with at most
// eight (LIVE = 2) two (48 contexts of MX4: 72 us without the gathering, 66 with).
// Bound by reading, and by starting: 48 contexts of 2048 to 65536 tokens, 8 kv heads of 64, 4 query heads each, MX4 (271 MB with old and new
// weights) take 66 us, 4.1 TB/s; 48 of 16384 59, 4.5, and of E4M3 90, 5.0. A short line's workgroups are a chain of offsets, lengths, block table,
// keys for one or two pairs. Not kept: two pairs ahead (66), the pairs of all lines in equal shares over the resident workgroups (72: finding a
// share's start takes longer than its lines' ends leave idle).
template <int D, int KIND, int LIVE>
__global__ __launch_bounds__(kThreads) void sp_weights_few_kernel(WeightArgs a)
{
    using B = Block<D, KIND, false>;
    constexpr bool E4M3 = KIND == SP_CACHE_E4M3, MX4 = KIND == SP_CACHE_MX4;
    constexpr int kSteps = D / 32;
    const int b = blockIdx.y / a.c.n_kv_heads, kvh = blockIdx.y % a.c.n_kv_heads, G = a.c.group;
    const Range rg = range_of(a, b);
    const int64_t rows = (int64_t)rg.n * G;
    const int pairs = (rg.len + 2 * kBlock - 1) / (2 * kBlock), lo = blockIdx.x * a.per * kWaves, hi = __builtin_amdgcn_readfirstlane(min(lo + a.per * kWaves, pairs));
    if (rows > kFewRows || lo >= hi) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    int pair = lo + wave;
    if (pair >= hi) return;
    const int64_t line_at = ((int64_t)b * a.c.n_kv_heads + kvh) * a.stride;
    const int older = older_of(a, rg);

    // this lane's part of row c for the products, and what it needs of the rows whose results it holds: 4 (g % LIVE) .. + 3
    bf16x8 q[kSteps];
    {
        // rows that are not there are copies of row 0: a key that makes its logit minus infinity makes theirs no NaN
        const int r = c < rows ? c : 0;
        const uint16_t *src = a.q + ((a.off[b] + r / G) * a.c.n_q_heads + kvh * G + r % G) * D;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int e = MX4 ? D / 4 * g + 8 * s : E4M3 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
            u32x4 w = {0, 0, 0, 0};
            if (rows > 0) w = *reinterpret_cast<const u32x4 *>(src + e);
            q[s] = __builtin_bit_cast(bf16x8, w);
        }
    }
    float ref[4];
    int first[4], last[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int r = 4 * (g % LIVE) + j;
        const Seen s(a, rg, r / G, r < rows);
        first[j] = s.first;
        last[j] = s.last;
        ref[j] = __builtin_huge_valf();
        if (r < rows) ref[j] = reference(a.lse[(a.off[b] + r / G) * a.c.n_q_heads + kvh * G + r % G]);
    }
    // every row sees the keys of [all_lo, all_hi); a request without rows has none that does
    const int all_lo = a.causal && a.window > 0 && rg.len - a.window > 0 ? rg.len - a.window : 0;
    const int all_hi = rows == 0 ? 0 : a.causal ? rg.len - rg.n + 1 : rg.len;

    const Line line(a, b, kvh, KIND, D);
    const uint32_t k_lane = MX4 ? 2 * c * line.row_bytes + D / 8 * g : c * line.row_bytes + 16 * g;
    const int last_block = __builtin_amdgcn_readfirstlane((rg.len - 1) / kBlock);           // the second of a last pair may not be there
    const auto load = [&](B &kv, const Entry &e) {
        Place at = e.place(a, line);
        at = {uniform(at.off), uniform(at.scale)};
        if constexpr (MX4) kv.load_keys(line, at, k_lane, c * (D / 16));
        else kv.load_keys(line, at, k_lane);
    };
    const float scale2 = a.scale * kLog2e;
    const int end = pair + (hi - 1 - pair) / kWaves * kWaves;
    B kv[2];
    const auto entry = [&](int blk) { return Entry(a, line, min(blk, last_block)); };
    Entry soon[2] = {entry(2 * min(pair + kWaves, end)), entry(2 * min(pair + kWaves, end) + 1)};
#pragma unroll
    for (int u = 0; u < 2; ++u) load(kv[u], entry(2 * pair + u));
    // key of column c of tile t (0, 1) of a block; the key of a pair whose weight this lane stores
    const auto key_in = [&](int t) { return MX4 ? 2 * c + t : 16 * t + c; };
    const int mine = LIVE == 2 ? kBlock * (g & 1) + key_in(g >> 1) : kBlock * (g >> 1) + key_in(g & 1);
    const auto weight_before = [&](int of) {
        const int key = 2 * kBlock * of + mine;
        return a.old && key < older ? a.old[line_at + key] : 0.f;
    };
    float was = weight_before(pair);
    for (;;) {
        const int key0 = pair * 2 * kBlock, then = 2 * min(pair + 2 * kWaves, end), own = key0 + mine;
        const Entry later[2] = {entry(then), entry(then + 1)};
        f32x4 x[4];                                         // tiles 0, 1 of the first block, then of the second
        float factor[2] = {scale2, scale2};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                x[2 * u + t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    bf16x8 k;
                    if constexpr (MX4) k = kv[u].key(t, s, g);
                    else k = kv[u].key(t, s);
                    x[2 * u + t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[s], k, x[2 * u + t], 0, 0, 0);
                }
            }
            if constexpr (E4M3) factor[u] = factor_of(scale2, kv[u].ks);
            load(kv[u], soon[u]);
            soon[u] = later[u];
        }
        const float will = weight_before(min(pair + kWaves, end));
        const bool whole = key0 >= all_lo && key0 + 2 * kBlock <= all_hi;
        // the key's logits of this lane's four rows become its part of the weight
        const auto part = [&](f32x4 y, float f, int key) {
            float p[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float x = y[j] * f - ref[j];
                if (!whole && (key < first[j] || key >= last[j])) x = neg_inf();        // whatever the key and its block's scale are
                p[j] = exp2_(x);
            }
            return (p[0] + p[1]) + (p[2] + p[3]);
        };
        float sum;
        if constexpr (LIVE == 1) {
            f32x4 y;
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = gather4(x[0][j], x[1][j], x[2][j], x[3][j]);
            sum = part(y, g < 2 ? factor[0] : factor[1], own);
        } else if constexpr (LIVE == 2) {
            float s[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                f32x4 y;
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = gather2(x[2 * u][j], x[2 * u + 1][j]);
                s[u] = part(y, factor[u], key0 + kBlock * u + key_in(g >> 1));
            }
            // lanes of even groups keep the first block's, those of odd ones the second's
            const float give = g & 1 ? s[0] : s[1], keep = g & 1 ? s[1] : s[0];
            sum = keep + __shfl_xor(give, 16);
        } else {
            float s[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) s[t] = part(x[t], factor[t >> 1], key0 + kBlock * (t >> 1) + key_in(t & 1));
            // tile t ends up in group t: its halves meet, then its quarters
            float half[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const float give = g & 2 ? s[t] : s[2 + t], keep = g & 2 ? s[2 + t] : s[t];
                half[t] = keep + __shfl_xor(give, 32);
            }
            const float give = g & 1 ? half[0] : half[1], keep = g & 1 ? half[1] : half[0];
            sum = keep + __shfl_xor(give, 16);
        }
        if (own < rg.len) a.weights[line_at + own] = was + sum;
        was = will;
        if (pair == end) break;
        pair += kWaves;
    }
}

// Requests with more rows: a wave holds 32 or 64 keys as bf16 and goes through tiles of 32 rows, which its workgroup brings to LDS, two buffers in
// turn. A block's E4M3 scale goes into the factor. R fours of waves have the same keys and take the tiles in turn; their sums are added in their
// order. The last 64 of 32768 tokens, 16 heads over 8 of 128, bf16: 67 MB of keys in 25 us. One read of the keys (11 us) and four tiles of rows (9
// us of products, and their exponentials) come after each other in a wave; four waves a SIMD fill in for one another (two, with twice the keys
// each: 27 us; all rows in LDS and the keys streamed past them: 29).
template <int D, int KIND, int R>
__global__ __launch_bounds__(kThreads * R, 4) void sp_weights_many_kernel(WeightArgs a)
{
    constexpr bool E4M3 = KIND == SP_CACHE_E4M3, MX4 = KIND == SP_CACHE_MX4;
    constexpr int kSteps = D / 16, kChunks = D / 8, kLoads = kManyRows * kChunks / kThreads;     // 16-byte pieces of a row; of a thread
    constexpr int kKeyLoads = (int)sp::cache_bytes(KIND, D) / 32;                       // 16-byte loads of half a key's row
    constexpr int W = many_blocks(D), kManyKeys = 32 * W;
    __shared__ u32x4 rows_lds[2][R][kManyRows * kChunks];
    __shared__ float ref_lds[2][R][kManyRows];
    __shared__ int first_lds[2][R][kManyRows], last_lds[2][R][kManyRows];
    __shared__ float sum_lds[R][kWaves][kManyKeys];

    const int b = blockIdx.y / a.c.n_kv_heads, kvh = blockIdx.y % a.c.n_kv_heads, G = a.c.group;
    const Range rg = range_of(a, b);
    const int64_t rows64 = (int64_t)rg.n * G;
    const int key_wg = blockIdx.x * kWaves * kManyKeys;
    if (rows64 <= kFewRows || key_wg >= rg.len) return;
    const int rows = (int)rows64;
    // four waves have the keys, R fours of them a tile of rows each
    const int tid = threadIdx.x % kThreads, wave = __builtin_amdgcn_readfirstlane(tid >> 6), four = __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
    const int lane = tid & 63, h = lane >> 5, c = lane & 31;
    const int key0 = key_wg + wave * kManyKeys, older = older_of(a, rg);
    const int64_t line_at = ((int64_t)b * a.c.n_kv_heads + kvh) * a.stride;
    const float scale2 = a.scale * kLog2e;

    // elements of step s of a lane's half of a key: E4M3 and MX4 loads bring more than one step's
    const auto piece = [&](int s) { return MX4 ? 8 * (s / 4) + 4 * h + s % 4 : E4M3 ? 4 * (s / 2) + 2 * h + s % 2 : 2 * s + h; };
    bf16x8 k[W][kSteps];
    float factor[W];
    const Line line(a, b, kvh, KIND, D);
#pragma unroll
    for (int w = 0; w < W; ++w) {
        // blocks behind the context are those of its last token: what they give is not stored
        const int blk = min(key0 + 32 * w, rg.len - 1) / kBlock;
        const Place at = Entry(a, line, blk).place(a, line);
        const uint8_t *src = line.k + at.off + (int64_t)c * line.row_bytes + 16 * h;
        factor[w] = scale2;
        if constexpr (E4M3) factor[w] = factor_of(scale2, line.ks[at.scale]);
#pragma unroll
        for (int i = 0; i < kKeyLoads; ++i) {
            const u32x4 x = *reinterpret_cast<const u32x4 *>(src + 32 * i);
            if constexpr (MX4) {
                const float s = __uint_as_float((uint32_t)line.ks4[at.scale * D + c * (D / 32) + 2 * i + h] << 23);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    k[w][4 * i + j] = __builtin_bit_cast(bf16x8, u32x4{widen4<0>(x[j], s), widen4<1>(x[j], s), widen4<2>(x[j], s), widen4<3>(x[j], s)});
            } else if constexpr (E4M3) {
                k[w][2 * i] = widen8(x[0], x[1]);
                k[w][2 * i + 1] = widen8(x[2], x[3]);
            } else
                k[w][i] = __builtin_bit_cast(bf16x8, x);
        }
    }

    // rows that may see a key of this workgroup: [from, to) in tiles
    int from = 0, to = rows;
    if (a.causal) {
        const int64_t p = (int64_t)rg.len - rg.n;                       // token t sees keys up to p + t
        const int64_t t0 = key_wg - p, t1 = a.window > 0 ? (int64_t)key_wg + kWaves * kManyKeys - 1 + a.window - p : rg.n;   // tokens [t0, t1)
        from = t0 > 0 ? (int)min(t0, (int64_t)rg.n) * G : 0;
        to = t1 < rg.n ? (t1 > 0 ? (int)t1 * G : 0) : rows;
    }
    const int tile0 = from / kManyRows, tiles = to > from ? (to + kManyRows - 1) / kManyRows : tile0;
    u32x4 next[kLoads];
    float next_ref = 0.f;
    Seen next_seen(a, rg, 0, false);
    const auto slot = [&](int r, int p) { return r * kChunks + (p ^ (r & (D == 128 ? 15 : 7))); };
    const auto fetch = [&](int tile) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            // behind the last row copies of it, which add nothing
            const int x = tid + i * kThreads, r = min(tile * kManyRows + x / kChunks, rows - 1);
            next[i] = reinterpret_cast<const u32x4 *>(a.q + ((a.off[b] + r / G) * a.c.n_q_heads + kvh * G + r % G) * D)[x % kChunks];
        }
        if (tid < kManyRows) {
            const int r = tile * kManyRows + tid;
            next_seen = Seen(a, rg, r / G, r < rows);
            next_ref = __builtin_huge_valf();
            if (r < rows) next_ref = reference(a.lse[(a.off[b] + r / G) * a.c.n_q_heads + kvh * G + r % G]);
        }
    };
    const auto put = [&](int buf) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int x = tid + i * kThreads;
            rows_lds[buf][four][slot(x / kChunks, x % kChunks)] = next[i];
        }
        if (tid < kManyRows) {
            ref_lds[buf][four][tid] = next_ref;
            first_lds[buf][four][tid] = next_seen.first;
            last_lds[buf][four][tid] = next_seen.last;
        }
    };
    float sum[W] = {};
    const auto multiply = [&](int tile, int buf) {
        f32x16 x[W];
#pragma unroll
        for (int w = 0; w < W; ++w)
#pragma unroll
            for (int e = 0; e < 16; ++e) x[w][e] = 0.f;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const bf16x8 q = __builtin_bit_cast(bf16x8, rows_lds[buf][four][slot(c, piece(s))]);
#pragma unroll
            for (int w = 0; w < W; ++w) x[w] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, k[w][s], x[w], 0, 0, 0);
        }
        // rows of a tile are in order: those in between see what its first and last row both see
        const int t_lo = tile * kManyRows / G, t_hi = min(tile * kManyRows + kManyRows - 1, rows - 1) / G;
        const int all_hi = a.causal ? rg.len - rg.n + t_lo + 1 : rg.len, all_lo = a.causal && a.window > 0 ? rg.len - rg.n + t_hi + 1 - a.window : 0;
        const bool whole = key0 >= all_lo && key0 + kManyKeys <= all_hi;
        float f[W];
#pragma unroll
        for (int w = 0; w < W; ++w) f[w] = whole ? factor[w] : 1.f;
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {                                // rows 8 e4 + 4 h + e
            const f32x4 ref = *reinterpret_cast<const f32x4 *>(&ref_lds[buf][four][8 * e4 + 4 * h]);
            if (!whole)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = 8 * e4 + 4 * h + e, first = first_lds[buf][four][r], last = last_lds[buf][four][r];
#pragma unroll
                    for (int w = 0; w < W; ++w) {
                        const int key = key0 + 32 * w + c;
                        x[w][4 * e4 + e] = key < first || key >= last ? neg_inf() : x[w][4 * e4 + e] * factor[w];    // whatever the key and its block's scale are
                    }
                }
#pragma unroll
            for (int w = 0; w < W; ++w) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = exp2_(x[w][4 * e4 + e] * f[w] - ref[e]);
                sum[w] += (p[0] + p[1]) + (p[2] + p[3]);
            }
        }
    };
    if (tile0 + four < tiles) {
        fetch(tile0 + four);
        put(0);
    }
    __syncthreads();
    for (int at = tile0, buf = 0; at < tiles; at += R, buf ^= 1) {
        const int tile = at + four;
        if (tile + R < tiles) fetch(tile + R);
        if (tile < tiles) multiply(tile, buf);
        if (tile + R < tiles) put(buf ^ 1);
        __syncthreads();
    }
#pragma unroll
    for (int w = 0; w < W; ++w) sum[w] += __shfl_xor(sum[w], 32);
    if constexpr (R > 1) {                                  // the fours' sums, in their order
#pragma unroll
        for (int w = 0; w < W; ++w)
            if (h == 0) sum_lds[four][wave][32 * w + c] = sum[w];
        __syncthreads();
        if (four != 0) return;
#pragma unroll
        for (int w = 0; w < W; ++w)
#pragma unroll
            for (int i = 1; i < R; ++i) sum[w] += sum_lds[i][wave][32 * w + c];
    }
    const int key = key0 + 32 * (W == 2 ? h : 0) + c;
    if (key < rg.len && (W == 2 || h == 0)) store_weight(a, line_at, key, older, W == 2 && h ? sum[W - 1] : sum[0]);
}

// few: rows of a kv head of the largest request that has few, -1 if none has; fours: of waves of a workgroup for many rows, 0 if none has many
template <int D, int KIND>
sp_status run(const WeightArgs &a, int few, int fours, hipStream_t st)
{
    const unsigned lines = (unsigned)(a.B * a.c.n_kv_heads);
    if (few >= 0) {
        const dim3 grid((unsigned)sp::ceil_div(sp::ceil_div(a.max_len, 2 * kBlock), (int64_t)a.per * kWaves), lines);
        if (few <= 4) hipLaunchKernelGGL((sp_weights_few_kernel<D, KIND, 1>), grid, dim3(kThreads), 0, st, a);
        else if (few <= 8) hipLaunchKernelGGL((sp_weights_few_kernel<D, KIND, 2>), grid, dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL((sp_weights_few_kernel<D, KIND, 4>), grid, dim3(kThreads), 0, st, a);
        SP_HIP_CHECK(hipGetLastError());
    }
    if (fours) {
        const dim3 grid((unsigned)sp::ceil_div(a.max_len, 32 * many_blocks(D) * kWaves), lines);
        if (fours == 4) hipLaunchKernelGGL((sp_weights_many_kernel<D, KIND, 4>), grid, dim3(4 * kThreads), 0, st, a);
        else if (fours == 2) hipLaunchKernelGGL((sp_weights_many_kernel<D, KIND, 2>), grid, dim3(2 * kThreads), 0, st, a);
        else hipLaunchKernelGGL((sp_weights_many_kernel<D, KIND, 1>), grid, dim3(kThreads), 0, st, a);
        SP_HIP_CHECK(hipGetLastError());
    }
    return SP_OK;
}

template <int D>
sp_status run_kind(const WeightArgs &a, int kind, int few, int fours, hipStream_t st)
{
    if (kind == SP_CACHE_MX4) return run<D, SP_CACHE_MX4>(a, few, fours, st);
    return kind == SP_CACHE_E4M3 ? run<D, SP_CACHE_E4M3>(a, few, fours, st) : run<D, SP_CACHE_BF16>(a, few, fours, st);
}

}  // namespace

extern "C" sp_status sp_attend_weights(const sp_cache_desc *desc, const void *q_dev, const int64_t *offsets_host, const int64_t *offsets_dev,
                                       int32_t B, const int32_t *lens_dev, int64_t max_len, const int32_t *block_table_dev, int64_t table_stride,
                                       const void *k_pool_dev, const void *k_scale_dev, float scale, int32_t causal, int64_t window,
                                       const float *lse_dev, const float *old_dev, float *weights_dev, int64_t weights_stride, void *hip_stream)
{
    if (sp_status rc = sp::check_cache(desc)) return rc;
    int64_t total, longest;
    if (sp_status rc = sp::check_ragged(offsets_host, B, &total, &longest)) return rc;
    if (max_len < 0 || max_len > kMaxLen) return sp::fail(SP_ERR_INVALID_ARG, "max_len = %lld outside 0..2^30", (long long)max_len);
    if (total > kMaxTokens) return sp::fail(SP_ERR_UNSUPPORTED, "%lld query tokens exceed 2^26", (long long)total);
    if (sp_status rc = check_masks(desc, max_len, table_stride, scale, causal, window)) return rc;
    if (weights_stride < max_len || weights_stride > (int64_t(1) << 40))
        return sp::fail(SP_ERR_INVALID_ARG, "weights_stride = %lld is less than max_len = %lld or above 2^40", (long long)weights_stride, (long long)max_len);
    if ((int64_t)B * desc->n_kv_heads > 65535)
        return sp::fail(SP_ERR_UNSUPPORTED, "%d requests of %d kv heads are more than a launch holds", B, desc->n_kv_heads);
    if (B == 0 || max_len == 0) return SP_OK;
    if (!offsets_dev || !lens_dev || !block_table_dev || !weights_dev)
        return sp::fail(SP_ERR_INVALID_ARG, "only old_dev may be null");
    if (total > 0 && (!q_dev || !lse_dev)) return sp::fail(SP_ERR_INVALID_ARG, "q_dev or lse_dev is null");
    if ((uintptr_t)q_dev % 16 != 0) return sp::fail(SP_ERR_INVALID_ARG, "q_dev must be 16-byte aligned");
    if (sp_status rc = sp::check_pools(*desc, k_pool_dev, k_pool_dev, k_scale_dev, k_scale_dev)) return rc;

    const int64_t G = desc->n_q_heads / desc->n_kv_heads;
    int few = -1;
    int64_t tiles = 0, longest_tiles = 0;       // of rows, of the requests with many
    for (int32_t b = 0; b < B; ++b) {
        const int64_t rows = (offsets_host[b + 1] - offsets_host[b]) * G, n = sp::ceil_div(rows, kManyRows);
        if (rows <= kFewRows) {
            few = rows > few ? (int)rows : few;
            continue;
        }
        tiles += n;
        longest_tiles = n > longest_tiles ? n : longest_tiles;
    }
    // A workgroup goes through the tiles of its line's rows, 1.1 us each; several fours of waves share them. That pays where the longest line, and
    // not the work of a compute unit, takes the time, and costs where there is work for all, since each four loads the keys. One, two, four fours
    // in us, at one longest line a unit's work: 8192 rows by 8192 keys, 8 heads of 64 284, 182, 132; at half of it: 4096 rows, 8 of 128 160, 118,
    // 128; at a quarter: 16 requests of 2048 rows by 2000 keys 142, 145, 160; few rows (128 by 32768, 8 of 128) 25, 32, 56.
    const int64_t unit = sp::ceil_div(max_len, 32 * many_blocks(desc->head_dim) * kWaves) * desc->n_kv_heads * tiles / kUnits;
    const int fours = tiles == 0 ? 0 : longest_tiles < 16 || 3 * longest_tiles < unit ? 1 : 4 * longest_tiles < 3 * unit ? 2 : 4;
    WeightArgs a{};
    static_cast<ContextArgs &>(a) = context_args(*desc, q_dev, offsets_dev, lens_dev, max_len, block_table_dev, table_stride, k_pool_dev, k_pool_dev,
                                                 k_scale_dev, k_scale_dev, scale, causal, window, B);
    a.lse = lse_dev;
    a.old = old_dev;
    a.weights = weights_dev;
    a.stride = weights_stride;
    // Pairs of blocks of a wave: as many as leave two waves a SIMD, at most 8. One, two, four, eight of them in us: 65536 keys, 8 heads of 64,
    // 10.6, 8.7, 9.0, 10.5; 16 times 16000 34, 26, 22, 20; 4 times 16000, 8 of 128, 43, 35, 32, 33; 48 of up to 65536 115, 74 to 81, 66, 67, and
    // 138 with sixteen.
    const int64_t pairs = sp::ceil_div(max_len, 2 * kBlock) * B * desc->n_kv_heads;
    a.per = 1;
    while (a.per < 8 && pairs > (int64_t)a.per * 2048) a.per *= 2;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return desc->head_dim == 64 ? run_kind<64>(a, desc->cache_type, few, fours, st) : run_kind<128>(a, desc->cache_type, few, fours, st);
}
