// sp_attend: attention of ragged queries over a paged cache (paper: Algorithm 1 ForwardWithAttn, a decoder layer's
// attention over the cache that the importance pass reads afterwards).
//
//   out = sum_j p_j v_j,  p_j = exp(x_j - m) / l,  x_j = scale <q, k_j>,  m = max_j x_j,  l = sum_j exp(x_j - m),
//   lse = m + log l,
// in one pass over the keys: a reference m and a sum l that run along, and the partial output, scaled whenever m moves.
//
// Rounded to fewer bits: the probabilities that go into the second product, to bf16 (2^-8 of each at most), since the matrix instructions take
// both operands in one type and the values are bf16, or 8-bit codes that bf16 holds exactly; fp32 operands would take a sixteenth of the rate. Their sum is taken
// before, in fp32, as are m, l, the logits and the partial outputs. The output is bf16 itself: its error against 64 bits is 0.0015 to 0.0017 of
// the 2-norm with the probabilities in fp32, 0.0016 to 0.0021 with these.
//
// Query rows of one request that share a kv head (n_b tokens of G heads) are taken together, so that a key is read once for
// all of them. Requests of up to few_rows_of() rows go to sp_attend_few_kernel, which is bound by the cache's bytes, others to
// sp_attend_many_kernel, tiles of 256 rows, which is bound by its operations.
//
// Shares. Contexts differ and only the device knows them, so work is shared out there: the blocks of all (request, kv head) lines
// are laid end to end, and workgroup i of N takes the i-th of N equal stretches. A line that lies in one stretch is finished there;
// of others every stretch leaves a partial result (reference, sum, unscaled output), at most two a workgroup, which a second
// launch joins. Nothing is added atomically: the order of every sum is fixed by the lengths.
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
// Query rows of a kv head that sp_attend_few_kernel takes at most. At head_dim 128 more of them leave it one wave a SIMD: 64 rows over two contexts of
// 20000 tokens take 38 us there and 35 in the other kernel (head_dim 64, four of 30000 to 64000: 60 and 125).
constexpr int few_rows_of(int d) { return d == 128 ? 32 : 64; }
constexpr int kManyList = 64;
constexpr int kBlock = sp::kCacheBlock;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// A block's key scale goes into its logits' factor, its value scale into the exponent (and out of the sum again): no operation for an element.
// The factor stays above zero, so that masked logits stay minus infinity, and finite, so that a product of zero stays a logit of zero; the value scale
// above 2^-64, so that exponents keep their range.
constexpr float kLeastScale = 5.42101086e-20f, kLeastFactor = 1.17549435e-38f, kMostFactor = 3.40282347e38f;
constexpr float kMostScale = 2.3e38f;      // of a call: times log2(e) it is finite

struct AttendArgs {
    sp::CacheView c;
    const uint16_t *q;
    const int64_t *off;
    const int32_t *lens;
    const uint8_t *k_pool, *v_pool;
    const float *k_scale, *v_scale;
    uint16_t *out;
    float *lse;
    int32_t max_len, window;            // a window is shorter than max_len, or 0
    int32_t B, causal;
    float scale;
    int32_t page_blocks, page_shift;    // blocks of 32 tokens in a page; their logarithm, or -1
    // sp_attend_few_kernel: workgroups that share the work (0: one for each request and kv head), rows of a partial result
    int32_t few_shares, few_rows, few_least;    // the last: blocks of a share
    f32x2 *few_ml;                      // [2 few_shares][few_rows]: reference (in units of log 2), sum
    float *few_o;                       // [2 few_shares][few_rows][head_dim]
    int64_t *few_before;                // [B + 1]: units of work before each request
    // sp_attend_many_kernel: tiles of query rows, workgroups that share the work (0: one for each tile and kv head)
    int32_t tiles, many_shares;
    f32x2 *many_ml;                     // as above, kManyRows rows
    float *many_o;
    int64_t *many_before;               // [tiles + 1]
};

// The requests with many rows and their first tiles, if there are at most kManyList of them (else count is 0). An argument of its own: the kernels for
// few rows, whose calls are short, need not be given it.
struct ManyList {
    int32_t count, b[kManyList], tile[kManyList];
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

// What a row's result is multiplied by, and its logarithm of the denominator (m in units of log 2). A row that saw no key has a sum of exactly
// zero; that of a row that saw a NaN is NaN and gets out.
__device__ __forceinline__ bool saw_nothing(float l) { return l == 0.f; }
__device__ __forceinline__ float inverse(float l) { return saw_nothing(l) ? 0.f : 1.f / l; }
__device__ __forceinline__ float lse_of(float m, float l) { return saw_nothing(l) ? neg_inf() : (m + log2_(l)) * kLn2; }

// ---- a few rows: single tokens, lookahead rows -----------------------------------------------------------------------

// What a request's rows see: row r (token r / G) keys [first(r), last(r)), all rows together [lo, hi). Key indices fit 32 bits:
// contexts are limited to 2^30 tokens, queries to 2^26.
struct Range {
    int len, n, lo, hi;
};

__device__ __forceinline__ Range range_of(const AttendArgs &a, int b)
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

__device__ __forceinline__ uint32_t page_of_block(const AttendArgs &a, uint32_t blk)
{
    return a.page_shift >= 0 ? blk >> a.page_shift : blk / (uint32_t)a.page_blocks;
}

// An entry of request b's row of the block table.
__device__ __forceinline__ int page_entry(const AttendArgs &a, int b, uint32_t i)
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
    int64_t page_bytes;
    uint32_t row_bytes, page_scales;

    const int32_t *table;

    __device__ __forceinline__ Line(const AttendArgs &a, int b, int kvh, int es)
    {
        table = a.c.table + b * a.c.table_stride;
        k = a.k_pool + kvh * a.c.stride_head * es;
        v = a.v_pool + kvh * a.c.stride_head * es;
        ks = a.k_scale + (int64_t)kvh * a.page_blocks;
        vs = a.v_scale + (int64_t)kvh * a.page_blocks;
        page_bytes = a.c.page_stride * es;
        row_bytes = (uint32_t)a.c.stride_token * es;
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

    __device__ __forceinline__ Entry(const AttendArgs &a, const Line &l, int blk)
    {
        const uint32_t i = page_of_block(a, (uint32_t)blk);
        page = l.table[i];
        in_page = (uint32_t)blk - i * (uint32_t)a.page_blocks;
    }

    __device__ __forceinline__ Place place(const AttendArgs &a, const Line &l) const
    {
        const int p = min(max(__builtin_amdgcn_readfirstlane(page), 0), (int)a.c.n_pages - 1);      // never outside the pools
        return {p * l.page_bytes + (int64_t)((uint64_t)in_page * (kBlock * l.row_bytes)), (int64_t)((uint64_t)(uint32_t)p * l.page_scales) + in_page};
    }
};

// One block of 32 tokens as a wave loads it, straight into the registers that the matrix instructions take it from.
// Lane l = 16 g + c. Keys: row c of 16-key tile t, the contraction's elements in an order that makes a lane's share of a row contiguous
// (queries are loaded in the same order). Values: elements [c D/16, (c+1) D/16) of the eight keys 4g + j and 16 + 4g + j, j < 4: the
// keys whose logits the lane holds after the first product.
// Loads that take whole lines of 128 bytes pass the caches by: values, unless their rows have 64 bytes, and keys whose rows do. 32 requests of bf16, head_dim
// 128, 172 us without and 160 with; 48 of E4M3, head_dim 64, 157 and 143 (200 of up to 4000 tokens 52 and 49, but 56 with values too). The latter only
// for contexts that no cache would hold until the next call: 64 of up to 2000 tokens, called again and again, take 15.7 us without and 18.7 with.
template <int D, bool E4M3, bool STREAM>
struct Block {
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
            const int key = first + 4 * g + (j & 3) + (j >> 2) * 16;
            if (key < lo || key >= hi)
#pragma unroll
                for (int i = 0; i < kLoads; ++i) v[j][i] = 0;
        }
    }
};

// Maximum over the four lanes that hold a query row's logits.
__device__ __forceinline__ float row_max(float x)
{
    x = larger(x, __shfl_xor(x, 16));
    return larger(x, __shfl_xor(x, 32));
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

    // x: products <q, k> of this lane's eight keys, factor: what makes logits in units of log 2 of them. Returns 2^vexp times the probabilities as bf16;
    // vinv = 2^-vexp by v_rcp_f32: exact for powers of two, 2^-23 of a block's part of the sum for others.
    __device__ __forceinline__ bf16x8 weigh(int t, const float (&x)[8], float factor, float vexp, float vinv)
    {
        const float top = factor * larger(larger(larger(x[0], x[1]), larger(x[2], x[3])), larger(larger(x[4], x[5]), larger(x[6], x[7])));
        if (__any(top > m[t] + kSlack)) {
            const float mx = larger(m[t], row_max(top));
            const float f = m[t] == neg_inf() ? 0.f : exp2_(m[t] - mx);
            l[t] *= f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[t][i] *= f;
            m[t] = mx;
        }
        const float ref = (m[t] == neg_inf() ? 0.f : m[t]) - vexp;
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = exp2_(x[i] * factor - ref);
        l[t] += (((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]))) * vinv;
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = pack2(p[2 * i], p[2 * i + 1]);
        return __builtin_bit_cast(bf16x8, r);
    }
};

// A value that is the same in all lanes, as a scalar.
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// Where a stretch of work begins: the unit `pos` lies in item `item`, whose units begin at `before`; all items have `total`.
struct Start {
    int item;
    int64_t pos, before, total, each;
};

// Items 0 .. count - 1 have units(item) units each; workgroup `share` of `shares` takes `each` of them (at least `least`). The first
// workgroup leaves the items' beginnings in before[0 .. count] for the joining launch.
template <int THREADS, class Units>
__device__ __forceinline__ Start start_of(int share, int shares, int count, int64_t times, int64_t least, int64_t *before, Units units)
{
    __shared__ int64_t wave_sum[THREADS / 64], found_before;
    __shared__ int found_item;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Start s;
    if (count <= 64) {                                      // every wave for itself
        const int64_t sum = lane < count ? units(lane) : 0;
        int64_t upto = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t y = __shfl_up(upto, o);
            if (lane >= o) upto += y;
        }
        s.total = uniform(__shfl(upto, 63));
        s.each = (s.total * times + shares - 1) / shares;
        s.each = s.each < least ? least : s.each;
        s.pos = share * s.each;
        const int64_t at = times == 1 || s.total == 0 ? s.pos : s.pos % s.total;
        const uint64_t in = __ballot(at >= upto - sum && at < upto);
        s.item = in ? __ffsll((unsigned long long)in) - 1 : 0;
        s.before = uniform(__shfl(upto - sum, s.item));
        if (share == 0 && tid < count) before[tid] = upto - sum;
        if (share == 0 && tid == 0) before[count] = s.total;
        return s;
    }
    const int each_items = (count + THREADS - 1) / THREADS, i0 = min(tid * each_items, count), i1 = min(i0 + each_items, count);
    int64_t sum = 0;
    for (int i = i0; i < i1; ++i) sum += units(i);
    int64_t upto = sum;                                     // inclusive within the wave
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = __shfl_up(upto, o);
        if (lane >= o) upto += y;
    }
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
    int64_t base = upto - sum, total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) base += wave_sum[w];
        total += wave_sum[w];
    }
    total = uniform(total);
    s.total = total;
    s.each = (total * times + shares - 1) / shares;
    s.each = s.each < least ? least : s.each;
    s.pos = share * s.each;
    const int64_t at = times == 1 || total == 0 ? s.pos : s.pos % total;
    if (at >= base && at < base + sum) {
        int64_t x = base;
        int i = i0;
        for (int64_t n = units(i); at >= x + n; n = units(i)) {
            x += n;
            ++i;
        }
        found_item = i;
        found_before = x;
    }
    if (share == 0) {
        int64_t x = base;
        for (int i = i0; i < i1; ++i) {
            before[i] = x;
            x += units(i);
        }
        if (tid == 0) before[count] = total;
    }
    __syncthreads();
    s.item = __builtin_amdgcn_readfirstlane(found_item);
    s.before = uniform(found_before);
    return s;
}

// Blocks of request b for sp_attend_few_kernel; one for a request that sees nothing, whose rows are still written.
template <int D>
__device__ __forceinline__ int few_blocks(const AttendArgs &a, int b)
{
    const Range g = range_of(a, b);
    if (g.n == 0 || g.n > few_rows_of(D) / a.c.group) return 0;
    const int n = (g.hi + kBlock - 1) / kBlock - g.lo / kBlock;
    return n < 1 ? 1 : n;
}

// Bound by the bytes of the cache: 48 single tokens over contexts of 2048 to 65536 (E4M3, head_dim 64) 143 us, 5.8 TB/s of the 6.3 that a streaming
// read reaches; 32 over 4001 to 12000 (bf16, 128) 159 us, 5.5. With 32 rows the operations on each logit come near it: 8 tokens of 4 heads a kv head
// over 131072, 36 us, 3.7 TB/s. Four waves take every fourth block of 32 tokens of a stretch; a wave holds its rows' statistics and output by itself
// and loads a block ahead, the four meet in LDS at the end. Blocks [k0, k1) of request b and kv head kvh; `slot` of the partial results, or -1 if
// that is all of them.
template <int D, bool E4M3, int MT, bool STREAM>
__device__ __forceinline__ void few_stretch(const AttendArgs &a, int b, int kvh, int k0, int k1, int slot)
{
    constexpr int kSteps = D / 32, kTiles = D / 16;
    __shared__ float merge_o[2][16 * MT][D + 4];       // padded: sixteen rows are written side by side
    __shared__ f32x2 merge_ml[2][16 * MT];
    const int G = a.c.group;
    const Range rg = range_of(a, b);
    const int rows = rg.n * G;
    const int blk_lo = rg.lo / kBlock, blk_hi = (rg.hi + kBlock - 1) / kBlock;
    const int from = blk_lo + k0, to = min(blk_lo + k1, blk_hi);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
    const float scale2 = a.scale * kLog2e;
    bf16x8 q[MT][kSteps];
    int last[MT];                           // row c of tile t sees keys [last - window or 0, last)
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int r = 16 * t + c, token = r / G, head = kvh * G + r % G;
        last[t] = a.causal ? rg.len - rg.n + token + 1 : rg.hi;
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
    const int all_lo = a.causal && a.window > 0 && rg.len - a.window > 0 ? rg.len - a.window : 0;
    const int all_hi = a.causal ? rg.len - rg.n + 1 : rg.hi;

    Rows<D, MT> acc;
    acc.clear();
    const Line line(a, b, kvh, E4M3 ? 1 : 2);
    const uint32_t k_lane = c * line.row_bytes + 16 * g, v_lane = 4 * g * line.row_bytes + c * (D / 16) * (E4M3 ? 1 : 2);
    // The next block's keys are loaded once this one's are in the first product, its values once these are in operand form. Block table entries
    // are requested two blocks ahead.
    Block<D, E4M3, STREAM> kv;
    int blk = from + wave;
    if (blk < to) {
        const int end = blk + (to - 1 - blk) / kWaves * kWaves;         // this wave's last block, loaded again behind it
        const Entry now(a, line, blk);
        Entry soon(a, line, min(blk + kWaves, end));
        const Place here = now.place(a, line);
        kv.load_keys(line, here, k_lane);
        kv.load_values(line, here, v_lane);
        for (;;) {
            const int key0 = blk * kBlock;
            const Entry later(a, line, min(blk + 2 * kWaves, end));
            const bool whole = key0 >= all_lo && key0 + kBlock <= all_hi;
            f32x4 s0[MT], s1[MT];
            {
                bf16x8 kf[2][kSteps];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) kf[t][s] = kv.key(t, s);
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    s0[t] = s1[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) {
                        s0[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[0][s], q[t][s], s0[t], 0, 0, 0);
                        s1[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[1][s], q[t][s], s1[t], 0, 0, 0);
                    }
                }
            }
            const Place there = soon.place(a, line);
            float factor = scale2, vexp = 0.f, vinv = 1.f;
            if (E4M3) {
                const float vs = larger(kv.vs, kLeastScale);
                factor = factor_of(scale2, kv.ks);
                vexp = log2_(vs);
                vinv = __builtin_amdgcn_rcpf(vs);
            }
            kv.load_keys(line, there, k_lane);
            bf16x8 vf[kTiles];
            if (!whole) kv.clear_values(g, key0, rg.lo, rg.hi);
            kv.values(vf);
            kv.load_values(line, there, v_lane);
            soon = later;
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                float x[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[j] = s0[t][j];
                    x[4 + j] = s1[t][j];
                }
                if (!whole)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int key = key0 + 4 * g + (j & 3) + (j >> 2) * 16;
                        if (key >= last[t] || (a.window > 0 && key < last[t] - a.window)) x[j] = neg_inf();
                    }
                const bf16x8 p = acc.weigh(t, x, factor, vexp, vinv);
#pragma unroll
                for (int i = 0; i < kTiles; ++i) acc.o[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i], p, acc.o[t][i], 0, 0, 0);
            }
            if (blk == end) break;
            blk += kWaves;
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
                const float mx = larger(acc.m[t], o[0]);
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
        if (slot >= 0) {
            const int64_t at = (int64_t)slot * a.few_rows + r;
            if (g == 0) a.few_ml[at] = f32x2{acc.m[t], acc.l[t]};
            float *dst = a.few_o + at * D + 4 * g * kTiles;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < kTiles; i += 4)
                    *reinterpret_cast<f32x4 *>(dst + j * kTiles + i) = f32x4{acc.o[t][i][j], acc.o[t][i + 1][j], acc.o[t][i + 2][j], acc.o[t][i + 3][j]};
        } else {
            const float inv = inverse(acc.l[t]);
            const int64_t row = (a.off[b] + r / G) * a.c.n_q_heads + kvh * G + r % G;
            uint32_t *dst = reinterpret_cast<uint32_t *>(a.out + row * D + 4 * g * kTiles);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < kTiles; i += 2) dst[(j * kTiles + i) / 2] = pack2(acc.o[t][i][j] * inv, acc.o[t][i + 1][j] * inv);
            if (a.lse && g == 0) a.lse[row] = lse_of(acc.m[t], acc.l[t]);
        }
    }
}

template <int D, bool E4M3, int MT, bool SHARED, bool STREAM>
__global__ __launch_bounds__(kThreads, D == 128 && MT > 1 ? 1 : 2) void sp_attend_few_kernel(AttendArgs a)
{
    const int kv = a.c.n_kv_heads, share = blockIdx.x;
    int64_t pos = 0, end, begin = 0;        // units of work; `begin` of them before request b
    int b;
    if constexpr (!SHARED) {                // a line each
        b = share / kv;
        const int n = few_blocks<D>(a, b);
        pos = (int64_t)(share % kv) * n;
        end = pos + n;
    } else {
        const Start s = start_of<kThreads>(share, a.few_shares, a.B, 1, a.few_least, a.few_before, [&](int i) { return (int64_t)few_blocks<D>(a, i) * kv; });
        b = s.item;
        begin = s.before;
        pos = s.pos;
        end = min(s.pos + s.each, s.total);
    }
    for (int part = 0; pos < end; ++part) {
        const int n = few_blocks<D>(a, b);
        if (pos >= begin + (int64_t)n * kv) {
            begin += (int64_t)n * kv;
            ++b;
            --part;
            continue;
        }
        const int rel = (int)(pos - begin), kvh = rel / n, k0 = rel % n, k1 = (int)min((int64_t)n, k0 + (end - pos));
        few_stretch<D, E4M3, MT, STREAM>(a, b, kvh, k0, k1, k0 == 0 && k1 == n ? -1 : 2 * share + (part > 0));
        pos += k1 - k0;
        __syncthreads();                    // the merge's LDS is used again
    }
}

// The partial results of a line of work, units [begin, end), `each` to a workgroup: workgroups first_share .. first_share + count - 1. A
// line that begins inside a workgroup's stretch is that workgroup's second partial result.
struct Parts {
    int first_share, count;
    bool second;

    __device__ __forceinline__ Parts(int64_t begin, int64_t end, int64_t each)
    {
        first_share = (int)(begin / each);
        count = (int)((end - 1) / each) - first_share + 1;
        second = begin != first_share * each;
    }

    __device__ __forceinline__ int slot(int s) const { return s == 0 ? 2 * first_share + second : 2 * (first_share + s); }
};

// Joins the partial results of one row, `rows` rows in each. WAVES waves share them out. The outputs are requested before the statistics
// have come, whose weights exp2(m_s - m) they wait for.
template <int D, int WAVES>
__device__ __forceinline__ void join_row(const AttendArgs &a, const f32x2 *ml, const float *po, int rows, int r, const Parts &parts, int64_t row)
{
    __shared__ float part[kWaves][D];
    constexpr int kAhead = WAVES == 1 ? 4 : 8;              // partial results under way
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, part_wave = wave % WAVES, count = parts.count;
    const auto at = [&](int s) { return (int64_t)parts.slot(s) * rows + r; };
    float x[kAhead][D / 64], acc[D / 64] = {}, m = neg_inf(), l = 0.f;
    const auto load = [&](int s) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const float *src = po + at(min(s + WAVES * k, count - 1)) * D + lane;
#pragma unroll
            for (int i = 0; i < D / 64; ++i) x[k][i] = src[64 * i];
        }
    };
    f32x2 mine = ml[at(min(lane, count - 1))];
    load(part_wave);
    if (lane < count) m = mine[0];
    for (int s = lane + 64; s < count; s += 64) m = larger(m, ml[at(s)][0]);
#pragma unroll
    for (int o = 32; o; o >>= 1) m = larger(m, __shfl_xor(m, o));
    for (int s0 = 0; s0 < count; s0 += 64) {
        if (s0 > 0) mine = ml[at(min(s0 + lane, count - 1))];
        const float w = s0 + lane >= count || mine[0] == neg_inf() ? 0.f : exp2_(mine[0] - m);
        if (s0 + lane < count) l += mine[1] * w;
        const int end = min(s0 + 64, count);
        for (int s = s0 + part_wave; s < end; s += WAVES * kAhead) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const float f = s + WAVES * k < end ? __shfl(w, s + WAVES * k - s0 & 63) : 0.f;
#pragma unroll
                for (int i = 0; i < D / 64; ++i) acc[i] += x[k][i] * f;
            }
            if (s + WAVES * kAhead < count) load(s + WAVES * kAhead);
        }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) l += __shfl_xor(l, o);
    const float inv = inverse(l);
    if (WAVES > 1) {
#pragma unroll
        for (int i = 0; i < D / 64; ++i) part[wave][lane + 64 * i] = acc[i];
        __syncthreads();
        if (wave != 0) return;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            acc[i] = part[0][lane + 64 * i];
            for (int w = 1; w < WAVES; ++w) acc[i] += part[w][lane + 64 * i];
        }
    }
#pragma unroll
    for (int i = 0; i < D / 64; ++i) a.out[row * D + lane + 64 * i] = __builtin_bit_cast(uint16_t, (__bf16)(acc[i] * inv));
    if (a.lse && lane == 0) a.lse[row] = lse_of(m, l);
}

// Every row of the kv heads and requests whose line lies in more than one stretch, WAVES waves a row.
template <int D, int WAVES>
__global__ __launch_bounds__(kThreads) void sp_attend_few_join_kernel(AttendArgs a)
{
    const int b = blockIdx.z, kvh = blockIdx.y, r = (blockIdx.x * kWaves + (threadIdx.x >> 6)) / WAVES, G = a.c.group;
    const int64_t before = a.few_before[b], total = a.few_before[a.B];
    const int n = (int)((a.few_before[b + 1] - before) / a.c.n_kv_heads), rows = (int)min((int64_t)few_rows_of(D) + 1, a.off[b + 1] - a.off[b]) * G;
    if (n == 0 || r >= rows) return;
    int64_t each = (total + a.few_shares - 1) / a.few_shares;
    each = each < a.few_least ? a.few_least : each;
    const int64_t begin = before + (int64_t)kvh * n;
    const Parts parts(begin, begin + n, each);
    if (parts.count == 1) return;
    join_row<D, WAVES>(a, a.few_ml, a.few_o, a.few_rows, r, parts, (a.off[b] + r / G) * a.c.n_q_heads + kvh * G + r % G);
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
    int lo, hi;
};

__device__ __forceinline__ bool tile_of(const AttendArgs &a, const ManyList &list, int few_rows, int x, Tile *t)
{
    const int G = a.c.group;
    int lo = 0, hi = list.count ? list.count : a.B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        const int64_t begin = list.count ? list.tile[mid] : a.off[mid] * G / kManyRows + mid;
        if (begin <= x) lo = mid; else hi = mid;
    }
    t->b = list.count ? list.b[lo] : lo;
    t->rg = range_of(a, t->b);
    const int64_t row0 = (x - (list.count ? list.tile[lo] : a.off[lo] * G / kManyRows + lo)) * kManyRows, rows = (int64_t)t->rg.n * G - row0;
    if (t->rg.n <= few_rows / G || rows <= 0) return false;
    t->row0 = (int)row0;
    t->rows = (int)(rows < kManyRows ? rows : kManyRows);
    t->lo = 0;
    t->hi = t->rg.len;
    if (a.causal) {
        const int p0 = t->rg.len - t->rg.n + t->row0 / G, p1 = t->rg.len - t->rg.n + (t->row0 + t->rows - 1) / G;
        t->hi = p1 + 1 > 0 ? p1 + 1 : 0;
        if (a.window > 0 && p0 - a.window + 1 > 0) t->lo = p0 - a.window + 1;
    }
    return true;
}

// Bound by what a SIMD issues: products of 32x32x16 and plain vector operations of two waves overlap by less than half (681 cycles of products and
// 717 of multiply-adds take 998 together), exponentials and products well. the last 2048 of 32768 tokens of 16 heads over 8, E4M3, head_dim 128, take
// 530 to 550 us, 1.0 PFLOP/s (a large matrix product reaches 1.3); a prompt of 8192 of 32 heads over 8, bf16, head_dim 64, where there is twice the
// softmax for a product, 345 us, 0.80. Eight waves of 32 rows share tiles of kKeys keys, which they bring to LDS as bf16: keys as they are, values
// transposed, so that both products take 16-byte operands from LDS. The transposed logits put a row into a lane column; the order of keys in a row of
// transposed values is the one in which a lane holds its probabilities, so these are the second product's operand as they are. Tiles are
// double-buffered, one barrier a tile; the next tile's loads are under way during the products.
template <int D, bool E4M3>
struct Stage {
    static constexpr int kKeys = 8192 / D, kBlocks = kKeys / kBlock;
    static constexpr int ES = E4M3 ? 1 : 2;
    static constexpr int kKeyLoads = E4M3 ? 1 : 2;              // 16-byte loads of a thread
    static constexpr int kKeyLanes = D * ES / 16;               // threads of a key's row
    static constexpr int kValueLanes = D / 4;                   // threads of four keys' values, four elements each
    struct Raw {                                                // what a thread loads of a tile
        u32x4 k[kKeyLoads];
        uint32_t v[4][ES];
        float scale;                                            // thread i < 2 kBlocks: key or value scale of a block
    };
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

    // Where a wave loads from, tile after tile. At a page's end the next table entry is requested, which the next tile's loads look at. Behind
    // the last page it goes back to that page's beginning: what is loaded there is masked.
    struct Cursor {
        int entry;
        uint32_t in, page;                                      // block of the page; place in the block table
    };

    __device__ __forceinline__ static Cursor cursor(const AttendArgs &a, const int32_t *table, uint32_t blk, uint32_t last_page)
    {
        Cursor c;
        c.page = page_of_block(a, blk);
        c.in = blk - c.page * (uint32_t)a.page_blocks;
        if (c.page > last_page) {                               // a tile's end behind the last page
            c.page = last_page;
            c.in = 0;
        }
        c.entry = table[c.page];
        return c;
    }

    // The address of the cursor's block; moves it to the next tile's.
    __device__ __forceinline__ static Moving next(const AttendArgs &a, const Line &l, const uint8_t *pool, uint32_t last_page, Cursor &c)
    {
        const int p = min(max(__builtin_amdgcn_readfirstlane(c.entry), 0), (int)a.c.n_pages - 1);       // never outside the pools
        const Moving at(pool + p * l.page_bytes + (int64_t)((uint64_t)c.in * (kBlock * l.row_bytes)));
        c.in += kBlocks;
        if (c.in >= (uint32_t)a.page_blocks) {
            do {
                c.in -= a.page_blocks;
                ++c.page;
            } while (c.in >= (uint32_t)a.page_blocks);
            if (c.page > last_page) {
                c.page = last_page;
                c.in = 0;
            }
            c.entry = l.table[c.page];
        }
        return at;
    }

    struct Cursors {
        Cursor key[kKeyLoads], value;
        const float *scale;                                     // of thread i < 2 kBlocks: key or value scale of block i % kBlocks
        uint32_t scale_in, scale_page;
    };

    __device__ __forceinline__ static const float *scale_place(const AttendArgs &a, int b, int kvh, const Cursors &c)
    {
        const float *scales = threadIdx.x < kBlocks ? a.k_scale : a.v_scale;
        return scales + ((int64_t)page_entry(a, b, c.scale_page) * a.c.n_kv_heads + kvh) * a.page_blocks + c.scale_in;
    }

    __device__ __forceinline__ Cursors cursors(const AttendArgs &a, const Line &l, int b, int kvh, uint32_t blk, uint32_t last_page) const
    {
        Cursors c;
#pragma unroll
        for (int i = 0; i < kKeyLoads; ++i)
            c.key[i] = cursor(a, l.table, blk + __builtin_amdgcn_readfirstlane((key_row + i * (kManyThreads / kKeyLanes)) / kBlock), last_page);
        c.value = cursor(a, l.table, blk + __builtin_amdgcn_readfirstlane(value_octet >> 2), last_page);
        if (E4M3) {
            const uint32_t mine = blk + threadIdx.x % kBlocks;
            c.scale_page = min(page_of_block(a, mine), last_page);
            c.scale_in = mine - page_of_block(a, mine) * (uint32_t)a.page_blocks;
            c.scale = scale_place(a, b, kvh, c);
        }
        return c;
    }

    // Loads the tile at the cursors and moves them to the next.
    __device__ __forceinline__ void load(const AttendArgs &a, const Line &l, int b, int kvh, uint32_t last_page, Cursors &c, Raw &w) const
    {
        Moving k[kKeyLoads];
#pragma unroll
        for (int i = 0; i < kKeyLoads; ++i) k[i] = next(a, l, l.k, last_page, c.key[i]);
        Moving v = next(a, l, l.v, last_page, c.value);
#pragma unroll
        for (int i = 0; i < kKeyLoads; ++i)
            w.k[i] = k[i].template load<u32x4>(opaque((key_row + i * (kManyThreads / kKeyLanes)) % kBlock * l.row_bytes + key_col * 16));
        const uint32_t lane = opaque(value_key % kBlock * l.row_bytes + value_col * 4 * ES);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (E4M3) w.v[j][0] = v.template load<uint32_t>(lane);
            else {
                const u32x2 x = v.template load<u32x2>(lane);
                w.v[j][0] = x[0];
                w.v[j][1] = x[1];
            }
            v.advance(l.row_bytes);
        }
        if (E4M3 && threadIdx.x < 2 * kBlocks) {
            w.scale = *c.scale;
            c.scale += kBlocks;
            c.scale_in += kBlocks;
            if (c.scale_in >= (uint32_t)a.page_blocks) {
                do {
                    c.scale_in -= a.page_blocks;
                    c.scale_page = min(c.scale_page + 1, last_page);
                } while (c.scale_in >= (uint32_t)a.page_blocks);
                c.scale = scale_place(a, b, kvh, c);
            }
        }
    }

    // 16-byte pieces: piece c of key row r, and octet o of element d's values, where their readers find them without bank conflicts.
    static __device__ __forceinline__ int key_slot(int r, int c) { return r * (D / 8) + (c ^ (D == 128 ? r & 15 : r & 7)); }
    static __device__ __forceinline__ int value_slot(int d, int o) { return d * (kKeys / 8) + (o ^ ((d ^ (d >> 2)) & 7)); }

    // Values of keys outside [lo, hi) become zero; `first` is the tile's first key.
    __device__ __forceinline__ void store(Raw &w, u32x4 *keys, u32x4 *values, float *scales, int first, int lo, int hi) const
    {
        auto &k = w.k;
        auto &v = w.v;
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
                const int key = first + value_key + j;
                if (key < lo || key >= hi)
#pragma unroll
                    for (int i = 0; i < ES; ++i) v[j][i] = 0;
            }
        u32x2 r[4];                                             // element 4 value_col + i of four keys
#pragma unroll
        for (int p = 0; p < 2; ++p)
            if constexpr (E4M3) {
                uint32_t pair[4];
                widen_pairs(v[2 * p][0], v[2 * p + 1][0], pair);
#pragma unroll
                for (int e = 0; e < 4; ++e) r[e][p] = pair[e];
            } else
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    r[2 * i][p] = __builtin_amdgcn_perm(v[2 * p + 1][i], v[2 * p][i], 0x05040100u);
                    r[2 * i + 1][p] = __builtin_amdgcn_perm(v[2 * p + 1][i], v[2 * p][i], 0x07060302u);
                }
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<u32x2 *>(values)[2 * value_slot(4 * value_col + i, value_octet) + value_half] = r[i];
        if (E4M3 && threadIdx.x < 2 * kBlocks) scales[threadIdx.x] = w.scale;
    }
};

// Tiles of keys that a tile of rows sees; one for a tile that sees nothing, whose rows are still written.
template <int D>
__device__ __forceinline__ int many_units(const Tile &t)
{
    constexpr int kKeys = 8192 / D;
    const int n = (t.hi + kKeys - 1) / kKeys - t.lo / kKeys;
    return t.hi <= t.lo || n < 1 ? 1 : n;
}

// Tiles [k0, k1) of the keys that tile t of query rows sees; `slot` of the partial results, or -1 if that is all of them.
template <int D, bool E4M3>
__device__ __forceinline__ void many_stretch(const AttendArgs &a, const Tile &t, int kvh, int k0, int k1, int slot)
{
    using S = Stage<D, E4M3>;
    constexpr int kKeys = S::kKeys, kBlocks = S::kBlocks, kSteps = D / 16, kOut = D / 32;
    constexpr float kSlack = 8.f;
    constexpr int kVectorOnly = 0x406;      // what may cross a scheduling barrier: vector, scalar and transcendental operations
    __shared__ u32x4 keys[2][1024], values[2][1024];            // 16 KB each
    __shared__ float scales[2][2 * kBlocks];
    const int from = (t.lo / kKeys + k0) * kKeys, to = min((t.lo / kKeys + k1) * kKeys, t.hi);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, h = lane >> 5, c = lane & 31;
    const int G = a.c.group, r = 32 * wave + c;                 // this lane's row of the tile
    const int token = (t.row0 + r) / G, head = kvh * G + (t.row0 + r) % G;
    const int64_t row = (a.off[t.b] + token) * a.c.n_q_heads + head;
    int last = t.rg.len;                    // this lane's row sees keys [first, last)
    // keys that every row of this wave sees: [all_lo, all_hi); that some row sees: [any_lo, any_hi)
    int all_lo = 0, all_hi = t.rg.len, any_hi = t.rg.len, any_lo = 0;
    if (a.causal) {
        const int p = t.rg.len - t.rg.n;
        last = p + token + 1;
        all_hi = p + (t.row0 + 32 * wave) / G + 1;
        any_hi = p + (t.row0 + 32 * wave + 31) / G + 1;
        if (a.window > 0) {
            all_lo = any_hi - a.window;
            any_lo = all_hi - a.window;
        }
    }
    const int first = a.causal && a.window > 0 && last > a.window ? last - a.window : 0;
    const uint32_t seen = last > first ? last - first : 0;      // keys of this lane's row
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
        const uint32_t last_page = page_of_block(a, last_blk);
        const int last_tile = (to - from + kKeys - 1) / kKeys - 1;
        typename S::Raw ra, rb;
        const Line line(a, t.b, kvh, S::ES);
        typename S::Cursors cur = st.cursors(a, line, t.b, kvh, (uint32_t)(from / kBlock), last_page);
        st.load(a, line, t.b, kvh, last_page, cur, ra);
        st.load(a, line, t.b, kvh, last_page, cur, rb);
        st.store(ra, keys[0], values[0], scales[0], from, t.lo, t.hi);
        __syncthreads();
        // Tile n is taken from buffer n % 2, while tile n + 1 lies in `ready`, loaded or under way, and tile n + 2 is requested into `fresh`.
        const auto take = [&](int n, int buf, typename S::Raw &ready, typename S::Raw &fresh) {
            const int key0 = from + n * kKeys;
            const bool more = n < last_tile;
            if (n + 2 <= last_tile) st.load(a, line, t.b, kvh, last_page, cur, fresh);
            if (busy && key0 < any_hi && key0 + kKeys > any_lo) {
                const bool whole = key0 >= all_lo && key0 + kKeys <= all_hi;
                // Of the two waves of a SIMD the one in its softmax goes first, then one that stores a tile, then one in the first product, so that
                // products run beside vector operations (four chunks of 512 rows over 8192 tokens at head_dim 64 170 us without, 166 with; a prompt
                // of 8192 at 128 277 and 276). Two blocks at a time: two independent chains of the first product, one look at the reference. Operands
                // are read from LDS a group of products ahead; the scheduling barriers keep the reads (not vector operations) from being moved behind
                // the products (2048 rows after 32K tokens 533 us without, 527 with). At head_dim 64 they gain nothing (341 both on a whole prompt of
                // 8192).
#pragma unroll
                for (int u = 0; u < kBlocks; u += 2) {
                    constexpr int kGroup = 2;                       // steps of the first product read at a time
                    bf16x8 kf[2][kGroup][2];
                    const auto read_keys = [&](int to, int s0) {
#pragma unroll
                        for (int s = 0; s < kGroup; ++s)
#pragma unroll
                            for (int w = 0; w < 2; ++w) kf[to][s][w] = __builtin_bit_cast(bf16x8, keys[buf][S::key_slot(32 * (u + w) + c, 2 * (s0 + s) + h)]);
                        if constexpr (D == 128) __builtin_amdgcn_sched_barrier(kVectorOnly);
                    };
                    f32x16 x[2];
#pragma unroll
                    for (int w = 0; w < 2; ++w)
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[w][e] = 0.f;
                    __builtin_amdgcn_s_setprio(0);
                    read_keys(0, 0);
#pragma unroll
                    for (int s0 = 0; s0 < kSteps; s0 += kGroup) {
                        if (s0 + kGroup < kSteps) read_keys(s0 / kGroup + 1 & 1, s0 + kGroup);
#pragma unroll
                        for (int s = 0; s < kGroup; ++s)
#pragma unroll
                            for (int w = 0; w < 2; ++w) x[w] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s0 / kGroup & 1][s][w], q[s0 + s], x[w], 0, 0, 0);
                        if constexpr (D == 128) __builtin_amdgcn_sched_barrier(kVectorOnly);
                    }
                    __builtin_amdgcn_s_setprio(3);
                    bf16x8 vf[2][kOut];
                    const auto read_values = [&](int to, int part) {        // part: 16 keys
#pragma unroll
                        for (int i = 0; i < kOut; ++i) vf[to][i] = __builtin_bit_cast(bf16x8, values[buf][S::value_slot(32 * i + c, 4 * u + 2 * part + h)]);
                        if constexpr (D == 128) __builtin_amdgcn_sched_barrier(kVectorOnly);
                    };
                    read_values(0, 0);
                    if (!whole) {
                        int at = key0 + 32 * u + 4 * h - first;
                        if constexpr (D == 128) asm volatile("" : "+v"(at));        // no register for each element: they are short
#pragma unroll
                        for (int w = 0; w < 2; ++w)
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                if ((uint32_t)(at + 32 * w + 8 * (e >> 2) + (e & 3)) >= seen) x[w][e] = neg_inf();
                    }
                    float sc[2], vexp[2], vinv[2], top = neg_inf();
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        sc[w] = scale2;
                        vexp[w] = 0.f;
                        vinv[w] = 1.f;
                        // blocks that no row of the tile sees may have any scale: they are masked, and take none
                        if (E4M3 && (whole || (key0 + 32 * (u + w) < t.hi && key0 + 32 * (u + w) + 32 > t.lo))) {
                            const float vs = larger(scales[buf][kBlocks + u + w], kLeastScale);
                            sc[w] = factor_of(scale2, scales[buf][u + w]);
                            vexp[w] = log2_(vs);
                            vinv[w] = __builtin_amdgcn_rcpf(vs);
                        }
                        float y = x[w][0];
#pragma unroll
                        for (int e = 1; e < 16; ++e) y = larger(y, x[w][e]);
                        top = larger(top, y * sc[w]);
                    }
                    if (__any(top > m + kSlack)) {
                        const float mx = larger(m, larger(top, __shfl_xor(top, 32)));
                        const float f = m == neg_inf() ? 0.f : exp2_(m - mx);
                        l *= f;
#pragma unroll
                        for (int i = 0; i < kOut; ++i) o[i] *= f;
                        m = mx;
                    }
                    float sum[2] = {0.f, 0.f};
#pragma unroll
                    for (int part = 0; part < 4; ++part) {
                        const int w = part >> 1, k = part & 1;
                        const float ref = (m == neg_inf() ? 0.f : m) - vexp[w];
                        u32x4 p;
                        if (k == 0) sum[0] = sum[1] = 0.f;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float a0 = exp2_(x[w][8 * k + 2 * e] * sc[w] - ref), a1 = exp2_(x[w][8 * k + 2 * e + 1] * sc[w] - ref);
                            p[e] = pack2(a0, a1);
                            sum[0] += a0;
                            sum[1] += a1;
                        }
                        if (part < 3) read_values(part + 1 & 1, part + 1);
#pragma unroll
                        for (int i = 0; i < kOut; ++i) o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[part & 1][i], __builtin_bit_cast(bf16x8, p), o[i], 0, 0, 0);
                        if constexpr (D == 128) __builtin_amdgcn_sched_barrier(kVectorOnly);
                        if (k == 1) l += (sum[0] + sum[1]) * vinv[w];
                    }
                }
            }
            __builtin_amdgcn_s_setprio(1);
            if (more) st.store(ready, keys[buf ^ 1], values[buf ^ 1], scales[buf ^ 1], key0 + kKeys, t.lo, t.hi);
            __syncthreads();
        };
        for (int n = 0; n <= last_tile; n += 2) {
            take(n, 0, rb, ra);
            if (n < last_tile) take(n + 1, 1, ra, rb);
        }
    }
    l += __shfl_xor(l, 32);
    if (r >= t.rows) return;
    if (slot >= 0) {
        const int64_t at = (int64_t)slot * kManyRows + r;
        if (h == 0) a.many_ml[at] = f32x2{m, l};
#pragma unroll
        for (int i = 0; i < kOut; ++i)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<f32x4 *>(a.many_o + at * D + 32 * i + 2 * e + 4 * h) = f32x4{o[i][e], o[i][e + 1], o[i][e + 2], o[i][e + 3]};
        return;
    }
    const float inv = inverse(l);
#pragma unroll
    for (int i = 0; i < kOut; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<u32x2 *>(a.out + row * D + 32 * i + 2 * e + 4 * h) =
                u32x2{pack2(o[i][e] * inv, o[i][e + 1] * inv), pack2(o[i][e + 2] * inv, o[i][e + 3] * inv)};
    if (a.lse && h == 0) a.lse[row] = lse_of(m, l);
}

template <int D, bool E4M3, bool SHARED>
__global__ __launch_bounds__(kManyThreads) void sp_attend_many_kernel(AttendArgs a, ManyList list)
{
    const int kv = a.c.n_kv_heads;
    Tile t;
    if constexpr (!SHARED) {
        // A line each. Neighbouring workgroups take different kv heads: with eight of them, each die's L2 holds one head's cache. Later
        // tiles of a prompt see more: they go first
        if (tile_of(a, list, few_rows_of(D), a.tiles - 1 - blockIdx.x / kv, &t)) many_stretch<D, E4M3>(a, t, blockIdx.x % kv, 0, many_units<D>(t), -1);
    } else {
        // stretches of one kv head lie on one die, as far as they divide
        const int per_die = a.many_shares / 8, x = blockIdx.x;
        const int share = x < 8 * per_die ? x % 8 * per_die + x / 8 : x;
        const Start s = start_of<kManyThreads>(share, a.many_shares, a.tiles, kv, 1, a.many_before, [&](int j) {
            Tile u;
            return tile_of(a, list, few_rows_of(D), j, &u) ? (int64_t)many_units<D>(u) : 0;
        });
        const int64_t all = s.total, end = min(s.pos + s.each, all * kv);   // units of a kv head; the stretch's end
        int64_t pos = s.pos, begin = s.before;
        int i = s.item, kvh = all > 0 ? (int)(pos / all) : 0;
        for (int part = 0; pos < end; ++part) {
            const int64_t rel = pos - kvh * all;
            if (rel >= all) {                           // the next kv head's first tile
                ++kvh;
                i = 0;
                begin = 0;
                --part;
                continue;
            }
            const int n = tile_of(a, list, few_rows_of(D), i, &t) ? many_units<D>(t) : 0;
            if (rel >= begin + n) {
                begin += n;
                ++i;
                --part;
                continue;
            }
            const int k0 = (int)(rel - begin), k1 = (int)min((int64_t)n, k0 + (end - pos));
            many_stretch<D, E4M3>(a, t, kvh, k0, k1, k0 == 0 && k1 == n ? -1 : 2 * share + (part > 0));
            pos += k1 - k0;
        }
    }
}

constexpr int join_rows(bool many_parts) { return many_parts ? 1 : 2 * kWaves; }      // of a workgroup

// Every row of the tiles whose line lies in more than one stretch: four waves a row where a line has many parts, else a wave for two rows (finding the
// parts takes longer than joining them).
template <int D, bool MANY_PARTS>
__global__ __launch_bounds__(kThreads) void sp_attend_many_join_kernel(AttendArgs a, ManyList list)
{
    constexpr int kRows = MANY_PARTS ? 1 : 2, kBlocksOfTile = kManyRows / join_rows(MANY_PARTS);
    const int x = blockIdx.x / kBlocksOfTile, kvh = blockIdx.y, G = a.c.group;
    const int r0 = blockIdx.x % kBlocksOfTile * join_rows(MANY_PARTS) + (MANY_PARTS ? 0 : (threadIdx.x >> 6) * kRows);
    const int64_t before = a.many_before[x], n = a.many_before[x + 1] - before, total = a.many_before[a.tiles];
    const int64_t each = (total * a.c.n_kv_heads + a.many_shares - 1) / a.many_shares;
    if (n == 0) return;
    const Parts parts(kvh * total + before, kvh * total + before + n, each);
    Tile t;
    if (parts.count == 1 || !tile_of(a, list, few_rows_of(D), x, &t)) return;
    for (int r = r0; r < min(r0 + kRows, t.rows); ++r)
        join_row<D, MANY_PARTS ? kWaves : 1>(a, a.many_ml, a.many_o, kManyRows, r, parts, (a.off[t.b] + (t.row0 + r) / G) * a.c.n_q_heads + kvh * G + (t.row0 + r) % G);
}

// How a call is laid out: which kernels run, and on how many workgroups.
struct Plan {
    int64_t total, most_few;            // query tokens in all; rows of a kv head of the largest request that has few
    bool few, many, stream;             // stream: contexts that no cache holds until the next call
    int32_t few_rows, few_shares, few_least, tiles, many_shares;
    ManyList list;
    size_t few_o, few_before, many_ml, many_o, many_before, bytes;      // where the workspace's parts begin (few_ml at 0)
};

constexpr int64_t kMaxLen = int64_t(1) << 30, kMaxTokens = int64_t(1) << 26;     // key indices and rows fit 32 bits
constexpr int64_t kUnits = 256;         // compute units
constexpr int64_t kStream = int64_t(1) << 28;                   // bytes that the last cache before memory holds
constexpr int64_t kMaxGroups = int64_t(1) << 23;                // a launch's threads fit 32 bits

sp_status make_plan(const sp_cache_desc *d, const int64_t *off, int32_t B, int64_t max_len, Plan *p)
{
    if (sp_status rc = sp::check_cache(d)) return rc;
    int64_t longest;
    if (sp_status rc = sp::check_ragged(off, B, &p->total, &longest)) return rc;
    if (max_len < 0 || max_len > kMaxLen)
        return sp::fail(SP_ERR_INVALID_ARG, "max_len = %lld outside 0..2^30", (long long)max_len);
    if (p->total > kMaxTokens) return sp::fail(SP_ERR_UNSUPPORTED, "%lld query tokens exceed 2^26", (long long)p->total);
    const int64_t G = d->n_q_heads / d->n_kv_heads, kv = d->n_kv_heads, D = d->head_dim;
    int64_t used = 0, requests = 0;     // tiles and requests with many rows
    p->most_few = 0;
    p->few = p->many = false;
    for (int32_t b = 0; b < B; ++b) {
        const int64_t rows = (off[b + 1] - off[b]) * G;
        if (rows > few_rows_of(d->head_dim)) {
            p->many = true;
            if (requests < kManyList) {
                p->list.b[requests] = b;
                p->list.tile[requests] = (int32_t)used;
            }
            ++requests;
            used += sp::ceil_div(rows, kManyRows);
        } else if (rows > 0) {
            p->few = true;
            p->most_few = rows > p->most_few ? rows : p->most_few;
        }
    }
    p->few_rows = p->most_few <= 16 ? 16 : (p->most_few <= 32 ? 32 : 64);
    const int64_t tiles = requests <= kManyList ? used : p->total * G / kManyRows + B;
    if (tiles * kv >= kMaxGroups || B * kv >= kMaxGroups)
        return sp::fail(SP_ERR_UNSUPPORTED, "%lld query rows of %d requests are more than a launch holds", (long long)(p->total * d->n_q_heads), B);
    p->tiles = (int32_t)tiles;
    p->list.count = requests <= kManyList ? (int32_t)requests : 0;

    // Few rows: shared out unless contexts are so short that a line is best taken whole. A block of a line takes 0.2 us (0.3 at head_dim 128), sharing out about
    // five for its second launch, and more with the number of lines. Single tokens over 8 kv heads of 64, whole and shared: 8 contexts of 1000 tokens 8.9 and
    // 10.7 us, of up to 4000 14.3 and 12.9; 64 of 1000 14.5 and 19.3, 200 of up to 4000 48 and 66. Of 128: 8 of 2000 22.7 and 18.3, 128 of up to 4000 77 and 90.
    // At most 128 blocks, since one long line among many short ones would then be what takes the time.
    const int64_t blocks = sp::ceil_div(max_len, kBlock) + 1, lines = B * kv, limit = 48 * 64 / D + lines / 4, whole = limit < 128 ? limit : 128;
    // Workgroups of a compute unit: with as many lines as units what is resident (by registers), so that one reads while another changes lines (32 requests of up to
    // 16000 tokens of E4M3, head_dim 128, 80 us with one, 74 with two); with fewer one less, which leaves fewer parts to join (8 tokens over 131072, head_dim 64,
    // 40.9 us with three, 36.5 with two), but for 64 rows (72 with one, 61 with two).
    const bool fill = lines >= kUnits || p->few_rows == 64;
    const int64_t spread = kUnits * ((D == 64 ? (p->few_rows == 16 ? 4 : p->few_rows == 32 ? 3 : 2) : p->few_rows == 16 ? 2 : 1) - (fill || (D == 128 && p->few_rows > 16) ? 0 : 1));
    // Joining takes longer with more parts of a line, its stretches with fewer: the best size grows with the root of the length (one context of 3000
    // tokens: at least 4 or 16 blocks 11.7 and 13.4 us; of 32768: 4 or 16 blocks 18.2 and 15.1).
    p->stream = 2 * max_len * B * kv * D * (sp::cache_is_e4m3(*d) ? 1 : 2) > kStream;
    p->few_least = 4;
    while (8 * p->few_least * p->few_least < blocks) p->few_least *= 2;
    const auto shares_of = [&](int64_t n, int64_t least) {
        const int64_t most = sp::ceil_div(n * lines, least);
        return (int32_t)(!p->few || n <= whole ? 0 : spread < most ? spread : most);
    };
    p->few_shares = shares_of(blocks, p->few_least);
    // Shorter contexts may be shared out over more workgroups, since their stretches are shorter: most of all at the lengths where few_least doubles. The
    // workspace holds the partial results of any of them.
    int32_t few_most = p->few_shares;
    for (int64_t least = 4; least < p->few_least; least *= 2) {
        const int32_t n = shares_of(8 * least * least, least);
        few_most = n > few_most ? n : few_most;
    }
    // Many rows: where compute units would be left over, unless lines are short. Whole and shared, 8 kv heads: 512 rows of head_dim 64 over 512 tokens (five
    // tiles of keys) 17 and 24 us, 128 rows of head_dim 128 over 500 (nine) 23 and 24, over 1500 51 and 25; but a prompt of 8192 (512 lines) 276 and 365.
    const int64_t spans = sp::ceil_div(max_len, 8192 / D) + 1, most_many = spans * tiles * kv;
    p->many_shares = 0;
    if (p->many && p->list.count && spans > 8 && tiles * kv < kUnits) p->many_shares = (int32_t)(kUnits < most_many ? kUnits : most_many);

    const size_t few = (size_t)2 * few_most * p->few_rows, many = (size_t)2 * p->many_shares * kManyRows;
    p->few_o = sp::align_up(few * sizeof(f32x2), 256);
    p->few_before = p->few_o + sp::align_up(few * D * sizeof(float), 256);
    p->many_ml = p->few_before + (few ? sp::align_up((size_t)(B + 1) * sizeof(int64_t), 256) : 0);
    p->many_o = p->many_ml + sp::align_up(many * sizeof(f32x2), 256);
    p->many_before = p->many_o + sp::align_up(many * D * sizeof(float), 256);
    p->bytes = p->many_before + (many ? sp::align_up((size_t)(tiles + 1) * sizeof(int64_t), 256) : 0);
    return SP_OK;
}

template <int D, bool E4M3, int MT, bool STREAM>
void few_of(const AttendArgs &a, dim3 grid, hipStream_t st)
{
    if (a.few_shares) hipLaunchKernelGGL((sp_attend_few_kernel<D, E4M3, MT, true, STREAM>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((sp_attend_few_kernel<D, E4M3, MT, false, STREAM>), grid, dim3(kThreads), 0, st, a);
}

template <int D, bool E4M3, int MT>
void few(const AttendArgs &a, bool stream, dim3 grid, hipStream_t st)
{
    if constexpr (D == 64 && E4M3)              // keys of 64 bytes: as they stand the only loads that the answer changes
        if (stream) return few_of<D, E4M3, MT, true>(a, grid, st);
    few_of<D, E4M3, MT, false>(a, grid, st);
}

template <int D, bool E4M3>
sp_status run(const AttendArgs &a, const Plan &p, hipStream_t st)
{
    const unsigned kv = (unsigned)a.c.n_kv_heads;
    if (p.few) {
        const dim3 grid(p.few_shares ? (unsigned)p.few_shares : (unsigned)a.B * kv);
        if (p.few_rows == 16) few<D, E4M3, 1>(a, p.stream, grid, st);
        else if (p.few_rows == 32) few<D, E4M3, 2>(a, p.stream, grid, st);
        else if constexpr (few_rows_of(D) > 32) few<D, E4M3, 4>(a, p.stream, grid, st);
        SP_HIP_CHECK(hipGetLastError());
        if (p.few_shares) {
            // four waves a row where a line has many parts
            if (p.few_shares > 8 * a.B * (int64_t)kv)
                hipLaunchKernelGGL((sp_attend_few_join_kernel<D, kWaves>), dim3((unsigned)p.most_few, kv, (unsigned)a.B), dim3(kThreads), 0, st, a);
            else
                hipLaunchKernelGGL((sp_attend_few_join_kernel<D, 1>), dim3((unsigned)sp::ceil_div(p.most_few, kWaves), kv, (unsigned)a.B), dim3(kThreads), 0, st, a);
            SP_HIP_CHECK(hipGetLastError());
        }
    }
    if (p.many) {
        const dim3 grid(p.many_shares ? (unsigned)p.many_shares : (unsigned)p.tiles * kv);
        if (p.many_shares) hipLaunchKernelGGL((sp_attend_many_kernel<D, E4M3, true>), grid, dim3(kManyThreads), 0, st, a, p.list);
        else hipLaunchKernelGGL((sp_attend_many_kernel<D, E4M3, false>), grid, dim3(kManyThreads), 0, st, a, p.list);
        SP_HIP_CHECK(hipGetLastError());
        if (p.many_shares) {
            const bool parts = p.many_shares > 8 * p.tiles * (int64_t)kv;
            const dim3 rows((unsigned)(p.tiles * (kManyRows / join_rows(parts))), kv);
            if (parts) hipLaunchKernelGGL((sp_attend_many_join_kernel<D, true>), rows, dim3(kThreads), 0, st, a, p.list);
            else hipLaunchKernelGGL((sp_attend_many_join_kernel<D, false>), rows, dim3(kThreads), 0, st, a, p.list);
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
    if (sp_status rc = make_plan(desc, offsets_host, B, max_len, &p)) return rc;
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
    if (sp_status rc = make_plan(desc, offsets_host, B, max_len, &p)) return rc;
    if (!(scale > 0.f) || scale > kMostScale) return sp::fail(SP_ERR_INVALID_ARG, "scale = %g must be > 0 and at most 2.3e38", (double)scale);
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
                 k_scale_dev, v_scale_dev, static_cast<uint16_t *>(out_dev), lse_dev, (int32_t)max_len,
                 window < max_len ? (int32_t)window : 0, B, causal, scale};      // a longer window takes no key from a row
    a.page_blocks = (int32_t)(desc->page_tokens / kBlock);
    a.page_shift = -1;
    for (int s = 0; s < 24; ++s)
        if (a.page_blocks == 1 << s) a.page_shift = s;
    a.tiles = p.tiles;
    uint8_t *ws = static_cast<uint8_t *>(ws_dev);
    a.few_shares = p.few_shares;
    a.few_rows = p.few_rows;
    a.few_least = p.few_least;
    a.few_ml = reinterpret_cast<f32x2 *>(ws);
    a.few_o = reinterpret_cast<float *>(ws + p.few_o);
    a.few_before = reinterpret_cast<int64_t *>(ws + p.few_before);
    a.many_shares = p.many_shares;
    a.many_ml = reinterpret_cast<f32x2 *>(ws + p.many_ml);
    a.many_o = reinterpret_cast<float *>(ws + p.many_o);
    a.many_before = reinterpret_cast<int64_t *>(ws + p.many_before);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool e4m3 = sp::cache_is_e4m3(*desc);
    if (desc->head_dim == 64) return e4m3 ? run<64, true>(a, p, st) : run<64, false>(a, p, st);
    return e4m3 ? run<128, true>(a, p, st) : run<128, false>(a, p, st);
}
