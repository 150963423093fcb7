// sp_attend: attention of ragged queries over a paged cache (paper: Algorithm 1 ForwardWithAttn, a decoder layer's
// attention over the cache that the importance pass reads afterwards).
//
//   out = sum_j p_j v_j,  p_j = exp(x_j - m) / l,  x_j = scale <q, k_j>,  m = max_j x_j,  l = sum_j exp(x_j - m),
//   lse = m + log l,
// in one pass over the keys: a running maximum m and sum l, and the partial output scaled by exp(m_old - m_new) whenever m grows.
//
// One workgroup takes one query row of one head, 256 keys at a time: a thread forms the logit of its key, the workgroup
// joins maximum and sum, and the threads then share out the output's elements.
#include "sp_cache.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

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
};

__device__ __forceinline__ float neg_inf() { return -__builtin_huge_valf(); }
__device__ __forceinline__ float bf16_to_f32(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

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

template <bool E4M3>
__device__ __forceinline__ float element(const uint8_t *pool, int64_t i)
{
    if (E4M3) return __builtin_amdgcn_cvt_f32_fp8((int)pool[i], 0);
    return bf16_to_f32(reinterpret_cast<const uint16_t *>(pool)[i]);
}

// Element offset of token j's row in a pool, and the index of its scale.
__device__ __forceinline__ int64_t row_of(const sp::CacheView &c, int b, int kvh, int64_t j, int64_t *scale_at)
{
    int64_t page = c.table[b * c.table_stride + j / c.page_tokens];
    page = page < 0 ? 0 : (page >= c.n_pages ? c.n_pages - 1 : page);       // never outside the pools
    const int64_t in_page = j % c.page_tokens;
    *scale_at = (page * c.n_kv_heads + kvh) * (c.page_tokens / sp::kCacheBlock) + in_page / sp::kCacheBlock;
    return page * c.page_stride + kvh * c.stride_head + in_page * c.stride_token;
}

template <int D, bool E4M3>
__global__ __launch_bounds__(kThreads) void sp_attend_row_kernel(AttendArgs a)
{
    __shared__ float query[D], prob[kThreads], part[kThreads], red[2][kWaves];
    __shared__ int64_t value_row[kThreads];
    const int64_t row = blockIdx.x;
    const int h = blockIdx.y, kvh = h / a.c.group, tid = threadIdx.x;
    int b = 0;
    for (int lo = 0, hi = a.B; lo < hi;) {              // the request that owns the row: the last with off[b] <= row
        const int mid = (lo + hi) >> 1;
        if (a.off[mid + 1] > row) hi = b = mid; else lo = b = mid + 1;
    }
    const int64_t n = a.off[b + 1] - a.off[b];
    int64_t len = a.lens[b];
    len = len < 0 ? 0 : (len > a.max_len ? a.max_len : len);
    int64_t first = 0, last = len;                      // the keys the row sees
    if (a.causal) {
        const int64_t p = len - n + (row - a.off[b]);
        last = p + 1 < 0 ? 0 : p + 1;
        if (a.window > 0 && p - a.window + 1 > 0) first = p - a.window + 1;
    }
    if (tid < D) query[tid] = bf16_to_f32(a.q[(row * a.c.n_q_heads + h) * D + tid]) * a.scale;
    constexpr int kParts = kThreads / D;                // the threads of one output element
    float m = neg_inf(), l = 0.f, acc = 0.f;
    for (int64_t base = first; base < last; base += kThreads) {
        const int64_t j = base + tid;
        float x = neg_inf();
        __syncthreads();
        if (j < last) {
            int64_t scale_at;
            const int64_t at = row_of(a.c, b, kvh, j, &scale_at);
            x = 0.f;
            for (int e = 0; e < D; ++e) x += query[e] * element<E4M3>(a.k_pool, at + e);
            if (E4M3) x *= a.k_scale[scale_at];
            value_row[tid] = at;
        }
        const float wm = wave_max(x);
        if ((tid & 63) == 0) red[0][tid >> 6] = wm;
        __syncthreads();
        float mx = m;
        for (int w = 0; w < kWaves; ++w) mx = fmaxf(mx, red[0][w]);
        const float p = __expf(x - mx), grow = __expf(m - mx);      // mx is finite: the chunk's first key is seen
        m = mx;
        const float ws = wave_sum(p);
        if ((tid & 63) == 0) red[1][tid >> 6] = ws;
        float vs = 1.f;
        if (E4M3 && j < last) {
            int64_t scale_at;
            row_of(a.c, b, kvh, j, &scale_at);
            vs = a.v_scale[scale_at];
        }
        prob[tid] = p * vs;
        __syncthreads();
        l = l * grow + red[1][0] + red[1][1] + red[1][2] + red[1][3];
        acc *= grow;
        const int count = (int)(last - base < kThreads ? last - base : kThreads);
        for (int i = tid / D; i < count; i += kParts) acc += prob[i] * element<E4M3>(a.v_pool, value_row[i] + tid % D);
    }
    part[tid] = acc;
    __syncthreads();
    if (tid < D) {
        float o = 0.f;
        for (int i = 0; i < kParts; ++i) o += part[i * D + tid];
        o = l > 0.f ? o / l : 0.f;
        const __bf16 r = (__bf16)o;
        a.out[(row * a.c.n_q_heads + h) * D + tid] = __builtin_bit_cast(uint16_t, r);
    }
    if (a.lse && tid == 0) a.lse[row * a.c.n_q_heads + h] = l > 0.f ? m + __logf(l) : neg_inf();
}

}  // namespace

extern "C" sp_status sp_attend_workspace(const sp_cache_desc *desc, const int64_t *offsets_host, int32_t B, int64_t max_len,
                                         size_t *bytes)
{
    if (!bytes) return sp::fail(SP_ERR_INVALID_ARG, "bytes is null");
    if (sp_status rc = sp::check_cache(desc)) return rc;
    int64_t total, longest;
    if (sp_status rc = sp::check_ragged(offsets_host, B, &total, &longest)) return rc;
    if (max_len < 0 || max_len >= (int64_t(1) << 31))
        return sp::fail(SP_ERR_INVALID_ARG, "max_len = %lld outside 0..2^31-1", (long long)max_len);
    *bytes = 0;
    return SP_OK;
}

extern "C" sp_status sp_attend(const sp_cache_desc *desc, const void *q_dev, const int64_t *offsets_host,
                               const int64_t *offsets_dev, int32_t B, const int32_t *lens_dev, int64_t max_len,
                               const int32_t *block_table_dev, int64_t table_stride, const void *k_pool_dev,
                               const void *v_pool_dev, const float *k_scale_dev, const float *v_scale_dev, float scale,
                               int32_t causal, int64_t window, void *out_dev, float *lse_dev, void *ws_dev,
                               size_t ws_bytes, void *hip_stream)
{
    size_t need;
    if (sp_status rc = sp_attend_workspace(desc, offsets_host, B, max_len, &need)) return rc;
    int64_t total, longest;
    if (sp_status rc = sp::check_ragged(offsets_host, B, &total, &longest)) return rc;
    if (!(scale > 0.f) || scale > 3.0e38f) return sp::fail(SP_ERR_INVALID_ARG, "scale must be finite and > 0");
    if (causal != 0 && causal != 1) return sp::fail(SP_ERR_INVALID_ARG, "causal = %d is neither 0 nor 1", causal);
    if (window < 0 || (window > 0 && !causal))
        return sp::fail(SP_ERR_INVALID_ARG, "window = %lld must be 0, or positive with causal = 1", (long long)window);
    if (table_stride < 1 || table_stride > (int64_t(1) << 31))
        return sp::fail(SP_ERR_INVALID_ARG, "table_stride = %lld outside 1..2^31", (long long)table_stride);
    if (max_len > table_stride * desc->page_tokens)
        return sp::fail(SP_ERR_INVALID_ARG, "max_len = %lld exceeds the block table's %lld tokens", (long long)max_len,
                        (long long)(table_stride * desc->page_tokens));
    if (total == 0) return SP_OK;
    if (!q_dev || !out_dev || !offsets_dev || !lens_dev || !block_table_dev)
        return sp::fail(SP_ERR_INVALID_ARG, "only lse_dev, and ws_dev where no workspace is needed, may be null");
    if ((uintptr_t)q_dev % 16 != 0 || (uintptr_t)out_dev % 16 != 0)
        return sp::fail(SP_ERR_INVALID_ARG, "q_dev and out_dev must be 16-byte aligned");
    if (sp_status rc = sp::check_pools(*desc, k_pool_dev, v_pool_dev, k_scale_dev, v_scale_dev)) return rc;
    if (need > 0) {
        if (!ws_dev) return sp::fail(SP_ERR_WORKSPACE, "ws_dev is null (%zu bytes needed)", need);
        if ((uintptr_t)ws_dev % 256 != 0) return sp::fail(SP_ERR_WORKSPACE, "ws_dev is not 256-byte aligned");
        if (ws_bytes < need) return sp::fail(SP_ERR_WORKSPACE, "workspace too small: %zu < %zu", ws_bytes, need);
    }

    AttendArgs a{sp::view_of(*desc, block_table_dev, table_stride), static_cast<const uint16_t *>(q_dev), offsets_dev,
                 lens_dev, static_cast<const uint8_t *>(k_pool_dev), static_cast<const uint8_t *>(v_pool_dev),
                 k_scale_dev, v_scale_dev, static_cast<uint16_t *>(out_dev), lse_dev, max_len, window, B, causal, scale};
    const dim3 grid((unsigned)total, (unsigned)desc->n_q_heads);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool e4m3 = sp::cache_is_e4m3(*desc);
    if (desc->head_dim == 64 && e4m3) hipLaunchKernelGGL((sp_attend_row_kernel<64, true>), grid, dim3(kThreads), 0, st, a);
    else if (desc->head_dim == 64) hipLaunchKernelGGL((sp_attend_row_kernel<64, false>), grid, dim3(kThreads), 0, st, a);
    else if (e4m3) hipLaunchKernelGGL((sp_attend_row_kernel<128, true>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((sp_attend_row_kernel<128, false>), grid, dim3(kThreads), 0, st, a);
    SP_HIP_CHECK(hipGetLastError());
    return SP_OK;
}
