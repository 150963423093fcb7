// sp_logprobs: log probabilities of given tokens, entropy and the likeliest tokens of rows of logits (paper: Algorithm 1
// ForwardWithAttn, the end of a draft model's forward pass, where the next lookahead token is picked).
//
// With m = max x, s = sum exp(x - m), u = sum (x - m) exp(x - m):
//   lse = m + log s,  lp_t = (x_t - m) - log s,  H = log s - u / s.
//
// One workgroup takes a row: one pass for m, s and u, then one pass for every alternative, which finds the best token
// behind the last one found (larger logit first, lower token first among equals).
#include "sp_common.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

constexpr float kFar = 1e4f;

__device__ __forceinline__ float neg_inf() { return -__builtin_huge_valf(); }

template <bool BF16>
__device__ __forceinline__ float logit(const void *row, int64_t i)
{
    if (BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t *>(row)[i] << 16);
    return static_cast<const float *>(row)[i];
}

// (m, s, u) of two parts of a row. A part without a finite logit is (-inf, 0, 0).
__device__ __forceinline__ void join(float &m, float &s, float &u, float m2, float s2, float u2)
{
    const float mm = fmaxf(m, m2);
    if (mm == neg_inf()) return;
    const float a = m == neg_inf() ? 0.f : __expf(m - mm), b = m2 == neg_inf() ? 0.f : __expf(m2 - mm);
    // what lies more than kFar below the maximum has no weight; the product below must not overflow for it (logits of the type's
    // lowest value)
    const float d = fmaxf(m - mm, -kFar), d2 = fmaxf(m2 - mm, -kFar);
    u = a * (u + d * s) + b * (u2 + d2 * s2);
    s = a * s + b * s2;
    m = mm;
}

// Whether (x, i) comes before (y, j).
__device__ __forceinline__ bool before(float x, int64_t i, float y, int64_t j) { return x > y || (x == y && i < j); }

template <bool BF16>
__global__ __launch_bounds__(kThreads) void sp_logprobs_row_kernel(const void *logits, int64_t vocab, int64_t row_stride,
                                                                   const int32_t *targets, int n_top, float *logprob,
                                                                   float *entropy, int32_t *top_ids, float *top_logprobs)
{
    __shared__ float sm[kWaves], ss[kWaves], su[kWaves];
    __shared__ int64_t si[kWaves];
    const int64_t r = blockIdx.x;
    const int tid = threadIdx.x;
    const void *row = static_cast<const uint8_t *>(logits) + r * row_stride * (BF16 ? 2 : 4);
    float m = neg_inf(), s = 0.f, u = 0.f;
    for (int64_t i = tid; i < vocab; i += kThreads) {
        const float x = logit<BF16>(row, i);
        if (x != neg_inf()) join(m, s, u, x, 1.f, 0.f);
    }
    for (int o = 32; o; o >>= 1) join(m, s, u, __shfl_xor(m, o), __shfl_xor(s, o), __shfl_xor(u, o));
    if ((tid & 63) == 0) {
        sm[tid >> 6] = m;
        ss[tid >> 6] = s;
        su[tid >> 6] = u;
    }
    __syncthreads();
    m = sm[0];
    s = ss[0];
    u = su[0];
    for (int w = 1; w < kWaves; ++w) join(m, s, u, sm[w], ss[w], su[w]);
    const float log_s = s > 0.f ? __logf(s) : 0.f;
    if (tid == 0) {
        if (logprob) {
            const int64_t t = targets[r];
            float lp = 0.f;
            if (t >= 0 && t < vocab) {
                const float x = logit<BF16>(row, t);
                lp = x == neg_inf() ? x : (x - m) - log_s;
            }
            logprob[r] = lp;
        }
        if (entropy) entropy[r] = s > 0.f ? log_s - u / s : 0.f;
    }
    float last = __builtin_huge_valf();
    int64_t last_i = -1;
    for (int k = 0; k < n_top; ++k) {
        float best = neg_inf();
        int64_t best_i = INT64_MAX;
        for (int64_t i = tid; i < vocab; i += kThreads) {
            const float x = logit<BF16>(row, i);
            if (before(last, last_i, x, i) && before(x, i, best, best_i)) {
                best = x;
                best_i = i;
            }
        }
        for (int o = 32; o; o >>= 1) {
            const float y = __shfl_xor(best, o);
            const int64_t j = __shfl_xor(best_i, o);
            if (before(y, j, best, best_i)) {
                best = y;
                best_i = j;
            }
        }
        __syncthreads();
        if ((tid & 63) == 0) {
            sm[tid >> 6] = best;
            si[tid >> 6] = best_i;
        }
        __syncthreads();
        last = sm[0];
        last_i = si[0];
        for (int w = 1; w < kWaves; ++w)
            if (before(sm[w], si[w], last, last_i)) {
                last = sm[w];
                last_i = si[w];
            }
        if (tid == 0) {
            top_ids[r * n_top + k] = (int32_t)last_i;
            top_logprobs[r * n_top + k] = last == neg_inf() ? last : (last - m) - log_s;
        }
    }
}

}  // namespace

extern "C" sp_status sp_logprobs_workspace(int64_t n_rows, int64_t vocab, int32_t n_top, size_t *bytes)
{
    if (!bytes) return sp::fail(SP_ERR_INVALID_ARG, "bytes is null");
    if (n_rows < 0 || n_rows >= (int64_t(1) << 31))
        return sp::fail(SP_ERR_INVALID_ARG, "n_rows = %lld outside 0..2^31-1", (long long)n_rows);
    if (vocab < 1 || vocab >= (int64_t(1) << 31))
        return sp::fail(SP_ERR_INVALID_ARG, "vocab = %lld outside 1..2^31-1", (long long)vocab);
    if (n_top < 0 || n_top > SP_LOGPROBS_MAX_TOP || n_top > vocab)
        return sp::fail(SP_ERR_INVALID_ARG, "n_top = %d outside 0..min(%d, vocab)", n_top, SP_LOGPROBS_MAX_TOP);
    *bytes = 0;
    return SP_OK;
}

extern "C" sp_status sp_logprobs(const void *logits_dev, int32_t dtype, int64_t n_rows, int64_t vocab, int64_t row_stride,
                                 const int32_t *targets_dev, int32_t n_top, float *logprob_dev, float *entropy_dev,
                                 int32_t *top_ids_dev, float *top_logprobs_dev, void *ws_dev, size_t ws_bytes,
                                 void *hip_stream)
{
    size_t need;
    if (sp_status rc = sp_logprobs_workspace(n_rows, vocab, n_top, &need)) return rc;
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
    if (need > 0) {
        if (!ws_dev) return sp::fail(SP_ERR_WORKSPACE, "ws_dev is null (%zu bytes needed)", need);
        if ((uintptr_t)ws_dev % 256 != 0) return sp::fail(SP_ERR_WORKSPACE, "ws_dev is not 256-byte aligned");
        if (ws_bytes < need) return sp::fail(SP_ERR_WORKSPACE, "workspace too small: %zu < %zu", ws_bytes, need);
    }
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const dim3 grid((unsigned)n_rows);
    if (dtype == SP_LOGITS_BF16)
        hipLaunchKernelGGL((sp_logprobs_row_kernel<true>), grid, dim3(kThreads), 0, st, logits_dev, vocab, row_stride,
                           targets_dev, (int)n_top, logprob_dev, entropy_dev, top_ids_dev, top_logprobs_dev);
    else
        hipLaunchKernelGGL((sp_logprobs_row_kernel<false>), grid, dim3(kThreads), 0, st, logits_dev, vocab, row_stride,
                           targets_dev, (int)n_top, logprob_dev, entropy_dev, top_ids_dev, top_logprobs_dev);
    SP_HIP_CHECK(hipGetLastError());
    return SP_OK;
}
