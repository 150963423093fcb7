// sp_mx4_quantise and sp_mx4_matmul: projections of the draft model in microscaled 4-bit elements (the forward pass of Algorithm 1, ForwardWithAttn).
//
//   y[m][n] = sum_b 2^(sa[m][b] + sw[n][b] - 254) sum_{k in group b} a[m][k] w[n][k]
// on the scaled matrix instructions, which take codes and scale bytes as they are stored: no element is ever widened.
#include "sp_mx4.hpp"

namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr int kThreads = 256;
constexpr int kGroup = sp::kMx4Group;

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}

// Four neighbouring lanes have a group, eight elements each.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void sp_mx4_quantise_kernel(const void *x, int64_t octets, int64_t row_octets, int64_t row_stride, uint32_t *codes,
                                                                    uint8_t *scales)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= octets) return;                                // whole groups
    const int64_t row = i / row_octets, at = row * row_stride + (i - row * row_octets) * 8;
    float y[8];
    if constexpr (BF16) {
        const u32x4 w = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(x) + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            y[2 * e] = __uint_as_float(w[e] << 16);
            y[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    } else {
        const f32x4 *src = reinterpret_cast<const f32x4 *>(static_cast<const float *>(x) + at);
        const f32x4 a = src[0], b = src[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            y[e] = a[e];
            y[4 + e] = b[e];
        }
    }
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, sp::mx4_magnitude(y[e]));
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const int b = sp::mx4_scale(top);
    codes[i] = sp::mx4_codes(y, b);
    if ((i & 3) == 0) scales[i >> 2] = (uint8_t)b;
}

struct MatmulArgs {
    const uint8_t *a, *as, *w, *ws;
    void *out;
    int64_t M, N, K, out_stride;
};

template <bool BF16>
__device__ __forceinline__ void store(const MatmulArgs &p, int64_t m, int64_t n, float y)
{
    if constexpr (BF16) static_cast<uint16_t *>(p.out)[m * p.out_stride + n] = __builtin_bit_cast(uint16_t, (__bf16)y);
    else static_cast<float *>(p.out)[m * p.out_stride + n] = y;
}

// A wave for 16 x 16 results.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void sp_mx4_matmul_kernel(MatmulArgs p)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int64_t tiles = (p.N + 15) / 16, x = (int64_t)blockIdx.x * (kThreads / 64) + wave, m0 = x / tiles * 16, n0 = x % tiles * 16;
    if (m0 >= p.M) return;
    const int64_t m = min(m0 + c, p.M - 1), n = min(n0 + c, p.N - 1), groups = p.K / kGroup;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int64_t k0 = 0; k0 < groups; k0 += 4) {
        const int64_t k = k0 + g;
        u32x4 u = {0, 0, 0, 0}, v = {0, 0, 0, 0};
        int su = 127, sv = 127;
        if (k < groups) {
            u = *reinterpret_cast<const u32x4 *>(p.w + (n * groups + k) * 16);
            v = *reinterpret_cast<const u32x4 *>(p.a + (m * groups + k) * 16);
            su = p.ws[n * groups + k];
            sv = p.as[m * groups + k];
        }
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(i32x8{(int)u[0], (int)u[1], (int)u[2], (int)u[3]}, i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3]},
                                                               acc, 4, 4, 0, su, 0, sv);
    }
    if (m0 + c < p.M)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (n0 + 4 * g + j < p.N) store<BF16>(p, m0 + c, n0 + 4 * g + j, acc[j]);
}

bool bad_kind(int32_t dtype) { return dtype != SP_LOGITS_F32 && dtype != SP_LOGITS_BF16; }

}  // namespace

extern "C" sp_status sp_mx4_quantise(const void *x_dev, int32_t dtype, int64_t rows, int64_t K, int64_t row_stride, void *codes_dev, void *scales_dev,
                                     void *hip_stream)
{
    if (bad_kind(dtype)) return sp::fail(SP_ERR_INVALID_ARG, "dtype = %d is neither SP_LOGITS_F32 nor SP_LOGITS_BF16", dtype);
    if (rows < 0 || rows >= (int64_t(1) << 31)) return sp::fail(SP_ERR_INVALID_ARG, "rows = %lld outside 0..2^31-1", (long long)rows);
    if (K < kGroup || K >= (int64_t(1) << 31) || K % kGroup != 0)
        return sp::fail(SP_ERR_INVALID_ARG, "K = %lld is not a positive multiple of %d below 2^31", (long long)K, kGroup);
    if (row_stride < K || row_stride % 8 != 0 || row_stride > (int64_t(1) << 40))
        return sp::fail(SP_ERR_INVALID_ARG, "row_stride = %lld is less than K = %lld, above 2^40 or no multiple of 8", (long long)row_stride, (long long)K);
    if (rows == 0) return SP_OK;
    if (!x_dev || !codes_dev || !scales_dev) return sp::fail(SP_ERR_INVALID_ARG, "x_dev, codes_dev or scales_dev is null");
    if ((uintptr_t)x_dev % 16 != 0 || (uintptr_t)codes_dev % 16 != 0 || (uintptr_t)scales_dev % 4 != 0)
        return sp::fail(SP_ERR_INVALID_ARG, "x_dev and codes_dev must be 16-byte, scales_dev 4-byte aligned");
    const int64_t octets = rows * (K / 8), groups = sp::ceil_div(octets, kThreads);
    if (groups >= (int64_t(1) << 24))
        return sp::fail(SP_ERR_UNSUPPORTED, "%lld rows of %lld elements are more than a launch holds", (long long)rows, (long long)K);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (dtype == SP_LOGITS_BF16)
        hipLaunchKernelGGL((sp_mx4_quantise_kernel<true>), dim3((unsigned)groups), dim3(kThreads), 0, st, x_dev, octets, K / 8, row_stride,
                           static_cast<uint32_t *>(codes_dev), static_cast<uint8_t *>(scales_dev));
    else
        hipLaunchKernelGGL((sp_mx4_quantise_kernel<false>), dim3((unsigned)groups), dim3(kThreads), 0, st, x_dev, octets, K / 8, row_stride,
                           static_cast<uint32_t *>(codes_dev), static_cast<uint8_t *>(scales_dev));
    SP_HIP_CHECK(hipGetLastError());
    return SP_OK;
}

extern "C" sp_status sp_mx4_matmul(const void *a_codes_dev, const void *a_scales_dev, int64_t M, const void *w_codes_dev, const void *w_scales_dev,
                                   int64_t N, int64_t K, void *out_dev, int32_t dtype, int64_t out_stride, void *hip_stream)
{
    const int64_t most = int64_t(1) << 31;
    if (bad_kind(dtype)) return sp::fail(SP_ERR_INVALID_ARG, "dtype = %d is neither SP_LOGITS_F32 nor SP_LOGITS_BF16", dtype);
    if (M < 0 || M >= most || N < 0 || N >= most) return sp::fail(SP_ERR_INVALID_ARG, "M = %lld or N = %lld outside 0..2^31-1", (long long)M, (long long)N);
    if (K < kGroup || K >= most || K % kGroup != 0)
        return sp::fail(SP_ERR_INVALID_ARG, "K = %lld is not a positive multiple of %d below 2^31", (long long)K, kGroup);
    if (out_stride < N || out_stride > (int64_t(1) << 40))
        return sp::fail(SP_ERR_INVALID_ARG, "out_stride = %lld is less than N = %lld or above 2^40", (long long)out_stride, (long long)N);
    if (M == 0 || N == 0) return SP_OK;
    if (!a_codes_dev || !a_scales_dev || !w_codes_dev || !w_scales_dev || !out_dev) return sp::fail(SP_ERR_INVALID_ARG, "a pointer is null");
    if ((uintptr_t)a_codes_dev % 16 != 0 || (uintptr_t)w_codes_dev % 16 != 0 || (uintptr_t)a_scales_dev % 4 != 0 || (uintptr_t)w_scales_dev % 4 != 0)
        return sp::fail(SP_ERR_INVALID_ARG, "codes must be 16-byte, scales 4-byte aligned");
    if ((uintptr_t)out_dev % (dtype == SP_LOGITS_F32 ? 4 : 2) != 0) return sp::fail(SP_ERR_INVALID_ARG, "out_dev is not aligned to its elements");
    const int64_t tiles = sp::ceil_div(M, 16) * sp::ceil_div(N, 16), groups = sp::ceil_div(tiles, kThreads / 64);
    if (groups >= (int64_t(1) << 24)) return sp::fail(SP_ERR_UNSUPPORTED, "%lld x %lld results are more than a launch holds", (long long)M, (long long)N);
    const MatmulArgs p{static_cast<const uint8_t *>(a_codes_dev), static_cast<const uint8_t *>(a_scales_dev), static_cast<const uint8_t *>(w_codes_dev),
                       static_cast<const uint8_t *>(w_scales_dev), out_dev, M, N, K, out_stride};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (dtype == SP_LOGITS_BF16) hipLaunchKernelGGL((sp_mx4_matmul_kernel<true>), dim3((unsigned)groups), dim3(kThreads), 0, st, p);
    else hipLaunchKernelGGL((sp_mx4_matmul_kernel<false>), dim3((unsigned)groups), dim3(kThreads), 0, st, p);
    SP_HIP_CHECK(hipGetLastError());
    return SP_OK;
}
