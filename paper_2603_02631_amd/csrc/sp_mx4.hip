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
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr int kThreads = 256;
constexpr int kGroup = sp::kMx4Group;

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}

// Four neighbouring lanes have a group, eight elements each. Bound by HBM: 8192 rows of 4096 in bf16, 85 MB read and written, 18 us, 4.7 TB/s, in fp32
// 26 us, 5.8 TB/s (three inputs in turn).
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
    int32_t tiles_m, tiles_n;
    bool wide;              // rows of results can be stored four at a time
};

template <bool BF16>
__device__ __forceinline__ void store(const MatmulArgs &p, int64_t m, int64_t n, float y)
{
    if constexpr (BF16) static_cast<uint16_t *>(p.out)[m * p.out_stride + n] = __builtin_bit_cast(uint16_t, (__bf16)y);
    else static_cast<float *>(p.out)[m * p.out_stride + n] = y;
}

// Results n .. n + 3 of row m.
template <bool BF16>
__device__ __forceinline__ void store4(const MatmulArgs &p, int64_t m, int64_t n, f32x4 y)
{
    if (p.wide && n + 4 <= p.N) {
        if constexpr (BF16)
            *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(p.out) + m * p.out_stride + n) = u32x2{pack2(y[0], y[1]), pack2(y[2], y[3])};
        else *reinterpret_cast<f32x4 *>(static_cast<float *>(p.out) + m * p.out_stride + n) = y;
    } else
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < p.N) store<BF16>(p, m, n + e, y[e]);
}

__device__ __forceinline__ i32x8 operand(u32x4 x) { return i32x8{(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0}; }

// Up to four scale bytes of a row from group k on, as they lie there (at any address). For groups that the row does not have 0: with the other
// operand's, which are 0 too, a factor of 2^-254, under which any codes vanish.
__device__ __forceinline__ uint32_t scales4(const uint8_t *row, int64_t k, int64_t groups)
{
    if (k + 4 <= groups) {
        uint32_t w;
        __builtin_memcpy(&w, row + k, 4);
        return w;
    }
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (k + i < groups) w |= (uint32_t)row[k + i] << (8 * i);
    return w;
}

// ---- few rows: the weights are read once ------------------------------------------------------------------------------

// The scales of a lane for sixteen groups of a row from group k on: of group k + 4 s + g in the lowest byte of word s.
struct Scales16 {
    uint32_t w[4];

    __device__ __forceinline__ void load(const uint8_t *row, int64_t k, int64_t groups, int g)
    {
        if (k + 16 <= groups) __builtin_memcpy(w, row + k, 16);         // at any address
        else
#pragma unroll
            for (int s = 0; s < 4; ++s) w[s] = scales4(row, k + 4 * s, groups);
#pragma unroll
        for (int s = 0; s < 4; ++s) w[s] >>= 8 * g;
    }
};

// Bound by reading the weights: one row by 32000 x 2048 (35 MB) 8 us, by 33000 x 8192 (144 MB) 36 us, 4.0 TB/s, past the caches 9 and 38 (with 64
// neighbouring bytes for a lane, loaded in four pieces, 13 and 55); by launching and one chain of loads where they are few (48 x 4096 x 4096, 9 MB:
// 8.4 us). Sixteen weight rows and 16 MT activation rows a workgroup. Its waves take stretches of 512 elements of the rows in turn, four
// instructions of 128 (of a row a lane has one group in each, so that a load takes 64 neighbouring bytes of sixteen rows), and add up in LDS.
template <bool BF16, int MT>
__global__ __launch_bounds__(kThreads) void sp_mx4_few_kernel(MatmulArgs p)
{
    constexpr int kWaves = kThreads / 64;
    __shared__ f32x4 part[kWaves][MT][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int64_t m0 = (int64_t)(blockIdx.x / p.tiles_n) * 16 * MT, n0 = (int64_t)(blockIdx.x % p.tiles_n) * 16, groups = p.K / kGroup;
    const int64_t n = min(n0 + c, p.N - 1);
    f32x4 acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int64_t k = 16 * wave; k < groups; k += 16 * kWaves) {
        const u32x4 *w = reinterpret_cast<const u32x4 *>(p.w) + n * groups + k + g;
        u32x4 u[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            u[s] = u32x4{0, 0, 0, 0};
            if (k + 4 * s + g < groups) u[s] = w[4 * s];
        }
        Scales16 su;
        su.load(p.ws + n * groups, k, groups, g);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            const int64_t m = min(m0 + 16 * t + c, p.M - 1);
            const u32x4 *a = reinterpret_cast<const u32x4 *>(p.a) + m * groups + k + g;
            u32x4 v[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                v[s] = u32x4{0, 0, 0, 0};
                if (k + 4 * s + g < groups) v[s] = a[4 * s];
            }
            Scales16 sv;
            sv.load(p.as + m * groups, k, groups, g);
#pragma unroll
            for (int s = 0; s < 4; ++s)
                acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(u[s]), operand(v[s]), acc[t], 4, 4, 0, (int)su.w[s], 0, (int)sv.w[s]);
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) part[wave][t][lane] = acc[t];
    __syncthreads();
    for (int t = wave; t < MT; t += kWaves) {
        f32x4 y = part[0][t][lane];
#pragma unroll
        for (int v = 1; v < kWaves; ++v) y += part[v][t][lane];
        const int64_t m = m0 + 16 * t + c;
        if (m < p.M) store4<BF16>(p, m, n0 + 4 * g, y);
    }
}

// ---- many rows: tiles in LDS -------------------------------------------------------------------------------------------

constexpr int kStep = 256;              // elements of a row that a tile takes at a time
constexpr int kRowBytes = kStep / 2, kPieces = kRowBytes / 16, kStepGroups = kStep / kGroup;
constexpr int64_t kMostTiledK = int64_t(1) << 22;       // offsets of a tile's rows fit 32 bits

// 64 lanes x 16 bytes from base + off (each lane its own) straight into LDS from byte `to` on. asm, since the compiler would wait for all of them
// before it reads anything else from LDS; the loop waits itself.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(const uint8_t *base, uint32_t off, uint32_t to)
{
    __asm__ volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(to) : "memory", "m0");
}
#pragma clang diagnostic pop

// WM x WN waves, each with FM x FN blocks of 32 x 32 results: columns are activation rows m, rows weight rows n.
template <bool BF16, int WM, int WN, int FM, int FN>
struct Tiled {
    static constexpr int kThreadsT = 64 * WM * WN, TM = 32 * WM * FM, TN = 32 * WN * FN, kRows = TM + TN;
    static constexpr int kLoads = kRows * kPieces / kThreadsT;
    static_assert(kRows == kThreadsT && TM % (kThreadsT / kPieces) == 0, "a thread has the scales of one row; a load is of activations or of weights");
    static constexpr int kCodes = kRows * kRowBytes, kScales = kRows * kStepGroups;
    static constexpr int kPad = 32 * FN + 4;
    static constexpr int kStaged = WM * WN * 32 * kPad * 4;             // results on their way out
    static constexpr int kLds = 2 * (kCodes + kScales) > kStaged ? 2 * (kCodes + kScales) : kStaged;
};

// The codes that a wave multiplies at a time: groups of 32 elements of its rows, one for each half of the wave.
template <int FM, int FN>
struct Codes {
    u32x4 x[FM], y[FN];

    __device__ __forceinline__ void read(const uint8_t *a, const uint8_t *w, uint32_t lane)
    {
#pragma unroll
        for (int i = 0; i < FM; ++i) x[i] = *reinterpret_cast<const u32x4 *>(a + 32 * i * kRowBytes + lane);
#pragma unroll
        for (int j = 0; j < FN; ++j) y[j] = *reinterpret_cast<const u32x4 *>(w + 32 * j * kRowBytes + lane);
    }

    template <int S>
    __device__ __forceinline__ void multiply(f32x16 (&acc)[FM][FN], const uint32_t (&sa)[FM], const uint32_t (&sw)[FN]) const
    {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int i = 0; i < FM; ++i)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(y[j]), operand(x[i]), acc[i][j], 4, 4, S, (int)sw[j], S, (int)sa[i]);
    }
};

// 8192 x 8192 x 4096 takes 172 to 195 us by the clock that the power leaves (calls behind each other, by events; the first ten after a pause 215 to
// 228, as in a profile), 2.8 to 3.2 PFLOP/s, where the instructions alone run at 6.7 on random data and a large bf16 product reaches 1.3. Copies without loads take 150, without products 136, without results 176: products, operands from LDS
// and tiles to LDS share the time, and the first operands of a step come after a barrier. The next step's loads are requested behind the first
// products, whose issue they would hold up (181 to 174). Not kept: buffers for four steps, steps in another order for each workgroup, 128 x 128
// results a wave (the same or slower); operands requested across the barrier, which takes all registers (168, but 128 x 128 tiles 15.4 to 16.3).
template <bool BF16, int WM, int WN, int FM, int FN>
__global__ __launch_bounds__(64 * WM * WN) void sp_mx4_tiled_kernel(MatmulArgs p)
{
    using T = Tiled<BF16, WM, WN, FM, FN>;
    __shared__ alignas(16) uint8_t lds[T::kLds];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, h = lane >> 5, c = lane & 31;
    // neighbouring tiles on one die: eight rows of tiles at a time
    int x = blockIdx.x;
    const int total = p.tiles_m * p.tiles_n, per = total / 8;
    if (x < 8 * per) x = x % 8 * per + x / 8;
    const int band = 8 * p.tiles_n, first = x / band * 8, deep = min(8, p.tiles_m - first);
    // the quotients come from vector operations: as scalars, so that the addresses made of them are scalars however little is optimised
    const int64_t m0 = (int64_t)__builtin_amdgcn_readfirstlane(first + x % band % deep) * T::TM, n0 = (int64_t)__builtin_amdgcn_readfirstlane(x % band / deep) * T::TN;
    const int64_t row_bytes = p.K / 2, groups = p.K / kGroup;
    const int steps = (int)((p.K + kStep - 1) / kStep), rest = (int)(p.K % kStep);       // elements of the last step, 0: all

    // this thread's pieces: row (of the activations, then of the weights) and place in it, swapped about so that sixteen lanes read sixteen places
    // of 16 bytes
    const int most_m = (int)min(p.M - 1 - m0, (int64_t)T::TM), most_n = (int)min(p.N - 1 - n0, (int64_t)T::TN);
    uint32_t off[T::kLoads];
    const int slot = tid % kPieces, piece = slot ^ (tid / kPieces >> 1 & 7);
#pragma unroll
    for (int i = 0; i < T::kLoads; ++i) {
        const int r = tid / kPieces + i * (T::kThreadsT / kPieces);
        const int row = r < T::TM ? min(r, most_m) : min(r - T::TM, most_n);
        off[i] = __umul24((uint32_t)row, (uint32_t)row_bytes) + 16 * piece;      // fewer than 2^9 rows of less than 2^22 bytes
    }
    const uint8_t *a_base = p.a + m0 * row_bytes, *w_base = p.w + n0 * row_bytes;
    const uint8_t *scale_row = tid < T::TM ? p.as + min(m0 + tid, p.M - 1) * groups : p.ws + min(n0 + tid - T::TM, p.N - 1) * groups;
    const uint32_t lds_at = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t *)lds);
    uint8_t *const scale_lds = lds + 2 * T::kCodes;

    // behind a row's end a thread takes the last step's first piece, whose product with the scales there vanishes
    const uint32_t past = rest != 0 && 32 * piece >= rest ? 16 * piece : 0;
    const auto load_codes = [&](int step, int buf) {
        const uint32_t back = step == steps - 1 ? past : 0;
#pragma unroll
        for (int i = 0; i < T::kLoads; ++i)
            load_to_lds((i * (T::kThreadsT / kPieces) < T::TM ? a_base : w_base) + (int64_t)step * kRowBytes, off[i] - back,
                        lds_at + buf * T::kCodes + i * T::kThreadsT * 16 + wave * 1024);
    };
    const auto load_scales = [&](int step) {
        const int64_t k = (int64_t)step * kStepGroups;
        return u32x2{scales4(scale_row, k, groups), scales4(scale_row, k + 4, groups)};
    };
    const auto put_scales = [&](u32x2 w, int buf) { *reinterpret_cast<u32x2 *>(scale_lds + buf * T::kScales + tid * kStepGroups) = w; };

    f32x16 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    const int wm = wave / WN, wn = wave % WN;
    const int row_a = 32 * FM * wm + c, row_w = T::TM + 32 * FN * wn + c;
    uint32_t at[4];             // a lane's place in its row: half h takes groups 4h .. 4h + 3 of a step, one after another
#pragma unroll
    for (int s = 0; s < 4; ++s) at[s] = 16 * ((4 * h + s) ^ (c >> 1 & 7));

    put_scales(load_scales(0), 0);
    u32x2 scales = load_scales(1);
    load_codes(0, 0);
    __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    for (int step = 0; step < steps; ++step) {
        const int buf = step & 1;
        put_scales(scales, buf ^ 1);                        // of the next step, loaded in the one before
        if (step + 1 < steps) {
            scales = load_scales(step + 2);
        }
        const uint8_t *a = lds + buf * T::kCodes + row_a * kRowBytes, *w = lds + buf * T::kCodes + row_w * kRowBytes;
        uint32_t sa[FM], sw[FN];
#pragma unroll
        for (int i = 0; i < FM; ++i) sa[i] = *reinterpret_cast<const uint32_t *>(scale_lds + buf * T::kScales + (row_a + 32 * i) * kStepGroups + 4 * h);
#pragma unroll
        for (int j = 0; j < FN; ++j) sw[j] = *reinterpret_cast<const uint32_t *>(scale_lds + buf * T::kScales + (row_w + 32 * j) * kStepGroups + 4 * h);
        // codes are read one group of products ahead; the scheduling barriers keep them from being read later, or further ahead, for which there
        // are no registers
        Codes<FM, FN> even, odd;
        even.read(a, w, at[0]);
        odd.read(a, w, at[1]);
        __builtin_amdgcn_sched_barrier(0);
        even.template multiply<0>(acc, sa, sw);
        __builtin_amdgcn_sched_barrier(0);
        if (step + 1 < steps) load_codes(step + 1, buf ^ 1);
        __builtin_amdgcn_sched_barrier(0);
        even.read(a, w, at[2]);
        __builtin_amdgcn_sched_barrier(0);
        odd.template multiply<1>(acc, sa, sw);
        __builtin_amdgcn_sched_barrier(0);
        odd.read(a, w, at[3]);
        __builtin_amdgcn_sched_barrier(0);
        even.template multiply<2>(acc, sa, sw);
        odd.template multiply<3>(acc, sa, sw);
        __builtin_amdgcn_sched_barrier(0);                  // products before the wait
        __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }

    // A wave's results go through LDS, 32 rows at a time, so that rows leave in pieces of 128 bytes and more.
    float *mine = reinterpret_cast<float *>(lds) + wave * 32 * T::kPad;
    constexpr int kLanes = 8 * FN;                          // of a row, four results each
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<f32x4 *>(mine + c * T::kPad + 32 * j + 2 * e + 4 * h) = f32x4{acc[i][j][e], acc[i][j][e + 1], acc[i][j][e + 2], acc[i][j][e + 3]};
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int r = 0; r < 32; r += 64 / kLanes) {
            const int row = r + lane / kLanes, col = 4 * (lane % kLanes);
            const f32x4 y = *reinterpret_cast<const f32x4 *>(mine + row * T::kPad + col);
            const int64_t m = m0 + 32 * (FM * wm + i) + row, n = n0 + 32 * FN * wn + col;
            if (m < p.M && n < p.N) store4<BF16>(p, m, n, y);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <bool BF16, int WM, int WN, int FM, int FN>
sp_status tiled(MatmulArgs p, hipStream_t st)
{
    using T = Tiled<BF16, WM, WN, FM, FN>;
    p.tiles_m = (int32_t)sp::ceil_div(p.M, T::TM);
    p.tiles_n = (int32_t)sp::ceil_div(p.N, T::TN);
    hipLaunchKernelGGL((sp_mx4_tiled_kernel<BF16, WM, WN, FM, FN>), dim3((unsigned)(p.tiles_m * p.tiles_n)), dim3(T::kThreadsT), 0, st, p);
    SP_HIP_CHECK(hipGetLastError());
    return SP_OK;
}

template <bool BF16, int MT>
sp_status few(MatmulArgs p, hipStream_t st)
{
    p.tiles_m = (int32_t)sp::ceil_div(p.M, 16 * MT);
    p.tiles_n = (int32_t)sp::ceil_div(p.N, 16);
    hipLaunchKernelGGL((sp_mx4_few_kernel<BF16, MT>), dim3((unsigned)((int64_t)p.tiles_m * p.tiles_n)), dim3(kThreads), 0, st, p);
    SP_HIP_CHECK(hipGetLastError());
    return SP_OK;
}

template <bool BF16>
sp_status run(const MatmulArgs &p, hipStream_t st)
{
    if (p.M <= 16) return few<BF16, 1>(p, st);
    if (p.M <= 32) return few<BF16, 2>(p, st);
    // Tiles take as long however few they are (0.35 us for 128 elements of K), the workgroups for few rows as long as what they read from L2, by
    // turns (us, few rows' and tiles'): 128 x 4096 x 4096 (32 tiles) 14.0 and 14.6, 700 x 300 x 4000 (18) 7.7 and 14.0; 384 x 2048 x 2048 (48) 10.4
    // and 9.4, 256 x 4096 x 4096 (64) 25 and 15, 632 x 2025 x 224 (80) 11.0 and 6.3. Large tiles need nearly one for each unit (us, of 128 x 128
    // and 256 x 256): 2048 x 4096 x 4096 (128 large ones) 33 and 39, 2560 x 4096 x 4096 (160) 47 and 40, 8192 x 8192 x 4096 235 and 184. Of up to 128 rows
    // half a large tile and more is rows that are not there, and still they are near: 128 x 40960 x 4096 (160) 42 and 39, 48 x 40960 x 4096 33 and
    // 34, 128 x 128256 x 4096 (501) 90 and 93, 48 x 128256 x 4096 79 and 85, but 48 x 65536 x 2048 (256) 16 and 21 (few rows' workgroups 50 to 360).
    if (p.K <= kMostTiledK) {
        if (sp::ceil_div(p.M, 256) * sp::ceil_div(p.N, 256) >= 160) return tiled<BF16, 2, 4, 4, 2>(p, st);
        if (sp::ceil_div(p.M, 128) * sp::ceil_div(p.N, 128) >= 48) return tiled<BF16, 2, 2, 2, 2>(p, st);
    }
    return few<BF16, 4>(p, st);
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
    if ((M / 16 + 1) * (N / 16 + 1) >= (int64_t(1) << 24))
        return sp::fail(SP_ERR_UNSUPPORTED, "%lld x %lld results are more than a launch holds", (long long)M, (long long)N);
    const MatmulArgs p{static_cast<const uint8_t *>(a_codes_dev), static_cast<const uint8_t *>(a_scales_dev), static_cast<const uint8_t *>(w_codes_dev),
                       static_cast<const uint8_t *>(w_scales_dev), out_dev, M, N, K, out_stride, 0, 0,
                       out_stride % 4 == 0 && (uintptr_t)out_dev % (dtype == SP_LOGITS_F32 ? 16 : 8) == 0};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return dtype == SP_LOGITS_BF16 ? run<true>(p, st) : run<false>(p, st);
}
