// The two steps of a decoder layer that end in the INT8 rows that its products read: the residual's addition with the root-mean-square norm,
// and the gated activation between an MLP's (or an expert's) two products.  Rows of x in FP16 or BF16:
//
//     h  = T(x + residual)                        (where there is a residual: what the next layer adds to, rounded to the type)
//     r  = fp32(1 / sqrt(mean(h^2) + eps))        (mean and root in FP64, rounded once)
//     y  = (h * weight) * r                       |     y = gate / (1 + exp(-gate)) * up
//     s  = max |y| / 127   (1 where that is zero),   Q = clamp(rint(y / s), -127, 127)
//
// The norm: squares of 11-bit (8-bit) numbers are exact in FP64 and their sum is right to 2^-50, so whatever the order of the additions r is the
// definition's but for one sum in 2^25 that lies that near a rounding border; everything behind it is single FP32 roundings, which makes the codes
// the definition's, bit for bit.  As r comes last, max |y| is max |h * weight| * r, rounded (a product by a positive number keeps the order): one
// reduction over the block for the sum and the maximum, one barrier.
//
// A block takes a row, which stays in registers between the two passes over it; rows beyond 32768 elements are read twice.  Bound by memory:
// 2 to 4 bytes in and 1 to 5 out an element (4093 rows of 8192 with residual and y in 56 us, 5.4 TB/s; the gate of 2039 rows of 28672 in 56.5, 5.2: the rate
// of a large copy).  Few rows: a launch, a load, a reduction and a store one after the other, 2.5 us for one row of 4096.
#include <algorithm>

#include "act_common.h"
#include "attn_common.h"

namespace lqq {

struct NormArgs {
    const void *x, *residual;
    const float *weight;
    void *h, *y;
    int8_t *q;
    float *scales;
    long long x_row, residual_row;  // elements
    int K;
    float eps;
    double inv_k;
};
struct GateArgs {
    const void *x;
    int8_t *q;
    float *scales;
    long long x_row;
    int K;
};

// A row's scale, from its largest value: 1 for a row of zeros, or of numbers too small for a scale
__device__ __forceinline__ float scale_of(float most)
{
    const float s = most / 127.0f;
    return s > 0.0f ? s : 1.0f;
}

template <class T>
__device__ __forceinline__ void widen(const u32x4 x, float (&f)[8])
{
    const auto v = __builtin_bit_cast(vec<T, 8>, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)v[e];
}
template <class T>
__device__ __forceinline__ u32x4 narrow(const float (&f)[8])
{
    vec<T, 8> v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (T)f[e];
    return __builtin_bit_cast(u32x4, v);
}

// sum over the wave, in lane 63 (the lanes' order is fixed)
template <int CTRL, int ROWS>
__device__ __forceinline__ double lane_shift_or_0(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xf, ROWS == 0xf);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xf, ROWS == 0xf);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double x)
{
    x += lane_shift_or_0<0x111, 0xf>(x);
    x += lane_shift_or_0<0x112, 0xf>(x);
    x += lane_shift_or_0<0x114, 0xf>(x);
    x += lane_shift_or_0<0x118, 0xf>(x);
    x += lane_shift_or_0<0x142, 0xa>(x);
    return x + lane_shift_or_0<0x143, 0xc>(x);
}

// 1 / sqrt(x) in FP64: two steps of Newton's from the approximate instruction
__device__ __forceinline__ double inverse_root(double x)
{
    double r = __builtin_amdgcn_rsq(x);
#pragma unroll
    for (int i = 0; i < 2; ++i) r = __builtin_fma(r * 0.5, __builtin_fma(-x * r, r, 1.0), r);
    return r;
}

// r and max |y| of the row from the threads' sums of squares and maxima of |h * weight|
template <int NWAVES>
__device__ __forceinline__ void norm_of_row(double sum, float &most, float &r, const NormArgs &a)
{
    __shared__ double s_sum[NWAVES];
    __shared__ float s_part[NWAVES];
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 63) s_sum[threadIdx.x >> 6] = sum;
    most = block_max<NWAVES>(most, s_part);  // (with the block's barrier)
    sum = s_sum[0];
#pragma unroll
    for (int w = 1; w < NWAVES; ++w) sum += s_sum[w];
    r = (float)inverse_root(__builtin_fma(sum, a.inv_k, (double)a.eps));
    most *= r;
}

template <class T, bool RESIDUAL>
__device__ __forceinline__ u32x4 stream_of(const NormArgs &a, int m, int piece)
{
    u32x4 x = reinterpret_cast<const u32x4 *>(static_cast<const T *>(a.x) + m * a.x_row)[piece];
    if constexpr (RESIDUAL) {
        const u32x4 b = reinterpret_cast<const u32x4 *>(static_cast<const T *>(a.residual) + m * a.residual_row)[piece];
        float f[8], g[8];
        widen<T>(x, f);
        widen<T>(b, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] += g[e];
        x = narrow<T>(f);
    }
    return x;
}
__device__ __forceinline__ void times_weight(float (&f)[8], const float *weight, int piece)
{
    if (!weight) return;
    const v4f *const w = reinterpret_cast<const v4f *>(weight) + 2 * (size_t)piece;
    const v4f w0 = w[0], w1 = w[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] *= w0[e], f[4 + e] *= w1[e];
}
__device__ __forceinline__ double squares(const float (&f)[8], double sum)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = __builtin_fma((double)f[e], (double)f[e], sum);
    return sum;
}

// Rows of up to ITERS * NT pieces of 8 elements, in registers
template <class T, bool RESIDUAL, int ITERS, int NT>
__global__ __launch_bounds__(NT) void norm_quantize_rows_kernel(const NormArgs a)
{
    const int m = blockIdx.x, n8 = a.K >> 3;
    float f[ITERS][8], most = 0.0f, r;
    double sum = 0.0;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int piece = it * NT + (int)threadIdx.x;
        const bool mine = piece < n8;
        u32x4 x{};
        if (mine) {
            x = stream_of<T, RESIDUAL>(a, m, piece);
            if (RESIDUAL) reinterpret_cast<u32x4 *>(static_cast<T *>(a.h) + (size_t)m * a.K)[piece] = x;
        }
        widen<T>(x, f[it]);
        sum = squares(f[it], sum);
        if (mine) times_weight(f[it], a.weight, piece);
        most = max_abs8(f[it], most);
    }
    norm_of_row<NT / 64>(sum, most, r, a);
    const float s = scale_of(most), rcp_s = __builtin_amdgcn_rcpf(s);
    if (threadIdx.x == 0) a.scales[m] = s;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int piece = it * NT + (int)threadIdx.x;
        if (piece >= n8) break;
#pragma unroll
        for (int e = 0; e < 8; ++e) f[it][e] *= r;
        if (a.y) reinterpret_cast<u32x4 *>(static_cast<T *>(a.y) + (size_t)m * a.K)[piece] = narrow<T>(f[it]);
        reinterpret_cast<uint2 *>(a.q + (size_t)m * a.K)[piece] = round8(f[it], s, rcp_s);
    }
}

// Rows of any length, gone through twice (the second time a thread reads what it has stored itself, where there is a residual)
constexpr int kLongRow = 1024;
template <class T, bool RESIDUAL>
__global__ __launch_bounds__(kLongRow) void norm_quantize_long_kernel(const NormArgs a)
{
    const int m = blockIdx.x, n8 = a.K >> 3;
    float f[8], most = 0.0f, r;
    double sum = 0.0;
    u32x4 *const h = RESIDUAL ? reinterpret_cast<u32x4 *>(static_cast<T *>(a.h) + (size_t)m * a.K) : nullptr;
    for (int piece = threadIdx.x; piece < n8; piece += kLongRow) {
        const u32x4 x = stream_of<T, RESIDUAL>(a, m, piece);
        if (RESIDUAL) h[piece] = x;
        widen<T>(x, f);
        sum = squares(f, sum);
        times_weight(f, a.weight, piece);
        most = max_abs8(f, most);
    }
    norm_of_row<kLongRow / 64>(sum, most, r, a);
    const float s = scale_of(most), rcp_s = __builtin_amdgcn_rcpf(s);
    if (threadIdx.x == 0) a.scales[m] = s;
    for (int piece = threadIdx.x; piece < n8; piece += kLongRow) {
        widen<T>(RESIDUAL ? h[piece] : stream_of<T, false>(a, m, piece), f);
        times_weight(f, a.weight, piece);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= r;
        if (a.y) reinterpret_cast<u32x4 *>(static_cast<T *>(a.y) + (size_t)m * a.K)[piece] = narrow<T>(f);
        reinterpret_cast<uint2 *>(a.q + (size_t)m * a.K)[piece] = round8(f, s, rcp_s);
    }
}

// gate / (1 + exp(-gate)) * up of a piece.  From a gate of -88.7 on exp(-gate) is infinite in FP32, and near it the reciprocal has fewer bits, while up may bring the
// product back among the ordinary numbers.  Gates under -80 take gate * exp(gate) * up instead, which there is the same to 2^-115, with 2^200 on the way: the exponential does not
// vanish (2^-126) unless the result does, nothing overflows (up * 2^-100 is below 2^28), and the result is rounded to a subnormal number once.  (A branch that rows seldom take: 1 us of
// 56 for 2039 rows of 28672.)
constexpr float kFarGate = -80.0f;
template <class T>
__device__ __forceinline__ void gated(const GateArgs &a, int m, int piece, float (&f)[8])
{
    const u32x4 *const row = reinterpret_cast<const u32x4 *>(static_cast<const T *>(a.x) + m * a.x_row);
    float g[8], u[8], least = 0.0f;
    widen<T>(row[piece], g);
    widen<T>(row[(a.K >> 3) + piece], u);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        f[e] = g[e] * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g[e] * -1.44269504f)) * u[e];
        least = fminf(least, g[e]);
    }
    if (__builtin_expect(least < kFarGate, 0)) {
        asm volatile("s_nop 0");  // (kept a branch)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float far = g[e] * __builtin_amdgcn_exp2f(__builtin_fmaf(g[e], 1.44269504f, 200.0f)) * (u[e] * 0x1p-100f) * 0x1p-100f;
            f[e] = g[e] < kFarGate ? far : f[e];
        }
    }
}

template <class T, int ITERS, int NT>
__global__ __launch_bounds__(NT) void swiglu_quantize_rows_kernel(const GateArgs a)
{
    __shared__ float s_part[NT / 64];
    const int m = blockIdx.x, n8 = a.K >> 3;
    float f[ITERS][8], most = 0.0f;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        gated<T>(a, m, min(it * NT + (int)threadIdx.x, n8 - 1), f[it]);  // (the last piece once more: no new maximum)
        most = max_abs8(f[it], most);
    }
    most = block_max<NT / 64>(most, s_part);
    const float s = scale_of(most), rcp_s = __builtin_amdgcn_rcpf(s);
    if (threadIdx.x == 0) a.scales[m] = s;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int piece = it * NT + (int)threadIdx.x;
        if (piece < n8) reinterpret_cast<uint2 *>(a.q + (size_t)m * a.K)[piece] = round8(f[it], s, rcp_s);
    }
}

template <class T>
__global__ __launch_bounds__(kLongRow) void swiglu_quantize_long_kernel(const GateArgs a)
{
    __shared__ float s_part[kLongRow / 64];
    const int m = blockIdx.x, n8 = a.K >> 3;
    float f[8], most = 0.0f;
    for (int piece = threadIdx.x; piece < n8; piece += kLongRow) {
        gated<T>(a, m, piece, f);
        most = max_abs8(f, most);
    }
    most = block_max<kLongRow / 64>(most, s_part);
    const float s = scale_of(most), rcp_s = __builtin_amdgcn_rcpf(s);
    if (threadIdx.x == 0) a.scales[m] = s;
    for (int piece = threadIdx.x; piece < n8; piece += kLongRow) {
        gated<T>(a, m, piece, f);
        reinterpret_cast<uint2 *>(a.q + (size_t)m * a.K)[piece] = round8(f, s, rcp_s);
    }
}

// Threads by the length of a row: the fewest pieces a thread that 512 of them need, and 256 or 1024 where that leaves none idle, or no more than two
// pieces each.  Measured (us, FP16, inputs that change; norm with residual | gate):
//     4096 rows of  1024   256 threads   8.8 |  7.4     512       11.4 | 10.4     1024            19.0 | 17.3
//                   4096   512          22.7 | 15.9     256, two  23.1 | 15.9     1024            27.2 | 21.4     twice read  32.9 |  26.7
//                   8192   512, two     40.6 | 29.3     256, four 43.4 | 30.8     1024            41.2 | 30.1                 55.4 |  41.1
//                  16384   1024, two    85.5 | 60.7     512, four 89.4 | 64.3     1024, four     102.4 | 68.1                105.0 |  82.6
//                  28672   1024, four  160.3 | 109.6                                                                         181.9 | 150.1
//     one row of    4096   512           2.8 |  2.5     256, two   3.1 |  2.6     1024             2.9 |  2.8                  3.2 |   3.0
//                  28672   1024, four    6.5 |  5.5                                                                            6.9 |   7.7
template <class T, bool RESIDUAL>
static void launch_norm(int M, const NormArgs &a, hipStream_t st)
{
    const int n8 = a.K >> 3;
    const auto go = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3((unsigned)M), dim3((unsigned)threads), 0, st, a); };
    if (n8 <= 256) return go(norm_quantize_rows_kernel<T, RESIDUAL, 1, 256>, 256);
    if (n8 <= 512) return go(norm_quantize_rows_kernel<T, RESIDUAL, 1, 512>, 512);
    if (n8 <= 1024) return go(norm_quantize_rows_kernel<T, RESIDUAL, 2, 512>, 512);
    if (n8 <= 2048) return go(norm_quantize_rows_kernel<T, RESIDUAL, 2, 1024>, 1024);
    if (n8 <= 4096) return go(norm_quantize_rows_kernel<T, RESIDUAL, 4, 1024>, 1024);
    go(norm_quantize_long_kernel<T, RESIDUAL>, kLongRow);
}
template <class T>
static void launch_swiglu(int M, const GateArgs &a, hipStream_t st)
{
    const int n8 = a.K >> 3;
    const auto go = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3((unsigned)M), dim3((unsigned)threads), 0, st, a); };
    if (n8 <= 256) return go(swiglu_quantize_rows_kernel<T, 1, 256>, 256);
    if (n8 <= 512) return go(swiglu_quantize_rows_kernel<T, 1, 512>, 512);
    if (n8 <= 1024) return go(swiglu_quantize_rows_kernel<T, 2, 512>, 512);
    if (n8 <= 2048) return go(swiglu_quantize_rows_kernel<T, 2, 1024>, 1024);
    if (n8 <= 4096) return go(swiglu_quantize_rows_kernel<T, 4, 1024>, 1024);
    go(swiglu_quantize_long_kernel<T>, kLongRow);
}

// A launch holds fewer than 2^32 threads, and a row takes up to 1024 of them
constexpr int kRowsPerLaunch = 1 << 21;

}  // namespace lqq

using namespace lqq;

extern "C" int w4a8_norm_quantize(int dtype, int M, int K, const void *x, long long x_row, const void *residual, long long residual_row,
                                  const float *weight, float eps, void *h, void *y, int8_t *X_i8, float *act_scales, void *hip_stream)
{
    if (dtype != LQ_F16 && dtype != LQ_BF16) return fail(LQ_ERR_INVALID, "dtype must be LQ_F16 or LQ_BF16, got %d", dtype);
    if (M < 0 || K <= 0 || K % 8 != 0 || K > (1 << 24)) return fail(LQ_ERR_INVALID, "bad shape M=%d K=%d (need M>=0, K>0, K%%8==0)", M, K);
    if (!(eps > 0.0f && eps < 1e30f)) return fail(LQ_ERR_INVALID, "eps must be positive and finite");
    if (M == 0) return LQ_OK;
    if (!x || !X_i8 || !act_scales) return fail(LQ_ERR_INVALID, "null pointer");
    if (!residual != !h) return fail(LQ_ERR_INVALID, "residual and h go together");
    if (((uintptr_t)x | (uintptr_t)residual | (uintptr_t)weight | (uintptr_t)h | (uintptr_t)y | (uintptr_t)X_i8 | (uintptr_t)act_scales) & 15)
        return fail(LQ_ERR_ALIGN, "device pointers must be 16-byte aligned");
    if (M > 1 && (x_row % 8 || (residual && residual_row % 8))) return fail(LQ_ERR_ALIGN, "strides of rows must be multiples of 8 elements");
    if (M == 1) x_row = residual_row = 0;
    (void)hipGetLastError();
    for (long long m = 0; m < M; m += kRowsPerLaunch) {
        const int rows = (int)std::min<long long>(kRowsPerLaunch, M - m);
        const auto at = [&](const void *p, long long elements) { return p ? static_cast<const char *>(p) + 2 * elements : nullptr; };
        const NormArgs a{at(x, m * x_row), at(residual, m * residual_row), weight, const_cast<char *>(at(h, m * K)), const_cast<char *>(at(y, m * K)),
                         X_i8 + m * K, act_scales + m, x_row, residual_row, K, eps, 1.0 / K};
        const hipStream_t st = static_cast<hipStream_t>(hip_stream);
        if (dtype == LQ_F16)
            residual ? launch_norm<f16, true>(rows, a, st) : launch_norm<f16, false>(rows, a, st);
        else
            residual ? launch_norm<bf16, true>(rows, a, st) : launch_norm<bf16, false>(rows, a, st);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LQ_OK : fail(LQ_ERR_HIP, "norm launch failed: %s", hipGetErrorString(e));
}

extern "C" int w4a8_swiglu_quantize(int dtype, int M, int K, const void *x, long long x_row, int8_t *X_i8, float *act_scales, void *hip_stream)
{
    if (dtype != LQ_F16 && dtype != LQ_BF16) return fail(LQ_ERR_INVALID, "dtype must be LQ_F16 or LQ_BF16, got %d", dtype);
    if (M < 0 || K <= 0 || K % 8 != 0 || K > (1 << 24)) return fail(LQ_ERR_INVALID, "bad shape M=%d K=%d (need M>=0, K>0, K%%8==0)", M, K);
    if (M == 0) return LQ_OK;
    if (!x || !X_i8 || !act_scales) return fail(LQ_ERR_INVALID, "null pointer");
    if (((uintptr_t)x | (uintptr_t)X_i8 | (uintptr_t)act_scales) & 15) return fail(LQ_ERR_ALIGN, "device pointers must be 16-byte aligned");
    if (M > 1 && x_row % 8) return fail(LQ_ERR_ALIGN, "strides of rows must be multiples of 8 elements");
    if (M == 1) x_row = 0;
    (void)hipGetLastError();
    for (long long m = 0; m < M; m += kRowsPerLaunch) {
        const int rows = (int)std::min<long long>(kRowsPerLaunch, M - m);
        const GateArgs a{static_cast<const char *>(x) + 2 * m * x_row, X_i8 + m * K, act_scales + m, x_row, K};
        dtype == LQ_F16 ? launch_swiglu<f16>(rows, a, static_cast<hipStream_t>(hip_stream)) : launch_swiglu<bf16>(rows, a, static_cast<hipStream_t>(hip_stream));
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LQ_OK : fail(LQ_ERR_HIP, "gated activation launch failed: %s", hipGetErrorString(e));
}
