// Pieces shared by the kernels that end in INT8 codes with a scale for each row: eight elements at a time, the block's maximum, the codes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lqq_device.h"

namespace lqq {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// 8 FP16 values (one 16-byte load) -> FP32
__device__ __forceinline__ void widen8(const u32x4 x, float (&f)[8])
{
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const uint32_t w = x[d];
        const f16x2 h = __builtin_bit_cast(f16x2, w);
        f[2 * d] = (float)h[0];
        f[2 * d + 1] = (float)h[1];
    }
}

__device__ __forceinline__ float max_abs8(const float (&f)[8], float m)
{
#pragma unroll
    for (int e = 0; e < 8; e += 2) m = fmaxf(fmaxf(m, fabsf(f[e])), fabsf(f[e + 1]));
    return m;
}

// Q = clamp(rint(f / s)) for 8 values.  The FP32 quotient is only needed to decide an integer, so
// the common case multiplies by an approximate reciprocal, in one FMA with 1.5 * 2^23: the sum is
// rounded to an integer, which is its low byte.  The exact product and the correctly rounded
// quotient both lie within 127 * (2^-23 + 2^-24) < 2.3e-5 of the exact quotient (|f / s| <= 127,
// reciprocal within one unit), hence they round to the same integer unless the product is within 3e-5
// of a tie.  Only then (or where a value is not finite) that value is redone with the IEEE division,
// so the result is always that of the division.  A wave of 512 values meets one 3 times in 100, and a small call
// lasts as long as its slowest wave, hence a branch for each of the lane's values: redoing all 8 takes 1.02 to 1.06 of the
// time (8000 calls).  Where most values are ties a loop over the lane's, one selected at a time, takes as long on
// Gaussian values and up to twice as long on these (1311 x 27584 of halves 63 us, all 8 35.7, here 36.8).
__device__ __forceinline__ uint2 round8(const float (&f)[8], float s, float rcp_s)
{
    constexpr float kMagic = 0x1.8p23f;
    uint32_t u[8], ties = 0;  // bit e: value e needs the division
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float t = __builtin_fmaf(f[e], rcp_s, kMagic);
        const float off = __builtin_fmaf(f[e], rcp_s, -(t - kMagic));
        ties |= fabsf(off) <= 0.5f - 3e-5f ? 0u : 1u << e;  // (set for NaN)
        u[e] = __builtin_bit_cast(uint32_t, t);
    }
    // (a branch the compiler must not turn into divisions and selects for everybody)
    if (__builtin_expect_with_probability(ties != 0, 0, 0.999)) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (__builtin_expect_with_probability((ties >> e) & 1, 0, 0.999))
                u[e] = (uint32_t)(int)fminf(fmaxf(__builtin_rintf(f[e] / s), -127.0f), 127.0f);
    }
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)  // the low bytes of four registers
        w[h] = __builtin_amdgcn_perm(u[4 * h + 1], u[4 * h], 0x0c0c0400u) |
               __builtin_amdgcn_perm(u[4 * h + 3], u[4 * h + 2], 0x04000c0cu);
    return uint2{w[0], w[1]};
}

// maximum (of values >= 0) over the block of NWAVES waves; every thread gets the result
template <int CTRL, int ROWS>
__device__ __forceinline__ float lane_shift_or_0(float m)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, m), CTRL, ROWS, 0xf, ROWS == 0xf));
}
template <int NWAVES>
__device__ __forceinline__ float block_max(float m, float *s_part)
{
    m = fmaxf(m, lane_shift_or_0<0x111, 0xf>(m));  // row_shr 1, 2, 4, 8: lane 15 of each row of 16
    m = fmaxf(m, lane_shift_or_0<0x112, 0xf>(m));
    m = fmaxf(m, lane_shift_or_0<0x114, 0xf>(m));
    m = fmaxf(m, lane_shift_or_0<0x118, 0xf>(m));
    m = fmaxf(m, lane_shift_or_0<0x142, 0xa>(m));  // row_bcast 15, 31: lane 63 of the wave
    m = fmaxf(m, lane_shift_or_0<0x143, 0xc>(m));
    if ((threadIdx.x & 63) == 63) s_part[threadIdx.x >> 6] = m;
    __syncthreads();
    float r = s_part[0];
#pragma unroll
    for (int w = 1; w < NWAVES; ++w) r = fmaxf(r, s_part[w]);
    return r;
}

}  // namespace lqq
