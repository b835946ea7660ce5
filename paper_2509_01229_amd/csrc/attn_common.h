// Pieces shared by the attention kernels: element types, the 4-bit cache's page format, reductions over lanes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lqq_common.h"
#include "lqq_device.h"

namespace lqq {

typedef _Float16 f16;
typedef __bf16 bf16;
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
template <class T, int N>
using vec = T __attribute__((ext_vector_type(N)));

// ------------------------------------------------------------------------- the cache's pages
// A page holds P tokens (a power of two, 16 .. 256); for each kv head, one after the other, P * (D + 8) bytes:
//   P * D/2   key codes, token by token; element 2i in the low half of byte i
//   P * D/2   value codes: for every four tokens 16 column groups of D/16 elements; in each the token pairs (0, 1) and
//             (2, 3); in each pair four elements at a time, two bytes for its first token, two for its second
//   4 P       key words:   FP32 scale (its low 12 bits are zero) | zero point (0 .. 15)
//   4 P       value words
// A key row is what one lane of each k block of a 16x16x32 MFMA loads at once, a group of four tokens of a column group is
// what a lane needs of the values: both operands come out of 16-byte loads (D = 128) without a lane taking another's.
__host__ __device__ constexpr int kv4_head_bytes(int P, int D) { return P * (D + 8); }
template <int D>
__device__ __forceinline__ int kv4_key_byte(int j) { return j * (D / 2); }
template <int D>
__device__ __forceinline__ int kv4_value_byte(int P, int j)  // of column group 0; the next one is D/8 bytes on
{
    return P * (D / 2) + (j >> 2) * (2 * D) + ((j >> 1) & 1) * (D / 16) + (j & 1) * 2;
}
template <int D>
__device__ __forceinline__ int kv4_word_byte(int P, int j, bool value) { return P * D + (value ? 4 * P : 0) + 4 * j; }

constexpr uint32_t kScaleMask = 0xFFFFF000u;

inline bool head_dim_ok(int D) { return D == 64 || D == 128; }
inline bool page_ok(int P) { return P >= 16 && P <= 256 && (P & (P - 1)) == 0; }
inline int log2_of(int v) { return 31 - __builtin_clz((unsigned)v); }

// --------------------------------------------------------------------- all-reduce in a row of lanes
// (quad_perm 1032 and 2301, then the mirrors of 8 and 16 lanes: every lane of the row gets the result)
template <int CTRL>
__device__ __forceinline__ float dpp(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int L, class F>
__device__ __forceinline__ float reduce_lanes(float x, F f)
{
    static_assert(L == 8 || L == 16, "");
    x = f(x, dpp<0xB1>(x));
    x = f(x, dpp<0x4E>(x));
    x = f(x, dpp<0x141>(x));
    if constexpr (L == 16) x = f(x, dpp<0x140>(x));
    return x;
}

// ----------------------------------------------------------------------------------- over the lanes of a wave
// lane i: f over lanes 0 .. i (f with 0 has to leave a value as it is)
template <class F>
__device__ __forceinline__ int lanes_up_to(int x, F f)
{
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true));  // row_shr 1, 2, 4, 8
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true));
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true));
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true));
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));  // row_bcast 15, 31
    return f(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
}
__device__ __forceinline__ int sums_up_to(int x) { return lanes_up_to(x, [](int a, int b) { return a + b; }); }

// The largest of three in one instruction: a NaN stays one
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }
// or is left out.  (Not for results of a matrix product: the compiler does not count their wait states into assembly.)
__device__ __forceinline__ float max3_numbers(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float power_of_two(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }  // -126 <= e <= 127

}  // namespace lqq
