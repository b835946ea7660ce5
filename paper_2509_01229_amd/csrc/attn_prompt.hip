// Attention over whole prompts: packed sequences of different lengths, grouped heads, causal or not.
//
//     o_i = sum_j softmax_j(scale * q_i . k_j) v_j,   j < len_k,   causal: j <= i + len_k - len_q
//
// One pass over the keys with a running maximum and sum (FP32).  A block takes 128 queries of one head (a wave 32 of them, held as
// MFMA operands) through the keys, 64 at a time, in LDS; both products on 32x32x16 MFMAs with the keys' side as the first operand
// (S^T = K Q^T, O^T = V^T P^T): a lane's scores are 32 keys of one query, and they are in the order in which the weights enter the
// second product.  The values are read from LDS transposed (ds_read_b64_tr_b16).  Weights are rounded to the type of the values.
//
// Keys are taken from the last to the first: the tiles that the causal mask cuts come first.  What is masked has no
// part in the result, whatever it holds: scores by selection, and values, where a masked one is not finite, by taking
// the tile's values that are not finite out of the product and adding them to the rows that see them.
#include "attn_common.h"

namespace lqq {

struct PromptArgs {
    const void *q, *k, *v;
    long long q_token, q_head, k_token, k_head, v_token, v_head;
    const int *starts_q, *starts_k;
    void *out;
    int n_seqs, total_q, total_k, Hq, group, causal;
    float scale_log2;
};

constexpr int kQueries = 128, kKeys = 64, kPromptWaves = 4;

template <class T>
__device__ __forceinline__ v16f mfma32(vec<T, 8> a, vec<T, 8> b, v16f c)
{
    if constexpr (__is_same(T, f16))
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint2 read_transposed(const void *lds)
{
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                         (__attribute__((address_space(3))) s16x4 *)reinterpret_cast<const s16x4 *>(lds)));
}

// Which halves of a dword are not finite: their sign bits
template <class T>
__device__ __forceinline__ uint32_t not_finite2(uint32_t x)
{
    constexpr uint32_t e = __is_same(T, f16) ? 0x7c007c00u : 0x7f807f80u, one = __is_same(T, f16) ? 0x04000400u : 0x00800080u;
    return ((x & e) + one) & 0x80008000u;
}

template <int D, class T>
__global__ __launch_bounds__(64 * kPromptWaves, 2) void attn_prompt_kernel(const PromptArgs a)
{
    constexpr int CHUNKS = D / 8;  // 16-byte pieces of a row
    __shared__ __attribute__((aligned(16))) u32x4 s_k[kKeys][CHUNKS], s_v[kKeys][CHUNKS];
    __shared__ int s_odd;  // a value of the tile is not finite
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int head = (int)blockIdx.y, hk = head / a.group;

    // the tile's sequence
    int tile = (int)blockIdx.x, seq = 0, q0 = 0, len_q = 0;
    for (; seq < a.n_seqs; ++seq) {
        q0 = min(max(a.starts_q[seq], 0), a.total_q);
        len_q = max(min(a.starts_q[seq + 1], a.total_q) - q0, 0);
        const int tiles = (len_q + kQueries - 1) / kQueries;
        if (tile < tiles) break;
        tile -= tiles;
    }
    if (seq == a.n_seqs) return;
    const int k0 = min(max(a.starts_k[seq], 0), a.total_k), len_k = max(min(a.starts_k[seq + 1], a.total_k) - k0, 0);
    const int first = tile * kQueries, before = len_k - len_q;  // of the block's rows; keys that every row sees, and one more each
    const int row = first + 32 * wave + n;
    const int limit = a.causal ? min(len_k, row + before + 1) : len_k;  // keys that this lane's row sees
    const int until = a.causal ? min(len_k, min(first + kQueries, len_q) + before) : len_k;  // that some row of the block sees
    // keys that all rows of the wave (of the block) see
    const int wave_all = a.causal ? min(len_k, first + 32 * wave + before + 1) : len_k;
    const int wave_any = a.causal ? min(len_k, first + 32 * wave + 32 + before) : len_k;
    const int block_all = a.causal ? min(len_k, first + before + 1) : len_k;

    vec<T, 8> q[D / 16];
    {
        const T *src = static_cast<const T *>(a.q) + (long long)(q0 + min(row, len_q - 1)) * a.q_token + head * a.q_head + 8 * h;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) q[i] = *reinterpret_cast<const vec<T, 8> *>(src + 16 * i);
    }
    v16f o[D / 32] = {};
    float m = -__builtin_inff(), l = 0.0f;

    for (int tile_k = (until + kKeys - 1) / kKeys - 1; tile_k >= 0; --tile_k) {
        const int key = tile_k * kKeys;
        const bool masked = key + kKeys > block_all;
        __syncthreads();
        if (threadIdx.x == 0) s_odd = 0;
        __syncthreads();
        uint32_t odd = 0;
        for (int i = threadIdx.x; i < kKeys * CHUNKS; i += 64 * kPromptWaves) {
            const int j = i / CHUNKS, c = i % CHUNKS;
            u32x4 kk = {}, vv = {};
            if (key + j < len_k) {
                const long long at = k0 + key + j;
                kk = *reinterpret_cast<const u32x4 *>(static_cast<const T *>(a.k) + at * a.k_token + hk * a.k_head + 8 * c);
                vv = *reinterpret_cast<const u32x4 *>(static_cast<const T *>(a.v) + at * a.v_token + hk * a.v_head + 8 * c);
            }
            s_k[j][c ^ (j & (CHUNKS - 1))] = kk;
            s_v[j][c ^ ((j & (CHUNKS / 2 - 1)) << 1)] = vv;
            if (masked)
#pragma unroll
                for (int e = 0; e < 4; ++e) odd |= not_finite2<T>(vv[e]);
        }
        if (odd) s_odd = 1;
        __syncthreads();
        if (key >= wave_any) continue;  // (no row of the wave sees any of them)

        float sc[2][16];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            v16f acc = {};
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const int j = 32 * t + n, c = 2 * i + h;
                acc = mfma32<T>(__builtin_bit_cast(vec<T, 8>, s_k[j][c ^ (j & (CHUNKS - 1))]), q[i], acc);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[t][i] = acc[i] * a.scale_log2;
        }
        if (key + kKeys > wave_all) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int j = key + 32 * t + 8 * (i >> 2) + 4 * h + (i & 3);
                    sc[t][i] = j < limit ? sc[t][i] : -__builtin_inff();
                }
        }
        float top = sc[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) top = fmaxf(top, sc[i >> 4][i & 15]);
        const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, top), __builtin_bit_cast(unsigned, top), false, false);
        top = fmaxf(__builtin_bit_cast(float, (unsigned)both[0]), __builtin_bit_cast(float, (unsigned)both[1]));
        if (__any(top > m)) {
            const float now = fmaxf(m, top), by = now == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= by;
#pragma unroll
            for (int e = 0; e < D / 32; ++e) o[e] *= by;
        }
        const float base = m == -__builtin_inff() ? 0.0f : m;
        vec<T, 8> p[4];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const float x = __builtin_amdgcn_exp2f(sc[i >> 4][i & 15] - base);
            l += x;
            p[i >> 3][i & 7] = (T)x;
        }
        const bool careful = masked && s_odd;
#pragma unroll
        for (int e = 0; e < D / 32; ++e)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                uint2 half[2];
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const int i = lane & 15, j = 16 * u + 8 * w + 4 * h + (i >> 2);
                    const int c = 4 * e + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
                    half[w] = read_transposed(reinterpret_cast<const char *>(&s_v[j][c ^ ((j & (CHUNKS / 2 - 1)) << 1)]) + 8 * (i & 1));
                    if (careful) {
                        const uint32_t bx = not_finite2<T>(half[w].x), by = not_finite2<T>(half[w].y);
                        half[w].x &= ~((bx >> 15) * 0xffffu);
                        half[w].y &= ~((by >> 15) * 0xffffu);
                    }
                }
                o[e] = mfma32<T>(__builtin_bit_cast(vec<T, 8>, u32x4{half[0].x, half[0].y, half[1].x, half[1].y}), p[u], o[e]);
            }
        if (careful) {
            for (int j = 0; j < kKeys; ++j) {
                const bool sees = key + j < limit;
#pragma unroll
                for (int e = 0; e < D / 32; ++e)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int d = 32 * e + 8 * (i >> 2) + 4 * h + (i & 3);
                        const T x = reinterpret_cast<const T *>(&s_v[j][(d >> 3) ^ ((j & (CHUNKS / 2 - 1)) << 1)])[d & 7];
                        const float f = (float)x;
                        if (sees && !(fabsf(f) < __builtin_inff())) o[e][i] += f;
                    }
            }
        }
    }
    const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, l), __builtin_bit_cast(unsigned, l), false, false);
    l = __builtin_bit_cast(float, (unsigned)both[0]) + __builtin_bit_cast(float, (unsigned)both[1]);
    if (row >= len_q) return;
    const float by = l == 0.0f ? 0.0f : 1.0f / l;
    T *dst = static_cast<T *>(a.out) + ((size_t)(q0 + row) * a.Hq + head) * D;
#pragma unroll
    for (int e = 0; e < D / 32; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            vec<T, 4> y;
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] = (T)(o[e][4 * i + r] * by);
            *reinterpret_cast<vec<T, 4> *>(dst + 32 * e + 8 * i + 4 * h) = y;
        }
}

}  // namespace lqq

using namespace lqq;

extern "C" int attn_prompt(int dtype, int n_seqs, int total_q, int total_k, int Hq, int Hkv, int head_dim, const void *q, long long q_token,
                           long long q_head, const void *k, long long k_token, long long k_head, const void *v, long long v_token,
                           long long v_head, const int *starts_q, const int *starts_k, float scale, int causal, void *out, void *hip_stream)
{
    if (dtype != LQ_F16 && dtype != LQ_BF16) return fail(LQ_ERR_INVALID, "dtype must be LQ_F16 or LQ_BF16, got %d", dtype);
    if (!head_dim_ok(head_dim)) return fail(LQ_ERR_INVALID, "head_dim must be 64 or 128, got %d", head_dim);
    if (n_seqs < 0 || n_seqs > (1 << 20) || total_q < 0 || total_q > (1 << 28) || total_k < 0 || Hkv < 1 || Hq < 1 || Hq > 4096 || Hq % Hkv)
        return fail(LQ_ERR_INVALID, "bad shape: %d sequences, %d queries, %d keys, %d heads, %d kv heads (heads a multiple of kv heads, up to 4096)",
                    n_seqs, total_q, total_k, Hq, Hkv);
    if (!(scale > -1e30f && scale < 1e30f)) return fail(LQ_ERR_INVALID, "scale must be finite");
    if (n_seqs == 0 || total_q == 0) return LQ_OK;
    if (!q || !out || !starts_q || !starts_k || (total_k && (!k || !v))) return fail(LQ_ERR_INVALID, "null pointer");
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)out) & 15) return fail(LQ_ERR_ALIGN, "q, k, v and out must be 16-byte aligned");
    if (((uintptr_t)starts_q | (uintptr_t)starts_k) & 3) return fail(LQ_ERR_ALIGN, "starts_q and starts_k must be 4-byte aligned");
    if ((total_q > 1 && q_token % 8) || (Hq > 1 && q_head % 8) || (total_k > 1 && (k_token % 8 || v_token % 8)) || (Hkv > 1 && (k_head % 8 || v_head % 8)))
        return fail(LQ_ERR_ALIGN, "strides must be multiples of 8 elements");
    const PromptArgs a{q, k, v, q_token, q_head, k_token, k_head, v_token, v_head, starts_q, starts_k, out, n_seqs, total_q, total_k, Hq,
                       Hq / Hkv, causal != 0, scale * 1.44269504f};
    const dim3 grid((unsigned)(total_q / kQueries + n_seqs), (unsigned)Hq);
    (void)hipGetLastError();
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * kPromptWaves), 0, static_cast<hipStream_t>(hip_stream), a); };
    if (dtype == LQ_F16)
        head_dim == 128 ? go(attn_prompt_kernel<128, f16>) : go(attn_prompt_kernel<64, f16>);
    else
        head_dim == 128 ? go(attn_prompt_kernel<128, bf16>) : go(attn_prompt_kernel<64, bf16>);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LQ_OK : fail(LQ_ERR_HIP, "attention launch failed: %s", hipGetErrorString(e));
}
