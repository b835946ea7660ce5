// Attention of one or a few new tokens a sequence over the 4-bit cache (page format: attn_common.h, its values: kvcache.hip).
//
//     o = sum_j softmax_j(scale * q . k_j) v_j,   k_j = (code - z) * s of the key, v_j likewise,   j < context - n_new + 1 + i
// for new token i of n_new.  The heads that share a kv head and the new tokens are the rows of one matrix: row = token * group +
// head, 16 of them at a time.
//
// What is read is 17/16 of 4 bits an element, so the arithmetic has to stay small: 3.2 instruction slots of a lane for each code at the
// rate of memory.  Both products run on 16x16x32 MFMAs with the cache as the first operand (S^T = K Q^T, O^T = V^T P^T):
//   - codes become FP16 integers in 9 instructions for 8 (and-or into 1024 + code or 64 + code, subtract 1024 + z or 64 + z: all
//     exact); the scales stay out of the operands, a key's is applied to its scores, a value's to its weights;
//   - the scores come out with 4 keys of one row in a lane, which is the order in which the weights go into the second product, so
//     nothing moves between lanes; the keys of a 16-byte piece of values are those of the lane's scores.
// Weights are rounded to FP16 (2^-11 of each; the sums are FP32), as 2^6 .. 2^14 where they count most, times the value's
// scale over a power of two that is at least the largest one so far.
#include "attn_common.h"

namespace lqq {

typedef f16 f16x2v __attribute__((ext_vector_type(2)));

struct DecodeArgs {
    const void *q;
    long long q_seq, q_token, q_head;
    const uint8_t *cache;
    const int *table, *context;
    void *out;
    int n_new, Hq, Hkv, group, rows, row_tiles, width, pages, lg_page;
    float scale_log2;  // softmax scale / ln 2
};

__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, (f16x2v)(__builtin_bit_cast(f16x2v, a) - __builtin_bit_cast(f16x2v, b)));
}
// 8 nibbles of a dword as 4 pairs of FP16 integers, the zero points taken off: pair r = nibbles r and r + 4.
// even = 0x6400 + z in both halves (1024 + z), odd = 0x5400 + (z << 4) (64 + z)
__device__ __forceinline__ void integers8(uint32_t w, uint32_t even, uint32_t odd, uint32_t (&o)[4])
{
    const uint32_t w8 = w >> 8;
    o[0] = sub_f16x2((w & 0x000f000fu) | 0x64006400u, even);
    o[1] = sub_f16x2((w & 0x00f000f0u) | 0x54005400u, odd);
    o[2] = sub_f16x2((w8 & 0x000f000fu) | 0x64006400u, even);
    o[3] = sub_f16x2((w8 & 0x00f000f0u) | 0x54005400u, odd);
}

// over the four groups of 16 lanes: every lane gets the result of its column
template <class F>
__device__ __forceinline__ float across_groups(float x, F f)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    x = f(__builtin_bit_cast(float, (unsigned)a[0]), __builtin_bit_cast(float, (unsigned)a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    return f(__builtin_bit_cast(float, (unsigned)b[0]), __builtin_bit_cast(float, (unsigned)b[1]));
}

// What a wave loads for 32 keys (two tiles of 16)
template <int D>
struct Loaded {
    uint32_t k[2][D / 32], v[2][D / 32];  // this lane's key (row), this lane's four keys of its column group
    u32x4 kw[2], vw[2];                   // words of the lane's four keys
    uint32_t kz[2];                       // word of the lane's key
    __device__ __forceinline__ void load(const uint8_t *head, int P, int j, int t, int lane)
    {
        const int n = lane & 15, g = lane >> 4;
        typedef uint32_t piece __attribute__((ext_vector_type(D / 32)));
        const piece a = *reinterpret_cast<const piece *>(head + (j + n) * (D / 2) + g * (D / 8));
        const piece b = *reinterpret_cast<const piece *>(head + P * (D / 2) + ((j >> 2) + g) * (2 * D) + n * (D / 8));
#pragma unroll
        for (int i = 0; i < D / 32; ++i) k[t][i] = a[i], v[t][i] = b[i];
        const uint8_t *words = head + P * D + 4 * j;
        kw[t] = *reinterpret_cast<const u32x4 *>(words + 16 * g);
        vw[t] = *reinterpret_cast<const u32x4 *>(words + 4 * P + 16 * g);
        kz[t] = *reinterpret_cast<const uint32_t *>(words + 4 * n);
    }
};

constexpr int kDecodeWaves = 4;
constexpr float kWeightBits = 6.0f;  // a row's largest weight is 2^6 when its maximum is up to date

template <int D, class T>
__global__ __launch_bounds__(64 * kDecodeWaves) void kv4_attention_kernel(const DecodeArgs a)
{
    constexpr int W = D / 16, STEPS = D / 32;  // elements of a column group; MFMAs of a key tile
    __shared__ float s_o[kDecodeWaves][16][D + 4], s_m[kDecodeWaves][16], s_l[kDecodeWaves][16];
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    int item = (int)blockIdx.x;
    const int rt = item % a.row_tiles;
    item /= a.row_tiles;
    const int hk = item % a.Hkv, seq = item / a.Hkv;
    const int P = 1 << a.lg_page;
    const size_t page_bytes = (size_t)a.Hkv * kv4_head_bytes(P, D);
    const uint8_t *const cache = a.cache + (size_t)hk * kv4_head_bytes(P, D);

    int ctx = a.context[seq];
    bool bad = ctx > a.width * P;  // more than the table has pages for
    ctx = min(max(ctx, 0), a.width * P);
    const int row = rt * 16 + n, token = min(row / a.group, a.n_new - 1), head = hk * a.group + row % a.group;
    const bool real = row < a.rows;
    const int limit = real ? ctx - a.n_new + 1 + token : 0;  // keys that this lane's row sees

    // queries: operand order of the keys (see integers8)
    vec<f16, 8> q[STEPS];
    float q_scale = a.scale_log2;
    {
        float f[STEPS][8];
        const T *src = static_cast<const T *>(a.q) + seq * a.q_seq + token * a.q_token + (real ? head : hk * a.group) * a.q_head + g * (D / 4);
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const vec<T, 8> x = *reinterpret_cast<const vec<T, 8> *>(src + 8 * i);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[i][e] = real ? (float)x[e] : 0.0f, most = fmaxf(most, fabsf(f[i][e]));
        }
        if (sizeof(T) == 2 && !__is_same(T, f16)) {
            // BF16: times a power of two that brings the row below 2 (exact down to 2^-14 of its largest element)
            most = across_groups(most, [](float x, float y) { return fmaxf(x, y); });
            const int e = min(max((int)(__builtin_bit_cast(uint32_t, most) >> 23), 27), 227) - 127;
            q_scale *= __builtin_ldexpf(1.0f, e);
#pragma unroll
            for (int i = 0; i < STEPS; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) f[i][j] = __builtin_ldexpf(f[i][j], -e);
        }
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) q[i][2 * r] = (f16)f[i][r], q[i][2 * r + 1] = (f16)f[i][r + 4];
    }

    v4f o[W] = {};
    float m = -__builtin_inff(), l = 0.0f;  // the row's maximum (of scores / ln 2), this lane's part of its sum
    float v_top = 0x1p-126f, v_inv = 0.0f;  // power of two that no value's scale so far is above, and 2^-.. of it
    const int last_page = max((ctx - 1) >> a.lg_page, 0);

    auto fetch = [&](Loaded<D> &x, int key) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int k0 = key + 16 * t;
            int page = a.table[(size_t)seq * a.width + min(k0 >> a.lg_page, last_page)];
            const bool out_of_range = page < 0 || page >= a.pages;
            bad |= out_of_range;
            page = out_of_range ? 0 : page;
            x.load(cache + (size_t)page * page_bytes, P, k0 & (P - 1), t, lane);
        }
    };
    auto step = [&](const Loaded<D> &x, int key) {
        float sc[2][4];  // scores
        float sv[2][4];  // scales of the values
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t z = x.kz[t] & 15u, zz = z | z << 16, even = 0x64006400u | zz, odd = 0x54005400u | zz << 4;
            v4f acc = {};
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                uint32_t k8[4];
                integers8(x.k[t][i], even, odd, k8);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(vec<f16, 8>, u32x4{k8[0], k8[1], k8[2], k8[3]}), q[i], acc, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sc[t][i] = acc[i] * (__builtin_bit_cast(float, x.kw[t][i] & kScaleMask) * q_scale);
                sv[t][i] = __builtin_bit_cast(float, x.vw[t][i] & kScaleMask);
            }
        }
        const bool tail = key + 32 > ctx - a.n_new + 1;  // some row does not see all of these keys
        if (tail) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = key + 16 * t + 4 * g + i;
                    sc[t][i] = j < limit ? sc[t][i] : -__builtin_inff();
                    sv[t][i] = j < ctx ? sv[t][i] : 0.0f;
                }
        }
        float top = sc[0][0], vt = sv[0][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, sc[i >> 2][i & 3]), vt = fmaxf(vt, sv[i >> 2][i & 3]);
        if (__any(top > m + (14.0f - kWeightBits))) {  // (first of all: m is minus infinity)
            top = across_groups(top, [](float u, float w) { return fmaxf(u, w); });
            const float now = fmaxf(m, top), by = now == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= by;
#pragma unroll
            for (int e = 0; e < W; ++e) o[e] *= by;
        }
        if (__any(vt > v_top)) {
            for (int d = 1; d < 64; d <<= 1) vt = fmaxf(vt, __shfl_xor(vt, d));
            // (the next power of two; scales above 2^126 keep it there and reach FP16's largest weights)
            const uint32_t e = min((__builtin_bit_cast(uint32_t, vt) >> 23) + 1u, 253u);
            const float next = __builtin_bit_cast(float, e << 23), by = v_top / next;
#pragma unroll
            for (int i = 0; i < W; ++i) o[i] *= by;
            v_top = next;
            v_inv = 1.0f / next;
        }
        const float base = m == -__builtin_inff() ? 0.0f : m - kWeightBits;
        uint32_t w[4];
        float p[2][4];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[t][i] = __builtin_amdgcn_exp2f(sc[t][i] - base);
                l += p[t][i];
                p[t][i] *= sv[t][i] * v_inv;
                if (tail) p[t][i] = key + 16 * t + 4 * g + i < limit ? p[t][i] : 0.0f;  // (whatever the scale there is)
            }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                w[2 * t + i] = __builtin_bit_cast(uint32_t, f16x2v{(f16)p[t][2 * i], (f16)p[t][2 * i + 1]});
        const auto weights = __builtin_bit_cast(vec<f16, 8>, u32x4{w[0], w[1], w[2], w[3]});
        uint32_t zz[4];  // zero points of the pairs of keys
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) zz[2 * t + i] = (x.vw[t][2 * i] & 15u) | (x.vw[t][2 * i + 1] & 15u) << 16;
#pragma unroll
        for (int h = 0; h < W / 4; ++h) {
            uint32_t v8[4][4];  // [pair][element of the four]
#pragma unroll
            for (int p2 = 0; p2 < 4; ++p2)
                integers8(x.v[p2 >> 1][(p2 & 1) * (W / 4) + h], 0x64006400u | zz[p2], 0x54005400u | zz[p2] << 4, v8[p2]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                o[4 * h + e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                    __builtin_bit_cast(vec<f16, 8>, u32x4{v8[0][e], v8[1][e], v8[2][e], v8[3][e]}), weights, o[4 * h + e], 0, 0, 0);
        }
    };

    Loaded<D> x[2];
    int key = 32 * wave;
    constexpr int STRIDE = 32 * kDecodeWaves;
    if (key < ctx) {
        fetch(x[0], key);
        for (;; key += 2 * STRIDE) {
            const bool more = key + STRIDE < ctx;
            if (more) fetch(x[1], key + STRIDE);
            step(x[0], key);
            if (!more) break;
            const bool more2 = key + 2 * STRIDE < ctx;
            if (more2) fetch(x[0], key + 2 * STRIDE);
            step(x[1], key + STRIDE);
            if (!more2) break;
        }
    }
    l = across_groups(l, [](float u, float w) { return u + w; });
    if (bad) l = __builtin_nanf("");
    // the waves' parts: sums of weights relative to 2^(m - kWeightBits), both over 2^16 so that values near the end of FP32's range stay in it
    if (g == 0) s_m[wave][n] = m, s_l[wave][n] = l * 0x1p-16f;
#pragma unroll
    for (int e = 0; e < W; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) s_o[wave][n][(4 * g + i) * W + e] = o[e][i] * 0x1p-16f * v_top;
    __syncthreads();
    // thread: 8 elements of a row
    constexpr int PIECES = 16 * D / 8;
    for (int i = threadIdx.x; i < PIECES; i += 64 * kDecodeWaves) {
        const int r = i / (D / 8), c = i % (D / 8) * 8, to = rt * 16 + r;
        if (to >= a.rows) continue;
        float most = s_m[0][r];
#pragma unroll
        for (int w = 1; w < kDecodeWaves; ++w) most = fmaxf(most, s_m[w][r]);
        float sum = 0.0f, f[8] = {};
#pragma unroll
        for (int w = 0; w < kDecodeWaves; ++w) {
            const float by = s_m[w][r] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(s_m[w][r] - most);
            sum += s_l[w][r] * by;
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] += s_o[w][r][c + e] * by;
        }
        vec<T, 8> y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (T)(sum == 0.0f ? 0.0f : f[e] / sum);
        T *dst = static_cast<T *>(a.out) + (((size_t)seq * a.n_new + to / a.group) * a.Hq + hk * a.group + to % a.group) * D + c;
        *reinterpret_cast<vec<T, 8> *>(dst) = y;
    }
}

}  // namespace lqq

using namespace lqq;

extern "C" size_t kv4_attention_workspace_size(int n_seqs, int n_new, int Hq, int Hkv, int head_dim)
{
    (void)n_seqs, (void)n_new, (void)Hq, (void)Hkv, (void)head_dim;
    return 0;
}

extern "C" int kv4_attention(int dtype, int n_seqs, int n_new, int Hq, int Hkv, int head_dim, const void *q, long long q_seq,
                             long long q_token, long long q_head, const void *cache, int num_pages, int page_size,
                             const int *block_table, int table_width, const int *context, float scale, void *out, void *workspace,
                             size_t workspace_bytes, void *hip_stream)
{
    if (dtype != LQ_F16 && dtype != LQ_BF16) return fail(LQ_ERR_INVALID, "dtype must be LQ_F16 or LQ_BF16, got %d", dtype);
    if (!head_dim_ok(head_dim)) return fail(LQ_ERR_INVALID, "head_dim must be 64 or 128, got %d", head_dim);
    if (n_seqs < 0 || n_new < 1 || Hkv < 1 || Hq < 1 || Hq > 4096 || Hq % Hkv)
        return fail(LQ_ERR_INVALID, "bad shape: %d sequences, %d new tokens, %d heads, %d kv heads (heads a multiple of kv heads, up to 4096)",
                    n_seqs, n_new, Hq, Hkv);
    if (!page_ok(page_size)) return fail(LQ_ERR_INVALID, "page_size must be a power of two from 16 to 256, got %d", page_size);
    if (num_pages < 1 || num_pages > INT32_MAX / page_size || table_width < 1 || table_width > INT32_MAX / page_size)
        return fail(LQ_ERR_INVALID, "num_pages and table_width times page_size must be from 1 to 2^31 - 1, got %d and %d times %d", num_pages,
                    table_width, page_size);
    if (!(scale > -1e30f && scale < 1e30f)) return fail(LQ_ERR_INVALID, "scale must be finite");
    const long long rows = (long long)n_new * (Hq / Hkv), tiles = (rows + 15) / 16;
    if (rows > (1 << 20) || tiles * Hkv * n_seqs > (1 << 22))
        return fail(LQ_ERR_INVALID, "too many rows: %d sequences, %d new tokens, %d heads", n_seqs, n_new, Hq);
    if (n_seqs == 0) return LQ_OK;
    if (!q || !cache || !block_table || !context || !out) return fail(LQ_ERR_INVALID, "null pointer");
    if (((uintptr_t)q | (uintptr_t)cache | (uintptr_t)out) & 15) return fail(LQ_ERR_ALIGN, "q, cache and out must be 16-byte aligned");
    if (((uintptr_t)block_table | (uintptr_t)context) & 3) return fail(LQ_ERR_ALIGN, "block_table and context must be 4-byte aligned");
    if ((n_seqs > 1 && q_seq % 8) || (n_new > 1 && q_token % 8) || (Hq > 1 && q_head % 8))
        return fail(LQ_ERR_ALIGN, "q: strides must be multiples of 8 elements, got %lld, %lld and %lld", q_seq, q_token, q_head);
    (void)workspace, (void)workspace_bytes;
    const DecodeArgs a{q, q_seq, q_token, q_head, static_cast<const uint8_t *>(cache), block_table, context, out, n_new, Hq, Hkv, Hq / Hkv,
                       (int)rows, (int)tiles, table_width, num_pages, log2_of(page_size), scale * 1.44269504f};
    const dim3 grid((unsigned)(tiles * Hkv * n_seqs));
    (void)hipGetLastError();
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * kDecodeWaves), 0, static_cast<hipStream_t>(hip_stream), a); };
    if (dtype == LQ_F16)
        head_dim == 128 ? go(kv4_attention_kernel<128, f16>) : go(kv4_attention_kernel<64, f16>);
    else
        head_dim == 128 ? go(kv4_attention_kernel<128, bf16>) : go(kv4_attention_kernel<64, bf16>);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LQ_OK : fail(LQ_ERR_HIP, "attention launch failed: %s", hipGetErrorString(e));
}
