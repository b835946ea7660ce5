// Between the qkv projection and the attention: the norms of queries and keys for each head and the rotary positions in one
// pass, the 4-bit cache as it is written, both in one launch for a decode step, and the cache read back.
//
// Norm and rotation of a head's vector x of D elements at a position p (all in FP32, one rounding at the end):
//     y  = x * rsqrt(mean(x^2) + eps) * w                     (where there is a weight w)
//     y'_a = y_a cos_i - y_b sin_i,   y'_b = y_b cos_i + y_a sin_i,   i < R/2, cos_i = table[p][i], sin_i = table[p][R/2 + i]
// for the pairs (a, b) = (i, i + R/2) or, interleaved, (2i, 2i + 1); elements from R on only take part in the norm.  Products
// and sums are rounded one by one (no fused multiply-add), so that the rotation without a norm is determined bit for bit.
//
// 4-bit form of a vector x (a token's keys or values of one head):
//     lo = min(0, x), hi = max(0, x)
//     s = (hi - lo) / 15 rounded to 12 significant bits (ties to even), at least 2^-100;  z = rint(-lo / s)
//     code = clamp(rint(x / s) + z, 0, 15),   value = (code - z) * s
// A quotient of an 11-bit x (FP16; 8 bits in BF16) and a 12-bit s is a tie, or at least 2^-13 away from one: with x = a 2^i, s = b 2^j,
// 2^11 <= b < 2^12, the distance of x / s from n + 1/2 is |a 2^(i-j+1) - (2n+1) b| / 2b, an integer over 2b (for i - j + 1 < 0
// the quotient is below 1/4).  So the product with an approximate reciprocal, first rounded to a multiple of 2^-14, rounds as
// the quotient does, ties included: the codes are determined bit for bit.
//
// A lane holds 8 elements (16 bytes), D/8 lanes a vector, a wave 64/(D/8) consecutive tokens of one head: it keeps its
// tokens' cosines and sines over the heads that it goes through, and the value codes of four tokens, which share 16-byte pieces of
// a page, are stored by one wave.  Bound by memory (2 bytes in, 2 or 17/32 out an element), by the launch for few tokens.  Measured, calls one
// after another: norms and rotation of 4096 tokens with 64/8 heads of 128 28.9 us (5.2 TB/s; a large copy 5.4), of one token 5.1; 32768 tokens
// of 8 kv heads written 34.2 us (5.0 TB/s), read back 28.7 (5.9), 6000 tokens 9.1 to 10.4 and 5.8 to 7.0 (5.8 at a copy's rate: a wave writes head
// after head with one load a lane in flight, and 1500 blocks do not cover its latency); 16 tokens appended 4.8, 32768 of 64/8 heads 244 us (5.1 TB/s).
#include "attn_common.h"

namespace lqq {

enum Mode { kRope, kAppend, kWrite };  // q, k -> q, k;  q, k, v -> q, cache;  k, v -> cache

struct Vectors {  // of one of q, k, v: strides in elements
    const void *p;
    long long token, head;
};
struct Pages {
    uint8_t *p;
    int slots, lg_page;  // pages * page size
};

template <class T>
__device__ __forceinline__ void widen8(const vec<T, 8> x, float (&f)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)x[e];
}
template <class T>
__device__ __forceinline__ vec<T, 8> narrow8(const float (&f)[8])
{
    vec<T, 8> x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (T)f[e];
    return x;
}

// code + zero point arithmetic: rint(x / s) for r = 1 / s to within one unit
__device__ __forceinline__ float quotient(float x, float r)
{
    constexpr float kGrid = 768.0f;  // one unit of it is 2^-14
    return __builtin_rintf(__builtin_fmaf(x, r, kGrid) - kGrid);
}

// 8 of a vector's elements (L lanes hold it) -> 8 codes in a dword, and the vector's word
template <int L>
__device__ __forceinline__ uint32_t quantise8(const float (&f)[8], uint32_t &word)
{
    float lo = 0.0f, hi = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        lo = __builtin_elementwise_minimum(lo, f[e]);  // (a NaN stays one)
        hi = __builtin_elementwise_maximum(hi, f[e]);
    }
    lo = reduce_lanes<L>(lo, [](float a, float b) { return __builtin_elementwise_minimum(a, b); });
    hi = reduce_lanes<L>(hi, [](float a, float b) { return __builtin_elementwise_maximum(a, b); });
    const float range = hi - lo;
    if (!(range < __builtin_inff())) {  // not finite: every element reads back as NaN
        word = 0x7fc00000u;
        return 0;
    }
    uint32_t bits = __builtin_bit_cast(uint32_t, range / 15.0f);
    bits = (bits + 0x7ffu + ((bits >> 12) & 1u)) & kScaleMask;
    const float s = fmaxf(__builtin_bit_cast(float, bits), 0x1p-100f), r = __builtin_amdgcn_rcpf(s);
    const float z = quotient(-lo, r);
    word = __builtin_bit_cast(uint32_t, s) | (uint32_t)z;
    uint32_t codes = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) codes |= (uint32_t)__builtin_amdgcn_fmed3f(quotient(f[e], r) + z, 0.0f, 15.0f) << (4 * e);
    return codes;
}

template <int D>
__device__ __forceinline__ void store_codes(uint8_t *head, int P, int j, int l, bool value, uint32_t codes, uint32_t word)
{
    if (value) {
        uint8_t *at = head + kv4_value_byte<D>(P, j) + l * 16;  // (8 elements: one column group, or two of D = 64)
        *reinterpret_cast<uint16_t *>(at) = (uint16_t)codes;
        *reinterpret_cast<uint16_t *>(at + (D == 128 ? 4 : 8)) = (uint16_t)(codes >> 16);
    } else {
        *reinterpret_cast<uint32_t *>(head + kv4_key_byte<D>(j) + l * 4) = codes;
    }
    if (l == 0) *reinterpret_cast<uint32_t *>(head + kv4_word_byte<D>(P, j, value)) = word;
}

// grid: (groups of tokens, groups of 4 heads); wave w of a block takes heads 4 * blockIdx.y + w, + 4 * gridDim.y, ...
// of the Hq + Hkv (kRope), Hq + 2 Hkv (kAppend) or 2 Hkv (kWrite: Hq = 0) vectors of a token.
template <class T, int D, Mode MODE, bool NORM>
__global__ __launch_bounds__(256) void qkv_kernel(int tokens, int Hq, int Hkv, int R, int interleaved, Vectors q, Vectors k, Vectors v,
                                                  const int *__restrict__ positions, const float *__restrict__ table, int max_positions,
                                                  const float *__restrict__ q_norm, const float *__restrict__ k_norm, float eps,
                                                  Vectors q_out, Vectors k_out, const int *__restrict__ slots, Pages pages)
{
    constexpr int L = D / 8, TOKENS = 64 / L;
    const int lane = threadIdx.x & 63, l = lane % L;
    const int t = (int)blockIdx.x * TOKENS + lane / L;
    const bool there = t < tokens;
    const int tc = there ? t : tokens - 1;  // (the last token once more, not stored)

    // this lane's cosines and sines; its partner in the pairs of halves
    float c[8], s[8];
    const int half = R / 2, turning = R / 8;  // lanes of a vector that take part
    const bool turns = l < turning, second = l >= turning / 2;
    const int partner = turns ? (second ? lane - turning / 2 : lane + turning / 2) : lane;
    if (MODE != kWrite) {
        const int p = positions[tc];
        const bool known = p >= 0 && p < max_positions;
        const float *row = table + (size_t)(known ? p : 0) * R;
        const int first = !turns ? 0 : interleaved ? 4 * l : 8 * (second ? l - turning / 2 : l);
        const v4f c0 = *reinterpret_cast<const v4f *>(row + first), s0 = *reinterpret_cast<const v4f *>(row + half + first);
        const int more = interleaved ? 0 : 4;
        const v4f c1 = *reinterpret_cast<const v4f *>(row + first + more), s1 = *reinterpret_cast<const v4f *>(row + half + first + more);
        const float bad = __builtin_nanf("");
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            c[e] = known ? c0[e] : bad, c[e + 4] = known ? c1[e] : bad;
            s[e] = known ? s0[e] : bad, s[e + 4] = known ? s1[e] : bad;
        }
    }
    const int slot = MODE != kRope ? slots[tc] : -1;
    const bool stored = MODE != kRope && there && slot >= 0 && slot < pages.slots;
    const int P = 1 << pages.lg_page;
    uint8_t *const page = MODE != kRope ? pages.p + (size_t)(stored ? slot >> pages.lg_page : 0) * Hkv * kv4_head_bytes(P, D) : nullptr;

    const int heads = Hq + (MODE == kRope ? Hkv : 2 * Hkv);
    for (int h = (int)blockIdx.y * 4 + ((int)threadIdx.x >> 6); h < heads; h += 4 * (int)gridDim.y) {
        const bool is_q = h < Hq, is_v = h >= Hq + Hkv;  // (wave-uniform)
        const int head = is_q ? h : is_v ? h - Hq - Hkv : h - Hq;
        const Vectors in = is_q ? q : is_v ? v : k;
        float f[8];
        widen8<T>(*reinterpret_cast<const vec<T, 8> *>(static_cast<const T *>(in.p) + tc * in.token + head * in.head + 8 * l), f);
        if (MODE != kWrite && !is_v) {
            if (NORM) {
                const float *w = is_q ? q_norm : k_norm;
                if (w) {
                    float sum = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum += f[e] * f[e];
                    sum = reduce_lanes<L>(sum, [](float a, float b) { return a + b; });
                    const float rstd = rsqrtf(sum * (1.0f / D) + eps);
                    const v4f w0 = *reinterpret_cast<const v4f *>(w + 8 * l), w1 = *reinterpret_cast<const v4f *>(w + 8 * l + 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) f[e] = f[e] * rstd * w0[e], f[e + 4] = f[e + 4] * rstd * w1[e];
                }
            }
            {
#pragma clang fp contract(off)
                if (interleaved) {
                    if (turns) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float a = f[2 * e], b = f[2 * e + 1];
                            const float ac = a * c[e], bs = b * s[e], bc = b * c[e], as = a * s[e];
                            f[2 * e] = ac - bs;
                            f[2 * e + 1] = bc + as;
                        }
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float other = __shfl(f[e], partner);
                        const float yc = f[e] * c[e], os = other * s[e];
                        const float turned = second ? yc + os : yc - os;
                        f[e] = turns ? turned : f[e];
                    }
                }
            }
        }
        const vec<T, 8> y = narrow8<T>(f);
        if (MODE == kRope || (MODE == kAppend && is_q)) {
            const Vectors out = is_q ? q_out : k_out;
            if (there)
                *reinterpret_cast<vec<T, 8> *>(static_cast<T *>(const_cast<void *>(out.p)) + t * out.token + head * out.head + 8 * l) = y;
        } else {
            widen8<T>(y, f);  // the keys as the rotation alone would have returned them
            uint32_t word;
            const uint32_t codes = quantise8<L>(f, word);
            if (stored) store_codes<D>(page + (size_t)head * kv4_head_bytes(P, D), P, slot & (P - 1), l, is_v, codes, word);
        }
    }
}

// Values of 8 codes
template <class T>
__device__ __forceinline__ vec<T, 8> values8(uint32_t codes, uint32_t word)
{
    const float s = __builtin_bit_cast(float, word & kScaleMask), z = (float)(word & 15u);
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = ((float)((codes >> (4 * e)) & 15u) - z) * s;
    return narrow8<T>(f);
}

// A lane takes 8 elements, as above: keys and values of four or eight tokens of a head a wave.  Bound by what it writes.
template <class T, int D>
__global__ __launch_bounds__(256) void kv4_read_kernel(int tokens, int Hkv, const int *__restrict__ slots, Pages pages, T *__restrict__ k, T *__restrict__ v)
{
    constexpr int L = D / 8, TOKENS = 64 / L;
    const int lane = threadIdx.x & 63, l = lane % L, t = (int)blockIdx.x * TOKENS + lane / L;
    if (t >= tokens) return;
    const int slot = slots[t], P = 1 << pages.lg_page, j = slot & (P - 1);
    const bool held = slot >= 0 && slot < pages.slots;
    const uint8_t *const page = pages.p + (size_t)(held ? slot >> pages.lg_page : 0) * Hkv * kv4_head_bytes(P, D);
    for (int head = (int)blockIdx.y * 4 + ((int)threadIdx.x >> 6); head < Hkv; head += 4 * (int)gridDim.y) {
        const uint8_t *const at = page + (size_t)head * kv4_head_bytes(P, D);
        uint32_t kc = 0, vc = 0, kw = 0, vw = 0;
        if (held) {
            kc = *reinterpret_cast<const uint32_t *>(at + kv4_key_byte<D>(j) + l * 4);
            const uint8_t *const vb = at + kv4_value_byte<D>(P, j) + l * 16;
            vc = *reinterpret_cast<const uint16_t *>(vb) | (uint32_t)*reinterpret_cast<const uint16_t *>(vb + (D == 128 ? 4 : 8)) << 16;
            kw = *reinterpret_cast<const uint32_t *>(at + kv4_word_byte<D>(P, j, false));
            vw = *reinterpret_cast<const uint32_t *>(at + kv4_word_byte<D>(P, j, true));
        }
        const size_t o = ((size_t)t * Hkv + head) * D + 8 * l;
        *reinterpret_cast<vec<T, 8> *>(k + o) = values8<T>(kc, kw);
        *reinterpret_cast<vec<T, 8> *>(v + o) = values8<T>(vc, vw);
    }
}

// Groups of heads that a wave's tokens are shared between: as many as make 2048 blocks (eight a CU), a wave's cosines and sines being loaded
// once a group.  (Norms and rotation, 64/8 heads: one token 5.1 us, with all heads in one group 12.8; 32768 tokens 240 us, with four heads a
// group 342; 1024 tokens with 512, 2048, 8192 blocks 13.2, 9.5 and 10.6 us.)
static unsigned head_groups(int token_groups, int heads)
{
    const int most = (heads + 3) / 4, want = std::max(1, 2048 / std::max(1, token_groups));
    return (unsigned)std::min(most, want);
}

template <class T, int D, Mode MODE>
static void launch_qkv(int tokens, int Hq, int Hkv, int R, int interleaved, Vectors q, Vectors k, Vectors v, const int *positions,
                       const float *table, int max_positions, const float *q_norm, const float *k_norm, float eps, Vectors q_out,
                       Vectors k_out, const int *slots, Pages pages, hipStream_t st)
{
    const int groups = (tokens + 512 / D - 1) / (512 / D), heads = Hq + (MODE == kRope ? Hkv : 2 * Hkv);
    const dim3 grid((unsigned)groups, head_groups(groups, heads));
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, tokens, Hq, Hkv, R, interleaved, q, k, v, positions, table, max_positions, q_norm,
                           k_norm, eps, q_out, k_out, slots, pages);
    };
    if constexpr (MODE != kWrite)
        if (q_norm || k_norm) return go(qkv_kernel<T, D, MODE, true>);
    go(qkv_kernel<T, D, MODE, false>);
}

// what the entry points below have in common
static int check_heads(int dtype, int tokens, int Hq, int Hkv, int D)
{
    if (dtype != LQ_F16 && dtype != LQ_BF16) return fail(LQ_ERR_INVALID, "dtype must be LQ_F16 or LQ_BF16, got %d", dtype);
    if (!head_dim_ok(D)) return fail(LQ_ERR_INVALID, "head_dim must be 64 or 128, got %d", D);
    if (tokens < 0 || tokens > (1 << 24) || Hkv < 1 || Hq < 1 || Hq > 4096 || Hkv > 4096)
        return fail(LQ_ERR_INVALID, "bad shape: %d tokens, %d heads, %d kv heads (need 0..2^24, 1..4096, 1..4096)", tokens, Hq, Hkv);
    return LQ_OK;
}
static int check_vectors(const char *name, const void *p, long long token, long long head, int tokens, int heads, int D)
{
    if (!p) return fail(LQ_ERR_INVALID, "%s: null pointer", name);
    if ((uintptr_t)p & 15) return fail(LQ_ERR_ALIGN, "%s must be 16-byte aligned", name);
    if ((tokens > 1 && token % 8) || (heads > 1 && head % 8))
        return fail(LQ_ERR_ALIGN, "%s: strides must be multiples of 8 elements, got %lld and %lld", name, token, head);
    return LQ_OK;
}
static int check_pages(const void *cache, int num_pages, int page_size, const void *slots)
{
    if (!page_ok(page_size)) return fail(LQ_ERR_INVALID, "page_size must be a power of two from 16 to 256, got %d", page_size);
    if (num_pages < 1 || num_pages > INT32_MAX / page_size)
        return fail(LQ_ERR_INVALID, "num_pages * page_size must be from 1 to 2^31 - 1, got %d * %d", num_pages, page_size);
    if (!cache || !slots) return fail(LQ_ERR_INVALID, "null pointer");
    if ((uintptr_t)cache & 15) return fail(LQ_ERR_ALIGN, "cache must be 16-byte aligned");
    if ((uintptr_t)slots & 3) return fail(LQ_ERR_ALIGN, "slots must be 4-byte aligned");
    return LQ_OK;
}
static int check_rotation(int R, int D, const void *positions, const void *table, int max_positions, const void *q_norm, const void *k_norm, float eps)
{
    if (R < 16 || R > D || R % 16) return fail(LQ_ERR_INVALID, "rot_dim must be a multiple of 16 from 16 to head_dim, got %d", R);
    if (max_positions < 1) return fail(LQ_ERR_INVALID, "the table needs at least one position, got %d", max_positions);
    if (!positions || !table) return fail(LQ_ERR_INVALID, "null pointer");
    if ((uintptr_t)positions & 3) return fail(LQ_ERR_ALIGN, "positions must be 4-byte aligned");
    if (((uintptr_t)table | (uintptr_t)q_norm | (uintptr_t)k_norm) & 15) return fail(LQ_ERR_ALIGN, "table and norm weights must be 16-byte aligned");
    if ((q_norm || k_norm) && !(eps > 0.0f && eps < 1e30f)) return fail(LQ_ERR_INVALID, "eps must be positive, got %g", (double)eps);
    return LQ_OK;
}
static int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LQ_OK : fail(LQ_ERR_HIP, "%s launch failed: %s", what, hipGetErrorString(e));
}

template <class F>
static void by_type(int dtype, int D, F f)  // f(an element, the head dimension's constant)
{
    using std::integral_constant;
    if (dtype == LQ_F16)
        D == 128 ? f(f16{}, integral_constant<int, 128>{}) : f(f16{}, integral_constant<int, 64>{});
    else
        D == 128 ? f(bf16{}, integral_constant<int, 128>{}) : f(bf16{}, integral_constant<int, 64>{});
}

}  // namespace lqq

using namespace lqq;

extern "C" {

int attn_qk_norm_rope(int dtype, int tokens, int Hq, int Hkv, int head_dim, const void *q, long long q_token, long long q_head,
                      const void *k, long long k_token, long long k_head, const int *positions, const float *table, int max_positions,
                      int rot_dim, int interleaved, const float *q_norm, const float *k_norm, float eps, void *q_out,
                      long long qo_token, long long qo_head, void *k_out, long long ko_token, long long ko_head, void *hip_stream)
{
    int rc = check_heads(dtype, tokens, Hq, Hkv, head_dim);
    if (rc || tokens == 0) return rc;
    if ((rc = check_vectors("q", q, q_token, q_head, tokens, Hq, head_dim)) || (rc = check_vectors("k", k, k_token, k_head, tokens, Hkv, head_dim)) ||
        (rc = check_vectors("q_out", q_out, qo_token, qo_head, tokens, Hq, head_dim)) ||
        (rc = check_vectors("k_out", k_out, ko_token, ko_head, tokens, Hkv, head_dim)) ||
        (rc = check_rotation(rot_dim, head_dim, positions, table, max_positions, q_norm, k_norm, eps)))
        return rc;
    (void)hipGetLastError();
    by_type(dtype, head_dim, [&](auto x, auto d) {
        launch_qkv<decltype(x), d.value, kRope>(tokens, Hq, Hkv, rot_dim, interleaved != 0, {q, q_token, q_head}, {k, k_token, k_head}, {},
                                                positions, table, max_positions, q_norm, k_norm, eps, {q_out, qo_token, qo_head},
                                                {k_out, ko_token, ko_head}, nullptr, {}, static_cast<hipStream_t>(hip_stream));
    });
    return launched("norm and rotation");
}

size_t kv4_page_bytes(int page_size, int Hkv, int head_dim)
{
    if (!page_ok(page_size) || !head_dim_ok(head_dim) || Hkv < 1 || Hkv > 4096) return 0;
    return (size_t)Hkv * kv4_head_bytes(page_size, head_dim);
}

int kv4_write(int dtype, int tokens, int Hkv, int head_dim, const void *k, long long k_token, long long k_head, const void *v,
              long long v_token, long long v_head, const int *slots, void *cache, int num_pages, int page_size, void *hip_stream)
{
    int rc = check_heads(dtype, tokens, 1, Hkv, head_dim);
    if (rc || tokens == 0) return rc;
    if ((rc = check_vectors("k", k, k_token, k_head, tokens, Hkv, head_dim)) || (rc = check_vectors("v", v, v_token, v_head, tokens, Hkv, head_dim)) ||
        (rc = check_pages(cache, num_pages, page_size, slots)))
        return rc;
    (void)hipGetLastError();
    by_type(dtype, head_dim, [&](auto x, auto d) {
        launch_qkv<decltype(x), d.value, kWrite>(tokens, 0, Hkv, 16, 0, {}, {k, k_token, k_head}, {v, v_token, v_head}, nullptr, nullptr, 0,
                                                 nullptr, nullptr, 0.0f, {}, {}, slots,
                                                 {static_cast<uint8_t *>(cache), num_pages * page_size, log2_of(page_size)},
                                                 static_cast<hipStream_t>(hip_stream));
    });
    return launched("cache write");
}

int kv4_append(int dtype, int tokens, int Hq, int Hkv, int head_dim, const void *q, long long q_token, long long q_head, const void *k,
               long long k_token, long long k_head, const void *v, long long v_token, long long v_head, const int *positions,
               const float *table, int max_positions, int rot_dim, int interleaved, const float *q_norm, const float *k_norm, float eps,
               void *q_out, long long qo_token, long long qo_head, const int *slots, void *cache, int num_pages, int page_size, void *hip_stream)
{
    int rc = check_heads(dtype, tokens, Hq, Hkv, head_dim);
    if (rc || tokens == 0) return rc;
    if ((rc = check_vectors("q", q, q_token, q_head, tokens, Hq, head_dim)) || (rc = check_vectors("k", k, k_token, k_head, tokens, Hkv, head_dim)) ||
        (rc = check_vectors("v", v, v_token, v_head, tokens, Hkv, head_dim)) ||
        (rc = check_vectors("q_out", q_out, qo_token, qo_head, tokens, Hq, head_dim)) ||
        (rc = check_rotation(rot_dim, head_dim, positions, table, max_positions, q_norm, k_norm, eps)) ||
        (rc = check_pages(cache, num_pages, page_size, slots)))
        return rc;
    (void)hipGetLastError();
    by_type(dtype, head_dim, [&](auto x, auto d) {
        launch_qkv<decltype(x), d.value, kAppend>(tokens, Hq, Hkv, rot_dim, interleaved != 0, {q, q_token, q_head}, {k, k_token, k_head},
                                                  {v, v_token, v_head}, positions, table, max_positions, q_norm, k_norm, eps,
                                                  {q_out, qo_token, qo_head}, {}, slots,
                                                  {static_cast<uint8_t *>(cache), num_pages * page_size, log2_of(page_size)},
                                                  static_cast<hipStream_t>(hip_stream));
    });
    return launched("rotation and cache write");
}

int kv4_read(int dtype, int tokens, int Hkv, int head_dim, const void *cache, int num_pages, int page_size, const int *slots, void *k,
             void *v, void *hip_stream)
{
    int rc = check_heads(dtype, tokens, 1, Hkv, head_dim);
    if (rc || tokens == 0) return rc;
    if ((rc = check_vectors("k", k, 0, 0, tokens, Hkv, head_dim)) || (rc = check_vectors("v", v, 0, 0, tokens, Hkv, head_dim)) ||
        (rc = check_pages(cache, num_pages, page_size, slots)))
        return rc;
    (void)hipGetLastError();
    by_type(dtype, head_dim, [&](auto x, auto d) {
        using T = decltype(x);
        const int groups = (tokens + 512 / d.value - 1) / (512 / d.value);
        hipLaunchKernelGGL((kv4_read_kernel<T, d.value>), dim3((unsigned)groups, head_groups(groups, Hkv)), dim3(256), 0,
                           static_cast<hipStream_t>(hip_stream), tokens, Hkv, slots,
                           Pages{const_cast<uint8_t *>(static_cast<const uint8_t *>(cache)), num_pages * page_size, log2_of(page_size)},
                           static_cast<T *>(k), static_cast<T *>(v));
    });
    return launched("cache read");
}

}  // extern "C"
