// Attention of chunks of new tokens over the 4-bit cache (page format: attn_common.h, its values: kvcache.hip): packed sequences, each with any
// number of new tokens that the cache holds already.
//
//     o_i = sum_j softmax_j(scale * q_i . k_j) v_j,   k_j = (code - z) * s of the key, v_j likewise,   j < context - n + 1 + i
// for new token i of a sequence's n.
//
// A block takes rows, queries times the heads that share a kv head, a wave 32 of them; it goes through the keys from the last to the first, 64 at
// a time: their codes are loaded while the tile before is in the making, unpacked into LDS as FP16 integers (code - z, exact) while
// the one before that is worked on, and go into 32x32x16 MFMAs with the keys' side as the first operand (S^T = K Q^T, O^T = V^T P^T): a lane's
// scores are 32 keys of one row, in the order in which the weights enter the second product.  Value codes lie in a page as pairs of tokens,
// and so they are unpacked to [element][keys]: both operands come out of LDS in 16-byte reads.
//
// The scales never meet the codes.  The keys' are applied to the scores; the values' enter as logarithms,
//     t_j = scale * q . (code - z) * s_j + log2(sv_j),   x_j = 2^(t_j - m),   o = sum x_j (code - z) / sum x_j / sv_j,
// one fused multiply-add each, so that what is rounded to FP16 for the second product is a weight times its value's scale, relative to the largest
// such product (2^6 .. 2^14), and the values have no rounding at all.  sum x_j / sv_j stays in FP32's range for all scales there are, 2^-100 .. 2^124; but
// where the scales of a sequence are further apart than 2^100 an x_j may vanish whose weight counts, and the terms of the sum are taken from the scores
// without the values' scales instead.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_common.h"
#include "workspace_turn.h"

namespace lqq {

struct ChunkArgs {
    const void *q;
    long long q_token, q_head;
    const int *starts, *table, *context;
    const uint8_t *cache;
    void *out;
    unsigned *tickets;
    float *parts;
    int n_seqs, total_q, Hq, Hkv, group, width, pages, lg_page, tiles, splits;
    float scale_log2;
};

constexpr int kFew = 64, kKeys = 64;
constexpr float kWeightBits = 6.0f;
typedef f16 f16x2v __attribute__((ext_vector_type(2)));

__device__ __forceinline__ v16f mfma32(vec<f16, 8> a, vec<f16, 8> b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// 8 nibbles of a dword as 4 pairs of integers in FP16, pair r = nibbles r and r + 4, less the pair of zero points z (1024 more of each): a nibble
// under the exponent of 1024 is 1024 + code, one four bits up 1024 + 16 code.
__device__ __forceinline__ void unpack8(uint32_t w, f16x2v z, f16x2v z64, uint32_t (&o)[4])
{
    const uint32_t w8 = w >> 8;
    const f16x2v sixteenth = {(f16)0.0625f, (f16)0.0625f};
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const uint32_t x = (r < 2 ? w : w8);
        if (r & 1)
            o[r] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(f16x2v, (x & 0x00f000f0u) | 0x64006400u), sixteenth, -z64));
        else
            o[r] = __builtin_bit_cast(uint32_t, (f16x2v)(__builtin_bit_cast(f16x2v, (x & 0x000f000fu) | 0x64006400u) - z));
    }
}
// 1024 + z and 64 + z of two words' zero points
__device__ __forceinline__ void zeros_of(uint32_t a, uint32_t b, f16x2v &z, f16x2v &z64)
{
    const uint32_t zz = (__builtin_amdgcn_perm(b, a, 0x0c040c00u) & 0x000f000fu);
    z = __builtin_bit_cast(f16x2v, zz | 0x64006400u);
    z64 = z - f16x2v{(f16)960.0f, (f16)960.0f};
}

// A wave's share of a tile's codes: 16 keys, or their values, or both; all from one page
template <int D>
struct Codes {
    uint32_t c[D / 32];
    u32x4 w;  // words: of the lane's key (the first), or of the lane's four tokens
};
typedef __amdgpu_buffer_rsrc_t buf_t;
template <int D>
__device__ __forceinline__ void load_codes(Codes<D> &x, buf_t head, int P, int j, int lane, bool value)
{
    const int at = (value ? P * (D / 2) : 0) + j * (D / 2);
    if constexpr (D == 128) {
        const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(head, lane * 16, at, 0);
        x.c[0] = v[0], x.c[1] = v[1], x.c[2] = v[2], x.c[3] = v[3];
    } else {
        const auto v = __builtin_amdgcn_raw_buffer_load_b64(head, lane * 8, at, 0);
        x.c[0] = v[0], x.c[1] = v[1];
    }
    if (value)
        x.w = __builtin_amdgcn_raw_buffer_load_b128(head, 16 * (lane >> 4), P * (D + 4) + 4 * j, 0);
    else
        x.w[0] = __builtin_amdgcn_raw_buffer_load_b32(head, 4 * (lane >> 2), P * D + 4 * j, 0);
}
// (not __syncthreads(): codes stay in flight)
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int D, class T, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void kv4_chunks_kernel(const ChunkArgs a)
{
    constexpr int CHUNKS = D / 8, ROWS = 32 * WAVES;
    constexpr bool BOTH = WAVES == 4;  // a wave unpacks keys and values; of eight, four each
    __shared__ __attribute__((aligned(16))) u32x4 s_k[2][kKeys][CHUNKS], s_v[2][D][kKeys / 8];
    __shared__ __attribute__((aligned(16))) float s_sk[2][kKeys], s_lv[2][kKeys], s_rv[2][kKeys];
    __shared__ __attribute__((aligned(16))) int s_far[2][4];  // scales that are far from 1, in a quarter of the tile (large ones: or before)
    __shared__ int s_bad, s_last, s_top;
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);

    // the block's tile: as in attn_prompt.hip
    const auto start_of = [&](int s) { return min(max(a.starts[s], 0), a.total_q); };
    const bool few = a.n_seqs <= kFew;
    int from = 0, len = 0, upto = 0, tiles = a.tiles;
    if (few) {
        if (lane < a.n_seqs) {
            from = start_of(lane);
            len = max(min(a.starts[lane + 1], a.total_q) - from, 0);
        }
        upto = sums_up_to((len * a.group + ROWS - 1) / ROWS);
        tiles = min(__builtin_amdgcn_readlane(upto, 63), a.tiles);
    }
    const int blocks = tiles * a.Hkv * a.splits, per = (blocks + 7) >> 3, id = ((int)blockIdx.x & 7) * per + ((int)blockIdx.x >> 3);
    if ((int)blockIdx.x >> 3 >= per || id >= blocks) return;
    const int whole = id / a.splits, part = id % a.splits;
    const int hk = whole / tiles;
    int tile = tiles - 1 - whole % tiles;
    int seq, q0, len_q;
    if (few) {
        seq = __builtin_ctzll(__ballot(upto > tile) | 1ull << 63);
        q0 = __builtin_amdgcn_readlane(from, seq);
        len_q = __builtin_amdgcn_readlane(len, seq);
        tile -= seq ? __builtin_amdgcn_readlane(upto, seq - 1) : 0;
    } else {
        const auto first_tile = [&](int s) { return (int)((unsigned)(start_of(s) * a.group) / (unsigned)ROWS) + s; };
        int end = a.n_seqs;
        seq = 0;
        while (end - seq > 1) {
            const int step = (end - seq + 63) >> 6, s = seq + step * lane;
            const uint64_t past = __ballot(s >= end || first_tile(min(s, end - 1)) > tile);
            const int at = past ? max(__builtin_ctzll(past) - 1, 0) : 63;
            seq += step * at;
            end = min(end, seq + step);
        }
        q0 = __builtin_amdgcn_readfirstlane(start_of(seq));
        len_q = __builtin_amdgcn_readfirstlane(max(min(a.starts[seq + 1], a.total_q) - q0, 0));
        tile -= __builtin_amdgcn_readfirstlane(first_tile(seq));
    }
    if (tile < 0 || tile * ROWS >= len_q * a.group) return;

    const int P = 1 << a.lg_page, longest = a.width << a.lg_page;
    const int context = __builtin_amdgcn_readfirstlane(a.context[seq]), ctx = min(max(context, 0), longest);
    const int first = tile * ROWS, first_w = first + 32 * wave, rows = len_q * a.group, before = ctx - len_q;
    const int row = first_w + n, query = min(row, rows - 1) / a.group, head = hk * a.group + min(row, rows - 1) % a.group;
    const auto sees = [&](int r) { return min(r, rows - 1) / a.group + before + 1; };  // keys (none where it is not above 0)
    const int limit = sees(row), until = sees(first + ROWS - 1);
    const int wave_all = __builtin_amdgcn_readfirstlane(sees(first_w)), wave_any = __builtin_amdgcn_readfirstlane(sees(first_w + 31));
    const bool any_row = first_w < rows;

    const auto turn_k = [](int j) { return D == 128 ? j & 15 : j >> 1 & 7; };
    const auto turn_v = [](int d) { return ((d >> 1) ^ (d >> 4)) & 7; };
    const int tiles_k = max((until + kKeys - 1) / kKeys, 0);
    const int t_last = (int)((unsigned)part * (unsigned)tiles_k / (unsigned)a.splits);
    int t = (int)((unsigned)(part + 1) * (unsigned)tiles_k / (unsigned)a.splits) - 1, buf = 0;

    // the codes of this wave's 16 keys of a tile
    typedef const __attribute__((address_space(4))) int *ints;
    const ints table = (ints)(uintptr_t)(a.table + (size_t)seq * a.width);
    const unsigned page_bytes = (unsigned)a.Hkv * (unsigned)kv4_head_bytes(P, D);
    const uint8_t *const cache = a.cache + (size_t)hk * kv4_head_bytes(P, D);
    const int last_page = max((ctx - 1) >> a.lg_page, 0), keys_w = 16 * (wave & 3);
    const bool value_wave = wave >= 4;
    bool bad = context > longest, large = false;
    Codes<D> ck, cv;  // (of eight waves each uses one)
    const auto page_of = [&](int t) { return (unsigned)table[min((max(t, 0) * kKeys + keys_w) >> a.lg_page, last_page)]; };
    const auto load = [&](int t, unsigned page) {
        const bool any = t >= t_last, out_of_range = page >= (unsigned)a.pages;
        bad |= any && out_of_range;
        const buf_t at = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(cache + (uint64_t)(out_of_range ? 0u : page) * page_bytes), 0,
                                                           any ? kv4_head_bytes(P, D) : 0, 0x00027000);
        const int j = (t * kKeys + keys_w) & (P - 1);
        if (BOTH || !value_wave) load_codes<D>(ck, at, P, j, lane, false);
        if (BOTH) load_codes<D>(cv, at, P, j, lane, true);
        if (!BOTH && value_wave) load_codes<D>(ck, at, P, j, lane, true);
    };
    unsigned page = 0;
    if (t >= t_last) {
        load(t, page_of(t));
        page = page_of(t - 1);
    }

    // Queries, in the keys' order within 8 elements (a pair of a dword's nibbles is four apart).  FP16 as they are; BF16 as FP16 numbers, over a power
    // of two for the block that brings its largest element to 2^14 .. 2^15, or one of its own for a row that is far smaller.
    vec<f16, 8> q[D / 16];
    float q_scale = fabsf(a.scale_log2), row_scale = 1.0f;
    bool uneven = false;
    {
        const T *src = static_cast<const T *>(a.q) + (long long)(q0 + query) * a.q_token + head * a.q_head + 8 * h;
        u32x4 raw[D / 16];
#pragma unroll
        for (int i = 0; i < D / 16; ++i) raw[i] = *reinterpret_cast<const u32x4 *>(src + 16 * i);
        const float sign = a.scale_log2 < 0.0f ? -1.0f : 1.0f;
        if (threadIdx.x == 0) s_bad = 0, s_top = 0;
        if constexpr (!__is_same(T, f16)) {
            int most = 0;  // bits of the row's largest finite element
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int lo = (int)(raw[i][e] & 0x7fffu), hi = (int)(raw[i][e] >> 16 & 0x7fffu);
                    most = max(most, max(lo < 0x7f80 ? lo : 0, hi < 0x7f80 ? hi : 0));
                }
            }
            const auto both = __builtin_amdgcn_permlane32_swap((unsigned)most, (unsigned)most, false, false);
            most = max((int)both[0], (int)both[1]);
            meet();
            if (row < rows) atomicMax(&s_top, most);
            meet();
            const auto exponent = [](int bits) { return max(bits >> 7, 1) - 127; };
            const int top = exponent(s_top), own = most && row < rows && exponent(most) < top - 14 ? exponent(most) : top;
            uneven = __any(own != top);
            const int down = 14 - own;  // up to 140: in two steps
            const float by0 = power_of_two(down / 2), by1 = power_of_two(down - down / 2);
            row_scale = power_of_two(max((own - top) / 2, -126)) * power_of_two(max(own - top - (own - top) / 2, -126));
            q_scale = fminf(fmaxf(q_scale * power_of_two(max(top - 14, -126)), 0x1p-126f), 0x1p127f);
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t x = raw[i][e >> 1];
                    q[i][2 * (e & 3) + (e >> 2)] = (f16)(__builtin_bit_cast(float, e & 1 ? x & 0xffff0000u : x << 16) * by0 * by1 * sign);
                }
        } else {
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) q[i][2 * (e & 3) + (e >> 2)] = __builtin_bit_cast(vec<f16, 8>, raw[i])[e] * (f16)sign;
        }
    }

    const auto unpack_keys = [&](const Codes<D> &x, int buf) {
        const int j = keys_w + (lane >> 2);
        f16x2v z, z64;
        zeros_of(x.w[0], x.w[0], z, z64);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            uint32_t o[4];
            unpack8(x.c[i], z, z64, o);
            s_k[buf][j][((D / 32) * (lane & 3) + i) ^ turn_k(j)] = u32x4{o[0], o[1], o[2], o[3]};
        }
        const uint32_t word = x.w[0] & kScaleMask;
        const float s = __builtin_bit_cast(float, word) * q_scale;
        if ((lane & 3) == 0) s_sk[buf][j] = s > 0x1p127f ? 0x1p127f : s;  // (NaN stays)
    };
    const auto unpack_values = [&](const Codes<D> &x, int buf) {
        constexpr int W = D / 16;  // elements of a column group
        const int four = lane >> 4, d0 = W * (lane & 15);
        f16x2v z[2], z64[2];
#pragma unroll
        for (int p = 0; p < 2; ++p) zeros_of(x.w[2 * p], x.w[2 * p + 1], z[p], z64[p]);
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            uint32_t o[2][4];
#pragma unroll
            for (int p = 0; p < 2; ++p) unpack8(x.c[p * (W / 4) + i], z[p], z64[p], o[p]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = d0 + 4 * i + r;
                reinterpret_cast<uint2 *>(&s_v[buf][d][(2 * (keys_w >> 4) + (four & 1)) ^ turn_v(d)])[four >> 1] = uint2{o[0][r], o[1][r]};
            }
        }
        v4f scale;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t word = x.w[e] & kScaleMask;
            const float s = __builtin_bit_cast(float, word);
            scale[e] = s < 0x1p-100f ? 0x1p-100f : s;  // (NaN stays; a place that nothing was written to counts as zeros)
        }
        large |= __any(fmaxf(fmaxf(scale[0], scale[1]), fmaxf(scale[2], scale[3])) > 0x1p60f);
        const bool small = __any(fminf(fminf(scale[0], scale[1]), fminf(scale[2], scale[3])) < 0x1p-40f);
        if (lane == 0) s_far[buf][keys_w >> 4] = large || small;
        if ((lane & 15) == 0) {
            v4f lv, rv;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                lv[e] = __builtin_amdgcn_logf(scale[e]);
                rv[e] = __builtin_amdgcn_rcpf(scale[e]);
            }
            *reinterpret_cast<v4f *>(&s_lv[buf][keys_w + 4 * four]) = lv;
            *reinterpret_cast<v4f *>(&s_rv[buf][keys_w + 4 * four]) = rv;
        }
    };
    const auto unpack = [&](int buf) {
        if (BOTH || !value_wave) unpack_keys(ck, buf);
        if (BOTH) unpack_values(cv, buf);
        if (!BOTH && value_wave) unpack_values(ck, buf);
    };

    v16f o[D / 32] = {};
    float m = -__builtin_inff(), m_up = m, base = 0.0f, l = 0.0f;  // maximum of t, from where it moves, kWeightBits - m; this lane's part of sum x / sv

    // Fragments: 32 keys (u) of elements 16 i ..; 32 elements (e) of 16 keys (u).  (Rows 32 apart turn their pieces alike, but for 2 e of the values'.)
    int v_at[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) v_at[x] = n * (kKeys / 8) + ((2 * x + h) ^ turn_v(n));
    const auto keys = [&](int u, int i) {
        const int c = 2 * i + h;
        return __builtin_bit_cast(vec<f16, 8>, s_k[buf][32 * u + n][c ^ turn_k(n)]);
    };
    const auto values = [&](int u, int e) { return __builtin_bit_cast(vec<f16, 8>, (&s_v[buf][32 * e][0])[v_at[u ^ e]]); };
    const auto step = [&](int key) {
        v16f s[2] = {};
        vec<f16, 8> frag[2][2] = {{keys(0, 0), keys(1, 0)}};
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            if (i + 1 < D / 16)
#pragma unroll
                for (int u = 0; u < 2; ++u) frag[(i + 1) & 1][u] = keys(u, i + 1);
#pragma unroll
            for (int u = 0; u < 2; ++u) s[u] = mfma32(frag[i & 1][u], q[i], s[u]);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (uneven) {
#pragma unroll
            for (int u = 0; u < 2; ++u) s[u] *= row_scale;
        }
        const bool masked = key + kKeys > wave_all;  // some row of the wave does not see all of these keys
        const int seen = limit - key - 4 * h;  // of the keys that a lane has from 4 h on
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const v4f sk = *reinterpret_cast<const v4f *>(&s_sk[buf][32 * u + 8 * g + 4 * h]), lv = *reinterpret_cast<const v4f *>(&s_lv[buf][32 * u + 8 * g + 4 * h]);
#pragma unroll
                for (int r = 0; r < 4; ++r) s[u][4 * g + r] = __builtin_fmaf(s[u][4 * g + r], sk[r], lv[r]);
                if (g & 1) __builtin_amdgcn_sched_barrier(0);
            }
        if (masked) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[u][i] = 32 * u + 8 * (i >> 2) + (i & 3) < seen ? s[u][i] : -__builtin_inff();
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < 32; i += 2) top = fmaxf(fmaxf(top, s[i >> 4][i & 15]), s[i >> 4][(i & 15) + 1]);
        if (__any(top > m_up)) {  // (first of all: m is minus infinity)
            const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, top), __builtin_bit_cast(unsigned, top), false, false);
            top = fmaxf(__builtin_bit_cast(float, (unsigned)both[0]), __builtin_bit_cast(float, (unsigned)both[1]));
            top = top > m_up ? top : m;  // (a row's results go by its own scores alone)
            // (in two steps for l: a factor of 2^-200 may still leave something of a sum that is 2^100)
            const float half = top == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((m - top) * 0.5f), by = half * half;
            m = top;
            m_up = top + (14.0f - kWeightBits);
            base = top == -__builtin_inff() ? 0.0f : kWeightBits - top;
            l = l * half * half;
#pragma unroll
            for (int e = 0; e < D / 32; ++e) o[e] *= by;
        }
        const v4i far4 = *reinterpret_cast<const v4i *>(s_far[buf]);
        if (masked || __builtin_amdgcn_readfirstlane(far4[0] | far4[1] | far4[2] | far4[3])) {
            // the sum from the scores themselves (2^16 of it, which is 2^-130 .. 2^122); what is masked has no part in it
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const v4f lv = *reinterpret_cast<const v4f *>(&s_lv[buf][32 * u + 8 * g + 4 * h]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float t = s[u][4 * g + r], p = __builtin_amdgcn_exp2f(t - lv[r] + (base + 16.0f));
                        l = __builtin_fmaf(32 * u + 8 * g + r < seen ? p : 0.0f, 0x1p-16f, l);
                        s[u][4 * g + r] = __builtin_amdgcn_exp2f(t + base);
                    }
                    if (g & 1) __builtin_amdgcn_sched_barrier(0);
                }
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const v4f rv = *reinterpret_cast<const v4f *>(&s_rv[buf][32 * u + 8 * g + 4 * h]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float x = __builtin_amdgcn_exp2f(s[u][4 * g + r] + base);
                        l = __builtin_fmaf(x, rv[r], l);
                        s[u][4 * g + r] = x;
                    }
                    if (g & 1) __builtin_amdgcn_sched_barrier(0);
                }
        }
        vec<f16, 8> p[4];
#pragma unroll
        for (int i = 0; i < 32; ++i) p[i >> 3][i & 7] = (f16)s[i >> 4][i & 15];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < D / 32; ++e) o[e] = mfma32(values(u, e), p[u], o[e]);
    };

    if (t >= t_last) {
        unpack(0);
        load(t - 1, page);
        page = page_of(t - 2);
    }
    for (; t >= t_last; --t, buf ^= 1) {
        meet();  // (the tile is there, and all waves have read the one before it)
        if (t > t_last) {  // the next tile's codes are unpacked, those of the one after it loaded
            unpack(buf ^ 1);
            load(t - 2, page);
            page = page_of(t - 3);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (any_row && t * kKeys < wave_any) step(t * kKeys);  // (else: no row of the wave sees any of them)
    }

    if (bad) s_bad = 1;
    meet();
    const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, l), __builtin_bit_cast(unsigned, l), false, false);
    l = __builtin_bit_cast(float, (unsigned)both[0]) + __builtin_bit_cast(float, (unsigned)both[1]);
    if (s_bad) l = __builtin_nanf("");
    if (a.splits > 1) {
        // every part leaves its maxima, sums and results, past the L2s; the last to arrive at the tile's ticket joins them, in their order
        constexpr int FLOATS = 64 * WAVES * (D / 2 + 4);  // of a part
        float *const parts = a.parts + (size_t)whole * a.splits * FLOATS;
        const auto all = __builtin_amdgcn_make_buffer_rsrc(parts, 0, a.splits * FLOATS * 4, 0x00027000);
        const int none = row < rows ? 0 : a.splits * FLOATS * 4;  // (a lane without a row leaves and reads nothing)
        const auto at = [&](int p, int piece) { return (p * FLOATS + (piece * 64 * WAVES + (int)threadIdx.x) * 4) * 4 + none; };
        constexpr int kShared = 16;  // sc1
#pragma unroll
        for (int e = 0; e < D / 32; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v4f{o[e][4 * i], o[e][4 * i + 1], o[e][4 * i + 2], o[e][4 * i + 3]}), all,
                                                       at(part, 4 * e + i), 0, kShared);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v4f{m, l, 0.0f, 0.0f}), all, at(part, D / 8), 0, kShared);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (threadIdx.x == 0) {
            const unsigned arrived = __hip_atomic_fetch_add(a.tickets + whole, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_last = arrived == (unsigned)a.splits - 1;
            if (s_last) __hip_atomic_store(a.tickets + whole, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (!s_last) return;
        m = -__builtin_inff();
        l = 0.0f;
#pragma unroll
        for (int e = 0; e < D / 32; ++e) o[e] = v16f{};
        for (int p = 0; p < a.splits; ++p) {
            const v4f ml = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(all, at(p, D / 8), 0, kShared));
            v4f x[D / 8];
#pragma unroll
            for (int i = 0; i < D / 8; ++i) x[i] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(all, at(p, i), 0, kShared));
            const float now = fmaxf(m, ml[0]);
            const float old = m == now ? 1.0f : __builtin_amdgcn_exp2f((m - now) * 0.5f);
            const float by = ml[0] == now ? 1.0f : __builtin_amdgcn_exp2f((ml[0] - now) * 0.5f);
            m = now;
            l = l * old * old + ml[1] * by * by;
#pragma unroll
            for (int e = 0; e < D / 32; ++e)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[e][i] = o[e][i] * (old * old) + x[4 * e + (i >> 2)][i & 3] * (by * by);
        }
    }
    if (row >= rows) return;
    const float by = l == 0.0f ? 0.0f : 1.0f / l;
    T *dst = static_cast<T *>(a.out) + ((size_t)(q0 + query) * a.Hq + head) * D;
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

namespace {
constexpr size_t kTickets = 32768;  // bytes at the head of the workspace, those of the GEMM's
// Waves of a block: eight where they have rows for most of the tiles
int waves_of(int total_q, int n_seqs, int group) { return (long long)total_q * group >= 256LL * n_seqs ? 8 : 4; }
// Tiles of a kv head, at most (more than 64 sequences: as they are searched for)
long long tiles_of(int total_q, int n_seqs, int group, int waves)
{
    const long long rows = (long long)total_q * group, each = 32 * waves;
    return n_seqs <= kFew ? (rows + (long long)n_seqs * (each - 1)) / each : rows / each + n_seqs;
}
// Parts of the keys, where the tiles are fewer than the blocks that run at a time: as many as fill the CUs, none with fewer than four tiles of keys where all
// contexts are as long as the table allows
int splits_of(long long blocks, int waves, int longest)
{
    const long long at_once = waves == 8 ? 256 : 512;
    if (blocks < 1 || blocks >= at_once) return 1;
    return (int)std::max<long long>(1, std::min<long long>({at_once / blocks, (long long)longest / (4 * kKeys), 32}));
}
size_t part_bytes(int head_dim, int waves) { return sizeof(float) * 64 * waves * (head_dim / 2 + 4); }
}  // namespace

extern "C" size_t kv4_attention_chunks_workspace_size(int n_seqs, int total_q, int Hq, int Hkv, int head_dim, int page_size, int table_width)
{
    if (n_seqs < 1 || total_q < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv || !head_dim_ok(head_dim) || !page_ok(page_size) || table_width < 1 || table_width > (1 << 30) / page_size)
        return 0;
    const int waves = waves_of(total_q, n_seqs, Hq / Hkv);
    const long long blocks = tiles_of(total_q, n_seqs, Hq / Hkv, waves) * Hkv;
    const int splits = splits_of(blocks, waves, table_width * page_size);
    return splits == 1 ? 0 : kTickets + (size_t)blocks * splits * part_bytes(head_dim, waves);
}

extern "C" int kv4_attention_chunks(int dtype, int n_seqs, int total_q, int Hq, int Hkv, int head_dim, const void *q, long long q_token, long long q_head,
                                    const int *starts_q, const void *cache, int num_pages, int page_size, const int *block_table, int table_width,
                                    const int *context, float scale, void *out, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (dtype != LQ_F16 && dtype != LQ_BF16) return fail(LQ_ERR_INVALID, "dtype must be LQ_F16 or LQ_BF16, got %d", dtype);
    if (!head_dim_ok(head_dim)) return fail(LQ_ERR_INVALID, "head_dim must be 64 or 128, got %d", head_dim);
    if (n_seqs < 0 || n_seqs > (1 << 20) || total_q < 0 || total_q > (1 << 28) || Hkv < 1 || Hkv > 4096 || Hq < 1 || Hq > 4096 || Hq % Hkv)
        return fail(LQ_ERR_INVALID, "bad shape: %d sequences, %d queries, %d heads, %d kv heads (heads a multiple of kv heads, up to 4096)",
                    n_seqs, total_q, Hq, Hkv);
    if (!page_ok(page_size)) return fail(LQ_ERR_INVALID, "page_size must be a power of two from 16 to 256, got %d", page_size);
    if (num_pages < 1 || num_pages > INT32_MAX / page_size || table_width < 1 || table_width > (1 << 30) / page_size)
        return fail(LQ_ERR_INVALID, "num_pages times page_size must be from 1 to below 2^31, table_width times it to 2^30, got %d and %d times %d",
                    num_pages, table_width, page_size);
    if (!(scale > -1e30f && scale < 1e30f)) return fail(LQ_ERR_INVALID, "scale must be finite");
    if (n_seqs == 0 || total_q == 0) return LQ_OK;
    if (!q || !starts_q || !cache || !block_table || !context || !out) return fail(LQ_ERR_INVALID, "null pointer");
    if (((uintptr_t)q | (uintptr_t)cache | (uintptr_t)out | (uintptr_t)workspace) & 15)
        return fail(LQ_ERR_ALIGN, "q, cache, out and workspace must be 16-byte aligned");
    if (((uintptr_t)starts_q | (uintptr_t)block_table | (uintptr_t)context) & 3) return fail(LQ_ERR_ALIGN, "starts_q, block_table and context must be 4-byte aligned");
    if ((total_q > 1 && q_token % 8) || (Hq > 1 && q_head % 8)) return fail(LQ_ERR_ALIGN, "q: strides must be multiples of 8 elements, got %lld and %lld", q_token, q_head);
    const int group = Hq / Hkv, waves = waves_of(total_q, n_seqs, group);
    const long long tiles = tiles_of(total_q, n_seqs, group, waves);
    if (tiles * Hkv > (1 << 22) || (long long)total_q * group > (1 << 30)) return fail(LQ_ERR_INVALID, "too many rows: %d queries of %d sequences, %d heads", total_q, n_seqs, Hq);
    const size_t need = kv4_attention_chunks_workspace_size(n_seqs, total_q, Hq, Hkv, head_dim, page_size, table_width);
    const int splits = need && workspace && workspace_bytes >= need ? splits_of(tiles * Hkv, waves, table_width * page_size) : 1;
    const ChunkArgs a{q, q_token, q_head, starts_q, block_table, context, static_cast<const uint8_t *>(cache), out,
                      static_cast<unsigned *>(workspace), splits > 1 ? reinterpret_cast<float *>(static_cast<char *>(workspace) + kTickets) : nullptr,
                      n_seqs, total_q, Hq, Hkv, group, table_width, num_pages, log2_of(page_size), (int)tiles, splits, scale * 1.44269504f};
    const dim3 grid((unsigned)((tiles * Hkv * splits + 7) / 8 * 8));
    (void)hipGetLastError();
    const WorkspaceTurn turn(splits > 1 ? workspace : nullptr, hip_stream);
    const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * waves), 0, static_cast<hipStream_t>(hip_stream), a); };
    const auto of = [&](auto x, auto d) {
        using T = decltype(x);
        constexpr int D = decltype(d)::value;
        waves == 8 ? go(kv4_chunks_kernel<D, T, 8>) : go(kv4_chunks_kernel<D, T, 4>);
    };
    using Wide = std::integral_constant<int, 128>;
    using Narrow = std::integral_constant<int, 64>;
    if (dtype == LQ_F16)
        head_dim == 128 ? of(f16{}, Wide{}) : of(f16{}, Narrow{});
    else
        head_dim == 128 ? of(bf16{}, Wide{}) : of(bf16{}, Narrow{});
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LQ_OK : fail(LQ_ERR_HIP, "attention launch failed: %s", hipGetErrorString(e));
}
