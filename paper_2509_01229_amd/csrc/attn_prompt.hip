// Attention over whole prompts: packed sequences of different lengths, grouped heads, causal or not.
//
//     o_i = sum_j softmax_j(scale * q_i . k_j) v_j,   j < len_k,   causal: j <= i + len_k - len_q
//
// One pass over the keys with a running maximum and sum (FP32).  A block takes 128 rows, queries times the heads that share a kv head (few
// queries fill it, and the causal mask cuts fewer of its tiles than for 128 queries of one head); a wave takes 32 of them, held as
// MFMA operands, through the keys, 64 at a time, which go straight into LDS while the 64 before them are worked on; both products
// on 32x32x16 MFMAs with the keys' side as the first operand (S^T = K Q^T, O^T = V^T P^T): a lane's scores are 32 keys of one query, and
// they are in the order in which the weights enter the second product.  The values are read from LDS transposed (ds_read_b64_tr_b16).
// Weights are rounded to the type of the values, as the matrix cores multiply one type; a row's largest is 2^6 .. 2^14, so that FP16 holds those
// down to 2^-20 of it in full, and their sum is that of the numbers before rounding (FP32).
//
// Keys are taken from the last to the first: the tiles that the causal mask cuts come first.  What is masked has no
// part in the result, whatever it holds: scores by selection, and values, where a masked one is not finite, by taking
// the tile's values that are not finite out of the product and adding them to the rows that see them.
//
// Measured (BF16, 64/8 heads of 128): 8192 tokens, not causal, 1980 us, 1110 TFLOP/s; three causal prompts of 12000 tokens together 795 us, 1020 (a
// product of 8192^3 in the library: 1400).  The matrix cores are busy in 55% of the cycles (counters); next to the 32 MFMAs of a wave's tile stand
// about 130 vector instructions and 32 exponentials at a quarter of their rate, 56% of a SIMD's cycles.  Neither is full: a wave's scores, softmax and second
// product follow one another, and the two waves of a SIMD overlap them little.  For short
// prompts the time is one of latencies: four of 256 tokens, 32/32 heads, 13.2 us.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_common.h"
#include "workspace_turn.h"

namespace lqq {

struct PromptArgs {
    const void *q, *k, *v;
    long long q_token, q_head, k_token, k_head, v_token, v_head;
    const int *starts_q, *starts_k;
    void *out;
    unsigned *tickets;
    float *parts;
    int n_seqs, total_q, total_k, Hq, Hkv, group, causal, tiles, splits;
    float scale_log2;
};

constexpr int kFew = 64, kRows = 128, kKeys = 64, kPromptWaves = 4;
constexpr float kWeightBits = 6.0f;  // a row's largest weight is 2^6 when its maximum is up to date (2^14 at most)

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

// 16 bytes for each lane straight into LDS, from a wave-uniform base plus the lane's offset to a wave-uniform place plus 16 * lane.  Written in
// assembly, so that the compiler does not wait for all of them before each LDS read; the kernel waits for them itself.
__device__ __forceinline__ void load_to_lds(uint32_t lane_offset, const char *base, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(lane_offset), "s"(base), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ void wait_and_meet() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int D, class T>
__global__ __launch_bounds__(64 * kPromptWaves, 2) void attn_prompt_kernel(const PromptArgs a)
{
    constexpr int CHUNKS = D / 8;                          // 16-byte pieces of a row
    constexpr int ROWS = 64 / CHUNKS, LOADS = kKeys / kPromptWaves / ROWS;  // rows that a load of a wave brings; loads of a wave's share of a tile
    __shared__ __attribute__((aligned(16))) u32x4 s_k[2][kKeys][CHUNKS], s_v[2][kKeys][CHUNKS];
    __shared__ int s_odd;  // the tile (plus 1) in which a value is not finite
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);

    // Up to 64 sequences: a lane looks at each, and `tiles` is the number of tiles that they have.  More of them: sequence s has the tiles from
    // floor(rows before it / kRows) + s on (enough for its rows, one more at times, which has none), and is searched for 64 ways at a time.
    // (1000 sequences of 100 tokens, 32/8 heads: looked at 64 at a time 1000 us, searched for 648; four of 256, 32/32 heads: the tiles that there are
    // 13.2 us, those from floor(...) 17.1.)
    const auto start_of = [&](int s) { return min(max(a.starts_q[s], 0), a.total_q); };
    const bool few = a.n_seqs <= kFew;
    int from = 0, len = 0, upto = 0, tiles = a.tiles;
    if (few) {
        if (lane < a.n_seqs) {
            from = start_of(lane);
            len = max(min(a.starts_q[lane + 1], a.total_q) - from, 0);
        }
        upto = sums_up_to((len * a.group + kRows - 1) / kRows);  // tiles of the sequences 0 .. lane
        tiles = min(__builtin_amdgcn_readlane(upto, 63), a.tiles);  // (more than there can be where sequences overlap)
    }
    // Blocks with ids 8 apart run on one XCD: each XCD gets consecutive kv heads, and goes through a head's tiles from the last
    // (the longest rows of keys) to the first, so that what runs at a time shares keys and values in the XCD's L2.  Blocks that the grid
    // has too many come last.
    const int blocks = tiles * a.Hkv * a.splits, per = (blocks + 7) >> 3, id = ((int)blockIdx.x & 7) * per + ((int)blockIdx.x >> 3);
    if ((int)blockIdx.x >> 3 >= per || id >= blocks) return;
    const int whole = id / a.splits, part = id % a.splits;  // a tile of a kv head, which part of its keys
    const int hk = whole / tiles;
    int tile = tiles - 1 - whole % tiles;

    // the tile's sequence
    int seq, q0, len_q;
    if (few) {
        seq = __builtin_ctzll(__ballot(upto > tile) | 1ull << 63);
        q0 = __builtin_amdgcn_readlane(from, seq);
        len_q = __builtin_amdgcn_readlane(len, seq);
        tile -= seq ? __builtin_amdgcn_readlane(upto, seq - 1) : 0;
    } else {
        const auto first_tile = [&](int s) { return (int)((unsigned)(start_of(s) * a.group) / (unsigned)kRows) + s; };
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
        len_q = __builtin_amdgcn_readfirstlane(max(min(a.starts_q[seq + 1], a.total_q) - q0, 0));
        tile -= __builtin_amdgcn_readfirstlane(first_tile(seq));
    }
    if (tile < 0 || tile * kRows >= len_q * a.group) return;
    const int k0 = min(max(a.starts_k[seq], 0), a.total_k), len_k = max(min(a.starts_k[seq + 1], a.total_k) - k0, 0);
    // Rows: the queries' heads of this kv head, row = query * group + head.  The first rows of the block and of the wave, how many there are
    const int first = tile * kRows, first_w = first + 32 * wave, rows = len_q * a.group, before = len_k - len_q;
    const int row = first_w + n, query = min(row, rows - 1) / a.group, head = hk * a.group + min(row, rows - 1) % a.group;
    const auto sees = [&](int r) { return a.causal ? min(len_k, min(r, rows - 1) / a.group + before + 1) : len_k; };  // keys
    const int limit = sees(row), until = sees(first + kRows - 1), block_all = sees(first);
    const int wave_all = __builtin_amdgcn_readfirstlane(sees(first_w)), wave_any = __builtin_amdgcn_readfirstlane(sees(first_w + 31));
    const bool any_row = first_w < rows;

    // A wave loads 16 rows of a tile of keys and of values.  A row's pieces lie at their number XOR what these give, so that lanes that read together
    // do not meet in a bank: 16 rows and the same piece of each (keys), four rows and four pieces of each (values).  256 bytes are one round of the
    // banks, a row or two of them.
    const auto turn_k = [](int j) { return D == 128 ? j & 15 : j >> 1 & 7; };
    const auto turn_v = [](int j) { return D == 128 ? (j & 3) << 2 : (j >> 1 & 1) << 2; };
    const char *const k_head = reinterpret_cast<const char *>(static_cast<const T *>(a.k) + k0 * a.k_token + hk * a.k_head);
    const char *const v_head = reinterpret_cast<const char *>(static_cast<const T *>(a.v) + k0 * a.v_token + hk * a.v_head);
    const uint32_t lds_k = (uint32_t)(size_t)(__attribute__((address_space(3))) void *)s_k, lds_v = (uint32_t)(size_t)(__attribute__((address_space(3))) void *)s_v;
    constexpr uint32_t TILE = kKeys * D * 2;  // bytes
    const uint32_t k_row = (uint32_t)a.k_token * 2, v_row = (uint32_t)a.v_token * 2;
    uint32_t k_at[LOADS], v_at[LOADS];
    const auto lane_offsets = [&](int last) {  // (rows behind `last`: that one once more; they are masked)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = 16 * wave + ROWS * i + lane / CHUNKS, p = lane % CHUNKS, from = min(r, last);
            k_at[i] = (uint32_t)from * k_row + 16 * (p ^ turn_k(r));
            v_at[i] = (uint32_t)from * v_row + 16 * (p ^ turn_v(r));
        }
    };
    const auto issue = [&](int t, int buf) {
        const char *const k = k_head + (long long)t * kKeys * a.k_token * 2, *const v = v_head + (long long)t * kKeys * a.v_token * 2;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load_to_lds(k_at[i], k, lds_k + buf * TILE + (16 * wave + ROWS * i) * (D * 2));
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load_to_lds(v_at[i], v, lds_v + buf * TILE + (16 * wave + ROWS * i) * (D * 2));
    };

    // this part's tiles of keys: from t down to t_last
    const int tiles_k = max((until + kKeys - 1) / kKeys, 0);
    const int t_last = (int)((unsigned)part * (unsigned)tiles_k / (unsigned)a.splits);
    int t = (int)((unsigned)(part + 1) * (unsigned)tiles_k / (unsigned)a.splits) - 1, buf = 0;
    if (t >= t_last) {
        lane_offsets(len_k - 1 - t * kKeys);
        issue(t, 0);
        lane_offsets(kKeys);
    }
    if (threadIdx.x == 0) s_odd = 0;

    vec<T, 8> q[D / 16];
    {
        const T *src = static_cast<const T *>(a.q) + (long long)(q0 + query) * a.q_token + head * a.q_head + 8 * h;
        const uint32_t sign = a.scale_log2 < 0.0f ? 0x80008000u : 0u;  // (the scale's)
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            u32x4 x = *reinterpret_cast<const u32x4 *>(src + 16 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] ^= sign;
            q[i] = __builtin_bit_cast(vec<T, 8>, x);
        }
    }
    const float scale = fmaxf(fabsf(a.scale_log2), 0x1p-126f);
    v16f o[D / 32] = {};
    float m = -__builtin_inff(), m_up = m, base = 0.0f, l = 0.0f;  // maximum (over scale), from where it moves, kWeightBits - m * scale; this lane's part of the sum

    // K fragment of 32 keys (u) for elements 16 i ..; V fragment of 16 keys (u) and elements 32 e ..
    const auto keys = [&](int u, int i) {
        const int j = 32 * u + n, c = 2 * i + h;
        return __builtin_bit_cast(vec<T, 8>, s_k[buf][j][c ^ turn_k(j)]);
    };
    const auto values = [&](int u, int e) {
        uint2 half[2];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int i = lane & 15, j = 16 * u + 8 * w + 4 * h + (i >> 2), c = 4 * e + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
            half[w] = read_transposed(reinterpret_cast<const char *>(&s_v[buf][j][c ^ turn_v(j)]) + 8 * (i & 1));
        }
        return __builtin_bit_cast(vec<T, 8>, u32x4{half[0].x, half[0].y, half[1].x, half[1].y});
    };
    // One tile.  CUT: some row of the block does not see all of its keys.
    const auto step = [&](auto cut, int key, bool careful) {
        constexpr bool CUT = decltype(cut)::value;
        // (the next fragments are read before the products of these: 2% on long prompts)
        v16f s[2] = {};
        vec<T, 8> frag[2][2] = {{keys(0, 0), keys(1, 0)}};
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            if (i + 1 < D / 16)
#pragma unroll
                for (int u = 0; u < 2; ++u) frag[(i + 1) & 1][u] = keys(u, i + 1);
#pragma unroll
            for (int u = 0; u < 2; ++u) s[u] = mfma32<T>(frag[i & 1][u], q[i], s[u]);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (CUT && key + kKeys > wave_all) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int j = key + 32 * u + 8 * (i >> 2) + 4 * h + (i & 3);
                    s[u][i] = j < limit ? s[u][i] : -__builtin_inff();
                }
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < 32; i += 2) top = max3(top, s[i >> 4][i & 15], s[i >> 4][(i & 15) + 1]);
        if (__any(top > m_up)) {  // (first of all: m is minus infinity)
            const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, top), __builtin_bit_cast(unsigned, top), false, false);
            top = fmaxf(__builtin_bit_cast(float, (unsigned)both[0]), __builtin_bit_cast(float, (unsigned)both[1]));
            top = top > m_up ? top : m;  // (a row's results go by its own scores alone)
            const float by = top == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((m - top) * scale);
            m = top;
            m_up = top == -__builtin_inff() ? top : top + (14.0f - kWeightBits) / scale;  // (a quotient of infinity: one maximum is enough)
            base = top == -__builtin_inff() ? 0.0f : kWeightBits - top * scale;
            l *= by;
#pragma unroll
            for (int e = 0; e < D / 32; ++e) o[e] *= by;
        }
        vec<T, 8> p[4];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 4][i & 15], scale, base));
            l += x;
            p[i >> 3][i & 7] = (T)x;
        }
        if (!CUT || !careful) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int e = 0; e < D / 32; ++e) o[e] = mfma32<T>(values(u, e), p[u], o[e]);
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int e = 0; e < D / 32; ++e) {
                    u32x4 x = __builtin_bit_cast(u32x4, values(u, e));
#pragma unroll
                    for (int w = 0; w < 4; ++w) x[w] &= ~((not_finite2<T>(x[w]) >> 15) * 0xffffu);
                    o[e] = mfma32<T>(__builtin_bit_cast(vec<T, 8>, x), p[u], o[e]);
                }
            for (int j = 0; j < kKeys; ++j) {
                const char *const at = reinterpret_cast<const char *>(s_v) + (buf * kKeys + j) * (D * 2) + 8 * h;
                const int turn = turn_v(j) << 4;
                const bool seen = key + j < limit;
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
                    const auto x = *reinterpret_cast<const vec<T, 4> *>(at + ((16 * c) ^ turn));
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float f = (float)x[r];
                        o[c >> 2][4 * (c & 3) + r] += seen && !(fabsf(f) < __builtin_inff()) ? f : 0.0f;
                    }
                }
            }
        }
    };

    // the tiles that are cut, with a look at their values
    for (; t >= t_last && (t + 1) * kKeys > block_all; --t, buf ^= 1) {
        wait_and_meet();  // (the tile is there, and all waves have read the one before it)
        uint32_t odd = 0;
#pragma unroll
        for (int i = 0; i < kKeys * CHUNKS / (64 * kPromptWaves); ++i) {
            const u32x4 x = (&s_v[buf][0][0])[i * 64 * kPromptWaves + (int)threadIdx.x];
#pragma unroll
            for (int e = 0; e < 4; ++e) odd |= not_finite2<T>(x[e]);
        }
        if (odd) s_odd = t + 1;
        wait_and_meet();
        if (t > t_last) issue(t - 1, buf ^ 1);
        if (any_row && t * kKeys < wave_any) step(std::true_type{}, t * kKeys, s_odd == t + 1);  // (else: no row of the wave sees any of them)
    }
    for (; t >= t_last; --t, buf ^= 1) {
        wait_and_meet();
        if (t > t_last) issue(t - 1, buf ^ 1);
        if (any_row) step(std::false_type{}, t * kKeys, false);
    }
    const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, l), __builtin_bit_cast(unsigned, l), false, false);
    l = __builtin_bit_cast(float, (unsigned)both[0]) + __builtin_bit_cast(float, (unsigned)both[1]);
    if (a.splits > 1) {
        // every part leaves its maxima, sums and unscaled results, past the L2s (the XCDs do not share them); the last to arrive at the
        // tile's ticket joins them, in their order
        constexpr int FLOATS = 64 * kPromptWaves * (D / 2 + 4);  // of a part
        float *const parts = a.parts + (size_t)whole * a.splits * FLOATS;
        const auto all = __builtin_amdgcn_make_buffer_rsrc(parts, 0, a.splits * FLOATS * 4, 0x00027000);
        const int none = row < rows ? 0 : a.splits * FLOATS * 4;  // (a lane without a row leaves and reads nothing)
        const auto at = [&](int p, int piece) { return (p * FLOATS + (piece * 64 * kPromptWaves + (int)threadIdx.x) * 4) * 4 + none; };
        constexpr int kShared = 16;  // sc1
#pragma unroll
        for (int e = 0; e < D / 32; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v4f{o[e][4 * i], o[e][4 * i + 1], o[e][4 * i + 2], o[e][4 * i + 3]}), all,
                                                       at(part, 4 * e + i), 0, kShared);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v4f{m, l, 0.0f, 0.0f}), all, at(part, D / 8), 0, kShared);
        wait_and_meet();
        if (threadIdx.x == 0) {
            const unsigned arrived = __hip_atomic_fetch_add(a.tickets + whole, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_odd = arrived == (unsigned)a.splits - 1;
            if (s_odd) __hip_atomic_store(a.tickets + whole, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        wait_and_meet();
        if (!s_odd) return;
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
            const float old = m == now ? 1.0f : __builtin_amdgcn_exp2f((m - now) * scale);
            const float by = ml[0] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((ml[0] - now) * scale);
            m = now;
            l = l * old + ml[1] * by;
#pragma unroll
            for (int e = 0; e < D / 32; ++e)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[e][i] = o[e][i] * old + x[4 * e + (i >> 2)][i & 3] * by;
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
// Parts of the keys, where the tiles of queries are fewer than the CUs: as many as give each CU a block.  A second one on a CU makes both nearly
// half as fast, and a part costs its tile's last block 1.2 us, about what 60 keys cost: two blocks a CU where the parts stay longer than
// 600 keys for each part that there is, and no more parts than parts of 60 keys for each.  `keys`: what a query sees on the average.  (FP16, 32/8 heads:
// 512 queries of two sequences over 6000 keys, one part 114 us, three 75, seven 85; 17 queries over 16000: one 258, eight 46.6, sixteen 36.5, 31
// 41; 200 queries over 3000: one 57, four 27.7, six 32.4; 200 queries, 64/8 heads, over 8000: two 83, four 73; 256 alone, 64/8 heads: one 11.1,
// two 13.7.)
int splits_of(long long blocks, int total_q, int total_k, int n_seqs)
{
    if (blocks < 1 || blocks > 256) return 1;
    const long long keys = std::max(total_k - total_q / 2, 0) / std::max(n_seqs, 1), one = 256 / blocks;
    return (int)std::max<long long>(1, std::min<long long>({keys > 600 * one * one ? 512 / blocks : one, (long long)std::sqrt((double)keys / 60.0), 32}));
}
// Tiles of a kv head, at most (more than 64 sequences: as they are searched for)
long long tiles_of(int total_q, int n_seqs, int group)
{
    const long long rows = (long long)total_q * group;
    return n_seqs <= kFew ? (rows + (long long)n_seqs * (kRows - 1)) / kRows : rows / kRows + n_seqs;
}
size_t part_bytes(int head_dim) { return sizeof(float) * 64 * kPromptWaves * (head_dim / 2 + 4); }
}  // namespace

extern "C" size_t attn_prompt_workspace_size(int n_seqs, int total_q, int total_k, int Hq, int Hkv, int head_dim)
{
    if (n_seqs < 1 || total_q < 1 || total_k < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv || !head_dim_ok(head_dim)) return 0;
    const long long blocks = tiles_of(total_q, n_seqs, Hq / Hkv) * Hkv;
    const int splits = splits_of(blocks, total_q, total_k, n_seqs);
    return splits == 1 ? 0 : kTickets + (size_t)blocks * splits * part_bytes(head_dim);
}

extern "C" int attn_prompt(int dtype, int n_seqs, int total_q, int total_k, int Hq, int Hkv, int head_dim, const void *q, long long q_token,
                           long long q_head, const void *k, long long k_token, long long k_head, const void *v, long long v_token,
                           long long v_head, const int *starts_q, const int *starts_k, float scale, int causal, void *out, void *workspace,
                           size_t workspace_bytes, void *hip_stream)
{
    if (dtype != LQ_F16 && dtype != LQ_BF16) return fail(LQ_ERR_INVALID, "dtype must be LQ_F16 or LQ_BF16, got %d", dtype);
    if (!head_dim_ok(head_dim)) return fail(LQ_ERR_INVALID, "head_dim must be 64 or 128, got %d", head_dim);
    if (n_seqs < 0 || n_seqs > (1 << 20) || total_q < 0 || total_q > (1 << 28) || total_k < 0 || Hkv < 1 || Hq < 1 || Hq > 4096 || Hq % Hkv)
        return fail(LQ_ERR_INVALID, "bad shape: %d sequences, %d queries, %d keys, %d heads, %d kv heads (heads a multiple of kv heads, up to 4096)",
                    n_seqs, total_q, total_k, Hq, Hkv);
    if (!(scale > -1e30f && scale < 1e30f)) return fail(LQ_ERR_INVALID, "scale must be finite");
    if (n_seqs == 0 || total_q == 0) return LQ_OK;
    if (!q || !out || !starts_q || !starts_k || (total_k && (!k || !v))) return fail(LQ_ERR_INVALID, "null pointer");
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)out | (uintptr_t)workspace) & 15)
        return fail(LQ_ERR_ALIGN, "q, k, v, out and workspace must be 16-byte aligned");
    if (((uintptr_t)starts_q | (uintptr_t)starts_k) & 3) return fail(LQ_ERR_ALIGN, "starts_q and starts_k must be 4-byte aligned");
    if ((total_q > 1 && q_token % 8) || (Hq > 1 && q_head % 8) || (total_k > 1 && (k_token % 8 || v_token % 8)) || (Hkv > 1 && (k_head % 8 || v_head % 8)))
        return fail(LQ_ERR_ALIGN, "strides must be multiples of 8 elements");
    if (total_k > 1 && (k_token < 0 || v_token < 0 || k_token > (1 << 24) || v_token > (1 << 24)))
        return fail(LQ_ERR_INVALID, "k and v: strides from token to token must be from 0 to 2^24 elements, got %lld and %lld", k_token, v_token);
    if (total_k <= 1) k_token = v_token = 0;
    const long long tiles = tiles_of(total_q, n_seqs, Hq / Hkv);
    if (tiles * Hkv > (1 << 23) || (long long)total_q * (Hq / Hkv) > (1 << 30)) return fail(LQ_ERR_INVALID, "too many rows: %d queries of %d sequences, %d heads", total_q, n_seqs, Hq);
    const size_t need = attn_prompt_workspace_size(n_seqs, total_q, total_k, Hq, Hkv, head_dim);
    const int splits = need && workspace && workspace_bytes >= need ? splits_of(tiles * Hkv, total_q, total_k, n_seqs) : 1;
    const PromptArgs a{q, k, v, q_token, q_head, k_token, k_head, v_token, v_head, starts_q, starts_k, out,
                       static_cast<unsigned *>(workspace), splits > 1 ? reinterpret_cast<float *>(static_cast<char *>(workspace) + kTickets) : nullptr,
                       n_seqs, total_q, total_k, Hq, Hkv, Hq / Hkv, causal != 0, (int)tiles, splits, scale * 1.44269504f};
    const dim3 grid((unsigned)((tiles * Hkv * splits + 7) / 8 * 8));
    (void)hipGetLastError();
    const WorkspaceTurn turn(splits > 1 ? workspace : nullptr, hip_stream);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * kPromptWaves), 0, static_cast<hipStream_t>(hip_stream), a); };
    if (dtype == LQ_F16)
        head_dim == 128 ? go(attn_prompt_kernel<128, f16>) : go(attn_prompt_kernel<64, f16>);
    else
        head_dim == 128 ? go(attn_prompt_kernel<128, bf16>) : go(attn_prompt_kernel<64, bf16>);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LQ_OK : fail(LQ_ERR_HIP, "attention launch failed: %s", hipGetErrorString(e));
}
