// Attention of chunks of new tokens over the 4-bit cache (page format: attn_common.h, its values: kvcache.hip): packed sequences, each with any
// number of new tokens that the cache holds already.
//
//     o_i = sum_j softmax_j(scale * q_i . k_j) v_j,   k_j = (code - z) * s of the key, v_j likewise,   j < context - n + 1 + i
// for new token i of a sequence's n.
//
// A block takes 128 rows, queries times the heads that share a kv head, a wave 32 of them; it goes through the keys from the last to the first, 64 at a
// time.  Their codes are loaded while the tile before the last is worked on, and unpacked into LDS next to the products of the tile before: a wave unpacks a
// quarter of them.  Both products run on 32x32x16 MFMAs with the cache as the first operand (S^T = K Q^T, O^T = V^T P^T): a lane's scores are 32
// keys of one row, in the order in which the weights enter the second product.  Value codes lie in a page as pairs of tokens, and so they are unpacked to
// [element][keys]: both operands come out of LDS in 16-byte reads.  Codes are masked out of their dword (5 instructions for 8) and go in as the subnormal FP16
// numbers that they then are, whose products the matrix cores form exactly (and cut, in sums of eight, below 2^-24 of the largest, in which a subnormal number counts as 2^-14: a
// key loses at most 2^-14 of the largest weight of its eight for each element); what the keys' zero points take off the scores is one more product, with the sum of a query's
// elements; the values' are taken off the codes (4 more instructions), as their sums may cancel.
//
// The scales never meet the codes.  The keys' are applied to the scores; the values' enter as logarithms,
//     t_j = scale * q . (code - z) * s_j + log2(sv_j),   x_j = 2^(t_j - m),   o = sum x_j (code - z) / sum x_j / sv_j,
// one fused multiply-add each, so that what is rounded to FP16 for the second product is a weight times its value's scale, relative to the largest
// such product (2^6 .. 2^14; what is below 2^-31 of the largest may vanish), and the values have no rounding at all.  sum x_j / sv_j stays in FP32's range for all
// scales there are, 2^-100 .. 2^124; but where the scales of a sequence are further apart than 2^100 an x_j may vanish whose weight counts, and the terms of the sum
// are taken from the scores without the values' scales instead.
//
// Tiles of at most 32 rows (single tokens, short chunks, ends of long ones) would leave three waves of four without products: there each wave has keys of its
// own, 32 at a time, straight from the cache into the operands' registers, and the waves' results are joined in LDS at the end.  (24 sequences, three of them
// chunks, 97 -> 73 us; 17 tokens of 517, 32 heads, 18.2 -> 15.6.)
//
// There, where the result is FP16, what the rounding of a weight leaves goes into the second product as a second number, so that a token has the same error as in a
// step of single tokens (attn_decode.hip): 2.1e-4 of the result, that of its own rounding, with one number 2.8 to 2.9e-4.  It costs 17 tokens of 517 12.5 -> 13.2 us, 64 single tokens over
// up to 4096, 32/8 heads, 51 -> 58, the 24 sequences 63.6 -> 64.5.  Tiles of more rows have one number a weight, as attn_prompt.hip's have: with two, chunks of FP16 take 2425 -> 3250 us
// (two of 2048 over up to 16384), the 24 sequences 76.  Beside the rounding of BF16 results neither shows (1.67e-3 for 1.66e-3).
//
// Heads of 64 leave room for three blocks a CU: two chunks of 2048 over up to 16384, 64/8 heads, 1516 us, with two 1620.  They have half the products of heads of 128 and the same
// softmax: vector instructions take 74% of a SIMD's cycles, MFMAs 34%, LDS 54% of a CU's (4096 tokens of two sequences over 16384 and 11253, BF16, 1206 us, 695 TFLOP/s).
// Measured, heads of 128 (by machine; the clock is 1.95 to 2.2 GHz under this load): two chunks of 2048 over up to 16384, 64/8 heads, BF16, 2210 to 2470 us (820 to 910
// TFLOP/s); 512 tokens over 1536 earlier ones, 32/8 heads, 39 us; 24 sequences with up to 4096 tokens, 640 new ones, 64; 17 of 517, 32/32 heads, 13.2.  A wave
// takes 34 MFMAs (1088 cycles) and 250 vector instructions with 34 exponentials or the like (1330) for 32 rows and 64 keys, and 56 reads of LDS of 16 bytes a lane
// (49% of its cycles, with the writes; none meet in a bank); two waves a SIMD make that in 2600 cycles each, so that MFMAs (43%) and vector instructions (51 to 57%) hardly overlap.  Tried, and slower or
// within 1% (2270 us beside them): two tiles of rows a wave with one wave a SIMD (3480 when this took 2660; halves the LDS reads); blocks of 8 waves and 256 rows, of which four
// unpack keys and four values (2524), the same half a tile apart with two barriers a tile (2461: a softmax alone takes a wave 2500 cycles, a quarter of them
// waiting for the keys' scales, and that is then the time of every half); fragments read two slices ahead; one of the two blocks of a CU ahead by priority; the maximum
// and the sum in four chains; the factors of the sum read before the maximum is known.
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
    int n_seqs, total_q, Hq, Hkv, group, width, pages, lg_page, tiles, slots;
    float scale_log2;
};

constexpr int kFew = 64, kLittle = 32, kLeast = 4, kKeys = 64, kWaves = 4, kRows = 32 * kWaves, kMostParts = 32;
constexpr float kWeightBits = 6.0f;
typedef f16 f16x2v __attribute__((ext_vector_type(2)));

__device__ __forceinline__ v16f mfma32(vec<f16, 8> a, vec<f16, 8> b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// 8 nibbles of a dword as 4 pairs of FP16 numbers: pair r = nibbles r and r + 4, which as subnormal numbers are 2^-24 of the code (r even) or
// 2^-20 of it (r odd)
__device__ __forceinline__ u32x4 halves8(uint32_t w)
{
    const uint32_t w8 = w >> 8;
    return u32x4{w & 0x000f000fu, w & 0x00f000f0u, w8 & 0x000f000fu, w8 & 0x00f000f0u};
}
// the same with the zero points of both halves taken off: exact, subnormal numbers all of them
__device__ __forceinline__ u32x4 halves8(uint32_t w, uint32_t zz)
{
    const u32x4 x = halves8(w);
    u32x4 o;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const uint32_t code = x[r], zero = r & 1 ? zz << 4 : zz;
        o[r] = __builtin_bit_cast(uint32_t, (f16x2v)(__builtin_bit_cast(f16x2v, code) - __builtin_bit_cast(f16x2v, zero)));
    }
    return o;
}

typedef __amdgpu_buffer_rsrc_t buf_t;
template <int N>
struct Dwords {
    uint32_t x[N];
    __device__ __forceinline__ void load(buf_t b, int lane_offset, int offset)
    {
        if constexpr (N == 4) {
            const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(b, lane_offset, offset, 0);
            x[0] = v[0], x[1] = v[1], x[2] = v[2], x[3] = v[3];
        } else if constexpr (N == 2) {
            const auto v = __builtin_amdgcn_raw_buffer_load_b64(b, lane_offset, offset, 0);
            x[0] = v[0], x[1] = v[1];
        } else {
            x[0] = __builtin_amdgcn_raw_buffer_load_b32(b, lane_offset, offset, 0);
        }
    }
};
// (not __syncthreads(): codes stay in flight)
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ int up(int a, int b) { return (int)(((unsigned)a + (unsigned)b - 1) / (unsigned)b); }

template <int D, class T>
__global__ __launch_bounds__(64 * kWaves, D == 64 ? 3 : 2) void kv4_chunks_kernel(const ChunkArgs a)
{
    constexpr int KW = kKeys / kWaves, DW = D / 32, STEPS = D / 16, W = D / 16;  // (a wave unpacks KW keys; a lane DW dwords of codes)
    constexpr bool kTwo = __is_same(T, f16);  // (two numbers a weight, in tiles of few rows)
    // Unpacked codes of two tiles (rows of keys are 16 bytes longer than they need be: lanes that read together meet in no bank); or, of a tile with
    // few rows, the waves' results
    struct Tiles {
        u32x4 k[2][kKeys][D / 8 + 1], v[2][D][kKeys / 8];
    };
    union Pool {
        Tiles tiles;
        float o[kWaves][32][D + 4];
    };
    __shared__ __attribute__((aligned(16))) Pool s_pool;
    auto &s_k = s_pool.tiles.k;
    auto &s_v = s_pool.tiles.v;
    __shared__ __attribute__((aligned(16))) float s_sk[4][kKeys], s_lv[4][kKeys], s_rv[4][kKeys], s_none[kKeys], s_row[kRows];
    __shared__ __attribute__((aligned(16))) uint32_t s_zk[4][kKeys];
    __shared__ __attribute__((aligned(16))) uint16_t s_zv[4][kKeys];
    __shared__ __attribute__((aligned(16))) int s_far[4][kWaves];  // scales that are far from 1, in a wave's keys of the tile (large ones: or before)
    __shared__ int s_bad, s_last, s_top;
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int P = 1 << a.lg_page, longest = a.width << a.lg_page;
    const auto within = [&](int context) { return min(max(context, 0), longest); };

    // The block's tile of rows and its part of the keys.  Up to 64 sequences: a lane looks at each; with a workspace (slots > 0) the tiles of a
    // sequence are cut into parts of at most `size` tiles of keys, the smallest size with which all parts run at a time.  More sequences are searched for
    // as in attn_prompt.hip, and their keys are not cut (8/1 heads, one context of 32768 among single tokens over 1024: 64 sequences 20 us, 65 252).
    const auto start_of = [&](int s) { return min(max(a.starts[s], 0), a.total_q); };
    const bool few = a.n_seqs <= kFew;
    int from = 0, len = 0, context = 0, mine = 0, parts = 1, upto = 0, all = a.tiles;
    if (few) {
        if (lane < a.n_seqs) {
            from = start_of(lane);
            len = max(min(a.starts[lane + 1], a.total_q) - from, 0);
            context = a.context[lane];
            mine = up(len * a.group, kRows);
        }
        const bool little = len * a.group <= kLittle;
        const int keys = up(within(context), little ? 4 * kKeys : kKeys);  // tiles of keys, by what they cost
        all = __builtin_amdgcn_readlane(sums_up_to(mine), 63);
        if (all > a.tiles) {  // (more than there can be: the sequences overlap)
            mine = min(mine, a.tiles / a.n_seqs);
            all = __builtin_amdgcn_readlane(sums_up_to(mine), 63);
        }
        if (a.slots > all * a.Hkv) {
            const int most = a.slots / a.Hkv;  // parts of a kv head
            // Joining a part costs about what a tile of keys does (1.4 us: 68 KB from behind the L2 for one CU), so that parts and tiles of each are as many.  (One
            // sequence of 2048 keys, 32/8 heads, 128 new tokens, tiles of a part: 2 42.5 us, 6 25.0, 9 27.5, 17 39.0; of 16384, 64 new ones: 8 76, 16 50.9, 24 59.1, 48
            // 85.8; of 1024, 64/8 heads, 64 new ones: 2 21.7, 4 21.1, 8 26.1.)  Few rows: from 1024 keys on (17 tokens of 517, 32 heads: one part 13.8 us, two 16.0,
            // three 15.8).
            const int least = little ? kLeast : max(2, (int)__builtin_sqrtf((float)keys));
            int size = max(up(__builtin_amdgcn_readlane(sums_up_to(mine * min(keys, 1 << 16)), 63), most), 1), sum;
            do {
                parts = min(max(up(keys, max(size, least)), 1), kMostParts);
                sum = __builtin_amdgcn_readlane(sums_up_to(mine * parts), 63);
                size += up(size, 8);
            } while (sum > most);  // (one part each fits, and comes before size overflows: keys is below 2^24)
            all = sum;
        }
        // Those of few rows come last: they are short, and fill what the others leave (a mixed step 67 -> 63 us)
        const int upto_long = sums_up_to(little ? 0 : mine * parts), upto_short = sums_up_to(little ? mine * parts : 0);
        upto = little ? __builtin_amdgcn_readlane(upto_long, 63) + upto_short : upto_long;
    }
    // Blocks with ids 8 apart run on one XCD: each XCD gets consecutive kv heads, and goes through a sequence's tiles from the last (the longest rows of
    // keys) to the first.  Blocks that the grid has too many come last.
    const int blocks = all * a.Hkv, per = (blocks + 7) >> 3, id = ((int)blockIdx.x & 7) * per + ((int)blockIdx.x >> 3);
    if ((int)blockIdx.x >> 3 >= per || id >= blocks) return;
    const int hk = __builtin_amdgcn_readfirstlane(id / all);
    int tile = few ? id % all : all - 1 - id % all, part = 0, n_parts = 1, seq, q0, len_q, whole = 0;
    if (few) {
        const int start = upto - mine * parts;
        seq = __builtin_ctzll(__ballot(start <= tile && upto > tile) | 1ull << 63);
        q0 = __builtin_amdgcn_readlane(from, seq);
        len_q = __builtin_amdgcn_readlane(len, seq);
        n_parts = __builtin_amdgcn_readlane(parts, seq);
        whole = hk * all + __builtin_amdgcn_readlane(start, seq);  // (the sequence's first part)
        tile -= whole - hk * all;
        part = tile % n_parts;
        tile = __builtin_amdgcn_readlane(mine, seq) - 1 - tile / n_parts;  // (the longest rows of keys first)
        whole += tile * n_parts;  // the tile's first part: its place in the workspace, and its ticket
        context = __builtin_amdgcn_readlane(context, seq);
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
        len_q = __builtin_amdgcn_readfirstlane(max(min(a.starts[seq + 1], a.total_q) - q0, 0));
        tile -= __builtin_amdgcn_readfirstlane(first_tile(seq));
        context = __builtin_amdgcn_readfirstlane(a.context[seq]);
    }
    const auto uniform = [](int &x) { x = __builtin_amdgcn_readfirstlane(x); };
    uniform(tile), uniform(part), uniform(n_parts), uniform(seq), uniform(q0), uniform(len_q), uniform(whole), uniform(context);
    if (tile < 0 || tile * kRows >= len_q * a.group) return;

    const int ctx = within(context), first = tile * kRows, rows = len_q * a.group, before = ctx - len_q;
    const auto sees = [&](int r) { return min(r, rows - 1) / a.group + before + 1; };  // keys (none where it is not above 0)
    const bool little = rows - first <= kLittle;  // all waves have the same rows, and keys of their own
    const int row = first + (little ? 0 : 32 * wave) + n, limit = sees(row), wave_all = __builtin_amdgcn_readfirstlane(sees(row - n));
    const bool any_row = first + 32 * wave < rows;
    // (computed again where it is needed again: registers that the loops do not have)
    const auto thread_again = []() __attribute__((always_inline)) {
        int thread = threadIdx.x;
        asm volatile("" : "+v"(thread));
        return thread;
    };
    const auto row_of = [&](int thread) { return first + (little ? 0 : 32 * wave) + (thread & 31); };

    // this part's tiles of keys: n_tiles of them, from t_first down (place p: tile t_first - p)
    const int tiles_k = __builtin_amdgcn_readfirstlane(max((sees(first + kRows - 1) + kKeys - 1) / kKeys, 0));
    const int t_first = (int)((unsigned)(part + 1) * (unsigned)tiles_k / (unsigned)n_parts) - 1;
    const int n_tiles = t_first + 1 - (int)((unsigned)part * (unsigned)tiles_k / (unsigned)n_parts);

    // the codes of this wave's keys of a tile: all from one page
    typedef const __attribute__((address_space(4))) int *ints;
    const ints table = (ints)(uintptr_t)(a.table + (size_t)seq * a.width);
    const unsigned page_bytes = (unsigned)a.Hkv * (unsigned)kv4_head_bytes(P, D);
    const uint8_t *const cache = a.cache + (size_t)hk * kv4_head_bytes(P, D);
    const int last_page = max((ctx - 1) >> a.lg_page, 0), keys_w = KW * wave;
    bool bad = context > longest, large = false;
    const auto page_of = [&](int p) __attribute__((always_inline)) { return (unsigned)table[min((max(t_first - p, 0) * kKeys + keys_w) >> a.lg_page, last_page)]; };
    const auto page_at = [&](int p, unsigned page) __attribute__((always_inline)) {
        const bool any = p < n_tiles, out_of_range = page >= (unsigned)a.pages;
        bad |= any && out_of_range;
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(cache + (uint64_t)(out_of_range ? 0u : page) * page_bytes), 0,
                                                 any ? kv4_head_bytes(P, D) : 0, 0x00027000);
    };
    Dwords<DW> ck, cv;
    uint32_t wk, wv;  // words of the lane's key, of its keys and its values
    // The lane's four keys and column group of the values (heads of 128: 16 lanes that write together have both halves of 8 pieces; for 64 it takes the register
    // that the third block of a CU needs)
    const int four = D == 128 ? (lane >> 2 & 2) | lane >> 5 : lane >> 4, column = D == 128 ? (lane & 7) | (lane >> 1 & 8) : lane & 15;
    const auto load_keys = [&](int p, unsigned page) __attribute__((always_inline)) {
        const buf_t b = page_at(p, page);
        const int j = ((t_first - p) * kKeys + keys_w) & (P - 1);
        ck.load(b, lane * (4 * DW), j * (D / 2));
        wk = __builtin_amdgcn_raw_buffer_load_b32(b, 4 * column, P * D + 4 * j, 0);
        wv = __builtin_amdgcn_raw_buffer_load_b32(b, 4 * column, P * (D + 4) + 4 * j, 0);
    };
    const auto load_values = [&](int p, unsigned page) __attribute__((always_inline)) {
        const buf_t b = page_at(p, page);
        const int j = ((t_first - p) * kKeys + keys_w) & (P - 1);
        cv.load(b, (D == 128 ? 16 * four + column : lane) * (4 * DW), (P + j) * (D / 2));
    };

    vec<f16, 8> q[STEPS + 1];
    float q_scale = fabsf(a.scale_log2);
    bool uneven = false;
    // (heads of 128: pieces 8 on lie at their number XOR 2, so that the eight lanes of two keys that write together meet in no bank)
    const int turn_k = D == 128 ? lane & 2 : 0, piece_low = DW * (lane & 3) + turn_k, piece_high = DW * (lane & 3) - turn_k;
    const auto unpack_keys = [&](int buf, int i) __attribute__((always_inline)) {
        s_k[buf][keys_w + (lane >> 2)][(i & 2 ? piece_high : piece_low) + i] = halves8(ck.x[i]);
    };
    // Values: [element][key]; a row's 16-byte pieces have the keys that a half of the lanes multiplies at once (two fours, 8 keys apart), and lie at
    // their number XOR turn_v
    const auto turn_v = [](int d) { return ((d >> 1) ^ (d >> 4)) & 7; };
    const auto unpack_values = [&](int buf, int slot, int i) __attribute__((always_inline)) {
        const uint2 zz = *reinterpret_cast<const uint2 *>(&s_zv[slot][keys_w + 4 * four]);
        const u32x4 o[2] = {halves8(cv.x[i], zz.x), halves8(cv.x[W / 4 + i], zz.y)};
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = W * column + 4 * i + r;
            reinterpret_cast<uint2 *>(&s_v[buf][d][(2 * wave + (four & 1)) ^ turn_v(d)])[four >> 1] = uint2{o[0][r], o[1][r]};
        }
    };
    const auto scales = [&](int slot, int key_w) __attribute__((always_inline)) {  // (lanes that have the same key write the same)
        const uint32_t word_k = wk & kScaleMask, word_v = wv & kScaleMask, z = wk & 15u;
        const float sk = __builtin_bit_cast(float, word_k) * q_scale;
        float sv = __builtin_bit_cast(float, word_v);
        sv = sv < 0x1p-100f ? 0x1p-100f : sv;                // (NaN stays; a place that nothing was written to counts as zeros)
        s_sk[slot][key_w] = sk > 0x1p127f ? 0x1p127f : sk;   // (here, too)
        s_zk[slot][key_w] = z | z << 16;
        s_zv[slot][key_w] = (uint16_t)(wv & 15u);
        s_lv[slot][key_w] = __builtin_amdgcn_logf(sv);
        s_rv[slot][key_w] = sv > 0.0f ? __builtin_amdgcn_rcpf(sv) : 0.0f;  // (of NaN 0: who does not see it has no part of it)
        large |= __any(sv > 0x1p60f);
        return (int)large | (int)__any(sv < 0x1p-40f);
    };
    // An eighth of what a wave unpacks next to the products of place p + 1: keys of place p + 2 (into p's buffer) and all its scales, values of place p + 1
    const auto unpack_part = [&](int p, int j) __attribute__((always_inline)) {
        if (j < DW) unpack_keys(p & 1, j);
        if (j == 4) s_far[(p + 2) & 3][wave] = scales((p + 2) & 3, keys_w + column);
        if (j >= 5 && j - 5 < W / 4) unpack_values(~p & 1, (p + 1) & 3, j - 5);
    };
    const auto next_loads = [&](int p, unsigned &page) __attribute__((always_inline)) {
        load_values(p + 2, page);
        page = page_of(p + 3);
        load_keys(p + 3, page);
    };

    // Fragments: 32 keys (u) of 16 elements (i); 32 elements (e) of 16 keys (u).  (Rows 32 apart turn their pieces alike, but for 2 e of the values'.)
    int v_at[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) v_at[x] = n * (kKeys / 8) + ((2 * x + h) ^ turn_v(n));
    const auto keys = [&](int buf, int u, int i) { return __builtin_bit_cast(vec<f16, 8>, s_k[buf][32 * u + n][(2 * i ^ (D == 128 && i >= STEPS / 2 ? 2 : 0)) + h]); };
    const auto values = [&](int buf, int u, int e) { return __builtin_bit_cast(vec<f16, 8>, (&s_v[buf][32 * e][0])[v_at[u ^ e]]); };
    const auto zeros = [&](int slot, int u) {
        const uint32_t zz = s_zk[slot][32 * u + n];
        return __builtin_bit_cast(vec<f16, 8>, u32x4{zz, zz, 0, 0});
    };

    v16f o[D / 32], s[2];
    vec<f16, 8> w[4], rest[2];  // weights as FP16 numbers, and what the rounding leaves of them
    float m = -__builtin_inff(), l = 0.0f;  // maximum of t, this lane's part of sum x / sv
    // The softmax of place p's scores: s -> w, l, m
    const auto softmax = [&](int slot, int key, int limit, bool far, auto n_u) __attribute__((always_inline)) {
        constexpr int U = decltype(n_u)::value;  // times 32 keys
        const auto at = [&](int i) { return 32 * (i >> 2) + 8 * (i & 3) + 4 * h; };  // the lane's keys 4 i ..
        if (uneven) {
            asm volatile("s_nop 0");  // (kept a branch)
#pragma unroll
            for (int u = 0; u < U; ++u) s[u] *= s_row[row - first];
        }
#pragma unroll
        for (int i = 0; i < 4 * U; ++i) {
            const v4f sk = *reinterpret_cast<const v4f *>(&s_sk[slot][at(i)]), lv = *reinterpret_cast<const v4f *>(&s_lv[slot][at(i)]);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[i >> 2][4 * (i & 3) + e] = __builtin_fmaf(s[i >> 2][4 * (i & 3) + e], sk[e], lv[e]);
        }
        if (key + 32 * U > wave_all) {  // some row of the wave does not see all of these keys
            const int seen = limit - key - 4 * h;  // of the keys that a lane has from 4 h on
            asm volatile("s_nop 0");
#pragma unroll
            for (int i = 0; i < 16 * U; ++i) s[i >> 4][i & 15] = 8 * (i >> 2) + (i & 3) < seen ? s[i >> 4][i & 15] : -__builtin_inff();
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < 16 * U; i += 2) top = fmaxf(fmaxf(top, s[i >> 4][i & 15]), s[i >> 4][(i & 15) + 1]);
        constexpr float kUp = 14.0f - kWeightBits;  // (from where the maximum moves)
        if (__any(top > m + kUp)) {                 // (first of all: m is minus infinity)
            const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, top), __builtin_bit_cast(unsigned, top), false, false);
            top = fmaxf(__builtin_bit_cast(float, (unsigned)both[0]), __builtin_bit_cast(float, (unsigned)both[1]));
            top = top > m + kUp ? top : m;  // (a row's results go by its own scores alone)
            // (in two steps for l: a factor of 2^-200 may still leave something of a sum that is 2^100)
            const float half = top == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((m - top) * 0.5f), by = half * half;
            m = top;
            l = l * half * half;
#pragma unroll
            for (int e = 0; e < D / 32; ++e) o[e] *= by;
        }
        const float base = m == -__builtin_inff() ? 0.0f : kWeightBits - m, *sums = s_rv[slot];
        if (far) {
            // the sum from the scores themselves (2^16 of it, which is 2^-130 .. 2^122); the factors below are then zeros
#pragma unroll
            for (int i = 0; i < 4 * U; ++i) {
                const v4f lv = *reinterpret_cast<const v4f *>(&s_lv[slot][at(i)]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = s[i >> 2][4 * (i & 3) + e], whole = __builtin_amdgcn_exp2f(x - lv[e] + (base + 16.0f));
                    l = __builtin_fmaf(x == -__builtin_inff() ? 0.0f : whole, 0x1p-16f, l);  // (whatever is there)
                }
            }
            sums = s_none;
        }
#pragma unroll
        for (int i = 0; i < 4 * U; ++i) {
            const v4f rv = *reinterpret_cast<const v4f *>(&sums[at(i)]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = __builtin_amdgcn_exp2f(s[i >> 2][4 * (i & 3) + e] + base);
                const f16 y = (f16)x;
                l = __builtin_fmaf(x, rv[e], l);
                w[i >> 1][4 * (i & 1) + e] = y;
                if constexpr (U == 1 && kTwo) rest[i >> 1][4 * (i & 1) + e] = (f16)__builtin_fmaf((float)y, -1.0f, x);
            }
        }
        if constexpr (U == 2) asm volatile("" : "+v"(l), "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));  // (here, not among the products, where the scores would have to stay)
    };
    // The second product of place p and the first one of place p + 1, next to which the codes behind them are unpacked: eight slices, whose fragments are read
    // one slice ahead.  The order is that of the statements between scheduling barriers.
    const auto products = [&](int p) __attribute__((always_inline)) {
        constexpr int E = D / 64;
        const int buf = p & 1;
        vec<f16, 8> kf[2][2], vf[2][E];
        const auto fragments = [&](int j) __attribute__((always_inline)) {
            if (j * STEPS % 8 == 0)
#pragma unroll
                for (int u = 0; u < 2; ++u) kf[j * STEPS / 8 & 1][u] = keys(buf ^ 1, u, j * STEPS / 8);
#pragma unroll
            for (int e = 0; e < E; ++e) vf[j & 1][e] = values(buf, j >> 1, (j & 1) * E + e);
        };
#pragma unroll
        for (int u = 0; u < 2; ++u) s[u] = mfma32(zeros((p + 1) & 3, u), q[STEPS], v16f{});
        fragments(0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = j * STEPS / 8;
            if (j < 7) fragments(j + 1);
            if (j * STEPS % 8 == 0)
#pragma unroll
                for (int u = 0; u < 2; ++u) s[u] = mfma32(kf[i & 1][u], q[i], s[u]);
#pragma unroll
            for (int e = 0; e < E; ++e) o[(j & 1) * E + e] = mfma32(vf[j & 1][e], w[j >> 1], o[(j & 1) * E + e]);
            unpack_part(p, j);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    // Results: a row's, and where a part of the keys leaves what it has (a lane without a row leaves and reads nothing)
    const auto write_row = [&]() __attribute__((always_inline)) {
        const float by = l == 0.0f ? 0.0f : 1.0f / l;
        const int thread = thread_again(), row = row_of(thread), h = thread >> 5 & 1;
        T *const dst = static_cast<T *>(a.out) + ((size_t)(q0 + row / a.group) * a.Hq + hk * a.group + row % a.group) * D;
        if (row >= rows) return;
#pragma unroll
        for (int e = 0; e < D / 32; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                vec<T, 4> y;
#pragma unroll
                for (int x = 0; x < 4; ++x) y[x] = (T)(o[e][4 * i + x] * (x & 1 ? 0x1p20f : 0x1p24f) * by);
                *reinterpret_cast<vec<T, 4> *>(dst + 32 * e + 8 * i + 4 * h) = y;
            }
    };
    constexpr int FLOATS = 64 * kWaves * (D / 2 + 4), kShared = 16;  // of a part; sc1
    const auto left_parts = __builtin_amdgcn_make_buffer_rsrc(a.parts + (size_t)whole * FLOATS, 0, n_parts * FLOATS * 4, 0x00027000);

    // Tiles of few rows: of 32 keys, a wave's own, which go from the cache into the products as they are: lane n, h has key n's dwords STEPS h on, and for
    // the second product elements D / 32 n on of the four keys 8 g + 4 h of both halves.
    const int tiles32 = __builtin_amdgcn_readfirstlane(max((sees(first + kLittle - 1) + 31) / 32, 0));
    const int from32 = (int)((unsigned)part * (unsigned)tiles32 / (unsigned)n_parts);
    int t = (int)((unsigned)(part + 1) * (unsigned)tiles32 / (unsigned)n_parts) - 1 - wave;
    const auto pages_of = [&](int t, int u) __attribute__((always_inline)) { return (unsigned)table[min((max(t, 0) * 32 + 16 * u) >> a.lg_page, last_page)]; };
    const auto head_of = [&](unsigned page) __attribute__((always_inline)) { return cache + (uint64_t)(page >= (unsigned)a.pages ? 0u : page) * page_bytes; };
    const auto place_of = [&](int t, int u) { return (max(t, 0) * 32 + 16 * u) & (P - 1); };
    uint32_t k[STEPS], v[2][2][2];
    unsigned pages[2];
    const auto load_own = [&](int t) __attribute__((always_inline)) {  // (of a tile that is not there: the first page's keys, which all waves have at hand)
        const bool any = t >= from32;
        const uint8_t *const head0 = any ? head_of(pages[0]) : cache, *const head1 = any ? head_of(pages[1]) : cache, *const head = n & 16 ? head1 : head0;
        const int j = (n & 16 ? place_of(t, 1) : place_of(t, 0)) + (n & 15);
        bad |= any && (pages[0] >= (unsigned)a.pages || pages[1] >= (unsigned)a.pages);
#pragma unroll
        for (int i = 0; i < STEPS; i += 4) {
            const u32x4 x = *reinterpret_cast<const u32x4 *>(head + j * (D / 2) + h * (D / 4) + 4 * i);
            k[i] = x[0], k[i + 1] = x[1], k[i + 2] = x[2], k[i + 3] = x[3];
        }
        wk = *reinterpret_cast<const uint32_t *>(head + P * D + 4 * j);
        wv = *reinterpret_cast<const uint32_t *>(head + P * (D + 4) + 4 * j);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const buf_t b = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(u ? head1 : head0), 0, any ? kv4_head_bytes(P, D) : 0, 0x00027000);
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const int at = (2 * g + h) * (2 * D) + (n >> 1) * (D / 8) + (D == 128 ? 4 * (n & 1) : 0), piece = (P + place_of(t, u)) * (D / 2);
                v[u][g][0] = __builtin_amdgcn_raw_buffer_load_b32(b, at, piece, 0);
                v[u][g][1] = __builtin_amdgcn_raw_buffer_load_b32(b, at + D / 16, piece, 0);
            }
        }
    };
    // (the first loads, before those of the queries)
    unsigned page = 0;
    if (little) {
        pages[0] = pages_of(t, 0), pages[1] = pages_of(t, 1);
        load_own(t);
        pages[0] = pages_of(t - kWaves, 0), pages[1] = pages_of(t - kWaves, 1);
    } else if (n_tiles > 0) {
        page = page_of(0);
        load_keys(0, page);
        load_values(0, page);
    }

    if (threadIdx.x == 0) s_bad = s_top = 0;
    s_none[lane] = 0.0f;
    // Queries, in the keys' order within 8 elements (a pair of a dword's nibbles is four apart), over a power of two for the block that brings its
    // largest element to 4 .. 8, what meets even pairs times 16: what is above 2^-17 of the largest is held exactly.  A row whose largest element is below
    // 2^-8 of the block's has a power of its own, and a factor for its scores.  A last operand holds what the zero points are multiplied with, minus 16 times
    // the sum of the row's elements, as three numbers (33 bits of it).
    {
        float f[STEPS][8];
        int most = 0;  // bits of the row's largest finite element
        {
            const int at = min(row, rows - 1);
            const T *src = static_cast<const T *>(a.q) + (long long)(q0 + at / a.group) * a.q_token + (hk * a.group + at % a.group) * a.q_head + (little ? D / 2 : 8) * h;
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const u32x4 raw = *reinterpret_cast<const u32x4 *>(src + (little ? 8 : 16) * i);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (__is_same(T, f16))
                        f[i][e] = (float)__builtin_bit_cast(vec<f16, 8>, raw)[e];
                    else
                        f[i][e] = __builtin_bit_cast(float, e & 1 ? raw[e >> 1] & 0xffff0000u : raw[e >> 1] << 16);
                    const int bits = __builtin_bit_cast(int, f[i][e]) & 0x7fffffff;
                    most = max(most, bits < 0x7f800000 ? bits : 0);
                }
            }
        }
        const auto both = __builtin_amdgcn_permlane32_swap((unsigned)most, (unsigned)most, false, false);
        most = max((int)both[0], (int)both[1]);
        int top_bits = __builtin_amdgcn_readlane(lanes_up_to(row < rows ? most : 0, [](int x, int y) { return max(x, y); }), 63);
        if (!little) {
            meet();
            if (lane == 0) atomicMax(&s_top, top_bits);
            meet();
            top_bits = __builtin_amdgcn_readfirstlane(s_top);
        }
        const auto exponent = [](int bits) { return max(bits >> 23, 1) - 129; };
        const int top = exponent(top_bits), own = most && exponent(most) < top - 8 ? exponent(most) : top;
        q_scale = fminf(fmaxf(q_scale * 0x1p20f * power_of_two(max(top, -126)), 0x1p-126f), 0x1p127f);
        s_row[row - first] = power_of_two(max(own - top, -126));
        uneven = __any(own != top);
        const float by0 = power_of_two(-own / 2) * (a.scale_log2 < 0.0f ? -1.0f : 1.0f), by1 = power_of_two(-own - -own / 2);  // (up to 2^128: in two steps)
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const f16 x = (f16)(f[i][e] * by0 * by1);
                sum += (float)x;
                q[i][2 * (e & 3) + (e >> 2)] = e & 1 ? x : x * (f16)16.0f;
            }
        const auto halves = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, sum), __builtin_bit_cast(unsigned, sum), false, false);
        sum = -16.0f * (__builtin_bit_cast(float, (unsigned)halves[0]) + __builtin_bit_cast(float, (unsigned)halves[1]));
        const f16 s0 = (f16)sum, s1 = (f16)(sum - (float)s0), s2 = (f16)(sum - (float)s0 - (float)s1);
        q[STEPS] = vec<f16, 8>{};
        if (h == 0) q[STEPS][0] = s0, q[STEPS][1] = s1, q[STEPS][2] = s2;
    }
#pragma unroll
    for (int e = 0; e < D / 32; ++e) o[e] = v16f{};
    if (little) {
        const int limit_again = sees(row_of(thread_again()));
        for (; t >= from32; t -= kWaves) {
            uint32_t v_now[2][2][2];
#pragma unroll
            for (int i = 0; i < 8; ++i) v_now[i >> 2][i >> 1 & 1][i & 1] = v[i >> 2][i >> 1 & 1][i & 1];
            const uint32_t zz = (wk & 15u) * 0x10001u;
            s[0] = mfma32(__builtin_bit_cast(vec<f16, 8>, u32x4{zz, zz, 0, 0}), q[STEPS], v16f{});
#pragma unroll
            for (int i = 0; i < STEPS; ++i) s[0] = mfma32(__builtin_bit_cast(vec<f16, 8>, halves8(k[i])), q[i], s[0]);
            asm volatile("" ::: "memory");  // (written and read by one wave, in the order that stands here, and as other types)
            const bool far = scales(wave, n);
            asm volatile("" ::: "memory");
            load_own(t - kWaves);
            pages[0] = pages_of(t - 2 * kWaves, 0), pages[1] = pages_of(t - 2 * kWaves, 1);
            softmax(wave, 32 * t, limit_again, far, std::integral_constant<int, 1>{});
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                u32x4 x[2][2];  // of four keys: pairs of them, elements
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const uint2 z4 = *reinterpret_cast<const uint2 *>(&s_zv[wave][16 * u + 8 * g + 4 * h]);
#pragma unroll
                    for (int i = 0; i < 2; ++i) x[g][i] = halves8(D == 128 ? v_now[u][g][i] : v_now[u][g][i] >> (8 * (n & 1)), i ? z4.y : z4.x);
                }
#pragma unroll
                for (int e = 0; e < D / 32; ++e) {
                    const auto codes = __builtin_bit_cast(vec<f16, 8>, u32x4{x[0][0][e], x[0][1][e], x[1][0][e], x[1][1][e]});
                    o[e] = mfma32(codes, w[u], o[e]);
                    if constexpr (kTwo) o[e] = mfma32(codes, rest[u], o[e]);
                }
            }
        }
    } else if (n_tiles > 0) {
        // the first two tiles' keys and scales, the first one's values
#pragma unroll
        for (int i = 0; i < DW; ++i) unpack_keys(0, i);
        s_far[0][wave] = scales(0, keys_w + column);
        page = page_of(1);
        load_keys(1, page);
        meet();  // (a wave writes the zero points that it reads, but the compiler has to know)
#pragma unroll
        for (int i = 0; i < W / 4; ++i) unpack_values(0, 0, i);
        load_values(1, page);
#pragma unroll
        for (int i = 0; i < DW; ++i) unpack_keys(1, i);
        s_far[1][wave] = scales(1, keys_w + column);
        page = page_of(2);
        load_keys(2, page);
        meet();
        if (any_row) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                s[u] = mfma32(zeros(0, u), q[STEPS], v16f{});
#pragma unroll
                for (int i = 0; i < STEPS; ++i) s[u] = mfma32(keys(0, u, i), q[i], s[u]);
            }
            // (what has products to issue goes first: 2332 -> 2294 us for two chunks of 2048, a mixed step 72 -> 68)
            for (int p = 0; p < n_tiles; ++p) {
                const v4i far = *reinterpret_cast<const v4i *>(s_far[p & 3]);
                softmax(p & 3, (t_first - p) * kKeys, limit, __builtin_amdgcn_readfirstlane(far[0] | far[1] | far[2] | far[3]), std::integral_constant<int, 2>{});
                meet();  // (what the next products read is there, and all waves are done with what they write over)
                __builtin_amdgcn_s_setprio(1);
                products(p);
                __builtin_amdgcn_s_setprio(0);
                next_loads(p, page);
            }
        } else {
            for (int p = 0; p < n_tiles; ++p) {
                meet();
#pragma unroll
                for (int j = 0; j < 8; ++j) unpack_part(p, j);
                next_loads(p, page);
            }
        }
    }
    if (!little) {
        if (bad) s_bad = 1;
        meet();
        bad = s_bad;
    }
    const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, l), __builtin_bit_cast(unsigned, l), false, false);
    l = __builtin_bit_cast(float, (unsigned)both[0]) + __builtin_bit_cast(float, (unsigned)both[1]);
    if (bad) l = __builtin_nanf("");
    // Every part leaves its maxima, sums and results, past the L2s; the last to arrive at the tile's ticket joins them, in their order
    const auto last_to_arrive = [&]() __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (threadIdx.x == 0) {
            const unsigned arrived = __hip_atomic_fetch_add(a.tickets + whole, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_last = arrived == (unsigned)n_parts - 1;
            if (s_last) __hip_atomic_store(a.tickets + whole, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        return __builtin_amdgcn_readfirstlane(s_last) != 0;
    };
    // what a maximum that moves to top takes off, as the root of it: a sum takes it in two steps (as above)
    const auto root_of = [](float m, float top) { return m == top ? 1.0f : __builtin_amdgcn_exp2f((m - top) * 0.5f); };
    if (little) {
        // the waves' results, and those of the parts: a thread has pieces of four elements of the rows
        if (h == 0) s_lv[wave][n] = m, s_rv[wave][n] = l;
        const auto top_of = [&](int r) { return fmaxf(fmaxf(s_lv[0][r], s_lv[1][r]), fmaxf(s_lv[2][r], s_lv[3][r])); };
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            vec<float, D / 32> x;
#pragma unroll
            for (int e = 0; e < D / 32; ++e) x[e] = o[e][i];
            *reinterpret_cast<vec<float, D / 32> *>(&s_pool.o[wave][n][(D / 32) * (8 * (i >> 2) + 4 * h + (i & 3))]) = x;
        }
        meet();
        constexpr int PIECES = D / 32, STRIDE = D + 4;
        const auto write = [&](int r, int c, v4f x, float l) __attribute__((always_inline)) {
            const float by = l == 0.0f ? 0.0f : 1.0f / l;
            vec<T, 4> y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (T)(x[e] * (e & 1 ? 0x1p20f : 0x1p24f) * by);
            const int at = first + r;
            if (at < rows) *reinterpret_cast<vec<T, 4> *>(static_cast<T *>(a.out) + ((size_t)(q0 + at / a.group) * a.Hq + hk * a.group + at % a.group) * D + 4 * c) = y;
        };
        const auto place = [&](int i, int &r, int &c) { r = ((int)threadIdx.x + 64 * kWaves * i) / (D / 4), c = ((int)threadIdx.x + 64 * kWaves * i) % (D / 4); };
        const auto at_part = [&](int p, int r, int c) { return first + r < rows && p < n_parts ? (p * FLOATS + r * STRIDE + 4 * c) * 4 : n_parts * FLOATS * 4; };
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            int r, c;
            place(i, r, c);
            const float top = top_of(r);
            v4f x{};
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                const float root = root_of(s_lv[k][r], top);
                sum += s_rv[k][r] * root * root;
                x += *reinterpret_cast<const v4f *>(&s_pool.o[k][r][4 * c]) * (root * root);
            }
            if (n_parts == 1) {
                write(r, c, x, sum);
                continue;
            }
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), left_parts, at_part(part, r, c), 0, kShared);
            if (c == 0) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v4f{top, sum, 0.0f, 0.0f}), left_parts, at_part(part, r, D / 4), 0, kShared);
        }
        if (n_parts == 1 || !last_to_arrive()) return;
        constexpr int kAtOnce = 8;  // parts whose loads are in flight together
        for (int i = 0; i < PIECES && first + 64 * kWaves * i / (D / 4) < rows; ++i) {
            int r, c;
            place(i, r, c);
            float top = -__builtin_inff(), sum = 0.0f;
            v4f x{};
            for (int p = 0; p < n_parts; p += kAtOnce) {
                vec<float, 2> ml[kAtOnce];
                v4f y[kAtOnce];
                float now = top;
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    ml[k] = __builtin_bit_cast(vec<float, 2>, __builtin_amdgcn_raw_buffer_load_b64(left_parts, at_part(p + k, r, D / 4), 0, kShared));
                    y[k] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(left_parts, at_part(p + k, r, c), 0, kShared));
                }
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    if (p + k >= n_parts) ml[k][0] = -__builtin_inff();
                    now = fmaxf(now, ml[k][0]);
                }
                const float old = root_of(top, now);
                top = now;
                sum = sum * old * old;
                x *= old * old;
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    const float by = root_of(ml[k][0], now);
                    sum += ml[k][1] * by * by;
                    x += y[k] * (by * by);
                }
            }
            write(r, c, x, sum);
        }
        return;
    }
    if (n_parts == 1) {
        write_row();
        return;
    }
    const bool there = row_of(thread_again()) < rows;
    const auto part_at = [&](int p, int piece) { return there ? (p * FLOATS + (piece * 64 * kWaves + (int)threadIdx.x) * 4) * 4 : n_parts * FLOATS * 4; };
#pragma unroll
    for (int e = 0; e < D / 32; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v4f{o[e][4 * i], o[e][4 * i + 1], o[e][4 * i + 2], o[e][4 * i + 3]}), left_parts,
                                                   part_at(part, 4 * e + i), 0, kShared);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v4f{m, l, 0.0f, 0.0f}), left_parts, part_at(part, D / 8), 0, kShared);
    if (!last_to_arrive()) return;
    m = -__builtin_inff();
    l = 0.0f;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) o[e] = v16f{};
    for (int p = 0; p < n_parts; ++p) {
        const v4f ml = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(left_parts, part_at(p, D / 8), 0, kShared));
        v4f x[D / 8];
#pragma unroll
        for (int i = 0; i < D / 8; ++i) x[i] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(left_parts, part_at(p, i), 0, kShared));
        const float now = fmaxf(m, ml[0]);
        const float old = root_of(m, now), by = root_of(ml[0], now);
        m = now;
        l = l * old * old + ml[1] * by * by;
#pragma unroll
        for (int e = 0; e < D / 32; ++e)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[e][i] = o[e][i] * (old * old) + x[4 * e + (i >> 2)][i & 3] * (by * by);
    }
    write_row();
}

}  // namespace lqq

using namespace lqq;

namespace {
constexpr size_t kTickets = 32768;  // bytes at the head of the workspace, those of the GEMM's
// Tiles of a kv head, at most (more than 64 sequences: as they are searched for)
long long tiles_of(int total_q, int n_seqs, int group)
{
    const long long rows = (long long)total_q * group;
    return n_seqs <= kFew ? (rows + (long long)n_seqs * (kRows - 1)) / kRows : rows / kRows + n_seqs;
}
// Blocks that run at a time: what the keys are cut into, where there are fewer tiles than that (0: they are not cut)
int slots_of(long long tiles, int n_seqs, int Hkv)
{
    constexpr int kSlots = 512;
    return n_seqs <= kFew && tiles * Hkv < kSlots ? kSlots : 0;
}
size_t part_bytes(int head_dim) { return sizeof(float) * 64 * kWaves * (head_dim / 2 + 4); }
}  // namespace

extern "C" size_t kv4_attention_chunks_workspace_size(int n_seqs, int total_q, int Hq, int Hkv, int head_dim, int page_size, int table_width)
{
    if (n_seqs < 1 || total_q < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv || !head_dim_ok(head_dim) || !page_ok(page_size) || table_width < 1 || table_width > (1 << 30) / page_size)
        return 0;
    const int slots = slots_of(tiles_of(total_q, n_seqs, Hq / Hkv), n_seqs, Hkv);
    return slots ? kTickets + slots * part_bytes(head_dim) : 0;
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
    const int group = Hq / Hkv;
    const long long tiles = tiles_of(total_q, n_seqs, group);
    if (tiles * Hkv > (1 << 22) || (long long)total_q * group > (1 << 30)) return fail(LQ_ERR_INVALID, "too many rows: %d queries of %d sequences, %d heads", total_q, n_seqs, Hq);
    const size_t need = kv4_attention_chunks_workspace_size(n_seqs, total_q, Hq, Hkv, head_dim, page_size, table_width);
    const int slots = need && workspace && workspace_bytes >= need ? slots_of(tiles, n_seqs, Hkv) : 0;
    const ChunkArgs a{q, q_token, q_head, starts_q, block_table, context, static_cast<const uint8_t *>(cache), out,
                      static_cast<unsigned *>(workspace), slots ? reinterpret_cast<float *>(static_cast<char *>(workspace) + kTickets) : nullptr,
                      n_seqs, total_q, Hq, Hkv, group, table_width, num_pages, log2_of(page_size), (int)tiles, slots, scale * 1.44269504f};
    const dim3 grid((unsigned)((std::max<long long>(tiles * Hkv, slots) + 7) / 8 * 8));
    (void)hipGetLastError();
    const WorkspaceTurn turn(slots ? workspace : nullptr, hip_stream);
    const auto go = [&](auto kernel) __attribute__((always_inline)) { hipLaunchKernelGGL(kernel, grid, dim3(64 * kWaves), 0, static_cast<hipStream_t>(hip_stream), a); };
    const auto of = [&](auto x, auto d) {
        using T = decltype(x);
        constexpr int D = decltype(d)::value;
        go(kv4_chunks_kernel<D, T>);
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
