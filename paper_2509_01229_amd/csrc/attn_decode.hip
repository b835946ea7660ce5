// Attention of one or a few new tokens a sequence over the 4-bit cache (page format: attn_common.h, its values: kvcache.hip).
//
//     o = sum_j softmax_j(scale * q . k_j) v_j,   k_j = (code - z) * s of the key, v_j likewise,   j < context - n_new + 1 + i
// for new token i of n_new.  The heads that share a kv head and the new tokens are the rows of one matrix: row = token * group +
// head, 16 of them at a time.
//
// What is read is 17/16 of 4 bits an element, so the arithmetic has to stay small: 3.2 instruction slots of a lane for each code at the
// rate of memory.  Both products run on 16x16x32 MFMAs with the cache as the first operand (S^T = K Q^T, O^T = V^T P^T):
//   - the codes go into them as they are: masked out of their dword (5 instructions for 8), they are subnormal FP16 numbers, which the matrix
//     cores multiply exactly; the scales are applied to the scores (keys) and to the weights (values).  The keys' zero points take an
//     MFMA of their own (with the sum of a query's elements); the values' are taken off the codes (4 more instructions), as their
//     sums may cancel;
//   - the scores come out with 4 keys of one row in a lane, which is the order in which the weights go into the second product, so
//     nothing moves between lanes; the keys of a 16-byte piece of values are those of the lane's scores.
// Weights go into the second product as FP16 numbers, 2^6 .. 2^14 where they count most, times the value's scale over a power of two that is at
// least the largest one so far; the sums are FP32.  Where the result is FP16, too, what the rounding leaves of a weight goes in as a second
// number (8 more MFMAs of 18 and 12 more vector instructions for 32 keys: the rounding alone made the result's error 1.4 to 1.6 times that
// of its own rounding); beside BF16's it does not show.
//
// Measured (FP16, heads of 128): 128 contexts of 8192 tokens, 32/8 heads, 185 to 193 us, 6.0 to 6.2 TB/s of the 7.0 that a pure read reaches; two of
// 131072, 64/8 heads, 60 us (4.7 TB/s, their 32 parts an item joined in 10 of them); 16 of 4096 21.7 us; one of 517, 32/32 heads, 8.7 us,
// which are latencies: contexts, page numbers, first keys, and the join of the parts one after the other.  With 32 rows a pass (four
// new tokens of 64/8 heads, BF16) two of up to 131072 67 us (3.8 TB/s).  There 32 keys take about 290 vector instructions (half of a SIMD's cycles; 58% with
// the exponentials' rate) and 36 MFMAs (a quarter): neither is full, and two waves a SIMD do not overlap them and the loads any better; with
// blocks of four waves 77 us instead of 70.5, three of these a CU instead of two 83, the unpacking between the MFMAs 76.
#include <algorithm>
#include <type_traits>

#include "attn_common.h"
#include "workspace_turn.h"

namespace lqq {

typedef f16 f16x2v __attribute__((ext_vector_type(2)));

struct DecodeArgs {
    const void *q;
    long long q_seq, q_token, q_head;
    const uint8_t *cache;
    const int *table, *context;
    void *out;
    unsigned *tickets;
    float *parts;
    u32x4 *plan;
    int n_seqs, n_new, Hq, Hkv, group, rows, row_tiles, width, pages, lg_page, split, target;
    float scale_log2;  // softmax scale / ln 2
};

// 8 nibbles of a dword as 4 pairs of FP16 numbers: pair r = nibbles r and r + 4, which as subnormal numbers are 2^-24 of the code (r
// even) or 2^-20 of it (r odd)
__device__ __forceinline__ void halves8(uint32_t w, uint32_t (&o)[4])
{
    const uint32_t w8 = w >> 8;
    o[0] = w & 0x000f000fu;
    o[1] = w & 0x00f000f0u;
    o[2] = w8 & 0x000f000fu;
    o[3] = w8 & 0x00f000f0u;
}
// the same with the zero points of both halves taken off: exact, subnormal numbers all of them
__device__ __forceinline__ void halves8(uint32_t w, uint32_t zz, uint32_t (&o)[4])
{
    halves8(w, o);
#pragma unroll
    for (int r = 0; r < 4; ++r)
        o[r] = __builtin_bit_cast(uint32_t, (f16x2v)(__builtin_bit_cast(f16x2v, o[r]) - __builtin_bit_cast(f16x2v, r & 1 ? zz << 4 : zz)));
}
// what the two halves of x, which are a and b rounded, leave of them (one instruction each: the halves are taken as they are)
__device__ __forceinline__ uint32_t rest_of(uint32_t x, float a, float b)
{
    float c, d;
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(c) : "v"(x), "v"(a));
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(d) : "v"(x), "v"(b));
    return __builtin_bit_cast(uint32_t, f16x2v{(f16)c, (f16)d});
}
__device__ __forceinline__ v4f mfma16(const uint32_t (&a)[4], vec<f16, 8> b, v4f c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(vec<f16, 8>, u32x4{a[0], a[1], a[2], a[3]}), b, c, 0, 0, 0);
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

// What a wave loads for 32 keys (two tiles of 16): the keys' part and the values'.  `head`: the kv head's bytes of the tile's page as a
// buffer, of length zero where nothing is to be loaded (so that a load is never behind a branch, and the compiler can count those in flight).
constexpr int kReadOnce = 2;  // (non-temporal)
typedef __amdgpu_buffer_rsrc_t buf_t;
template <int N>
__device__ __forceinline__ void load_dwords(uint32_t (&x)[N], buf_t b, int lane_offset, int offset)
{
    if constexpr (N == 4) {
        const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(b, lane_offset, offset, kReadOnce);
        x[0] = v[0], x[1] = v[1], x[2] = v[2], x[3] = v[3];
    } else {
        const auto v = __builtin_amdgcn_raw_buffer_load_b64(b, lane_offset, offset, kReadOnce);
        x[0] = v[0], x[1] = v[1];
    }
}
template <int D>
struct Keys {
    uint32_t k[2][D / 32];  // this lane's key (row)
    u32x4 w[2];             // words of the lane's four keys
    uint32_t z[2];          // word of the lane's key
    __device__ __forceinline__ void load(buf_t head, int P, int j, int t, int lane)
    {
        const int n = lane & 15, g = lane >> 4;
        load_dwords(k[t], head, n * (D / 2) + g * (D / 8), j * (D / 2));
        w[t] = __builtin_amdgcn_raw_buffer_load_b128(head, 16 * g, P * D + 4 * j, 0);
        z[t] = __builtin_amdgcn_raw_buffer_load_b32(head, 4 * n, P * D + 4 * j, 0);
    }
};
template <int D>
struct Values {
    uint32_t v[2][D / 32];  // the lane's four keys of its column group
    u32x4 w[2];             // their words
    __device__ __forceinline__ void load(buf_t head, int P, int j, int t, int lane)
    {
        const int n = lane & 15, g = lane >> 4;
        w[t] = __builtin_amdgcn_raw_buffer_load_b128(head, 16 * g, P * (D + 4) + 4 * j, 0);
        load_dwords(v[t], head, g * (2 * D) + n * (D / 8), (P + j) * (D / 2));
    }
};

constexpr int blocks_per_cu(int row_tiles, int waves) { return (row_tiles == 1 ? 16 : 8) / waves; }
constexpr int unit_keys(int waves) { return 32 * waves; }  // keys that a block goes through at once
constexpr float kWeightBits = 6.0f;                        // a row's largest weight is 2^6 when its maximum is up to date

// The work is units of kUnit keys.  With split = 1 an item (sequence, kv head, tile of rows) is cut into chunks of the same number of
// units for all sequences, so many that about `target` blocks have work, and a block takes a chunk.  The chunks of an item are joined by the
// last of its blocks to arrive at its ticket: each leaves its maxima, sums and unscaled results in the workspace (written and read past
// the L2s, which the XCDs do not share), in the order of the split chunks of all items; the ticket is that of the item's first.
// A sequence without keys has one unit all the same (its zeros are written there).  With split = 0 a block is an item.  Each block finds its
// chunk from all context lengths (1.2 us for up to 64 sequences), or reads it from what one block found before.
// Every item rounds its own number of chunks up, so there can be more than `target`, by up to one an item.  Where all chunks are as
// long, the last of them then start when the others end: with four new tokens, 64/8 heads, BF16, where 256 blocks run at a time, 32 contexts of 8192
// make 256 chunks (77 us, inputs that change) and 33 make 264 (117); two of 131072 make 256 (82), three 264 (160).
constexpr int kMaxParts = 32, kLongChunk = 1024;
constexpr size_t kTickets = 32768;  // bytes at the head of the workspace, those of the GEMM's
__host__ __device__ constexpr int part_floats(int rows, int D) { return rows * (D + 4); }

template <int WAVES>
__device__ __forceinline__ int units_of(int ctx)
{
    return max(1, (ctx + unit_keys(WAVES) - 1) / unit_keys(WAVES));
}
// Units of a chunk, for `total` units in all (of all items), `most` of one sequence: as many as would cut all of them, end to end, into `target` chunks,
// half as many chunks while they have at most kLongChunk keys (a block's start and end cost as much as some units); and joining a part costs the last block
// about as much as 32 keys of a block of four waves where there are few, more than kMaxParts of them are never ahead.  (16 contexts of 4096,
// 64/8 heads: 8 units 21.3 us, 4 units 24.2; two of 131072: 32 units 56.8, 16 units 71.5.)
template <int WAVES>
__device__ __forceinline__ int units_of_chunk(int total, int most, int target)
{
    return max(max(max((total + target - 1) / target, min((2 * total + target - 1) / target, kLongChunk / unit_keys(WAVES))),
                   (int)__builtin_sqrtf((float)most / (float)WAVES)),
               (most + kMaxParts - 1) / kMaxParts);
}
// Where there are many items, a kernel of one block finds the chunks before the others start and puts long ones first; entry i has those of
// blocks items * i on: the sequence, the place of its first chunk among the split ones (over items), chunk | chunks << 16, the
// sequence's context.  A sequence of -1: no chunk.
__host__ __device__ constexpr long long plan_entries(long long n_seqs, long long items, int target) { return target / items + n_seqs; }
constexpr int kPlanThreads = 1024, kPlanClasses = 256;
template <int WAVES>
__global__ __launch_bounds__(kPlanThreads) void kv4_attention_plan_kernel(const DecodeArgs a)
{
    __shared__ int s_total[kPlanThreads / 64], s_most[kPlanThreads / 64], s_place[2][kPlanClasses];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, items = a.Hkv * a.row_tiles;
    const int longest = a.width << a.lg_page;
    const auto units = [&](int s) { return units_of<WAVES>(min(max(a.context[s], 0), longest)); };
    int total = 0, most = 0;
    for (int s = threadIdx.x; s < a.n_seqs; s += kPlanThreads) {
        const int u = units(s);
        total += u;
        most = max(most, u);
    }
    total = sums_up_to(total);
    most = lanes_up_to(most, [](int x, int y) { return max(x, y); });
    if (lane == 63) s_total[wave] = total, s_most[wave] = most;
    for (int i = threadIdx.x; i < 2 * kPlanClasses; i += kPlanThreads) s_place[0][i] = 0;
    __syncthreads();
    total = most = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) total += s_total[w], most = max(most, s_most[w]);
    const int size = units_of_chunk<WAVES>(total * items, most, a.target);
    // classes by the length of a sequence's chunks, long ones first
    const float by_size = (float)kPlanClasses / (float)size;
    const auto class_of = [&](int u, int c) { return min(max(kPlanClasses - (int)((float)u * by_size / (float)c), 0), kPlanClasses - 1); };
    for (int s = threadIdx.x; s < a.n_seqs; s += kPlanThreads) {
        const int u = units(s), c = (u + size - 1) / size, k = class_of(u, c);
        atomicAdd(&s_place[0][k], c);
        if (c > 1) atomicAdd(&s_place[1][k], c);
    }
    __syncthreads();
    // first places: chunks (wave 0), split chunks (wave 1)
    if (wave < 2) {
        constexpr int EACH = kPlanClasses / 64;
        int c[EACH], sum = 0;
        for (int i = 0; i < EACH; ++i) c[i] = s_place[wave][EACH * lane + i], sum += c[i];
        int place = sums_up_to(sum) - sum;
        for (int i = 0; i < EACH; ++i) s_place[wave][EACH * lane + i] = place, place += c[i];
        if (lane == 63) s_total[wave] = place;
    }
    __syncthreads();
    const int entries = (int)plan_entries(a.n_seqs, items, a.target);
    for (int s = threadIdx.x; s < a.n_seqs; s += kPlanThreads) {
        const int u = units(s), c = (u + size - 1) / size, k = class_of(u, c);
        const int at = atomicAdd(&s_place[0][k], c), part = c > 1 ? atomicAdd(&s_place[1][k], c) : 0;
        for (int i = 0; i < c; ++i) a.plan[at + i] = u32x4{(unsigned)s, (unsigned)part, (unsigned)(i | c << 16), (unsigned)a.context[s]};
    }
    for (int i = s_total[0] + (int)threadIdx.x; i < entries; i += kPlanThreads) a.plan[i] = u32x4{~0u, 0, 0, 0};
}
// 16 bytes past the L2 (device scope)
constexpr int kShared = 16;  // sc1
__device__ __forceinline__ __amdgpu_buffer_rsrc_t shared_buffer(float *p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc(p, 0, bytes, 0x00027000); }

// (RT: tiles of 16 rows that share a pass over the keys; WAVES: of a block, the keys of a unit shared between them)
template <int D, class T, int RT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, (RT == 1 ? 4 : 2)) void kv4_attention_kernel(const DecodeArgs a)
{
    constexpr int W = D / 16, STEPS = D / 32;  // elements of a column group; MFMAs of a key tile
    constexpr int ROWS = 16 * RT;
    constexpr bool TWO = __is_same(T, f16);
    constexpr int kUnit = unit_keys(WAVES);
    __shared__ float s_o[WAVES][16][D + 4], s_m[WAVES][ROWS], s_l[WAVES][ROWS];
    __shared__ int s_last;
    __shared__ float s_scale[RT][16];
    __shared__ vec<f16, 8> s_q[RT][STEPS + 1][64];  // (the waves have the same queries)
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int P = 1 << a.lg_page, items = a.Hkv * a.row_tiles;
    const unsigned page_bytes = (unsigned)a.Hkv * (unsigned)kv4_head_bytes(P, D);
    const int longest = a.width << a.lg_page;
    // (integers that no kernel writes meanwhile: scalar loads)
    typedef const __attribute__((address_space(4))) int *ints;
    const ints table = (ints)(uintptr_t)a.table, contexts = (ints)(uintptr_t)a.context;
    const auto within = [&](int context) { return min(max(context, 0), longest); };

    // this block's sequence, item and units; the item's chunks, and where they are among the split ones
    int seq, context, item, unit = 0, units = 1, count, chunks = 1, chunk = 0, first_part = 0;
    if (a.plan) {
        const u32x4 *const plan = a.plan + blockIdx.x / (unsigned)items;
        const u32x4 x = *(const __attribute__((address_space(4))) u32x4 *)(uintptr_t)plan;
        seq = (int)x[0];
        if ((unsigned)seq >= (unsigned)a.n_seqs) return;
        item = (int)(blockIdx.x % (unsigned)items);
        chunk = (int)(x[2] & 0xffffu);
        chunks = (int)(x[2] >> 16);
        context = (int)x[3];
        units = units_of<WAVES>(within(context));
        first_part = (int)x[1] * items + item * chunks;
        unit = (int)((unsigned)chunk * (unsigned)units / (unsigned)chunks);
        count = (int)((unsigned)(chunk + 1) * (unsigned)units / (unsigned)chunks) - unit;
    } else if (a.split) {
        int total = 0, most = 0;
        const auto context64 = [&](int s0) { return s0 + lane < a.n_seqs ? contexts[s0 + lane] : 0; };
        const int first64 = context64(0);
        const auto units64 = [&](int s0, int c) { return s0 + lane < a.n_seqs ? units_of<WAVES>(within(c)) : 0; };
        for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
            const int u = units64(s0, s0 ? context64(s0) : first64);
            total += __builtin_amdgcn_readlane(sums_up_to(u), 63);
            most = max(most, __builtin_amdgcn_readlane(lanes_up_to(u, [](int x, int y) { return max(x, y); }), 63));
        }
        total *= items;
        const int size = units_of_chunk<WAVES>(total, most, a.target);
        int before = 0, parts = 0;  // chunks, split chunks of the sequences that come before
        seq = -1;
        for (int s0 = 0; seq < 0 && s0 < a.n_seqs; s0 += 64) {
            const int keys = s0 ? context64(s0) : first64, u = units64(s0, keys), c = (u + size - 1) / size, sum = sums_up_to(c), split = sums_up_to(c > 1 ? c : 0);
            const uint64_t past = __ballot((before + sum) * items > (int)blockIdx.x);
            const int at = past ? __builtin_ctzll(past) : 63;
            before += __builtin_amdgcn_readlane(sum, at);
            parts += __builtin_amdgcn_readlane(split, at);
            if (past) {
                seq = s0 + at;
                context = __builtin_amdgcn_readlane(keys, at);
                units = __builtin_amdgcn_readlane(u, at);
                chunks = __builtin_amdgcn_readlane(c, at);
                before -= chunks;
                if (chunks > 1) parts -= chunks;
            }
        }
        if (seq < 0) return;
        const int inside = (int)blockIdx.x - before * items;
        item = inside / chunks;
        chunk = inside % chunks;
        first_part = parts * items + item * chunks;
        unit = (int)((unsigned)chunk * (unsigned)units / (unsigned)chunks);
        count = (int)((unsigned)(chunk + 1) * (unsigned)units / (unsigned)chunks) - unit;
    } else {
        seq = (int)blockIdx.x / items;
        item = (int)blockIdx.x % items;
        context = contexts[seq];
        count = units_of<WAVES>(within(context));
    }

    {
        const int rt = item % a.row_tiles, hk = item / a.row_tiles;
        const uint8_t *const cache = a.cache + (size_t)hk * kv4_head_bytes(P, D);
        bool bad = context > longest;  // more than the table has pages for
        const int ctx = within(context), end = min(ctx, (unit + count) * kUnit);
        int limit[RT];                        // keys that this lane's rows see

        const unsigned last_page = max((ctx - 1) >> a.lg_page, 0);

        // the pages of 32 keys: numbers first, then addresses
        struct Place {
            unsigned page[2];
        };
        typedef const __attribute__((address_space(4))) char *bytes;
        const bytes pages = (bytes)(table + (size_t)seq * a.width);
        const auto pages_of = [&](int key) {
            Place p;
#pragma unroll
            for (int t = 0; t < 2; ++t) p.page[t] = *(ints)(pages + 4 * min((unsigned)(key + 16 * t) >> a.lg_page, last_page));
            return p;
        };
        buf_t head[2];
        const auto go_to = [&](Place p, bool any) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const bool out_of_range = p.page[t] >= (unsigned)a.pages;
                bad |= out_of_range;
                head[t] = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(cache + (uint64_t)(out_of_range ? 0u : p.page[t]) * page_bytes), 0,
                                                            any ? kv4_head_bytes(P, D) : 0, 0x00027000);
            }
        };
        const auto load = [&](auto &x, int key) {
#pragma unroll
            for (int t = 0; t < 2; ++t) x.load(head[t], P, (key + 16 * t) & (P - 1), t, lane);
        };
        Keys<D> xk;
        Values<D> xv;
        // the queries, then the first keys and values: in flight together
        vec<T, 8> raw[RT][STEPS];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = rt * ROWS + r * 16 + n, token = min(row / a.group, a.n_new - 1), head = hk * a.group + row % a.group;
            const bool real = row < a.rows;
            limit[r] = real ? ctx - a.n_new + 1 + token : 0;
            const T *src = static_cast<const T *>(a.q) + seq * a.q_seq + token * a.q_token + (real ? head : hk * a.group) * a.q_head + g * (D / 4);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) raw[r][i] = *reinterpret_cast<const vec<T, 8> *>(src + 8 * i);
        }
        int key = unit * kUnit + 32 * wave;
        Place next{};
        if (key < end) {
            go_to(pages_of(key), true);
            __builtin_amdgcn_sched_barrier(0);
            load(xk, key);
            __builtin_amdgcn_sched_barrier(0);  // (in the order of the loop's)
            load(xv, key);
            __builtin_amdgcn_sched_barrier(0);
            next = pages_of(key + kUnit);
        }
        // Queries in the keys' operand order, times a power of two that brings the row's largest element to 4 .. 8 (exact down to 2^-16 of
        // it), those that meet even pairs (halves8) times 16.  A last operand holds what the zero points are multiplied with, minus 16 times
        // the sum of the row's elements, as three numbers (33 bits of it).  Of two tiles each is one wave's (one context of 2000, 32 rows: 16.1 us instead
        // of 17.5); of one tile every wave writes the same, and no wave waits (one of 517: 8.8 instead of 9.0).
        constexpr int Q = STEPS + 1;
        float q_scale[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            if (RT == 2 && wave != (int)((blockIdx.x + r) % WAVES)) continue;
            const bool real = rt * ROWS + r * 16 + n < a.rows;
            float f[STEPS][8];
            const float sign = a.scale_log2 < 0.0f ? -1.0f : 1.0f;  // (the scale's)
            float most = 0.0f;
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
#pragma unroll
                for (int e = 0; e < 8; ++e) f[i][e] = real ? (float)raw[r][i][e] * sign : 0.0f, most = fmaxf(most, fabsf(f[i][e]));
            }
            most = across_groups(most, [](float x, float y) { return fmaxf(x, y); });
            const int e = min(max((int)(__builtin_bit_cast(uint32_t, most) >> 23), 29), 254) - 129;
            // (neither zero nor infinite, whatever the scale and the row: minus infinity times it stays that, and zero stays zero)
            q_scale[r] = fminf(fmaxf(fabsf(a.scale_log2) * 0x1p20f * power_of_two(e), 0x1p-126f), 0x1p127f);
            vec<f16, 8> q[Q];
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < STEPS; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const f16 x = (f16)(f[i][j] * power_of_two(-e));
                    sum += (float)x;
                    q[i][2 * (j & 3) + (j >> 2)] = j & 1 ? x : x * (f16)16.0f;
                }
            sum = -16.0f * across_groups(sum, [](float x, float y) { return x + y; });
            const f16 s0 = (f16)sum, s1 = (f16)(sum - (float)s0), s2 = (f16)(sum - (float)s0 - (float)s1);
            q[STEPS] = vec<f16, 8>{};
            if (g == 0) q[STEPS][0] = s0, q[STEPS][1] = s1, q[STEPS][2] = s2;
#pragma unroll
            for (int i = 0; i < Q; ++i) s_q[r][i][lane] = q[i];
            if (RT == 2 && g == 0) s_scale[r][n] = q_scale[r];
        }
        if (RT == 2) {
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // (not __syncthreads(): the keys stay in flight)
#pragma unroll
            for (int r = 0; r < RT; ++r) q_scale[r] = s_scale[r][n];
        }
        const auto query = [&](int r, int i) { return s_q[r][i][lane]; };

        v4f o[RT][W] = {};
        float m[RT], l[RT] = {};   // a row's maximum (as sc), this lane's part of its sum
        float m_up[RT], base[RT];  // the score from which the maximum moves; see below
#pragma unroll
        for (int r = 0; r < RT; ++r) m[r] = m_up[r] = -__builtin_inff(), base[r] = 0.0f;
        // Weights are over 2^v_exp, a power of two that no value's scale so far is above: 2^v_in of it in the exponent (and in l), the rest,
        // where v_exp is very far from 0, by a factor.
        int v_exp = -126, v_in = -90;
        float v_top = power_of_two(v_exp);
        const auto base_of = [&](int r) { return m[r] == -__builtin_inff() ? 0.0f : kWeightBits - (float)v_in - m[r] * q_scale[r]; };
        // a step takes 32 keys; the next ones' registers are those that it has just used
        const auto step = [&](int key, bool more, Place &next) {
            float sc[RT][2][4];  // scores over q_scale
            float sv[2][4];      // scales of the values (with the zero points still in their last bits: 2^-19 of them)
            float vt = 0.0f;
            const bool tail = key + 32 > ctx - a.n_new + 1;  // some row does not see all of these keys
            v4f acc[2][RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const auto qi = query(r, STEPS);
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const uint32_t z = xk.z[t] & 15u, zz = z | z << 16, zeros[4] = {zz, zz, 0, 0};
                    acc[t][r] = mfma16(zeros, qi, v4f{});
                }
            }
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                uint32_t k8[2][4];
#pragma unroll
                for (int t = 0; t < 2; ++t) halves8(xk.k[t][i], k8[t]);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const auto qi = query(r, i);
#pragma unroll
                    for (int t = 0; t < 2; ++t) acc[t][r] = mfma16(k8[t], qi, acc[t][r]);
                }
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float sk = __builtin_bit_cast(float, xk.w[t][i] & kScaleMask);
#pragma unroll
                    for (int r = 0; r < RT; ++r) sc[r][t][i] = acc[t][r][i] * sk;
                }
            go_to(next, more);
            load(xk, key + kUnit);
            next = pages_of(key + 2 * kUnit);
            __builtin_amdgcn_sched_barrier(0);
            asm("" : "+v"(xv.w[0]), "+v"(xv.w[1]));  // (nothing of the values is looked at before)
            if (tail) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int j = key + 16 * t + 4 * g + i;
#pragma unroll
                        for (int r = 0; r < RT; ++r) sc[r][t][i] = j < limit[r] ? sc[r][t][i] : -__builtin_inff();
                        xv.w[t][i] = j < ctx ? xv.w[t][i] : 0u;
                    }
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t word = xv.w[t][i];  // (a bit cast of a vector's element takes its first)
                    sv[t][i] = __builtin_bit_cast(float, word);
                }
#pragma unroll
            for (int i = 0; i < 8; i += 2) vt = max3_numbers(vt, sv[i >> 2][i & 3], sv[i >> 2][(i & 3) + 1]);
            float top[RT];
            bool up = false;
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                top[r] = m[r];
#pragma unroll
                for (int i = 0; i < 8; i += 2) top[r] = max3_numbers(top[r], sc[r][i >> 2][i & 3], sc[r][i >> 2][(i & 3) + 1]);
                up |= top[r] > m_up[r];
            }
            if (__any(up)) {  // (first of all: m is minus infinity)
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    top[r] = across_groups(top[r], [](float u, float w) { return fmaxf(u, w); });
                    const float now = top[r] > m_up[r] ? top[r] : m[r];  // (a row's results go by its own scores alone)
                    const float by = now == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((m[r] - now) * q_scale[r]);
                    m[r] = now;
                    m_up[r] = now == -__builtin_inff() ? now : now + (14.0f - kWeightBits) / q_scale[r];  // (a quotient of infinity: one maximum is enough)
                    base[r] = base_of(r);
                    l[r] *= by;
#pragma unroll
                    for (int e = 0; e < W; ++e) o[r][e] *= by;
                }
            }
            if (__any(vt > v_top)) {
                for (int d = 1; d < 64; d <<= 1) vt = fmaxf(vt, __shfl_xor(vt, d));
                const int e = __builtin_amdgcn_readfirstlane(min((int)(__builtin_bit_cast(uint32_t, vt) >> 23) - 126, 126));  // the next power of two
                const int in = min(max(e, -90), 90);
                const float by = power_of_two(max(v_exp - e, -126)), by_l = power_of_two(max(v_in - in, -126));
                v_exp = e;
                v_in = in;
                v_top = power_of_two(e);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    base[r] = base_of(r);
                    l[r] *= by_l;
#pragma unroll
                    for (int i = 0; i < W; ++i) o[r][i] *= by;
                }
            }
            vec<f16, 8> weights[RT], rest[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                uint32_t w[4], w2[4];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    float p[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[r][t][i], q_scale[r], base[r]));
                        l[r] += p[i];
                        p[i] *= sv[t][i];
                    }
                    if (v_exp != v_in) {
                        asm volatile("");
#pragma unroll
                        for (int i = 0; i < 4; ++i) p[i] *= power_of_two(v_in - v_exp);
                    }
                    if (tail) {  // (whatever the scale there is)
                        asm volatile("");
#pragma unroll
                        for (int i = 0; i < 4; ++i) p[i] = sc[r][t][i] == -__builtin_inff() ? 0.0f : p[i];
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        w[2 * t + i] = __builtin_bit_cast(uint32_t, f16x2v{(f16)p[2 * i], (f16)p[2 * i + 1]});
                        if constexpr (TWO) w2[2 * t + i] = rest_of(w[2 * t + i], p[2 * i], p[2 * i + 1]);
                    }
                }
                weights[r] = __builtin_bit_cast(vec<f16, 8>, u32x4{w[0], w[1], w[2], w[3]});
                if constexpr (TWO) rest[r] = __builtin_bit_cast(vec<f16, 8>, u32x4{w2[0], w2[1], w2[2], w2[3]});
            }
            uint32_t zz[4];  // zero points of the pairs of keys (the low bytes of their words)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 2; ++i) zz[2 * t + i] = __builtin_amdgcn_perm(xv.w[t][2 * i + 1], xv.w[t][2 * i], 0x0c040c00u) & 0x000f000fu;
#pragma unroll
            for (int h = 0; h < W / 4; ++h) {
                uint32_t v8[4][4];  // [pair of keys][element of the four]
#pragma unroll
                for (int p2 = 0; p2 < 4; ++p2) halves8(xv.v[p2 >> 1][(p2 & 1) * (W / 4) + h], zz[p2], v8[p2]);
#pragma unroll
                for (int two = TWO ? 0 : 1; two < 2; ++two)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t x[4] = {v8[0][e], v8[1][e], v8[2][e], v8[3][e]};
#pragma unroll
                        for (int r = 0; r < RT; ++r) o[r][4 * h + e] = mfma16(x, two ? weights[r] : rest[r], o[r][4 * h + e]);
                    }
            }
            load(xv, key + kUnit);
            __builtin_amdgcn_sched_barrier(0);
        };

        for (; key < end; key += kUnit) step(key, key + kUnit < end, next);
        // the waves' parts: sums of weights relative to 2^(m - kWeightBits), both over 2^16 so that values near the end of FP32's range stay in it
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            l[r] = across_groups(l[r], [](float u, float w) { return u + w; });
            if (bad) l[r] = __builtin_nanf("");
            if (g == 0) s_m[wave][16 * r + n] = m[r] * q_scale[r], s_l[wave][16 * r + n] = l[r] * (0x1p-16f * power_of_two(v_in));
        }
        // thread: 8 elements of a row of each tile; the waves' results one tile at a time
        float most[RT], sum[RT], f[RT][8];
        constexpr int STEP = 64 * WAVES;
        static_assert(16 * D / 8 <= STEP, "");
        const int c = (int)threadIdx.x % (D / 8) * 8;
        int r16 = (int)threadIdx.x / (D / 8);
        bool mine = threadIdx.x < 16 * D / 8;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            if (r) __syncthreads();
#pragma unroll
            for (int e = 0; e < W; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) s_o[wave][n][(4 * g + i) * W + e] = o[r][e][i] * (e & 1 ? 0x1p4f : 0x1p8f) * v_top;
            __syncthreads();
            if (!mine) continue;
            most[r] = s_m[0][16 * r + r16];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) most[r] = fmaxf(most[r], s_m[w][16 * r + r16]);
            sum[r] = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) f[r][e] = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float mw = s_m[w][16 * r + r16], by = mw == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(mw - most[r]);
                sum[r] += s_l[w][16 * r + r16] * by;
#pragma unroll
                for (int e = 0; e < 8; ++e) f[r][e] += s_o[w][r16][c + e] * by;
            }
        }
        if (chunks > 1) {
            // the results of this block, in the place of chunk `to`
            constexpr int PART = part_floats(ROWS, D) * 4;
            const auto all = shared_buffer(a.parts + (size_t)first_part * part_floats(ROWS, D), chunks * PART);
            const auto store = [&](int to) {
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    if (!mine || rt * ROWS + 16 * r + r16 >= a.rows) continue;
                    const int at = to * PART + ((16 * r + r16) * D + c) * 4;
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v4f{f[r][0], f[r][1], f[r][2], f[r][3]}), all, at, 0, kShared);
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v4f{f[r][4], f[r][5], f[r][6], f[r][7]}), all, at + 16, 0, kShared);
                    if (c == 0)
                        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v4f{most[r], sum[r], 0.0f, 0.0f}), all,
                                                               to * PART + (ROWS * D + (16 * r + r16) * 4) * 4, 0, kShared);
                }
            };
            // whether this block is the last of `count` to arrive at the ticket of chunk `to`
            const auto last_at = [&](int to, int count) {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
                if (threadIdx.x == 0) {
                    unsigned *const ticket = a.tickets + first_part + to;
                    const unsigned before = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    s_last = before == (unsigned)count - 1;
                    if (before == (unsigned)count - 1) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
                __syncthreads();
                return s_last != 0;
            };
            // threads: piece (8 elements) of a real row, and as many groups of threads as there are for the parts
            const int left = a.rows - rt * ROWS, rows16 = left >= 9 ? 16 : left >= 5 ? 8 : left >= 3 ? 4 : left;  // (a power of two)
            const int pieces = rows16 * (D / 8), groups = 64 * WAVES / pieces, group = (int)threadIdx.x / pieces;
            float *const s_f = &s_o[0][0][0];
            // the results of `count` chunks, from `from` on in steps of `by`, joined in their order
            const auto join = [&](int from, int by, int count) {
                r16 = (int)threadIdx.x / (D / 8) % rows16;
                constexpr int U = 8 / RT;  // parts whose loads are in flight together
                const auto add = [&](int r, float m, float l, const float (&x)[8]) {
                    const float now = fmaxf(most[r], m);
                    const float old = most[r] == now ? 1.0f : __builtin_amdgcn_exp2f(most[r] - now);
                    const float by = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m - now);
                    most[r] = now;
                    sum[r] = sum[r] * old + l * by;
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[r][e] = f[r][e] * old + x[e] * by;
                };
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    most[r] = -__builtin_inff();
                    sum[r] = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[r][e] = 0.0f;
                }
                for (int w = group; w < count; w += U * groups) {
                    v4f x[U][RT][2], ml[U][RT];
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int r = 0; r < RT; ++r) {  // (past the last: nothing is loaded)
                            const int at = (w + u * groups < count ? from + by * (w + u * groups) : chunks) * PART;
                            ml[u][r] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(all, at + (ROWS * D + (16 * r + r16) * 4) * 4, 0, kShared));
                            x[u][r][0] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(all, at + ((16 * r + r16) * D + c) * 4, 0, kShared));
                            x[u][r][1] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(all, at + ((16 * r + r16) * D + c) * 4 + 16, 0, kShared));
                        }
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (w + u * groups < count)
#pragma unroll
                            for (int r = 0; r < RT; ++r) {
                                const v4f a = x[u][r][0], b = x[u][r][1];
                                const float x8[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
                                add(r, ml[u][r][0], ml[u][r][1], x8);
                            }
                }
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    if (groups == 1) break;
                    float *const to = s_f + threadIdx.x * 10;
                    to[0] = most[r], to[1] = sum[r];
#pragma unroll
                    for (int e = 0; e < 8; ++e) to[2 + e] = f[r][e];
                    __syncthreads();
                    if (group == 0)
                        for (int w = 1; w < min(groups, count); ++w) {
                            const float *const o = s_f + (threadIdx.x + w * pieces) * 10;
                            const float x8[8] = {o[2], o[3], o[4], o[5], o[6], o[7], o[8], o[9]};
                            add(r, o[0], o[1], x8);
                        }
                    __syncthreads();
                }
                mine = group == 0;
            };
            // kJoin chunks at a time, then their results, so that what is left to do when the last chunk is done is short (32 chunks, 32 rows:
            // 94.5 us instead of 101.3; 16 chunks of 8 rows, whose loads are all in flight together, in one go 10.9 us, in two 12.6)
            constexpr int kJoin = RT == 1 || WAVES == 8 ? 16 : 8;
            const int g0 = chunk / kJoin * kJoin, n = min(kJoin, chunks - g0), sets = (chunks + kJoin - 1) / kJoin;
            store(chunk);
            if (!last_at(g0, n)) return;
            join(g0, 1, n);
            if (sets > 1) {
                store(g0);
                if (!last_at(1, sets)) return;  // (a ticket that no set has)
                join(0, kJoin, sets);
            }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int to = rt * ROWS + 16 * r + r16;
            if (!mine || to >= a.rows) continue;
            vec<T, 8> y;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = (T)(sum[r] == 0.0f ? 0.0f : f[r][e] / sum[r]);
            T *dst = static_cast<T *>(a.out) + (((size_t)seq * a.n_new + to / a.group) * a.Hq + hk * a.group + to % a.group) * D + c;
            *reinterpret_cast<vec<T, 8> *>(dst) = y;
        }
    }
}

}  // namespace lqq

using namespace lqq;

// Rows that share a pass: one tile of 16, or two
static int row_tiles_of(int rows) { return rows <= 16 ? 1 : 2; }
// Waves of a block: four, two or four of which a CU holds; with two tiles of rows and few items eight, which leave half as many parts to join.  (64/8
// heads, 4 new tokens: two contexts of 131072 76.7 us with four waves, 70.5 with eight; 32 of 8192 69.6 and 67; 64 of 400 to 4000 62.6 and 51.5; but 128 of
// these 88 and 97, and 300 of 50 to 500 62.6 and 103, as nothing else runs on a CU while a block starts and ends; one
// of 2000 15.6 and 16.6.  The two and the 32 contexts make as many chunks as run at a time.  Blocks of 16 waves with one tile:
// 59 and 54.6 for two contexts of 131072, but 8.9 and 13.4 for one of 517.)
static int waves_of(long long n_seqs, long long items, int row_tiles) { return row_tiles == 2 && n_seqs * items <= 512 ? 8 : 4; }
// Blocks that have work where the keys can be split, about: as many as the CUs hold at a time
static int target_of(int row_tiles, int waves) { return 256 * blocks_per_cu(row_tiles, waves); }
static size_t parts_bytes(int row_tiles, int head_dim, int target) { return sizeof(float) * 2 * target * part_floats(16 * row_tiles, head_dim); }
// Whether the chunks are found by a kernel of their own: where there are as many items as blocks at a time.  Measured with and without, 8 kv
// heads: 128 contexts of 400 to 8192 tokens 112 and 125 us, of 8192 each 193 and 190; 256 of 512 to 1024 48.5 and 55; 1000 of 100 to 1000
// 146 and 221; with a quarter of the items, where most blocks run at once, it costs what it saves (32 contexts of 400 to 4096: 28.0 and
// 26.1; 64 of 200 to 2048: 25.8 and 27.5).
static bool planned(long long n_seqs, long long items, int target) { return n_seqs * items >= target; }

extern "C" size_t kv4_attention_workspace_size(int n_seqs, int n_new, int Hq, int Hkv, int head_dim)
{
    if (n_seqs < 1 || n_new < 1 || Hkv < 1 || Hq < 1 || Hq % Hkv || !head_dim_ok(head_dim)) return 0;
    const long long rows = (long long)n_new * (Hq / Hkv);
    const int RT = row_tiles_of((int)std::min(rows, 1LL << 20));
    const long long items = (rows + 16 * RT - 1) / (16 * RT) * Hkv;
    const int target = target_of(RT, waves_of(n_seqs, items, RT));
    return kTickets + parts_bytes(RT, head_dim, target) + (planned(n_seqs, items, target) ? 16 * plan_entries(n_seqs, items, target) : 0);
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
    if (num_pages < 1 || num_pages > INT32_MAX / page_size || table_width < 1 || table_width > (1 << 30) / page_size)
        return fail(LQ_ERR_INVALID, "num_pages times page_size must be from 1 to below 2^31, table_width times it to 2^30, got %d and %d times %d",
                    num_pages, table_width, page_size);
    if (!(scale > -1e30f && scale < 1e30f)) return fail(LQ_ERR_INVALID, "scale must be finite");
    const long long rows = (long long)n_new * (Hq / Hkv);
    if (rows > (1 << 20)) return fail(LQ_ERR_INVALID, "too many rows: %d new tokens, %d heads a kv head", n_new, Hq / Hkv);
    const int RT = row_tiles_of((int)rows);
    const long long tiles = (rows + 16 * RT - 1) / (16 * RT), items = tiles * Hkv;
    if (items * n_seqs > (1 << 22)) return fail(LQ_ERR_INVALID, "too many rows: %d sequences, %d new tokens, %d heads", n_seqs, n_new, Hq);
    if (n_seqs == 0) return LQ_OK;
    if (!q || !cache || !block_table || !context || !out) return fail(LQ_ERR_INVALID, "null pointer");
    if (((uintptr_t)q | (uintptr_t)cache | (uintptr_t)out | (uintptr_t)workspace) & 15)
        return fail(LQ_ERR_ALIGN, "q, cache, out and workspace must be 16-byte aligned");
    if (((uintptr_t)block_table | (uintptr_t)context) & 3) return fail(LQ_ERR_ALIGN, "block_table and context must be 4-byte aligned");
    if ((n_seqs > 1 && q_seq % 8) || (n_new > 1 && q_token % 8) || (Hq > 1 && q_head % 8))
        return fail(LQ_ERR_ALIGN, "q: strides must be multiples of 8 elements, got %lld, %lld and %lld", q_seq, q_token, q_head);
    // units are counted in 32 bits; no more of them than this
    const int waves = waves_of(n_seqs, items, RT), target = target_of(RT, waves);
    const long long most = items * n_seqs * (((long long)table_width * page_size + unit_keys(waves) - 1) / unit_keys(waves));
    const bool split = workspace && workspace_bytes >= kv4_attention_workspace_size(n_seqs, n_new, Hq, Hkv, head_dim) && most < (1LL << 30);
    const DecodeArgs a{q, q_seq, q_token, q_head, static_cast<const uint8_t *>(cache), block_table, context, out,
                       static_cast<unsigned *>(workspace), split ? reinterpret_cast<float *>(static_cast<char *>(workspace) + kTickets) : nullptr,
                       split && planned(n_seqs, items, target) ? reinterpret_cast<u32x4 *>(static_cast<char *>(workspace) + kTickets + parts_bytes(RT, head_dim, target)) : nullptr,
                       n_seqs, n_new, Hq, Hkv, Hq / Hkv, (int)rows, (int)tiles, table_width, num_pages, log2_of(page_size), split,
                       target, scale * 1.44269504f};
    const dim3 grid((unsigned)(a.plan  ? plan_entries(n_seqs, items, target) * items
                               : split ? std::min<long long>(target + items * n_seqs, most)
                                       : items * n_seqs));
    (void)hipGetLastError();
    const WorkspaceTurn turn(split ? workspace : nullptr, hip_stream);  // (the list of chunks is the next kernel's, and no other call's)
    if (a.plan)
        hipLaunchKernelGGL(waves == 4 ? kv4_attention_plan_kernel<4> : kv4_attention_plan_kernel<8>, dim3(1), dim3(kPlanThreads), 0,
                           static_cast<hipStream_t>(hip_stream), a);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * waves), 0, static_cast<hipStream_t>(hip_stream), a); };
    auto by_dim = [&](auto x) {
        using T = decltype(x);
        const auto of = [&](auto D) {
            constexpr int d = decltype(D)::value;
            RT == 1 ? go(kv4_attention_kernel<d, T, 1, 4>) : waves == 4 ? go(kv4_attention_kernel<d, T, 2, 4>) : go(kv4_attention_kernel<d, T, 2, 8>);
        };
        head_dim == 128 ? of(std::integral_constant<int, 128>{}) : of(std::integral_constant<int, 64>{});
    };
    dtype == LQ_F16 ? by_dim(f16{}) : by_dim(bf16{});
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LQ_OK : fail(LQ_ERR_HIP, "attention launch failed: %s", hipGetErrorString(e));
}
