// Around the grouped product of a mixture of experts: tokens sorted by expert, their results brought back with weights, and the gradients of that.
//
// A pair p = token * k + j is a token and its j-th expert e_p.  Its row is
//     place(p) = #{p' : e_p' < e_p} + #{p' < p : e_p' = e_p},    offsets(e) = #{p' : e_p' < e}
// over the pairs whose expert is one of 0 .. E - 1 (other pairs have the place -1 and no row): sorted by expert, in the pairs' order.  Then
//     rows[place(p)] = X[token],     out[t] = sum_j w[t][j] Y[place(t, j)],     dY[place(t, j)] = w[t][j] g[t],     dw[t][j] = g[t] . Y[place(t, j)]
// (sums in FP32, in the order of j, or of the elements' pieces; no atomics).
//
// The places are counted, not sorted: blocks of each expert look at all pairs, for those before its own, and then number its own (ballots).  Up to kFewPairs of
// them each token's block counts its own pairs' places itself and copies the row in the same launch.
//
// Bound by memory, or by the launch where there are few tokens.  Measured (by run; inputs that change): 8191 FP16 rows of 4096, 8 of 64 experts each, half of them here,
// 75 to 83 us to sort (12.9 of them the places, the copy 4.9 to 5.1 TB/s), 60 to 69 us to bring back (BF16, 4.9 to 5.6 TB/s); gradients of 2047 tokens of 8192, 4 experts each, 62
// to 64 us (4.7 TB/s).  16 tokens: kernels of 2.5 to 2.8 us.
#include <algorithm>

#include "attn_common.h"

namespace lqq {

constexpr int kMostExperts = 256, kMostEach = 64, kFewPairs = 2048;

struct DispatchArgs {
    const char *x;
    const float *scales;
    const int *experts;
    char *rows;
    float *row_scales;
    int *offsets, *places;
    long long x_row;  // bytes
    int tokens, each, n_experts, pieces, segments;
};

__device__ __forceinline__ int lanes_set_below(uint64_t mask) { return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0u)); }

// The row of a token to its places, of which lane j of each wave has the j-th (so that no store waits for one to be loaded)
__device__ __forceinline__ void copy_row(const DispatchArgs &a, int token, int place, int thread, int threads)
{
    const u32x4 *const from = reinterpret_cast<const u32x4 *>(a.x + token * a.x_row);
    if (a.scales && thread < a.each && place >= 0) a.row_scales[place] = a.scales[token];
    for (int i = thread; i - (thread & 63) < a.pieces; i += threads) {  // (whole waves: lanes hold what others take)
        const bool any = i < a.pieces;
        u32x4 x{};
        if (any) x = from[i];
        for (int j = 0; j < a.each; ++j) {
            const int to = __builtin_amdgcn_readlane(place, j);
            if (to >= 0 && any) reinterpret_cast<u32x4 *>(a.rows)[(size_t)to * a.pieces + i] = x;
        }
    }
}

// Few pairs, up to 64 * IDS of them: block t < tokens counts the places of its pairs and copies the row, the last block counts the experts' pairs.  All pairs are
// looked at, whether they are there or not: 32 pairs take 2.6 us as up to 128, 3.4 as up to 1024 and 4.9 as up to 2048; 1600 pairs 8.6 as up to 2048, 10.4 by the
// kernels for many (16 and 64 experts, rows of 4096 INT8), 13.7 as up to 4096.
constexpr int kSmallThreads = 256;
template <int IDS>
__global__ __launch_bounds__(kSmallThreads) void moe_dispatch_small_kernel(const DispatchArgs a)
{
    __shared__ int s_places[kMostEach], s_count[kMostExperts];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), pairs = a.tokens * a.each, token = blockIdx.x;
    constexpr int WAVES = kSmallThreads / 64;
    if (token == a.tokens) {
        for (int e = threadIdx.x; e < kMostExperts; e += kSmallThreads) s_count[e] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < pairs; i += kSmallThreads) {
            const int e = a.experts[i];
            if ((unsigned)e < (unsigned)a.n_experts) atomicAdd(&s_count[e], 1);
        }
        __syncthreads();
        if (wave == 0) {
            int before = 0;
            for (int e0 = 0; e0 < a.n_experts; e0 += 64) {
                const int n = e0 + lane < a.n_experts ? s_count[e0 + lane] : 0, upto = sums_up_to(n);
                if (e0 + lane < a.n_experts) a.offsets[e0 + lane] = before + upto - n;
                before += __builtin_amdgcn_readlane(upto, 63);
            }
            if (lane == 0) a.offsets[a.n_experts] = before;
        }
        return;
    }
    int ids[IDS];
#pragma unroll
    for (int i = 0; i < IDS; ++i) ids[i] = 64 * i + lane < pairs ? a.experts[64 * i + lane] : -1;
    for (int j = wave; j < a.each; j += WAVES) {
        const int p = token * a.each + j, e = a.experts[p];
        int before = 0;
#pragma unroll
        for (int i = 0; i < IDS; ++i) {
            const bool counts = ids[i] >= 0 && (ids[i] < e || (ids[i] == e && 64 * i + lane < p));
            before += __popcll(__ballot(counts));
        }
        if (lane == 0) {
            const int place = (unsigned)e < (unsigned)a.n_experts ? before : -1;
            s_places[j] = place;
            a.places[p] = place;
        }
    }
    __syncthreads();
    copy_row(a, token, lane < a.each ? s_places[lane] : -1, threadIdx.x, kSmallThreads);
}

// Many pairs: each expert has `segments` blocks, which number its pairs of a segment each (of whole batches).  All of them look at all pairs: 262 KB for
// 65528, at what a CU gets from its L2; so that is done once, with sums of the lanes' own, and only the segment is looked at again.  (65528 pairs of 64 experts:
// a load for every 64 pairs, one after the other, twice, by a block for each expert 41 us; 16 loads together 15.6; four blocks an expert 12.6)
constexpr int kSortThreads = 1024, kBatch = 16, kBatchPairs = kBatch * kSortThreads;
__global__ __launch_bounds__(kSortThreads) void moe_places_kernel(const DispatchArgs a)
{
    constexpr int WAVES = kSortThreads / 64;
    __shared__ int s_sum[3][WAVES], s_own[2][WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), pairs = a.tokens * a.each;
    const int e = blockIdx.x % (unsigned)a.n_experts, segment = blockIdx.x / (unsigned)a.n_experts, batches = (pairs + kBatchPairs - 1) / kBatchPairs;
    const long long from = (long long)segment * batches / a.segments * kBatchPairs, to = std::min<long long>((segment + 1LL) * batches / a.segments * kBatchPairs, pairs);
    // 16 pairs of the thread's, `step` apart (-1: not there)
    const auto batch = [&](long long at, int step, int (&ids)[kBatch]) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i, at += step) ids[i] = at < pairs ? a.experts[at] : -1;
    };
    int ids[kBatch], less = 0, before = 0, own = 0;
    for (long long i0 = 0; i0 < pairs; i0 += kBatchPairs) {
        batch(i0 + threadIdx.x, kSortThreads, ids);
        int here = 0;
#pragma unroll
        for (int i = 0; i < kBatch; ++i) less += (unsigned)ids[i] < (unsigned)e, here += ids[i] == e;
        own += here;
        before += i0 < from ? here : 0;
    }
    const auto of_wave = [](int x) { return __builtin_amdgcn_readlane(sums_up_to(x), 63); };
    less = of_wave(less), before = of_wave(before), own = of_wave(own);
    if (lane == 0) s_sum[0][wave] = less, s_sum[1][wave] = before, s_sum[2][wave] = own;
    __syncthreads();
    less = before = own = 0;
    for (int w = 0; w < WAVES; ++w) less += s_sum[0][w], before += s_sum[1][w], own += s_sum[2][w];
    if (threadIdx.x == 0 && segment == 0) a.offsets[e] = less;
    if (threadIdx.x == 0 && segment == 0 && e == a.n_experts - 1) a.offsets[e + 1] = less + own;
    int first = less + before, turn = 0;
    for (long long i0 = from; i0 < to; i0 += kBatchPairs, turn ^= 1) {
        // a wave's pairs are consecutive
        const long long at = i0 + wave * (kBatchPairs / WAVES) + lane;
        batch(at, 64, ids);
        int mine = 0;
#pragma unroll
        for (int i = 0; i < kBatch; ++i) mine += __popcll(__ballot(ids[i] == e));
        if (lane == 0) s_own[turn][wave] = mine;
        __syncthreads();
        int place = first;
        for (int w = 0; w < WAVES; ++w) {
            const int n = s_own[turn][w];
            if (w < wave) place += n;
            first += n;
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const uint64_t mask = __ballot(ids[i] == e);
            if (ids[i] == e) a.places[at + 64 * i] = place + lanes_set_below(mask);
            if (e == 0 && (unsigned)ids[i] >= (unsigned)a.n_experts && at + 64 * i < to) a.places[at + 64 * i] = -1;
            place += __popcll(mask);
        }
    }
}
// A block copies a token's row.  Threads: 512, and 1024 for rows of more than 8 KB (4096 tokens of 8 experts: rows of 8 KB 72 us, with 256 threads 79; of
// 16 KB 133, with 512 138 to 144, with 256 145 to 154; of 4 KB 40, with 256 and with 1024 41).
constexpr int kCopyThreads = 1024;
__global__ __launch_bounds__(kCopyThreads) void moe_copy_kernel(const DispatchArgs a)
{
    const int lane = threadIdx.x & 63;
    copy_row(a, blockIdx.x, lane < a.each ? a.places[(long long)blockIdx.x * a.each + lane] : -1, threadIdx.x, blockDim.x);
}

struct CombineArgs {
    const void *y, *grad;
    const int *places, *used;
    const float *weights;
    void *out;
    float *grad_weights;
    long long y_row, grad_row;  // elements
    int tokens, each, rows, pieces;
};
// 8 elements of row `place`
template <class T>
__device__ __forceinline__ vec<T, 8> piece_of(const CombineArgs &a, int place, int piece)
{
    return reinterpret_cast<const vec<T, 8> *>(static_cast<const T *>(a.y) + place * a.y_row)[piece];
}

// Pair j's place, which is -1 where it has no row, and weight, which is then 0 (whatever is there)
struct Pair {
    int place;
    float weight;
};
__device__ __forceinline__ Pair pair_of(const CombineArgs &a, int token, int j)
{
    Pair p{-1, 0.0f};
    if (j < a.each) {
        const long long at = (long long)token * a.each + j;
        p.place = a.places[at];
        p.weight = a.weights[at];
        if ((unsigned)p.place >= (unsigned)a.rows) p = Pair{-1, 0.0f};
    }
    return p;
}

constexpr int kCombineThreads = 256;
template <class T>
__global__ __launch_bounds__(kCombineThreads) void moe_combine_kernel(const CombineArgs a)
{
    const int chunks = (a.pieces + kCombineThreads - 1) / kCombineThreads, token = (int)(blockIdx.x / (unsigned)chunks);
    const int piece = (int)(blockIdx.x % (unsigned)chunks) * kCombineThreads + (int)threadIdx.x;
    // (places and weights are scalar loads, and waves enough are there to hide a row's: 8191 tokens of 8 experts, half of them here, 64 us; with four rows
    // of a thread in flight 68)
    if (piece >= a.pieces) return;
    const int *const places = a.places + (long long)token * a.each;
    const float *const weights = a.weights ? a.weights + (long long)token * a.each : nullptr;
    float sum[8] = {};
    for (int j = 0; j < a.each; ++j) {
        const int place = places[j];
        if ((unsigned)place >= (unsigned)a.rows) continue;
        const float w = weights ? weights[j] : 1.0f;
        const auto x = piece_of<T>(a, place, piece);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = __builtin_fmaf((float)x[e], w, sum[e]);
    }
    vec<T, 8> out;
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = (T)sum[e];
    reinterpret_cast<vec<T, 8> *>(a.out)[(size_t)token * a.pieces + piece] = out;
}

// The gradients: a block takes a token; the blocks behind the tokens clear the rows that no expert has
// Threads: 512, and 256 where a row has no more pieces than that (2047 tokens of 8192 elements, 4 experts each, 65 us, with 256 threads 70, with 1024 63; 4096 of 1024, 8 each,
// with 256 32, with 512 36; 4096 of 4096, 2 each, 36, 37 and 39).
constexpr int kGradThreads = 512;
template <class T>
__global__ __launch_bounds__(kGradThreads) void moe_combine_backward_kernel(const CombineArgs a)
{
    constexpr int kPairs = 4;  // (rows in flight)
    __shared__ float s_dot[kGradThreads / 64][kMostEach];
    const int threads = blockDim.x;
    const int lane = threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    vec<T, 8> *const out = static_cast<vec<T, 8> *>(a.out);
    if ((int)blockIdx.x >= a.tokens) {
        const int used = min(max(*a.used, 0), a.rows);
        for (long long i = (long long)used * a.pieces + (long long)(blockIdx.x - a.tokens) * threads + threadIdx.x; i < (long long)a.rows * a.pieces;
             i += (long long)(gridDim.x - a.tokens) * threads)
            out[i] = vec<T, 8>{};
        return;
    }
    const int token = blockIdx.x;
    const vec<T, 8> *const grad = reinterpret_cast<const vec<T, 8> *>(static_cast<const T *>(a.grad) + token * a.grad_row);
    const Pair pair = pair_of(a, token, lane);
    for (int j0 = 0; j0 < a.each; j0 += kPairs) {
        int place[kPairs];
        float w[kPairs], dot[kPairs] = {};
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            place[j] = __builtin_amdgcn_readlane(pair.place, (j0 + j) & 63);
            w[j] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, pair.weight), (j0 + j) & 63));
        }
        for (int piece = threadIdx.x; piece < a.pieces; piece += threads) {
            const auto g = grad[piece];
            vec<T, 8> y[kPairs];
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                y[j] = vec<T, 8>{};
                if (place[j] >= 0) y[j] = piece_of<T>(a, place[j], piece);
            }
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                if (place[j] < 0) continue;
                vec<T, 8> d;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    dot[j] = __builtin_fmaf((float)g[e], (float)y[j][e], dot[j]);
                    d[e] = (T)((float)g[e] * w[j]);
                }
                out[(size_t)place[j] * a.pieces + piece] = d;
            }
        }
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            for (int d = 32; d; d >>= 1) dot[j] += __shfl_xor(dot[j], d);
            if (lane == 0 && j0 + j < a.each) s_dot[wave][j0 + j] = dot[j];
        }
    }
    __syncthreads();
    if ((int)threadIdx.x < a.each) {
        float dot = s_dot[0][threadIdx.x];
        for (int w = 1; w < threads / 64; ++w) dot += s_dot[w][threadIdx.x];
        a.grad_weights[(long long)token * a.each + threadIdx.x] = dot;
    }
}

}  // namespace lqq

using namespace lqq;

namespace {
constexpr int kMostTokens = 1 << 23;
// A launch holds fewer than 2^32 threads: so many blocks of a size are one (half of what there could be)
constexpr long long blocks_of_launch(int threads) { return (1LL << 31) / threads; }
// launch(first, n) for the tokens, as many at a time as a launch holds
template <class F>
void in_launches(int tokens, long long at_once, F launch)
{
    for (long long first = 0; first < tokens; first += at_once) launch(first, (int)std::min<long long>(at_once, tokens - first));
}
int type_bytes(int type) { return type == LQ_I8 ? 1 : type == LQ_F16 || type == LQ_BF16 ? 2 : 0; }
bool pairs_ok(int tokens, int each) { return tokens >= 0 && each >= 1 && each <= kMostEach && (long long)tokens * each < (1LL << 31) - kBatchPairs; }
}  // namespace

extern "C" int moe_dispatch(int type, int tokens, int each, int n_experts, int K, const void *X, long long x_row, const float *act_scales,
                            const int *experts, void *rows, float *row_scales, int *row_offsets, int *places, void *hip_stream)
{
    const int size = type_bytes(type);
    if (!size) return fail(LQ_ERR_INVALID, "type must be LQ_F16, LQ_BF16 or LQ_I8, got %d", type);
    if (!pairs_ok(tokens, each) || tokens >= kMostTokens) return fail(LQ_ERR_INVALID, "bad shape: %d tokens of %d experts each (1 to %d; up to 2^23 tokens)", tokens, each, kMostEach);
    if (n_experts < 1 || n_experts > kMostExperts) return fail(LQ_ERR_INVALID, "n_experts must be 1 to %d, got %d", kMostExperts, n_experts);
    if (K < 1 || K > (1 << 24) || K * size % 16) return fail(LQ_ERR_INVALID, "bad shape: rows of %d elements (a multiple of 16 bytes)", K);
    if (!row_offsets || (tokens && (!X || !experts || !rows || !places))) return fail(LQ_ERR_INVALID, "null pointer");
    if (!act_scales != !row_scales && tokens) return fail(LQ_ERR_INVALID, "act_scales and row_scales go together");
    if (((uintptr_t)X | (uintptr_t)rows) & 15) return fail(LQ_ERR_ALIGN, "X and rows must be 16-byte aligned");
    if (((uintptr_t)act_scales | (uintptr_t)row_scales | (uintptr_t)experts | (uintptr_t)row_offsets | (uintptr_t)places) & 3)
        return fail(LQ_ERR_ALIGN, "scales, experts, row_offsets and places must be 4-byte aligned");
    if (tokens > 1 && x_row * size % 16) return fail(LQ_ERR_ALIGN, "the stride of X's rows must be a multiple of 16 bytes, got %lld elements", x_row);
    const DispatchArgs a{static_cast<const char *>(X), act_scales, experts, static_cast<char *>(rows), row_scales, row_offsets, places,
                         tokens > 1 ? x_row * size : 0, tokens, each, n_experts, K * size / 16,
                         std::max(1, std::min(256 / n_experts, (tokens * each + kBatchPairs - 1) / kBatchPairs))};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();
    if (tokens * (long long)each <= kFewPairs) {
        const int pairs = tokens * each;
        hipLaunchKernelGGL(pairs <= 128 ? moe_dispatch_small_kernel<2> : pairs <= 1024 ? moe_dispatch_small_kernel<16> : moe_dispatch_small_kernel<kFewPairs / 64>,
                           dim3((unsigned)tokens + 1), dim3(kSmallThreads), 0, st, a);
    } else {
        hipLaunchKernelGGL(moe_places_kernel, dim3((unsigned)(n_experts * a.segments)), dim3(kSortThreads), 0, st, a);
        const int threads = a.pieces > 512 ? kCopyThreads : kCopyThreads / 2;
        in_launches(tokens, blocks_of_launch(threads), [&](long long first, int n) {
            DispatchArgs b = a;
            b.x += first * a.x_row;
            if (a.scales) b.scales += first;
            b.places += first * each;
            hipLaunchKernelGGL(moe_copy_kernel, dim3((unsigned)n), dim3((unsigned)threads), 0, st, b);
        });
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LQ_OK : fail(LQ_ERR_HIP, "dispatch launch failed: %s", hipGetErrorString(e));
}

static int combine_shape(int dtype, int tokens, int each, int rows, int N)
{
    if (dtype != LQ_F16 && dtype != LQ_BF16) return fail(LQ_ERR_INVALID, "dtype must be LQ_F16 or LQ_BF16, got %d", dtype);
    if (!pairs_ok(tokens, each) || rows < 0) return fail(LQ_ERR_INVALID, "bad shape: %d tokens of %d rows each (1 to %d), %d rows", tokens, each, kMostEach, rows);
    if (N < 1 || N > (1 << 24) || N % 8) return fail(LQ_ERR_INVALID, "bad shape: rows of %d elements (a multiple of 8)", N);
    return LQ_OK;
}

extern "C" int moe_combine(int dtype, int tokens, int each, int rows, int N, const void *Y, long long y_row, const int *places, const float *weights,
                           void *out, void *hip_stream)
{
    if (const int rc = combine_shape(dtype, tokens, each, rows, N); rc != LQ_OK) return rc;
    const int pieces = N / 8, chunks = (pieces + kCombineThreads - 1) / kCombineThreads;  // (up to 2^13 blocks a token)
    if (tokens == 0) return LQ_OK;
    if ((rows && !Y) || !places || !out) return fail(LQ_ERR_INVALID, "null pointer");
    if (((uintptr_t)Y | (uintptr_t)out) & 15) return fail(LQ_ERR_ALIGN, "Y and out must be 16-byte aligned");
    if (((uintptr_t)places | (uintptr_t)weights) & 3) return fail(LQ_ERR_ALIGN, "places and weights must be 4-byte aligned");
    if (rows > 1 && y_row % 8) return fail(LQ_ERR_ALIGN, "the stride of Y's rows must be a multiple of 8 elements, got %lld", y_row);
    const CombineArgs a{Y, nullptr, places, nullptr, weights, out, nullptr, rows > 1 ? y_row : 0, 0, tokens, each, rows, pieces};
    (void)hipGetLastError();
    in_launches(tokens, blocks_of_launch(kCombineThreads) / chunks, [&](long long first, int n) {
        CombineArgs b = a;
        b.places += first * each;
        if (weights) b.weights += first * each;
        b.out = static_cast<char *>(out) + 2 * first * N;
        hipLaunchKernelGGL(dtype == LQ_F16 ? moe_combine_kernel<f16> : moe_combine_kernel<bf16>, dim3((unsigned)n * (unsigned)chunks), dim3(kCombineThreads), 0,
                           static_cast<hipStream_t>(hip_stream), b);
    });
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LQ_OK : fail(LQ_ERR_HIP, "combine launch failed: %s", hipGetErrorString(e));
}

extern "C" int moe_combine_backward(int dtype, int tokens, int each, int rows, int N, const void *grad, long long grad_row, const void *Y, long long y_row,
                                    const int *places, const float *weights, const int *rows_used, void *grad_Y, float *grad_weights, void *hip_stream)
{
    if (const int rc = combine_shape(dtype, tokens, each, rows, N); rc != LQ_OK) return rc;
    if (tokens >= kMostTokens) return fail(LQ_ERR_INVALID, "too large: %d tokens (up to 2^23)", tokens);
    if ((tokens && (!grad || !places || !weights || !grad_weights)) || (rows && (!Y || !grad_Y))) return fail(LQ_ERR_INVALID, "null pointer");
    if (((uintptr_t)grad | (uintptr_t)Y | (uintptr_t)grad_Y) & 15) return fail(LQ_ERR_ALIGN, "grad, Y and grad_Y must be 16-byte aligned");
    if (((uintptr_t)places | (uintptr_t)weights | (uintptr_t)rows_used | (uintptr_t)grad_weights) & 3)
        return fail(LQ_ERR_ALIGN, "places, weights, rows_used and grad_weights must be 4-byte aligned");
    if ((rows > 1 && y_row % 8) || (tokens > 1 && grad_row % 8)) return fail(LQ_ERR_ALIGN, "strides of rows must be multiples of 8 elements");
    const int pieces = N / 8, clearing = rows_used && rows ? 256 : 0;
    if (tokens + clearing == 0) return LQ_OK;
    const CombineArgs a{Y, grad, places, rows_used, weights, grad_Y, grad_weights, rows > 1 ? y_row : 0, tokens > 1 ? grad_row : 0, tokens, each, rows, pieces};
    (void)hipGetLastError();
    const int threads = pieces > 256 ? kGradThreads : 256;
    const auto go = [&](long long first, int n) {
        CombineArgs b = a;
        b.grad = static_cast<const char *>(grad) + 2 * first * a.grad_row;
        b.places += first * each;
        b.weights += first * each;
        b.grad_weights += first * each;
        b.tokens = n;
        hipLaunchKernelGGL(dtype == LQ_F16 ? moe_combine_backward_kernel<f16> : moe_combine_backward_kernel<bf16>, dim3((unsigned)(n + (first ? 0 : clearing))),
                           dim3((unsigned)threads), 0, static_cast<hipStream_t>(hip_stream), b);
    };
    if (tokens)
        in_launches(tokens, blocks_of_launch(threads), go);
    else
        go(0, 0);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LQ_OK : fail(LQ_ERR_HIP, "gradient launch failed: %s", hipGetErrorString(e));
}
