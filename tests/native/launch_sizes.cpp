// The launches of the calls that sort tokens by expert and bring them back, without a GPU: the runtime's launch is replaced by one that
// refuses what a GPU refuses (2^32 threads or more) and counts the blocks.
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <cstring>
#include <vector>

#include "liquidgemm.h"

namespace {
struct Launch {
    unsigned long long blocks, threads;
};
std::vector<Launch> launches;
hipError_t status = hipSuccess;
struct {
    dim3 grid, block;
    size_t lds;
    hipStream_t stream;
} asked;
}  // namespace

extern "C" {
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) { return asked = {grid, block, lds, stream}, hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream)
{
    return *grid = asked.grid, *block = asked.block, *lds = asked.lds, *stream = asked.stream, hipSuccess;
}
hipError_t hipLaunchKernel(const void *, dim3 grid, dim3 block, void **, size_t, hipStream_t)
{
    launches.push_back({(unsigned long long)grid.x * grid.y * grid.z, (unsigned long long)block.x * block.y * block.z});
    if (launches.back().blocks * launches.back().threads >> 32) return status = hipErrorInvalidConfiguration;
    return hipSuccess;
}
hipError_t hipGetLastError()
{
    const hipError_t e = status;
    return status = hipSuccess, e;
}
}

int main()
{
    char *const p = reinterpret_cast<char *>(1 << 20);  // an address that is aligned and never followed
    int *const ints = reinterpret_cast<int *>(p);
    int wrong = 0;
    // a call's launches from the first-th on have to have `blocks` blocks together
    const auto check = [&](const char *what, int tokens, int K, int rc, size_t first, unsigned long long blocks) {
        unsigned long long sum = 0;
        for (size_t i = first; i < launches.size(); ++i) sum += launches[i].blocks;
        const bool ok = rc == LQ_OK && sum == blocks;
        if (!ok) printf("%s of %d tokens, rows of %d: returned %d (%s), %llu blocks of %llu\n", what, tokens, K, rc, rc ? w4a8_last_error() : "", sum, blocks);
        wrong += !ok;
        launches.clear();
    };
    for (const int tokens : {1 << 11, (1 << 21) - 1, 1 << 21, (1 << 22) - 1, 1 << 22, (1 << 22) + 1, 6000001, (1 << 23) - 1025, (1 << 23) - 1}) {
        for (const int K : {16, 4096, 4104, 8200, 1 << 20})
            for (const int x_row : {K, 0}) {
                const int rc = moe_dispatch(LQ_F16, tokens, 2, 8, K, p, x_row, nullptr, ints, p, nullptr, ints, ints, nullptr);
                check("dispatch", tokens, K, rc, 1, tokens);
            }
    }
    // (back: as many blocks a token as its row has pieces of 256 times 16 bytes; the gradients: 256 blocks clear what no expert has)
    for (const int tokens : {0, 1, (1 << 21) + 3, 1 << 22, 5000000, (1 << 23) - 1025, (1 << 23) - 1024, (1 << 23) - 1, 1 << 23, (1 << 24) + 5}) {
        for (const int N : {8, 2048, 2056, 4096, 8200, 1 << 24}) {
            if ((long long)tokens * ((N + 2047) / 2048) < 1LL << 31) {
                const int rc = moe_combine(LQ_BF16, tokens, 2, 100, N, p, N, ints, nullptr, p, nullptr);
                check("combine", tokens, N, rc, 0, (unsigned long long)tokens * ((N + 2047) / 2048));
            }
            if (tokens < 1 << 23) {
                const int rc = moe_combine_backward(LQ_F16, tokens, 2, 100, N, p, N, p, N, ints, reinterpret_cast<float *>(p), ints, p, reinterpret_cast<float *>(p), nullptr);
                check("gradients", tokens, N, rc, 0, tokens + 256ull);
            }
        }
    }
    if (wrong) return 1;
    printf("launch_sizes ok\n");
    return 0;
}
