// Host threads that enqueue on one stream with one workspace, without a GPU: the runtime's launch is replaced by one that writes
// down who launched, and takes its time.  The launches of a call have to stand together; calls on another stream do not wait.
#include <hip/hip_runtime_api.h>

#include <atomic>
#include <chrono>
#include <condition_variable>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <mutex>
#include <thread>
#include <vector>

#include "liquidgemm.h"

namespace {
struct Launch {
    hipStream_t stream;
    int call;
};
std::mutex mutex;
std::condition_variable logged;
std::vector<Launch> launches;
thread_local int call = 0;
hipStream_t const kOne = reinterpret_cast<hipStream_t>(0x1000), kOther = reinterpret_cast<hipStream_t>(0x2000);
bool waited_for_the_other = false, the_other_came = false;

int launches_on(hipStream_t s)
{
    int n = 0;
    for (const Launch &l : launches) n += l.stream == s;
    return n;
}
}  // namespace

extern "C" {
// (what a launch hands to its kernel's stub, which hands it on)
thread_local struct {
    dim3 grid, block;
    size_t lds;
    hipStream_t stream;
} asked;
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) { return asked = {grid, block, lds, stream}, hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream)
{
    return *grid = asked.grid, *block = asked.block, *lds = asked.lds, *stream = asked.stream, hipSuccess;
}
hipError_t hipLaunchKernel(const void *, dim3, dim3 block, void **, size_t, hipStream_t stream)
{
    std::unique_lock<std::mutex> lock(mutex);
    launches.push_back({stream, call});
    logged.notify_all();
    if (stream == kOne && block.x == 1024 && !waited_for_the_other) {  // (the first list of chunks: held until the other stream has a launch)
        waited_for_the_other = true;
        const int before = launches_on(kOther);
        the_other_came = logged.wait_for(lock, std::chrono::seconds(20), [&] { return launches_on(kOther) > before; });
    }
    lock.unlock();
    if (stream == kOne) std::this_thread::sleep_for(std::chrono::milliseconds(3));
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipFuncSetAttribute(const void *, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipGetDevice(int *device) { return *device = 0, hipSuccess; }
hipError_t hipDeviceGetAttribute(int *value, hipDeviceAttribute_t, int) { return *value = 256, hipSuccess; }
}

int main()
{
    char *const p = reinterpret_cast<char *>(1 << 20);  // an address that is aligned and never followed
    int *const ints = reinterpret_cast<int *>(p);
    const size_t all = (size_t)1 << 40;
    const auto decode = [&](int seqs, hipStream_t s) {
        return kv4_attention(LQ_F16, seqs, 1, 32, 8, 128, p, 4096, 4096, 128, p, 10, 16, ints, 5, ints, 0.1f, p, p, all, s);
    };
    const auto prompt = [&](hipStream_t s) {
        return attn_prompt(LQ_F16, 2, 200, 8000, 8, 2, 128, p, 1024, 128, p, 256, 128, p, 256, 128, ints, ints, 0.1f, 1, p, p, all, s);
    };
    const auto gemm = [&](const char *name, int M, int N, int K, hipStream_t s) {
        for (int v = 0; v < w4a8_variant_count(); ++v)
            if (!strcmp(w4a8_variant_name(v), name))
                return w4a8_gemm_variant(v, M, N, K, 64, reinterpret_cast<int8_t *>(p), reinterpret_cast<float *>(p), p, reinterpret_cast<uint8_t *>(p),
                                         reinterpret_cast<float *>(p), reinterpret_cast<uint16_t *>(p), nullptr, p, all, s);
        return -1;
    };
    const std::vector<std::function<int()>> calls = {
        [&] { return decode(128, kOne); },  // two launches each
        [&] { return decode(300, kOne); },
        [&] { return gemm("solo16_g2_m256_s4", 256, 256, 16384, kOne); },
        [&] { return decode(2, kOne); },    // one launch each, which write to the workspace too
        [&] { return prompt(kOne); },
        [&] { return gemm("duo_m64_s2", 64, 256, 4096, kOne); },
    };
    std::atomic<int> failed{0}, running{(int)calls.size()};
    std::vector<std::thread> threads;
    for (size_t i = 0; i < calls.size(); ++i)
        threads.emplace_back([&, i] {
            for (int n = 0; n < 8; ++n) {
                call = (int)i * 100 + n;
                if (const int rc = calls[i]()) ++failed, fprintf(stderr, "call %zu: %d %s\n", i, rc, w4a8_last_error());
            }
            --running;
        });
    threads.emplace_back([&] {
        call = 10000;
        while (running > 0) {
            if (decode(2, kOther)) ++failed;
            std::this_thread::sleep_for(std::chrono::milliseconds(1));
        }
    });
    for (std::thread &t : threads) t.join();

    std::vector<Launch> one;
    for (const Launch &l : launches)
        if (l.stream == kOne) one.push_back(l);
    int torn = 0, pairs = 0;
    for (size_t i = 0; i < one.size(); ++i)
        for (size_t j = i + 1; j < one.size(); ++j)
            if (one[i].call == one[j].call) ++pairs, torn += j != i + 1;
    printf("%zu launches on the stream, %d calls of two, %d of these torn apart; the other stream %s\n", one.size(), pairs, torn,
           the_other_came ? "went on" : "waited");
    if (failed || one.size() != 72 || pairs != 24 || torn || !the_other_came) return 1;
    printf("stream_turns ok\n");
    return 0;
}
