// Four host threads call gpd_adapter at once, each with sizes and a stream of its own.  Prints how many calls were refused and ends with
// status 1 if any was, or if a result is wrong.
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <thread>
#include <vector>

#include "gpd.h"

namespace {

template <typename T>
T* upload(const std::vector<T>& v) {
    T* p = nullptr;
    if (cudaMalloc(reinterpret_cast<void**>(&p), v.size() * sizeof(T)) != cudaSuccess ||
        cudaMemcpy(p, v.data(), v.size() * sizeof(T), cudaMemcpyHostToDevice) != cudaSuccess)
        std::exit(2);
    return p;
}
constexpr uint16_t kOne = 0x3f80;                      // 1 in BF16

// T segments of one row.  x, A and B are ones, so that h = K and out = 16 K, a power of two.
struct Caller {
    int T, r = 16;
    int64_t K, N;
    uint16_t *x, *A, *B, *out;
    float* h;
    int32_t *offsets, *index;
    cudaStream_t stream;
    Caller(int T, int64_t K, int64_t N) : T(T), K(K), N(N) {
        std::vector<int32_t> o(T + 1), i(T, 0);
        for (int t = 0; t <= T; ++t) o[t] = t;
        x = upload(std::vector<uint16_t>(T * K, kOne));
        A = upload(std::vector<uint16_t>(r * K, kOne));
        B = upload(std::vector<uint16_t>(N * r, kOne));
        out = upload(std::vector<uint16_t>(T * N, 0));
        h = upload(std::vector<float>(T * r, 0.f));
        offsets = upload(o);
        index = upload(i);
        if (cudaStreamCreateWithFlags(&stream, cudaStreamNonBlocking) != cudaSuccess) std::exit(2);
    }
    gpd_status call() const {
        return gpd_adapter(GPD_DT_BF16, x, K, 1, r, A, K, r * K, B, r, N * r, nullptr, 4, offsets, index, T, h, GPD_DT_BF16, nullptr, 0, out, N, T, K, N,
                           stream);
    }
    bool right() const {
        std::vector<uint16_t> o(T * N);
        if (cudaMemcpy(o.data(), out, o.size() * 2, cudaMemcpyDeviceToHost) != cudaSuccess) return false;
        float want = (float)(r * K);
        uint32_t bits;
        __builtin_memcpy(&bits, &want, 4);
        for (uint16_t v : o)
            if (v != bits >> 16) return false;
        return true;
    }
};

}  // namespace

int main() {
    const std::vector<Caller> callers = {{1, 128, 128}, {40, 512, 1024}, {3, 4096, 4096}, {64, 256, 512}};
    cudaDeviceSynchronize();
    std::atomic<int> refused{0};
    std::vector<std::thread> threads;
    for (const Caller& c : callers)
        threads.emplace_back([&refused, &c] {
            cudaFree(nullptr);
            for (int i = 0; i < 20000; ++i)
                if (c.call() != GPD_OK) ++refused;
        });
    for (auto& t : threads) t.join();
    bool right = cudaDeviceSynchronize() == cudaSuccess;
    for (const Caller& c : callers) right = right && c.right();
    std::printf("refused %d of %d, results %s\n", refused.load(), 20000 * (int)callers.size(), right ? "right" : "wrong");
    return refused || !right;
}
