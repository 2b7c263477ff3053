// Gradients of low-rank adapters' factors: dW_i[c][k] = scale_i sum_t y[t][c] h[t][k] over the rows t of adapter i.
//
// Bound by reading y, 128 columns of which a CTA takes over a run of the adapter's rows (its segments' rows one after the
// other); the r columns of h are few.  Long adapters are cut into runs, whose sums meet in a second kernel in a fixed order.  h is
// FP32 and goes through the tensor cores as a sum of 16-bit parts, two for 16-bit gradients and FP16, three for FP32
// gradients of BF16; FP16 parts are taken of a column of 64 rows over a power of two.  The chain of the tensor cores'
// additions is cut every 64 rows.
#include <algorithm>
#include <type_traits>

#include "adapter_common.h"

namespace gpd {
namespace adapter {

namespace {

constexpr int kThreads = 256, kCols = 128, kRows = 64, kStages = 3, kMostRows = 2048;
constexpr int kYPitch = 2 * kCols + 16, kYStage = kRows * kYPitch;

struct Job {
    GradArgs two[2];
    Segments seg;
    const int32_t* slots;                              // [n + 1]: adapter i has the runs slots[i] .. slots[i + 1] - 1
    float* parts;                                      // [runs][part_size]
    int64_t part_size, run;                            // floats of a run's sums; rows of a run
    unsigned first_tiles;                              // column tiles of two[0]
    int r, max_slots;
    bool accumulate;
};

// Runs of every adapter.  One CTA; counts: n numbers of scratch.
__global__ void __launch_bounds__(256) plan_kernel(const __grid_constant__ Segments s, int64_t run, int max_slots, unsigned long long* counts,
                                                   int32_t* slots) {
    __shared__ int warp_sum[8];
    __shared__ int carry;
    after_previous();
    for (int i = threadIdx.x; i < s.n; i += 256) counts[i] = 0;
    if (threadIdx.x == 0) carry = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < s.S; i += 256) {
        const int64_t id = number(s.index, i, s.wide), rows = offset_at(s, i + 1) - offset_at(s, i);
        if (id >= 0 && id < s.n && rows > 0) atomicAdd(counts + id, (unsigned long long)rows);     // whole numbers: any order
    }
    __threadfence_block();
    __syncthreads();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int base = 0; base < s.n; base += 256) {
        const int i = base + threadIdx.x;
        const int64_t want = i < s.n ? max((int64_t)1, ((int64_t)counts[i] + run - 1) / run) : 0;
        const int own = (int)min(want, (int64_t)max_slots);
        int scan = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += v;
        }
        if (lane == 31) warp_sum[warp] = scan;
        __syncthreads();
        int before = carry;
        for (int k = 0; k < warp; ++k) before += warp_sum[k];
        if (i < s.n) slots[i] = min(before + scan - own, max_slots);
        __syncthreads();
        if (threadIdx.x == 255) carry = min(before + scan, max_slots);
        __syncthreads();
    }
    if (threadIdx.x == 0) slots[s.n] = carry;
}

// Rows v0 .. v0 + count - 1 of the adapter's rows, in `rows`; returns how many there are.  One warp.
__device__ __forceinline__ int list_rows(const Segments& s, int64_t id, int64_t v0, int count, int32_t* rows) {
    const int lane = threadIdx.x & 31;
    int64_t seen = 0;
    for (int64_t base = 0; base < s.S && seen < v0 + count; base += 32) {
        const int64_t i = base + lane;
        int64_t at = 0, len = 0;
        if (i < s.S && number(s.index, i, s.wide) == id) {
            at = offset_at(s, i);
            len = max((int64_t)0, offset_at(s, i + 1) - at);
        }
        uint32_t mine = __ballot_sync(0xffffffffu, len > 0);
        while (mine) {
            const int who = __ffs(mine) - 1;
            mine &= mine - 1;
            const int64_t start = __shfl_sync(0xffffffffu, at, who), n = __shfl_sync(0xffffffffu, len, who);
            const int64_t lo = max((int64_t)0, v0 - seen), hi = min(n, v0 + count - seen);
            for (int64_t j = lo + lane; j < hi; j += 32) rows[seen + j - v0] = (int32_t)(start + j);
            seen += n;
        }
    }
    return (int)min((int64_t)count, max((int64_t)0, seen - v0));
}

__device__ __forceinline__ void add_to(float* p, float v, bool accumulate) { *p = accumulate ? *p + v : v; }
__device__ __forceinline__ void add_to(__nv_bfloat16* p, float v, bool accumulate) { *p = from_f32<__nv_bfloat16>(accumulate ? to_f32(*p) + v : v); }
__device__ __forceinline__ void add_to(__half* p, float v, bool accumulate) { *p = from_f32<__half>(accumulate ? to_f32(*p) + v : v); }

template <int MT, int PARTS>
struct Shape {
    static constexpr int RP = 16 * MT, PITCH = 2 * RP + 16, PLANE = kRows * PITCH;
    static constexpr int SMEM = kStages * kYStage + PARTS * PLANE;
    static constexpr int PER = kRows * RP / kThreads;  // elements of h that a thread brings per stage
};

// MT: 16 columns of h each.  A warp has all of them and 16 columns of y.
template <typename T, typename O, int MT, int PARTS>
__global__ void __launch_bounds__(kThreads) grad_kernel(const __grid_constant__ Job job) {
    using S = Shape<MT, PARTS>;
    constexpr bool kScaled = std::is_same<T, __half>::value;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int32_t rows[kMostRows];
    __shared__ int n_rows;
    __shared__ int most[2][S::RP];                     // FP16: bits of the largest magnitude of every column of h in a stage
    after_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int slot = blockIdx.y, n = job.seg.n;
    if (slot >= job.slots[n]) return;
    int lo = 0, hi = n - 1;                            // the last adapter whose first run is <= slot
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (job.slots[mid] <= slot) lo = mid;
        else hi = mid - 1;
    }
    const int first = job.slots[lo], runs = job.slots[lo + 1] - first;
    const bool second = blockIdx.x >= job.first_tiles;
    const GradArgs& a = job.two[second];
    const int64_t c0 = (int64_t)(blockIdx.x - (second ? job.first_tiles : 0)) * kCols;
    if (warp == 0) {
        const int have = list_rows(job.seg, lo, (slot - first) * job.run, (int)job.run, rows);
        if (lane == 0) n_rows = have;
    }
    for (int i = threadIdx.x; i < 2 * S::RP; i += kThreads) (&most[0][0])[i] = 0;
    __syncthreads();
    const int count = n_rows, stages = (count + kRows - 1) / kRows;
    const uint32_t ring = smem_at(smem), planes = ring + kStages * kYStage;
    const T* y = static_cast<const T*>(a.y) + c0;
    auto fetch = [&](int k) {
        if (k < stages) {
            const uint32_t at = ring + k % kStages * kYStage;
#pragma unroll
            for (int i = 0; i < kRows * kCols / 8 / kThreads; ++i) {
                const int e = threadIdx.x + i * kThreads, row = e / (kCols / 8), c = e % (kCols / 8) * 8, v = k * kRows + row;
                const int left = v < count ? (int)min((int64_t)8, a.C - c0 - c) : 0;
                stage8<T>(at + row * kYPitch + 2 * c, left > 0 ? y + (int64_t)rows[v] * a.ldy + c : y, left, a.y_vec);
            }
        }
        copies_end();
    };
    const int hc = threadIdx.x % S::RP, hr = threadIdx.x / S::RP;      // column of h, first row
    float hv[S::PER];
    auto fetch_h = [&](int k) {
#pragma unroll
        for (int i = 0; i < S::PER; ++i) {
            const int v = k * kRows + hr + i * (kThreads / S::RP);
            hv[i] = v < count && hc < job.r ? a.h[(int64_t)rows[v] * job.r + hc] : 0.f;
        }
    };
    float sum[MT][2][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[m][j][i] = 0.f;
    for (int i = 0; i < kStages - 1; ++i) fetch(i);
    fetch_h(0);
    for (int k = 0; k < stages; ++k) {
        if (kScaled) {
            float m = 0.f;
#pragma unroll
            for (int i = 0; i < S::PER; ++i) m = fmaxf(m, fabsf(hv[i]));
            atomicMax(&most[k & 1][hc], __float_as_int(m));
            __syncthreads();
        }
        const float by = kScaled ? power2(-exponent_of(__int_as_float(most[k & 1][hc]))) : 1.f;
#pragma unroll
        for (int i = 0; i < S::PER; ++i) {
            uint32_t parts[PARTS];
            split2<T, PARTS>(hv[i] * by, 0.f, parts);
            const uint32_t at = planes + (hr + i * (kThreads / S::RP)) * S::PITCH + 2 * hc;
#pragma unroll
            for (int p = 0; p < PARTS; ++p) asm volatile("st.shared.u16 [%0], %1;" ::"r"(at + p * S::PLANE), "h"((unsigned short)parts[p]) : "memory");
        }
        copies_wait<kStages - 2>();
        __syncthreads();
        fetch(k + kStages - 1);
        fetch_h(k + 1);
        float acc[MT][2][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][j][i] = 0.f;
        const uint32_t ys = ring + k % kStages * kYStage;
#pragma unroll
        for (int s = 0; s < kRows / 16; ++s) {
            uint32_t b[4];
            ldmatrix4<true>(b, ys + (16 * s + (lane & 15)) * kYPitch + 2 * (16 * warp + (lane >> 4) * 8));
#pragma unroll
            for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    uint32_t h[4];
                    ldmatrix4<true>(h, planes + p * S::PLANE + (16 * s + (lane & 7) + (lane >> 4) * 8) * S::PITCH + 2 * (16 * m + (lane >> 3 & 1) * 8));
                    mma(acc[m][0], h, b[0], b[1], T());
                    mma(acc[m][1], h, b[2], b[3], T());
                }
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float undo = kScaled ? power2(exponent_of(__int_as_float(most[k & 1][16 * m + (lane >> 2) + 8 * (i >> 1)]))) : 1.f;
#pragma unroll
                for (int j = 0; j < 2; ++j) sum[m][j][i] = fmaf(acc[m][j][i], undo, sum[m][j][i]);
            }
        __syncthreads();
        if (kScaled)
            for (int i = threadIdx.x; i < S::RP; i += kThreads) most[k & 1][i] = 0;
    }
    copies_wait<0>();
    const float scale = a.scale ? a.scale[lo] : 1.f;
    O* dw = static_cast<O*>(a.dw) + lo * a.next;
    float* part = job.parts + slot * job.part_size + (second ? job.two[0].C * job.r : 0);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int kr = 16 * m + (lane >> 2) + 8 * (i >> 1);
                const int64_t c = c0 + 16 * warp + 8 * j + 2 * (lane & 3) + (i & 1);
                if (kr >= job.r || c >= a.C) continue;
                const float v = sum[m][j][i] * scale;
                if (runs == 1) add_to(dw + (a.transposed ? kr * a.ldw + c : c * a.ldw + kr), v, job.accumulate);
                else part[a.transposed ? kr * a.C + c : c * job.r + kr] = v;
            }
}

// Sums of the runs of the adapters that have several.
template <typename O>
__global__ void __launch_bounds__(256) runs_kernel(const __grid_constant__ Job job) {
    after_previous();
    const int i = blockIdx.y, first = job.slots[i], runs = job.slots[i + 1] - first;
    if (runs == 1) return;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < job.part_size; e += (int64_t)gridDim.x * 256) {
        float v = 0.f;
        const float* p = job.parts + first * job.part_size + e;
#pragma unroll 4
        for (int k = 0; k < runs; ++k) v += p[k * job.part_size];
        const bool second = e >= job.two[0].C * job.r;
        const GradArgs& a = job.two[second];
        const int64_t at = e - (second ? job.two[0].C * job.r : 0), width = a.transposed ? a.C : job.r;
        add_to(static_cast<O*>(a.dw) + i * a.next + at / width * a.ldw + at % width, v, job.accumulate);
    }
}

// Rows of a run: enough runs that three CTAs per SM (of 148) are busy, of 256 rows at least.
int64_t run_rows(int64_t T, int64_t K, int64_t N) {
    const int64_t tiles = (K + kCols - 1) / kCols + (N + kCols - 1) / kCols, runs = std::max<int64_t>(1, (3 * 148 + tiles - 1) / std::max<int64_t>(tiles, 1));
    const int64_t rows = ((T + runs - 1) / runs + kRows - 1) / kRows * kRows;
    return std::min<int64_t>(kMostRows, std::max<int64_t>(256, rows));
}
int64_t slots_of(int64_t T, int64_t n, int64_t K, int64_t N) { return T / run_rows(T, K, N) + n; }
int64_t up(int64_t bytes) { return (bytes + 255) / 256 * 256; }

template <typename T, typename O, int MT>
gpd_status launch(const Job& job, cudaStream_t st) {
    constexpr int PARTS = sizeof(O) == 4 && std::is_same<T, __nv_bfloat16>::value ? 3 : 2;
    using S = Shape<MT, PARTS>;
    auto kernel = grad_kernel<T, O, MT, PARTS>;
    if (S::SMEM > 40960 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) != cudaSuccess) return GPD_ERR_CUDA;
    const int64_t tiles = job.first_tiles + (job.two[1].C + kCols - 1) / kCols;
    if (tiles == 0 || job.seg.n == 0) return GPD_OK;
    gpd_status rc = launch_after(kernel, dim3((unsigned)tiles, (unsigned)job.max_slots), dim3(kThreads), S::SMEM, 1, st, job);
    if (rc != GPD_OK || job.max_slots == job.seg.n) return rc;         // as many runs as adapters: each has one
    const unsigned blocks = (unsigned)std::min<int64_t>((job.part_size + 255) / 256, 16 * sm_count());
    return launch_after(runs_kernel<O>, dim3(blocks, (unsigned)job.seg.n), dim3(256), 0, 1, st, job);
}
template <typename T, typename O>
gpd_status launch_rank(const Job& job, cudaStream_t st) {
    if (job.r <= 16) return launch<T, O, 1>(job, st);
    if (job.r <= 32) return launch<T, O, 2>(job, st);
    return job.r <= 64 ? launch<T, O, 4>(job, st) : launch<T, O, 8>(job, st);
}

}  // namespace

// Counts, runs, their sums
int64_t grad_workspace(int64_t T, int64_t n, int64_t r, int64_t K, int64_t N) {
    const int64_t slots = slots_of(T, n, K, N);
    return up(8 * n) + up(4 * (n + 1)) + (slots > n ? up(4 * slots * r * (K + N)) : 0);
}

gpd_status gradients(int type, int grad_type, bool accumulate, const Segments& seg, int r, const GradArgs (&two)[2], void* workspace,
                     cudaStream_t st) {
    Job job;
    job.two[0] = two[0];
    job.two[1] = two[1];
    job.seg = seg;
    job.r = r;
    job.accumulate = accumulate;
    job.run = run_rows(seg.T, two[0].C, two[1].C);
    const int64_t slots = slots_of(seg.T, seg.n, two[0].C, two[1].C);
    if (slots > 65535) return GPD_ERR_SHAPE;
    job.max_slots = (int)slots;
    job.part_size = (two[0].C + two[1].C) * r;
    job.first_tiles = (unsigned)((two[0].C + kCols - 1) / kCols);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    unsigned long long* counts = reinterpret_cast<unsigned long long*>(ws);
    int32_t* runs = reinterpret_cast<int32_t*>(ws + up(8 * seg.n));
    job.slots = runs;
    job.parts = reinterpret_cast<float*>(ws + up(8 * seg.n) + up(4 * ((int64_t)seg.n + 1)));
    const gpd_status rc = launch_after(plan_kernel, dim3(1), dim3(256), 0, 1, st, seg, job.run, job.max_slots, counts, runs);
    if (rc != GPD_OK) return rc;
    if (type == GPD_DT_BF16)
        return grad_type == GPD_DT_F32 ? launch_rank<__nv_bfloat16, float>(job, st) : launch_rank<__nv_bfloat16, __nv_bfloat16>(job, st);
    return grad_type == GPD_DT_F32 ? launch_rank<__half, float>(job, st) : launch_rank<__half, __half>(job, st);
}

}  // namespace adapter
}  // namespace gpd
