// Gradients of low-rank adapters' factors: dW_i[c][k] = scale_i sum_t y[t][c] h[t][k] over the rows t of adapter i.
//
// Bound by reading y, 128 columns of which a CTA takes over a part of the adapter's rows (its segments' rows one after the
// other); the r columns of h are few.  The parts' sums meet in a fixed order.  h is FP32 and goes through the tensor cores as a
// sum of 16-bit parts, three, or two for FP16 gradients of FP16.  The chain of the tensor cores' additions is cut every 64 rows
// (every 256 for FP16 gradients of FP16 by TMA: 32 steps, of at most 2^-22 each).
// Two forms.  Rows on 16-byte boundaries and segments that are not short: a first kernel cuts h into its parts, once for all
// columns of y, and tiles of both come by TMA, 64 rows of one segment each; the CTAs of a cluster share an adapter's rows and
// add up over distributed shared memory; FP16 parts are taken of an adapter's column over a power of two.  Otherwise
// rows are gathered by their numbers in runs, whose sums go through memory, and h is cut by every CTA; FP16 parts are then taken
// of a column of 64 rows over a power of two.
//
// Measured: 8192 x 4096 and 4096 columns, one adapter of rank 16, FP32 gradients: 34 us of 21 at the copy bandwidth (DRAM 50 %,
// tensor pipe 11 %), 40 before the tensor memory form.  At rank 128 the parts of h, which every 128 columns of y read again, bound it: 4868
// rows x 10560 and 1408 columns 108 us, 0.47 GB through L2; more CTAs that share the rows do not help (three: 125 us).
#include <cooperative_groups.h>

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
    const int32_t* slots;                              // [n + 1]: adapter i has the runs (chunks) slots[i] .. slots[i + 1] - 1
    int2* chunks;                                      // by TMA: first row and rows of the adapters' chunks, up to 64 rows of a segment
    float* parts;                                      // [runs][tiles]: a tile's sums, as the threads hold them
    int64_t run;                                       // rows of a run, a multiple of 64
    const int32_t* most;                               // FP16: bits of the largest magnitudes of h's columns, [2][n][RP]
    unsigned first_tiles, tiles;                       // column tiles of two[0], of both
    int r, max_slots;
    bool accumulate;
};

// Runs of every adapter, `least` or more.  One CTA; counts: n numbers of scratch.  Segments take up whole multiples of `unit` rows.
__device__ __forceinline__ void plan_runs(const Segments& s, int64_t run, int unit, int least, int max_slots, unsigned long long* counts, int32_t* slots) {
    __shared__ long long warp_sum[8], carry;           // offsets that mean nothing may add up to anything
    for (int i = threadIdx.x; i < s.n; i += 256) counts[i] = 0;
    if (threadIdx.x == 0) carry = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < s.S; i += 256) {
        const int64_t id = number(s.index, i, s.wide), rows = (offset_at(s, i + 1) - offset_at(s, i) + unit - 1) / unit * unit;
        if (id >= 0 && id < s.n && rows > 0) atomicAdd(counts + id, (unsigned long long)rows);     // whole numbers: any order
    }
    __threadfence_block();
    __syncthreads();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int base = 0; base < s.n; base += 256) {
        const int i = base + threadIdx.x;
        const int64_t want = i < s.n ? max((int64_t)least, ((int64_t)__ldcg(counts + i) + run - 1) / run) : 0;
        const long long own = min(want, (int64_t)max_slots);
        long long scan = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += v;
        }
        if (lane == 31) warp_sum[warp] = scan;
        __syncthreads();
        long long before = carry;
        for (int k = 0; k < warp; ++k) before += warp_sum[k];
        if (i < s.n) slots[i] = (int)min(before + scan - own, (long long)max_slots);
        __syncthreads();
        if (threadIdx.x == 255) carry = min(before + scan, (long long)max_slots);
        __syncthreads();
    }
    if (threadIdx.x == 0) slots[s.n] = (int)carry;
}
__global__ void __launch_bounds__(256) plan_kernel(const __grid_constant__ Segments s, int64_t run, int max_slots, unsigned long long* counts,
                                                   int32_t* slots) {
    after_previous();
    plan_runs(s, run, 1, 1, max_slots, counts, slots);
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

// A tile's sums: sum[m][j] are rows 16 m + g and g + 8 (columns of h), columns 8 (NT warp + j) + 2 q and the next, of 128.
template <int WARPS>
__device__ __forceinline__ void tile_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(32 * WARPS) : "memory"); }
// They leave through shared memory (16 MT rows of 132 floats), so that neighbours leave together.
constexpr int kTileWidth = kCols + 4;
template <int MT, int NT>
__device__ __forceinline__ void put_tile(const float (&sum)[MT][NT][4], float* tile) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            float* p = tile + (16 * m + (lane >> 2)) * kTileWidth + 8 * (NT * warp + j) + 2 * (lane & 3);
            *reinterpret_cast<float2*>(p) = make_float2(sum[m][j][0], sum[m][j][1]);
            *reinterpret_cast<float2*>(p + 8 * kTileWidth) = make_float2(sum[m][j][2], sum[m][j][3]);
        }
}
// Writes a tile where it belongs: four of its numbers at (row k of h, column c) come from get(k, c).  Of `threads` threads this is
// number `first`.
template <typename O, typename F>
__device__ __forceinline__ void write_tile(const Job& job, const GradArgs& a, int64_t id, int64_t c0, int first, int threads, F get) {
    const int cols = (int)min((int64_t)kCols, a.C - c0), r = job.r;
    O* dw = static_cast<O*>(a.dw) + id * a.next;
    if (a.transposed) {
        O* to = dw + c0;
        const bool vec = a.ldw % 4 == 0 && (reinterpret_cast<uintptr_t>(to) & (4 * sizeof(O) - 1)) == 0 && !job.accumulate;
#pragma unroll 1
        for (int e = first; e < r * (kCols / 4); e += threads) {
            const int k = e / (kCols / 4), c = e % (kCols / 4) * 4;
            if (c >= cols) continue;
            const float4 v = get(k, c);
            O* p = to + k * a.ldw + c;
            if (vec && c + 4 <= cols) {
                if constexpr (sizeof(O) == 4) *reinterpret_cast<float4*>(p) = v;
                else *reinterpret_cast<uint2*>(p) = make_uint2(pack2(v.x, v.y, O()), pack2(v.z, v.w, O()));
            } else {
                const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (c + i < cols) add_to(p + i, f[i], job.accumulate);
            }
        }
    } else {
        // four columns of y (rows of dW) at one column of h
#pragma unroll 1
        for (int e = first; e < r * (kCols / 4); e += threads) {
            const int g = e / r, k = e - g * r, c = 4 * g;
            if (c >= cols) continue;
            const float4 v = get(k, c);
            const float f[4] = {v.x, v.y, v.z, v.w};
            O* p = dw + (c0 + c) * a.ldw + k;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + i < cols) add_to(p + i * a.ldw, f[i], job.accumulate);
        }
    }
}
// The first 32 WARPS threads call it: a tile that is whole in their registers.
template <typename O, int MT, int NT, int WARPS>
__device__ __forceinline__ void finish_tile(const float (&sum)[MT][NT][4], const Job& job, const GradArgs& a, int id, int64_t c0, float* tile) {
    tile_barrier<WARPS>();                             // what was in the memory has been read
    put_tile<MT, NT>(sum, tile);
    tile_barrier<WARPS>();
    write_tile<O>(job, a, id, c0, threadIdx.x, 32 * WARPS, [&](int k, int c) { return *reinterpret_cast<const float4*>(tile + k * kTileWidth + c); });
}
template <int MT, int NT, int WARPS>
__device__ __forceinline__ float4* part_of(const Job& job, int slot, unsigned tile) {
    return reinterpret_cast<float4*>(job.parts) + ((int64_t)slot * job.tiles + tile) * (MT * NT * 32 * WARPS) + threadIdx.x;
}
template <int MT, int NT, int WARPS>
__device__ __forceinline__ void keep_tile(const float (&sum)[MT][NT][4], float4* part) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < NT; ++j) part[(m * NT + j) * 32 * WARPS] = make_float4(sum[m][j][0], sum[m][j][1], sum[m][j][2], sum[m][j][3]);
}

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
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[m][j][i] *= scale;
    if (runs == 1) finish_tile<O, MT, 2, kThreads / 32>(sum, job, a, lo, c0, reinterpret_cast<float*>(smem));
    else keep_tile<MT, 2, kThreads / 32>(sum, part_of<MT, 2, kThreads / 32>(job, slot, blockIdx.x));
}

// Sums of the runs of the adapters that have several.
template <typename O, int MT, int NT, int WARPS>
__global__ void __launch_bounds__(32 * WARPS) runs_kernel(const __grid_constant__ Job job) {
    extern __shared__ __align__(128) unsigned char smem[];
    after_previous();
    const int id = blockIdx.y, first = job.slots[id], runs = job.slots[id + 1] - first;
    if (runs <= 1) return;
    const bool second = blockIdx.x >= job.first_tiles;
    float sum[MT][NT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[m][j][i] = 0.f;
    const float4* part = part_of<MT, NT, WARPS>(job, first, blockIdx.x);
#pragma unroll 1
    for (int k = 0; k < runs; ++k, part += (int64_t)job.tiles * (MT * NT * 32 * WARPS))
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const float4 v = part[(m * NT + j) * 32 * WARPS];
                sum[m][j][0] += v.x;
                sum[m][j][1] += v.y;
                sum[m][j][2] += v.z;
                sum[m][j][3] += v.w;
            }
    finish_tile<O, MT, NT, WARPS>(sum, job, job.two[second], id, (int64_t)(blockIdx.x - (second ? job.first_tiles : 0)) * kCols,
                                  reinterpret_cast<float*>(smem));
}

// ---- parts of h made once, tiles by TMA ----------------------------------------------------------------------
__device__ int g_grad_status = 0;                      // GPD_ERR_TIMEOUT if a bounded wait expired

// FP16: the largest magnitudes of the columns of u and h (blockIdx.y), for every adapter; `most` is zero before.
__global__ void __launch_bounds__(256) most_kernel(const __grid_constant__ Job job, int RP, int32_t* most) {
    __shared__ int32_t here[kMaxRank];
    after_previous();
    const float* h = job.two[blockIdx.y].h;
    const int r = job.r;
    if (threadIdx.x < RP) here[threadIdx.x] = 0;
    __syncthreads();
    for (int s = blockIdx.z; s < job.seg.S; s += gridDim.z) {
        const int64_t id = number(job.seg.index, s, job.seg.wide);
        if (id < 0 || id >= job.seg.n) continue;
        const int64_t from = offset_at(job.seg, s), to = offset_at(job.seg, s + 1);
        // a thread keeps to one column
        const int c = threadIdx.x % RP, step = 256 / RP;
        float m = 0.f;
        if (c < r)
#pragma unroll 4
            for (int64_t t = from + (int64_t)blockIdx.x * step + threadIdx.x / RP; t < to; t += (int64_t)gridDim.x * step) m = fmaxf(m, fabsf(h[t * r + c]));
        if (m > 0.f) atomicMax(here + c, __float_as_int(m));           // order does not matter
        __syncthreads();
        if (threadIdx.x < RP) {
            const int32_t all = here[threadIdx.x];
            if (all > 0) atomicMax(most + ((int64_t)blockIdx.y * job.seg.n + id) * RP + threadIdx.x, all);
            here[threadIdx.x] = 0;
        }
        __syncthreads();
    }
}
// The adapter's chunks, `count` at most.  One warp.
__device__ __forceinline__ void list_chunks(const Segments& s, int64_t id, int count, int2* list) {
    const int lane = threadIdx.x & 31;
    int64_t seen = 0;
    for (int64_t base = 0; base < s.S && seen < count; base += 32) {
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
            const int64_t start = __shfl_sync(0xffffffffu, at, who), rows = __shfl_sync(0xffffffffu, len, who), n = (rows + kRows - 1) / kRows;
            for (int64_t j = lane; j < n && seen + j < count; j += 32)
                list[seen + j] = make_int2((int)(start + j * kRows), (int)min((int64_t)kRows, rows - j * kRows));
            seen += n;
        }
    }
}

// planes[2][PARTS][T][RP]: u and h as parts.  The last CTA lists the chunks.
template <typename T, int PARTS>
__global__ void __launch_bounds__(256) split_kernel(const __grid_constant__ Job job, int RP, T* planes, int max_chunks, unsigned long long* counts, int32_t* slots) {
    after_previous();
    if (blockIdx.x == gridDim.x - 1) {
        plan_runs(job.seg, kRows, kRows, 0, max_chunks, counts, slots);
        __syncthreads();
        for (int id = threadIdx.x >> 5; id < job.seg.n; id += 8) list_chunks(job.seg, id, slots[id + 1] - slots[id], job.chunks + slots[id]);
        return;
    }
    constexpr bool kScaled = std::is_same<T, __half>::value;
    const int64_t n = job.seg.T * (RP / 2), all = 2 * n;               // pairs
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < all; e += (int64_t)(gridDim.x - 1) * 256) {
        const bool second = e >= n;
        const int64_t at = e - (second ? n : 0), t = at / (RP / 2);
        const int c = (int)(at - t * (RP / 2)) * 2;
        const float* h = job.two[second].h + t * job.r + c;
        float x = c < job.r ? h[0] : 0.f, y = c + 1 < job.r ? h[1] : 0.f;
        if (kScaled) {
            // the row's adapter: the last segment that begins at or before it (rows of no segment: anything will do)
            int lo = 0, hi = job.seg.S - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if (offset_at(job.seg, mid) <= t) lo = mid;
                else hi = mid - 1;
            }
            const int64_t id = job.seg.S > 0 ? number(job.seg.index, lo, job.seg.wide) : -1;
            if (id >= 0 && id < job.seg.n) {
                const int32_t* m = job.most + ((int64_t)second * job.seg.n + id) * RP + c;
                x *= power2(-exponent_of(__int_as_float(m[0])));
                y *= power2(-exponent_of(__int_as_float(m[1])));
            }
        }
        uint32_t parts[PARTS];
        split2<T, PARTS>(x, y, parts);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) *reinterpret_cast<uint32_t*>(planes + ((second * PARTS + p) * job.seg.T + t) * RP + c) = parts[p];
    }
}

// The tensor cores take both tiles as TMA leaves them, rows of y and h being the depth of the product: D (128 columns of y x
// RP columns of h) in tensor memory, two accumulators in turn.  One warp issues copies, one the products, four pull a finished
// accumulator into registers and add it up to nearest: the chain of truncating additions in tensor memory is cut every chunk (three
// parts: 12 steps) or every fourth (two: 32).
template <int MT, int PARTS>
struct TmaShape {
    static constexpr int RP = 16 * MT, GROUP = PARTS == 3 ? 1 : 4, COLS = 2 * RP < 32 ? 32 : 2 * RP;      // columns of tensor memory
    using Y = WTile<kRows, kCols>;
    using H = WTile<kRows, RP>;
    static constexpr int STAGE = Y::BYTES + PARTS * H::BYTES;
    static constexpr int STAGES = MT == 8 ? (PARTS == 3 ? 3 : 4) : MT == 4 ? 2 : 3;
    static constexpr int SMEM = STAGES * STAGE + 1024, PER_SM = per_sm(SMEM) < 3 ? per_sm(SMEM) : 3;
};
struct GradMaps { CUtensorMap y[2], h[2]; };
constexpr int kTmaThreads = 192;

// Tile of [depth][PITCH / 2 elements] rows: eight rows of PITCH bytes make a swizzled group, the next eight follow; further
// columns lie `part` bytes on.
template <int PITCH>
__device__ __forceinline__ uint64_t depth_first(uint32_t at, uint32_t part) {
    const uint64_t layout = PITCH == 128 ? 2 : PITCH == 64 ? 4 : 6;
    return (uint64_t)(at >> 4 & 0x3fff) | (uint64_t)(part >> 4 & 0x3fff) << 16 | (uint64_t)(8 * PITCH >> 4) << 32 | (uint64_t)1 << 46 | layout << 61;
}
__device__ __forceinline__ void umma_16(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(what), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t at, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(at) : "memory");
}

template <typename T, typename O, int MT, int PARTS>
__global__ void __launch_bounds__(kTmaThreads, TmaShape<MT, PARTS>::PER_SM)
grad_tma_kernel(const __grid_constant__ GradMaps maps, const __grid_constant__ Job job, int splits) {
    using S = TmaShape<MT, PARTS>;
    constexpr int RP = S::RP;
    constexpr bool kScaled = std::is_same<T, __half>::value;
    extern __shared__ unsigned char raw[];
    __shared__ Ring<S::STAGES> ring;
    __shared__ uint64_t acc_full[2], acc_empty[2], done;
    __shared__ uint32_t tmem_slot;
    __shared__ int rows_of[S::STAGES];                 // rows of the stages' chunks
    unsigned char* smem = raw + (1024 - (smem_at(raw) & 1023)) % 1024;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(&acc_full[i], 1);
            tc::mbar_init(&acc_empty[i], 4);
        }
        tc::mbar_init(&done, 1);
        ring.init(1, 1);
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&tmem_slot)), "r"(S::COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // The kernel behind this one may want tensor memory too, and hold it while it waits for this one's end: it is let in only when
    // this CTA has its own.
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    after_previous();
    // the cluster's adapter; this CTA's chunks of it
    const int id = blockIdx.x / splits, rank = blockIdx.x % splits, first = job.slots[id], have = job.slots[id + 1] - first;
    const int from = (int)((int64_t)have * rank / splits), n = (int)((int64_t)have * (rank + 1) / splits) - from;
    const bool second = blockIdx.y >= job.first_tiles;
    const GradArgs& a = job.two[second];
    const int c0 = (int)(blockIdx.y - (second ? job.first_tiles : 0)) * kCols;
    const float scale = a.scale ? a.scale[id] : 1.f;
    const uint32_t tmem = tmem_slot;
    float sum[RP];
    if (warp == 0) {
        int k = 0;
        int2 next = make_int2(0, 0);
        for (; k < n; ++k) {
            if (k % 32 == 0 && k + lane < n) next = job.chunks[first + from + k + lane];
            const int row = __shfl_sync(0xffffffffu, next.x, k % 32), rows = __shfl_sync(0xffffffffu, next.y, k % 32);
            if (!ring.wait_empty(k, &g_grad_status)) break;
            if (lane == 0) {
                unsigned char* at = smem + k % S::STAGES * S::STAGE;
                uint64_t* bar = &ring.full[k % S::STAGES];
                rows_of[k % S::STAGES] = rows;
                tc::mbar_expect_tx(bar, S::STAGE);
                S::Y::load(at, &maps.y[second], c0, row, 0, bar);
#pragma unroll
                for (int p = 0; p < PARTS; ++p) S::H::load(at + S::Y::BYTES + p * S::H::BYTES, &maps.h[second], 0, row, p, bar);
            }
        }
        __syncwarp();
        if (lane == 0) ring.drain(k, &g_grad_status);
    } else if (warp == 1) {
        // FP32 sums of two BF16 or FP16 operands, both depth first, 128 x RP
        constexpr uint32_t kType = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
        constexpr uint32_t what = 1u << 4 | kType << 7 | kType << 10 | 1u << 15 | 1u << 16 | (uint32_t)(RP >> 3) << 17 | (uint32_t)(kCols >> 4) << 24;
        for (int k = 0; k < n; ++k) {
            const int buf = k / S::GROUP & 1, s = k % S::STAGES;
            const bool fresh = k % S::GROUP == 0;
            bool live = ring.wait_full(k, &g_grad_status);
            if (live && fresh) live = tc::mbar_wait(&acc_empty[buf], (k / S::GROUP >> 1 & 1) ^ 1, &ring.abort, &g_grad_status);
            if (!__all_sync(0xffffffffu, live)) break;
            unsigned char* stage = smem + s * S::STAGE;
            const int rows = rows_of[s];
            if (rows < kRows) {                        // rows behind the segment's end are another's, whatever they hold
                auto clear = [&](unsigned char* part, int pitch) {
                    for (int i = rows * pitch / 16 + lane; i < kRows * pitch / 16; i += 32) reinterpret_cast<uint4*>(part)[i] = make_uint4(0, 0, 0, 0);
                };
                for (int i = 0; i < S::Y::PARTS; ++i) clear(stage + i * kRows * 128, 128);
                for (int p = 0; p < PARTS; ++p)
                    for (int i = 0; i < S::H::PARTS; ++i) clear(stage + S::Y::BYTES + p * S::H::BYTES + i * kRows * 128, S::H::PITCH);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            if (lane == 0) {
                const uint32_t ys = smem_at(stage), hs = ys + S::Y::BYTES;
#pragma unroll
                for (int d = 0; d < kRows / 16; ++d)
#pragma unroll
                    for (int p = PARTS - 1; p >= 0; --p)               // the small parts first
                        umma_16(tmem + buf * RP, depth_first<128>(ys + d * 16 * 128, kRows * 128),
                                depth_first<S::H::PITCH>(hs + p * S::H::BYTES + d * 16 * S::H::PITCH, kRows * 128), what, !(fresh && d == 0 && p == PARTS - 1));
                tc::umma_commit(&ring.empty[s]);
                if (k % S::GROUP == S::GROUP - 1 || k == n - 1) tc::umma_commit(&acc_full[buf]);
            }
            __syncwarp();
        }
        if (lane == 0) {                               // nothing is under way when the memory gets another use
            int never = 0;
            tc::umma_commit(&done);
            tc::mbar_wait(&done, 0, &never, &g_grad_status);
        }
        __syncwarp();
    } else {
#pragma unroll
        for (int c = 0; c < RP; ++c) sum[c] = 0.f;
        const uint32_t mine = tmem + ((uint32_t)(warp & 3) * 32 << 16);
        for (int i = 0; i * S::GROUP < n; ++i) {
            const int buf = i & 1;
            const bool live = tc::mbar_wait(&acc_full[buf], i >> 1 & 1, &ring.abort, &g_grad_status);
            if (!__all_sync(0xffffffffu, live)) break; // loads from tensor memory are the whole warp's
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
            for (int c = 0; c < RP; c += 16) {
                uint32_t r[16];
                tmem_ld16(mine + buf * RP + c, r);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                for (int j = 0; j < 16; ++j) sum[c + j] += __uint_as_float(r[j]);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&acc_empty[buf]);
        }
    }
    float* tile = reinterpret_cast<float*>(smem);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();                                   // every stage and accumulator has been read
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::COLS) : "memory");
    if (warp >= 2) {
        const int32_t* most = job.most + ((int64_t)second * job.seg.n + id) * RP;
#pragma unroll
        for (int c = 0; c < RP; ++c) tile[c * kTileWidth + (warp & 3) * 32 + lane] = (kScaled ? sum[c] * power2(exponent_of(__int_as_float(most[c]))) : sum[c]) * scale;
    }
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    if (splits > 1) cluster.sync();
    else __syncthreads();
    write_tile<O>(job, a, id, c0, rank * kTmaThreads + threadIdx.x, splits * kTmaThreads, [&](int k, int c) {
        const int at = k * kTileWidth + c;
        float4 v = *reinterpret_cast<const float4*>(tile + at);
        if (splits > 1) {                              // all CTAs' numbers under way before the first is added
            float4 x[8];
#pragma unroll
            for (int s = 0; s < 8; ++s) x[s] = s < splits ? *reinterpret_cast<const float4*>(cluster.map_shared_rank(tile, s) + at) : make_float4(0.f, 0.f, 0.f, 0.f);
            v = x[0];
#pragma unroll
            for (int s = 1; s < 8; ++s) {
                v.x += x[s].x;
                v.y += x[s].y;
                v.z += x[s].z;
                v.w += x[s].w;
            }
        }
        return v;
    });
    if (splits > 1) cluster.sync();                    // the others have read this CTA's sums
}

int64_t tiles_of(int64_t K, int64_t N) { return (K + kCols - 1) / kCols + (N + kCols - 1) / kCols; }
// Rows of a run where rows are gathered: so many runs that two CTAs per SM are busy, of 256 rows at least.  148 SMs as a constant: the
// workspace's size is asked for without a device.
int64_t run_rows(int64_t T, int64_t K, int64_t N) {
    const int64_t runs = std::max<int64_t>(1, 2 * 148 / tiles_of(K, N));
    const int64_t rows = ((T + runs - 1) / runs + kRows - 1) / kRows * kRows;
    return std::min<int64_t>(kMostRows, std::max<int64_t>(256, rows));
}
int64_t slots_of(int64_t T, int64_t n, int64_t K, int64_t N) { return T / run_rows(T, K, N) + n; }    // most runs there can be
// Segments of less than 32 rows on average would leave half of their tiles empty.
bool long_segments(int64_t T, int64_t S) { return S > 0 && T >= 32 * S; }
bool by_tma(const Segments& s, const GradArgs (&two)[2]) { return two[0].y_vec && two[1].y_vec && long_segments(s.T, s.S); }
int64_t chunks_of(int64_t T, int64_t S) { return T / kRows + S; }      // most chunks there can be
// CTAs that share an adapter's rows: as many as are resident at once, if as many adapters as there are segments have rows; each has
// four chunks at least.
int splits_of(int64_t T, int64_t S, int64_t n, int64_t tiles, int resident) {
    const int64_t active = std::min(n, S), most = std::min<int64_t>(8, std::max<int64_t>(1, T / active / (4 * kRows)));
    return (int)std::min(most, std::max<int64_t>(1, resident / (tiles * active)));
}
int64_t up(int64_t bytes) { return (bytes + 255) / 256 * 256; }
int padded_rank(int64_t r) { return r <= 16 ? 16 : r <= 32 ? 32 : r <= 64 ? 64 : 128; }

template <typename T, typename O, int MT>
gpd_status launch(const Job& job, T* planes, unsigned long long* counts, int32_t* slots, int32_t* most, bool tma, cudaStream_t st) {
    constexpr int PARTS = kParts<T, O>;
    constexpr int TILE = 16 * MT * kTileWidth * 4;     // a tile's sums on their way out
    gpd_status rc;
    if (tma) {
        using S = TmaShape<MT, PARTS>;
        auto kernel = grad_tma_kernel<T, O, MT, PARTS>;
        GradMaps maps;
        for (int i = 0; i < 2; ++i)
            if (!make_map(&maps.y[i], job.two[i].y, 2, 1, job.seg.T, job.two[i].C, job.two[i].ldy, 0, kRows, 64) ||
                !make_map(&maps.h[i], planes + i * PARTS * job.seg.T * S::RP, 2, PARTS, job.seg.T, S::RP, S::RP, job.seg.T * S::RP, kRows, S::H::PITCH / 2))
                return GPD_ERR_CUDA;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) != cudaSuccess) return GPD_ERR_CUDA;
        if (std::is_same<T, __half>::value) {
            const int RP = S::RP;
            const unsigned z = (unsigned)std::min<int64_t>(job.seg.S, 64), x = (unsigned)std::max<int64_t>(1, std::min<int64_t>(1024 / z, job.seg.T / z * RP / 1024));
            rc = launch_after(most_kernel, dim3(x, 2, z), dim3(256), 0, 1, st, job, RP, most);
            if (rc != GPD_OK) return rc;
        }
        const unsigned blocks = (unsigned)std::min<int64_t>((job.seg.T * S::RP + 255) / 256, 8 * sm_count()) + 1;
        const int RP = S::RP;
        const int most_chunks = (int)chunks_of(job.seg.T, job.seg.S);
        rc = launch_after(split_kernel<T, PARTS>, dim3(blocks), dim3(256), 0, 1, st, job, RP, planes, most_chunks, counts, slots);
        if (rc != GPD_OK) return rc;
        const int splits = splits_of(job.seg.T, job.seg.S, job.seg.n, job.tiles, S::PER_SM * sm_count());
        return launch_after(kernel, dim3((unsigned)(job.seg.n * splits), job.tiles), dim3(kTmaThreads), S::SMEM, splits, st, maps, job, splits);
    }
    {
        using S = Shape<MT, PARTS>;
        static_assert(S::SMEM >= TILE && TmaShape<MT, PARTS>::SMEM - 1024 >= TILE, "a tile's sums leave through the stages' memory");
        auto kernel = grad_kernel<T, O, MT, PARTS>;
        if (S::SMEM > 40960 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) != cudaSuccess) return GPD_ERR_CUDA;
        rc = launch_after(plan_kernel, dim3(1), dim3(256), 0, 1, st, job.seg, job.run, job.max_slots, counts, slots);
        if (rc != GPD_OK) return rc;
        rc = launch_after(kernel, dim3(job.tiles, (unsigned)job.max_slots), dim3(kThreads), S::SMEM, 1, st, job);
    }
    if (rc != GPD_OK || job.max_slots == job.seg.n) return rc;         // as many runs as adapters: each has one
    auto join = runs_kernel<O, MT, 2, kThreads / 32>;
    if (TILE > 49152 && cudaFuncSetAttribute(join, cudaFuncAttributeMaxDynamicSharedMemorySize, TILE) != cudaSuccess) return GPD_ERR_CUDA;
    return launch_after(join, dim3(job.tiles, (unsigned)job.seg.n), dim3(kThreads), TILE, 1, st, job);
}
template <typename T, typename O, typename... A>
gpd_status launch_rank(const Job& job, T* planes, A... more) {
    if (job.r <= 16) return launch<T, O, 1>(job, planes, more...);
    if (job.r <= 32) return launch<T, O, 2>(job, planes, more...);
    return job.r <= 64 ? launch<T, O, 4>(job, planes, more...) : launch<T, O, 8>(job, planes, more...);
}

// Parts of the workspace, in bytes from its beginning
struct Workspace {
    int64_t counts, slots, most, planes, chunks, parts, bytes;
    Workspace(int64_t T, int64_t n, int64_t r, int64_t K, int64_t N) {
        const int64_t RP = padded_rank(r), runs = slots_of(T, n, K, N);
        counts = 0;
        slots = counts + up(8 * n);
        most = slots + up(4 * (n + 1));
        planes = most + up(8 * n * RP);
        chunks = planes + up(2 * 3 * 2 * T * RP);
        parts = chunks + up(8 * chunks_of(T, T / 32));
        bytes = parts + (runs > n ? up(4 * runs * tiles_of(K, N) * RP * kCols) : 0);
    }
};

}  // namespace

int64_t grad_workspace(int64_t T, int64_t n, int64_t r, int64_t K, int64_t N) { return Workspace(T, n, r, K, N).bytes; }

int grad_status_fetch_and_clear() {
    int v = 0, zero = 0;
    if (cudaMemcpyFromSymbol(&v, g_grad_status, sizeof(int)) != cudaSuccess) return (int)GPD_ERR_CUDA;
    if (v != 0) cudaMemcpyToSymbol(g_grad_status, &zero, sizeof(int));
    return v;
}

// Whether a launch's grid has room: all column tiles beside all adapters (by TMA), or beside all runs.
bool gradients_fit(const Segments& seg, const GradArgs (&two)[2]) {
    const int64_t K = two[0].C, N = two[1].C;
    return by_tma(seg, two) ? tiles_of(K, N) <= 65535 && (int64_t)seg.n * 8 <= 0x7fffffff : slots_of(seg.T, seg.n, K, N) <= 65535;
}

gpd_status gradients(int type, int grad_type, bool accumulate, const Segments& seg, int r, const GradArgs (&two)[2], void* workspace,
                     cudaStream_t st) {
    const Workspace at(seg.T, seg.n, r, two[0].C, two[1].C);
    const bool tma = by_tma(seg, two);
    Job job;
    job.two[0] = two[0];
    job.two[1] = two[1];
    job.seg = seg;
    job.r = r;
    job.accumulate = accumulate;
    job.run = run_rows(seg.T, two[0].C, two[1].C);
    job.max_slots = (int)slots_of(seg.T, seg.n, two[0].C, two[1].C);
    job.first_tiles = (unsigned)((two[0].C + kCols - 1) / kCols);
    job.tiles = (unsigned)tiles_of(two[0].C, two[1].C);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    auto* counts = reinterpret_cast<unsigned long long*>(ws + at.counts);
    int32_t *slots = reinterpret_cast<int32_t*>(ws + at.slots), *most = reinterpret_cast<int32_t*>(ws + at.most);
    job.slots = slots;
    job.most = most;
    job.chunks = reinterpret_cast<int2*>(ws + at.chunks);
    job.parts = reinterpret_cast<float*>(ws + at.parts);
    if (tma && type == GPD_DT_F16 && cudaMemsetAsync(most, 0, 8 * (size_t)seg.n * padded_rank(r), st) != cudaSuccess) return GPD_ERR_CUDA;
    auto* bf16 = reinterpret_cast<__nv_bfloat16*>(ws + at.planes);
    auto* f16 = reinterpret_cast<__half*>(ws + at.planes);
    if (type == GPD_DT_BF16)
        return grad_type == GPD_DT_F32 ? launch_rank<__nv_bfloat16, float>(job, bf16, counts, slots, most, tma, st)
                                       : launch_rank<__nv_bfloat16, __nv_bfloat16>(job, bf16, counts, slots, most, tma, st);
    return grad_type == GPD_DT_F32 ? launch_rank<__half, float>(job, f16, counts, slots, most, tma, st)
                                   : launch_rank<__half, __half>(job, f16, counts, slots, most, tma, st);
}

}  // namespace adapter
}  // namespace gpd
