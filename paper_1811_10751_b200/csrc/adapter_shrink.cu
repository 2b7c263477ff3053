// First factor of low-rank adapters: h[t] = scale_i W_i x[t] for the rows of every segment, i its adapter.
//
// Bound by reading x (many rows) or the adapters (one row per segment); the r columns of the result are few.  A CTA takes
// 64 rows of one segment, or 16 where segments are short, and a part of the columns of x; the CTAs of a cluster have the
// other parts and add up their sums over distributed shared memory, in a fixed order.  Tiles of x and W come through a
// ring of asynchronous copies.
//
// Measured (BF16): 16384 x 8192, rank 32, 53 us of 42 at the copy bandwidth; 4001 x 4096, rank 64, 25 us cold; 8192 x 4096, rank
// 16 (factors transposed), 20 us.  What the larger ranks cost beside the copies are mma.sync's operands: every warp loads all of W's tile.
#include <cooperative_groups.h>

#include <algorithm>

#include "adapter_common.h"

namespace gpd {
namespace adapter {

namespace {

constexpr int kThreads = 128, kDeep = 64, kXPitch = 2 * kDeep + 16;    // columns of x per stage

template <int NT, int WM, bool TRANS>
struct Shape {
    static constexpr int TM = 16 * WM, RP = 8 * NT, STAGES = WM == 4 ? 4 : NT == 16 ? 3 : NT == 8 ? 4 : 6;     // room for three CTAs per SM or more
    static constexpr int W_ROWS = TRANS ? kDeep : RP, W_COLS = TRANS ? RP : kDeep, W_PITCH = 2 * W_COLS + 16;
    static constexpr int STAGE = TM * kXPitch + W_ROWS * W_PITCH;
    static constexpr int SUMS = 64 * RP * 4;           // FP32 sums: of 64 rows, or of 16 rows four times
    static constexpr int SMEM = STAGES * STAGE > SUMS ? STAGES * STAGE : SUMS;
};

// WM = 4: a warp has 16 rows of the tile.  WM = 1: all warps have the same 16 rows, and each a quarter of every stage.
template <typename T, int NT, int WM, bool TRANS>
__global__ void __launch_bounds__(kThreads) shrink_kernel(const __grid_constant__ ShrinkArgs a, int splits) {
    using S = Shape<NT, WM, TRANS>;
    extern __shared__ __align__(128) unsigned char smem[];
    after_previous();
    const int rank = blockIdx.x % splits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const RowTile tile = find_tile<S::TM>(a.seg, (int)(blockIdx.x / splits));
    if (tile.rows == 0) return;                        // the whole cluster
    float* out = a.h + (int64_t)tile.row * a.r;
    if (tile.id < 0 || tile.id >= a.seg.n) {
        const float v = tile.id < 0 ? 0.f : __int_as_float(0x7fffffff);
        if (rank == 0)
            for (int i = threadIdx.x; i < tile.rows * a.r; i += kThreads) out[i] = v;
        return;
    }
    const T* x = static_cast<const T*>(a.x) + (int64_t)tile.row * a.ldx;
    const T* w = static_cast<const T*>(a.w) + (int64_t)tile.id * a.next;
    const int64_t stages = (a.C + kDeep - 1) / kDeep;
    const int64_t from = stages * rank / splits, to = stages * (rank + 1) / splits;
    const uint32_t ring = smem_at(smem);
    auto fetch = [&](int64_t k) {
        if (k < to) {
            const uint32_t at = ring + (uint32_t)((k - from) % S::STAGES) * S::STAGE;
            const int64_t c = k * kDeep;
            stage_tile<T, S::TM, kDeep, kThreads>(at, kXPitch, x + c, a.ldx, tile.rows, a.C - c, a.x_vec);
            if (TRANS) stage_tile<T, S::W_ROWS, S::W_COLS, kThreads>(at + S::TM * kXPitch, S::W_PITCH, w + c * a.ldw, a.ldw, a.C - c, a.r, a.w_vec);
            else stage_tile<T, S::W_ROWS, S::W_COLS, kThreads>(at + S::TM * kXPitch, S::W_PITCH, w + c, a.ldw, a.r, a.C - c, a.w_vec);
        }
        copies_end();
    };
    float sum[NT][4], acc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[n][i] = acc[n][i] = 0.f;
    auto cut = [&]() {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum[n][i] += acc[n][i];
                acc[n][i] = 0.f;
            }
    };
    for (int i = 0; i < S::STAGES - 1; ++i) fetch(from + i);
    for (int64_t k = from; k < to; ++k) {
        copies_wait<S::STAGES - 2>();
        __syncthreads();
        fetch(k + S::STAGES - 1);
        const uint32_t xs = ring + (uint32_t)((k - from) % S::STAGES) * S::STAGE, ws = xs + S::TM * kXPitch;
        auto step = [&](int ks) {
            uint32_t xa[4];
            ldmatrix4<false>(xa, xs + ((WM == 4 ? 16 * warp : 0) + (lane & 15)) * kXPitch + 2 * (16 * ks + (lane >> 4) * 8));
#pragma unroll
            for (int p = 0; p < NT / 2; ++p) {
                uint32_t b[4];
                if (TRANS) ldmatrix4<true>(b, ws + (16 * ks + (lane & 15)) * S::W_PITCH + 2 * (16 * p + (lane >> 4) * 8));
                else ldmatrix4<false>(b, ws + (16 * p + (lane & 7) + (lane >> 4) * 8) * S::W_PITCH + 2 * (16 * ks + (lane >> 3 & 1) * 8));
                mma(acc[2 * p], xa, b[0], b[1], T());
                mma(acc[2 * p + 1], xa, b[2], b[3], T());
            }
        };
        if (WM == 4) {
#pragma unroll
            for (int ks = 0; ks < kDeep / 16; ++ks) step(ks);
            cut();
        } else {
            step(warp);
            if (((k - from) & 3) == 3) cut();
        }
    }
    cut();
    copies_wait<0>();
    __syncthreads();
    float* sums = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float* s = sums + (16 * warp + (lane >> 2)) * S::RP + 8 * n + 2 * (lane & 3);
        *reinterpret_cast<float2*>(s) = make_float2(sum[n][0], sum[n][1]);
        *reinterpret_cast<float2*>(s + 8 * S::RP) = make_float2(sum[n][2], sum[n][3]);
    }
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    if (splits > 1) cluster.sync();
    else __syncthreads();
    const float scale = a.scale ? a.scale[tile.id] : 1.f;
    for (int e = rank * kThreads + threadIdx.x; e < S::TM * S::RP; e += splits * kThreads) {
        const int row = e / S::RP, c = e % S::RP;
        if (row >= tile.rows || c >= a.r) continue;
        float v = 0.f;
#pragma unroll 2
        for (int s = 0; s < splits; ++s) {
            const float* other = splits > 1 ? cluster.map_shared_rank(sums, s) : sums;
#pragma unroll
            for (int q = 0; q < (WM == 1 ? 4 : 1); ++q) v += other[e + q * 16 * S::RP];
        }
        out[(int64_t)row * a.r + c] = v * scale;
    }
    if (splits > 1) cluster.sync();                    // the others have read this CTA's sums
}

template <typename T, int NT, int WM, bool TRANS>
gpd_status launch(const ShrinkArgs& a, cudaStream_t st) {
    using S = Shape<NT, WM, TRANS>;
    const int64_t tiles = tiles_of(a.seg, S::TM), stages = (a.C + kDeep - 1) / kDeep;
    // until two CTAs per SM are busy, or four where loads are awaited in line, but four stages each at least
    const int64_t busy = (a.x_vec && a.w_vec ? 2 : 4) * sm_count();
    int splits = 1;
    while (splits < 8 && tiles * splits < busy && stages >= 8 * splits) splits *= 2;
    if (tiles * splits > 0x7fffffff) return GPD_ERR_SHAPE;
    auto kernel = shrink_kernel<T, NT, WM, TRANS>;
    if (S::SMEM > 49152 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) != cudaSuccess) return GPD_ERR_CUDA;
    return launch_after(kernel, dim3((unsigned)(tiles * splits)), dim3(kThreads), S::SMEM, splits, st, a, splits);
}
// ---- the same with tiles by TMA: many rows, x on 16-byte boundaries --------------------------------------------
__device__ int g_shrink_status = 0;                    // GPD_ERR_TIMEOUT if a bounded wait expired

template <int NT, bool TRANS>
struct TmaShape {
    static constexpr int TM = 64, RP = 8 * NT, STAGES = 4, X_BYTES = TM * 128;
    using W = WTile<TRANS ? kDeep : RP, TRANS ? RP : kDeep>;
    static constexpr int STAGE = X_BYTES + W::BYTES, SUMS = TM * RP * 4;
    static constexpr int SMEM = (STAGES * STAGE > SUMS ? STAGES * STAGE : SUMS) + 1024;
};

// Four warps with 16 rows each, and one that issues the copies.
template <typename T, int NT, bool TRANS>
__global__ void __launch_bounds__(kThreads + 32, per_sm(TmaShape<NT, TRANS>::SMEM)) shrink_tma_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                                                                   const __grid_constant__ ShrinkArgs a, int splits) {
    using S = TmaShape<NT, TRANS>;
    extern __shared__ unsigned char raw[];
    __shared__ Ring<S::STAGES> ring;
    unsigned char* smem = raw + (1024 - (smem_at(raw) & 1023)) % 1024;
    const int rank = blockIdx.x % splits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) ring.init(a.w_vec ? 1 : 33, 4);
    after_previous();
    const RowTile tile = find_tile<S::TM>(a.seg, (int)(blockIdx.x / splits));
    if (tile.rows == 0) return;                        // the whole cluster
    float* out = a.h + (int64_t)tile.row * a.r;
    if (tile.id < 0 || tile.id >= a.seg.n) {
        const float v = tile.id < 0 ? 0.f : __int_as_float(0x7fffffff);
        if (rank == 0)
            for (int i = threadIdx.x; i < tile.rows * a.r; i += kThreads + 32) out[i] = v;
        return;
    }
    const int64_t stages = (a.C + kDeep - 1) / kDeep;
    const int64_t from = stages * rank / splits;
    const int n = (int)(stages * (rank + 1) / splits - from);
    if (!a.w_vec)                                      // columns and rows of W that do not exist
        for (int i = threadIdx.x; i < S::STAGES * S::STAGE / 16; i += kThreads + 32) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
    if (!a.w_vec) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    float sum[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[i][j] = 0.f;
    if (warp == kThreads / 32) {
        int k = 0;
        for (; k < n && ring.wait_empty(k, &g_shrink_status); ++k) {
            unsigned char* at = smem + k % S::STAGES * S::STAGE;
            const int64_t c = (from + k) * kDeep;
            uint64_t* bar = &ring.full[k % S::STAGES];
            if (lane == 0) {
                tc::mbar_expect_tx(bar, S::X_BYTES + (a.w_vec ? S::W::BYTES : 0));
                tc::tma_load_3d(at, &map_x, (int)c, (int)tile.row, 0, bar);
                if (a.w_vec) S::W::load(at + S::X_BYTES, &map_w, TRANS ? 0 : (int)c, TRANS ? (int)c : 0, (int)tile.id, bar);
            }
            if (!a.w_vec) {
                const T* w = static_cast<const T*>(a.w) + (int64_t)tile.id * a.next + (TRANS ? c * a.ldw : c);
                if (TRANS) S::W::template copy<true>(at + S::X_BYTES, w, a.ldw, a.C - c, a.r, a.r);
                else S::W::template copy<false>(at + S::X_BYTES, w, a.ldw, a.r, a.C - c, a.r);
                tc::mbar_arrive(bar);
            }
        }
        __syncwarp();
        if (lane == 0) ring.drain(k, &g_shrink_status);
    } else {
        for (int k = 0; k < n && ring.wait_full(k, &g_shrink_status); ++k) {
            const uint32_t stage = smem_at(smem) + k % S::STAGES * S::STAGE;
            const uint32_t xs = WTile<S::TM, kDeep>::lane_at(stage, row_first(), row_first_col()) + 16 * warp * 128;
            const uint32_t ws = TRANS ? S::W::lane_at(stage + S::X_BYTES, row_first(), row_first_col())
                                      : S::W::lane_at(stage + S::X_BYTES, col_first_row(), col_first());
            float acc[NT][4];
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
#pragma unroll
            for (int ks = 0; ks < kDeep / 16; ++ks) {
                uint32_t xa[4];
                ldmatrix4<false>(xa, WTile<S::TM, kDeep>::on(xs, 0, 16 * ks));
#pragma unroll
                for (int p = 0; p < NT / 2; ++p) {
                    uint32_t b[4];
                    if (TRANS) ldmatrix4<true>(b, S::W::on(ws, 16 * ks, 16 * p));
                    else ldmatrix4<false>(b, S::W::on(ws, 16 * p, 16 * ks));
                    mma(acc[2 * p], xa, b[0], b[1], T());
                    mma(acc[2 * p + 1], xa, b[2], b[3], T());
                }
            }
            // every load of the stage has its data before copies may write there: an arrival alone does not hold matrix loads
            // back that nothing has waited for yet
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&ring.empty[k % S::STAGES]);
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[i][j] += acc[i][j];
        }
    }
    __syncthreads();                                   // every stage has been read
    float* sums = reinterpret_cast<float*>(smem);
    if (warp < kThreads / 32) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            float* s = sums + (16 * warp + (lane >> 2)) * S::RP + 8 * i + 2 * (lane & 3);
            *reinterpret_cast<float2*>(s) = make_float2(sum[i][0], sum[i][1]);
            *reinterpret_cast<float2*>(s + 8 * S::RP) = make_float2(sum[i][2], sum[i][3]);
        }
    }
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    if (splits > 1) cluster.sync();
    else __syncthreads();
    const float scale = a.scale ? a.scale[tile.id] : 1.f;
    for (int e = rank * (kThreads + 32) + threadIdx.x; e < S::TM * S::RP; e += splits * (kThreads + 32)) {
        const int r = e / S::RP, c = e % S::RP;
        if (r >= tile.rows || c >= a.r) continue;
        float v = sums[e];
        if (splits > 1) {                              // all CTAs' numbers under way before the first is added
            float x[8];
#pragma unroll
            for (int s = 0; s < 8; ++s) x[s] = s < splits ? cluster.map_shared_rank(sums, s)[e] : 0.f;
            v = x[0];
#pragma unroll
            for (int s = 1; s < 8; ++s) v += x[s];
        }
        out[(int64_t)r * a.r + c] = v * scale;
    }
    if (splits > 1) cluster.sync();                    // the others have read this CTA's sums
}

template <typename T, int NT, bool TRANS>
gpd_status launch_tma(const ShrinkArgs& a, cudaStream_t st) {
    using S = TmaShape<NT, TRANS>;
    const int64_t tiles = tiles_of(a.seg, S::TM), stages = (a.C + kDeep - 1) / kDeep;
    // The parts of a tile's columns with which the busiest SM is done first, a CTA costing about six stages beside its own:
    // an SM that has one CTA more than the others holds all up, and one that has less than three does not reach its share
    // of the bandwidth (16384 x 8192, rank 32, 280 tiles: two parts 165 us for both products, one 175).
    int splits = 1;
    int64_t best = 0;
    for (int s = 1; s <= 8; s *= 2) {
        const int64_t per = (tiles * s + sm_count() - 1) / sm_count(), time = std::max<int64_t>(per, 3) * ((stages + s - 1) / s + 6);
        if (s == 1 || time < best) {
            best = time;
            splits = s;
        }
    }
    if (tiles * splits > 0x7fffffff) return GPD_ERR_SHAPE;
    CUtensorMap map_x, map_w;
    if (!make_map(&map_x, a.x, 2, 1, a.seg.T, a.C, a.ldx, 0, S::TM, kDeep)) return GPD_ERR_CUDA;
    if (a.w_vec && a.seg.n > 0) {
        const bool ok = TRANS ? make_map(&map_w, a.w, 2, a.seg.n, a.C, a.r, a.ldw, a.next, kDeep, S::W::PITCH / 2)
                              : make_map(&map_w, a.w, 2, a.seg.n, a.r, a.C, a.ldw, a.next, S::RP, kDeep);
        if (!ok) return GPD_ERR_CUDA;
    } else {
        map_w = map_x;                                 // not used
    }
    auto kernel = shrink_tma_kernel<T, NT, TRANS>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) != cudaSuccess) return GPD_ERR_CUDA;
    return launch_after(kernel, dim3((unsigned)(tiles * splits)), dim3(kThreads + 32), S::SMEM, splits, st, map_x, map_w, a, splits);
}

template <typename T, int NT, bool TRANS>
gpd_status launch_rows(const ShrinkArgs& a, cudaStream_t st) {
    // Segments of 16 rows and less on average: tiles of 16 rows.
    if (a.seg.T <= 16 * (int64_t)a.seg.S) return launch<T, NT, 1, TRANS>(a, st);
    return a.x_vec ? launch_tma<T, NT, TRANS>(a, st) : launch<T, NT, 4, TRANS>(a, st);
}
template <typename T, bool TRANS>
gpd_status launch_rank(const ShrinkArgs& a, cudaStream_t st) {
    if (a.r <= 16) return launch_rows<T, 2, TRANS>(a, st);
    if (a.r <= 32) return launch_rows<T, 4, TRANS>(a, st);
    return a.r <= 64 ? launch_rows<T, 8, TRANS>(a, st) : launch_rows<T, 16, TRANS>(a, st);
}

}  // namespace

int shrink_status_fetch_and_clear() {
    int v = 0, zero = 0;
    if (cudaMemcpyFromSymbol(&v, g_shrink_status, sizeof(int)) != cudaSuccess) return (int)GPD_ERR_CUDA;
    if (v != 0) cudaMemcpyToSymbol(g_shrink_status, &zero, sizeof(int));
    return v;
}

gpd_status shrink(int type, bool transposed, const ShrinkArgs& a, cudaStream_t st) {
    if (type == GPD_DT_BF16) return transposed ? launch_rank<__nv_bfloat16, true>(a, st) : launch_rank<__nv_bfloat16, false>(a, st);
    return transposed ? launch_rank<__half, true>(a, st) : launch_rank<__half, false>(a, st);
}

}  // namespace adapter
}  // namespace gpd
