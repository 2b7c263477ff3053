// Low-rank adapters over short segments (a token each, or a few), both products in one launch:
//   h[t] = A_i x[t],   out[t] = base[t] + scale_i B_i h[t]
//
// Bound by reading the adapters, and where that is little by latency.  A cluster takes 16 rows of one segment.  Each of its CTAs
// has a part of the columns of A and of the rows of B, all of which it asks for at once (they fit in shared memory); it
// computes its share of h, gives it to every CTA of the cluster, and after one barrier each has h and computes its columns of out.
// Nothing but that barrier and the segment's numbers stands between the launch and the loads.
//
// Measured: 64 rows with an adapter each, 4096 x 4096, rank 16, BF16: 8.3 us, in two launches 21; reading the adapters takes 2.8.
// The columns' loads, the meeting of the CTAs and the rows' loads are 2 to 3 us each.  Many more segments run in waves of clusters: 256
// of them 33 us, reading takes 10.4.
#include <cooperative_groups.h>

#include <algorithm>

#include "adapter_rows.h"

namespace gpd {
namespace adapter {

namespace {

constexpr int kThreads = 128, kWarps = 4, kBlockCols = 64, kMostSplits = 8;

__device__ int g_short_status = 0;                     // GPD_ERR_TIMEOUT if a bounded wait expired

struct ShortArgs {
    ShrinkArgs down;
    ExpandArgs above;
    int blocks_a, blocks_b;                            // blocks of 64 columns of A and rows of B that a CTA has at most
    int all_a, all_b;                                  // and all of them
};
template <int NT>
struct Shape {
    static constexpr int RP = 8 * NT;
    using A = WTile<RP, kBlockCols>;
    using B = WTile<kBlockCols, RP>;
    static constexpr int SUMS = 16 * RP;               // floats: a share of h
    static_assert(A::BYTES >= SUMS * 4, "a warp's share fits in its first block of A");
    // A (a block for every warp at least), B, the CTAs' shares and h
    static int bytes(int blocks_a, int blocks_b, int splits) {
        return std::max(blocks_a, kWarps) * A::BYTES + blocks_b * B::BYTES + (splits + 1) * SUMS * 4 + 1024;
    }
};

template <typename T, typename O, int NT, int PARTS>
__global__ void __launch_bounds__(kThreads, NT == 2 && sizeof(O) == 2 ? 5 : 1) short_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                         const __grid_constant__ ShortArgs s, int log_splits) {
    using S = Shape<NT>;
    constexpr int KT = S::RP / 16;
    extern __shared__ unsigned char raw[];
    __shared__ uint64_t ready_a[kWarps], ready_b[kWarps];
    __shared__ int abort;
    unsigned char* smem = raw + (1024 - (smem_at(raw) & 1023)) % 1024;
    const int splits = 1 << log_splits, rank = blockIdx.x & (splits - 1), lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2;
    if (threadIdx.x < kWarps) {
        tc::mbar_init(&ready_a[threadIdx.x], 1);
        tc::mbar_init(&ready_b[threadIdx.x], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 0) abort = 0;
    __syncthreads();
    after_previous();
    const ShrinkArgs& down = s.down;
    const ExpandArgs& above = s.above;
    const RowTile tile = find_tile<16>(down.seg, blockIdx.x >> log_splits);
    if (tile.rows == 0) return;                        // the whole cluster
    const bool none = tile.id < 0 || tile.id >= down.seg.n;
    // the CTAs of a cluster write to each other only when all of them have come this far
    if (!none) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const bool has[2] = {g < tile.rows, g + 8 < tile.rows};
    // this CTA's blocks of A's columns and of B's rows; a warp has every fourth
    const int a0 = s.all_a * rank >> log_splits, na = (s.all_a * (rank + 1) >> log_splits) - a0;
    const int b0 = s.all_b * rank >> log_splits, nb = (s.all_b * (rank + 1) >> log_splits) - b0;
    unsigned char* as = smem;
    unsigned char* bs = as + max(s.blocks_a, kWarps) * S::A::BYTES;
    float* given = reinterpret_cast<float*>(bs + s.blocks_b * S::B::BYTES);            // [splits][16][RP]
    float* h = given + splits * S::SUMS;               // [16][RP]
    // A warp's share of h takes the place of its first block of A, which no other warp reads.
    auto share_of = [&](int w) { return reinterpret_cast<float*>(as + w * S::A::BYTES); };
    if (!none && lane == 0) {
        tc::mbar_expect_tx(&ready_a[warp], (na - warp + kWarps - 1) / kWarps * S::A::BYTES);
        tc::mbar_expect_tx(&ready_b[warp], (nb - warp + kWarps - 1) / kWarps * S::B::BYTES);
#pragma unroll 1
        for (int i = warp; i < na; i += kWarps) S::A::load(as + i * S::A::BYTES, &map_a, (a0 + i) * kBlockCols, 0, tile.id, &ready_a[warp]);
#pragma unroll 1
        for (int i = warp; i < nb; i += kWarps) S::B::load(bs + i * S::B::BYTES, &map_b, 0, (b0 + i) * kBlockCols, tile.id, &ready_b[warp]);
    }
    __syncwarp();
    const O* base = above.base ? static_cast<const O*>(above.base) + (int64_t)(tile.row + g) * above.ldb : nullptr;
    O* out = static_cast<O*>(above.out) + (int64_t)(tile.row + g) * above.ldo;
    auto columns = [&](int i) { return i < nb ? (int)min((int64_t)kBlockCols, above.C - (int64_t)(b0 + i) * kBlockCols) : 0; };
    Share<O> next;
    load_share<O>(next, base ? base + (int64_t)(b0 + warp) * kBlockCols : nullptr, above.ldb, has, columns(warp), above.io_vec);
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    if (!none) {
        float sum[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[n][i] = 0.f;
        // the lane's elements of x: rows g and g + 8, columns 2 q and the next, and eight on, of sixteen; a block ahead
        uint32_t x[2][kBlockCols / 16][4];
        const T* row = static_cast<const T*>(down.x) + (int64_t)(tile.row + g) * down.ldx + 2 * (lane & 3);
        auto load_x = [&](int i, uint32_t (&to)[kBlockCols / 16][4]) {
            const int64_t c = (int64_t)(a0 + i) * kBlockCols;
            const T* p = row + c;
            if (i < na && c + kBlockCols <= down.C) {
#pragma unroll
                for (int k = 0; k < kBlockCols / 16; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        to[k][j] = has[j & 1] ? *reinterpret_cast<const uint32_t*>(p + 8 * (j & 1) * down.ldx + 16 * k + 8 * (j >> 1)) : 0u;
            } else {
                const int left = i < na ? (int)(down.C - c) - 2 * (lane & 3) : 0;
#pragma unroll
                for (int k = 0; k < kBlockCols / 16; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int at = 16 * k + 8 * (j >> 1);
                        const unsigned short* e = reinterpret_cast<const unsigned short*>(p + 8 * (j & 1) * down.ldx + at);
                        to[k][j] = has[j & 1] && at < left ? e[0] : 0u;
                        if (has[j & 1] && at + 1 < left) to[k][j] |= (uint32_t)e[1] << 16;
                    }
            }
        };
        load_x(warp, x[0]);
        bool live = tc::mbar_wait(&ready_a[warp], 0, &abort, &g_short_status);
        for (int i = warp; live && i < na; i += kWarps) {
            if (i + kWarps < na) load_x(i + kWarps, x[1]);
            const uint32_t aa = S::A::lane_at(smem_at(as + i * S::A::BYTES), col_first_row(), col_first());
            float acc[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[n][j] = 0.f;
#pragma unroll
            for (int k = 0; k < kBlockCols / 16; ++k) {
#pragma unroll
                for (int p = 0; p < NT / 2; ++p) {
                    uint32_t b[4];
                    ldmatrix4<false>(b, S::A::on(aa, 16 * p, 16 * k));
                    mma(acc[2 * p], x[0][k], b[0], b[1], T());
                    mma(acc[2 * p + 1], x[0][k], b[2], b[3], T());
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[n][j] += acc[n][j];
#pragma unroll
            for (int k = 0; k < kBlockCols / 16; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[0][k][j] = x[1][k][j];
        }
        __syncwarp();                                  // its blocks have been read
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float* p = share_of(warp) + g * S::RP + 8 * n + 2 * (lane & 3);
            *reinterpret_cast<float2*>(p) = make_float2(sum[n][0], sum[n][1]);
            *reinterpret_cast<float2*>(p + 8 * S::RP) = make_float2(sum[n][2], sum[n][3]);
        }
        __syncthreads();
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        for (int e = threadIdx.x; e < tile.rows * S::RP; e += kThreads) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) v += share_of(w)[e];
            for (int c = 0; c < splits; ++c) *cluster.map_shared_rank(given + rank * 16 * S::RP + e, c) = v;
        }
        // no CTA writes to another after this barrier, so none has to wait for the others at its end
        cluster.sync();
        for (int e = threadIdx.x; e < 16 * S::RP; e += kThreads) {
            float v = 0.f;
            if (e < tile.rows * S::RP && e % S::RP < down.r)           // behind the rank: zeros, where x has infinities too
                for (int c = 0; c < splits; ++c) v += given[c * 16 * S::RP + e];
            h[e] = v;
        }
        __syncthreads();
    }
    if (rank == 0)
        for (int e = threadIdx.x; e < tile.rows * down.r; e += kThreads) {
            const int row = e / down.r, c = e - row * down.r;
            down.h[(int64_t)tile.row * down.r + e] = none ? (tile.id < 0 ? 0.f : __int_as_float(0x7fffffff)) : h[row * S::RP + c];
        }
    uint32_t ha[PARTS][KT][4];
    float undo[2];
    load_parts<T, KT, PARTS>(h + g * S::RP, none ? 0 : S::RP, none || !above.scale ? 1.f : above.scale[tile.id], has, ha, undo);
    const float nothing = tile.id >= down.seg.n ? __int_as_float(0x7fffffff) : 0.f;
    const bool live = none || tc::mbar_wait(&ready_b[warp], 0, &abort, &g_short_status);
    for (int i = warp; live && i < nb; i += kWarps) {
        const Share<O> share = next;
        if (i + kWarps < nb) load_share<O>(next, base ? base + (int64_t)(b0 + i + kWarps) * kBlockCols : nullptr, above.ldb, has, columns(i + kWarps), above.io_vec);
        float acc[8][4];
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[n][j] = nothing;
        if (!none) {
            const uint32_t bb = S::B::lane_at(smem_at(bs + i * S::B::BYTES), col_first_row(), col_first());
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    uint32_t b[4];
                    ldmatrix4<false>(b, S::B::on(bb, 16 * p, 16 * k));
#pragma unroll
                    for (int j = PARTS - 1; j >= 0; --j) {             // the small parts first
                        mma(acc[2 * p], ha[j][k], b[0], b[1], T());
                        mma(acc[2 * p + 1], ha[j][k], b[2], b[3], T());
                    }
                }
            if (std::is_same<T, __half>::value) {
#pragma unroll
                for (int n = 0; n < 8; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[n][j] *= undo[j >> 1];
            }
        }
        const int64_t c = (int64_t)(b0 + i) * kBlockCols;
        store_sum<O>(share, acc, out + c, above.ldo, has, columns(i), above.io_vec, tile.rows > 8);
    }
    if (!none && *static_cast<volatile int*>(&abort)) {                // given up: copies in flight land before the CTA ends
        int never = 0;
        tc::mbar_wait(&ready_a[warp], 0, &never, &g_short_status);
        tc::mbar_wait(&ready_b[warp], 0, &never, &g_short_status);
    }
}

template <typename T, typename O, int NT>
gpd_status launch(const ShrinkArgs& down, const ExpandArgs& above, bool* taken, cudaStream_t st) {
    using S = Shape<NT>;
    constexpr int PARTS = kParts<T, O>;
    const int64_t tiles = tiles_of(down.seg, 16), all_a = (down.C + kBlockCols - 1) / kBlockCols, all_b = (above.C + kBlockCols - 1) / kBlockCols;
    // Eight CTAs per tile while all of them are resident at once, fewer for more tiles as long as their parts fit.
    constexpr int kRoom = 220 * 1024;                  // of shared memory, and a fifth of it
    auto bytes = [&](int n) {
        const int64_t a = (all_a + n - 1) / n, b = (all_b + n - 1) / n;
        return a > 4096 || b > 4096 ? INT32_MAX : S::bytes((int)a, (int)b, n);
    };
    int splits = kMostSplits, log_splits = 0;
    while (splits > 1 && tiles * splits > 4 * sm_count() && bytes(splits / 2) <= kRoom / 5) splits /= 2;
    while (splits > 1 && (all_a < splits || all_b < splits)) splits /= 2;
    while (1 << log_splits < splits) ++log_splits;
    // One CTA per SM waits for its loads alone: beyond two waves of such the pipelines of two launches are faster (4096 x 4096, rank
    // 64, segments of a row, this and two launches: 24 of them 15 and 20 us, 32 24 and 25, 48 34 and 28, 256 147 and 81; two CTAs per SM, rank
    // 32: 64 of them 20 and 28 us, 256 70 and 69).
    int smem = bytes(splits);
    *taken = smem <= kRoom / 2 || (smem <= kRoom && tiles * splits <= 2 * sm_count());
    if (!*taken) return GPD_OK;
    if (tiles * splits > 0x7fffffff) return GPD_ERR_SHAPE;
    // Where all CTAs are resident at once, no SM gets more of them than an even share (64 segments: 8.1 us, else 9.0).
    const int64_t even = (tiles * splits + sm_count() - 1) / sm_count();
    if (even < kRoom / smem) smem = (int)(kRoom / even);
    ShortArgs s{down, above, (int)((all_a + splits - 1) / splits), (int)((all_b + splits - 1) / splits), (int)all_a, (int)all_b};
    CUtensorMap map_a{}, map_b{};                      // without adapters they are not used
    if (down.seg.n > 0 && (!make_map(&map_a, down.w, 2, down.seg.n, down.r, down.C, down.ldw, down.next, S::RP, kBlockCols) ||
                           !make_map(&map_b, above.w, 2, down.seg.n, above.C, above.r, above.ldw, above.next, kBlockCols, S::B::PITCH / 2)))
        return GPD_ERR_CUDA;
    auto kernel = short_kernel<T, O, NT, PARTS>;
    // the limit is the kernel's, not the call's: always the largest, so that calls of other host threads do not meet a lower one
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRoom) != cudaSuccess) return GPD_ERR_CUDA;
    return launch_after(kernel, dim3((unsigned)(tiles * splits)), dim3(kThreads), smem, splits, st, map_a, map_b, s, log_splits);
}
template <typename T, typename O>
gpd_status launch_rank(const ShrinkArgs& down, const ExpandArgs& above, bool* taken, cudaStream_t st) {
    if (down.r <= 16) return launch<T, O, 2>(down, above, taken, st);
    if (down.r <= 32) return launch<T, O, 4>(down, above, taken, st);
    return down.r <= 64 ? launch<T, O, 8>(down, above, taken, st) : launch<T, O, 16>(down, above, taken, st);
}

}  // namespace

int short_status_fetch_and_clear() {
    int v = 0, zero = 0;
    if (cudaMemcpyFromSymbol(&v, g_short_status, sizeof(int)) != cudaSuccess) return (int)GPD_ERR_CUDA;
    if (v != 0) cudaMemcpyToSymbol(g_short_status, &zero, sizeof(int));
    return v;
}

// Segments of 16 rows and less on average, everything but base and out on 16-byte boundaries; *taken: it was done here.
gpd_status short_segments(int type, int out_type, const ShrinkArgs& down, const ExpandArgs& above, bool* taken, cudaStream_t st) {
    *taken = false;
    if (down.seg.T > 16 * (int64_t)down.seg.S || !down.x_vec || !down.w_vec || !above.w_vec) return GPD_OK;
    if (type == GPD_DT_BF16)
        return out_type == GPD_DT_F32 ? launch_rank<__nv_bfloat16, float>(down, above, taken, st)
                                      : launch_rank<__nv_bfloat16, __nv_bfloat16>(down, above, taken, st);
    return out_type == GPD_DT_F32 ? launch_rank<__half, float>(down, above, taken, st) : launch_rank<__half, __half>(down, above, taken, st);
}

}  // namespace adapter
}  // namespace gpd
