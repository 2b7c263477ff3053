// 8-bit matrix product with a power-of-two scale for each block of 128 along the contraction:
//
//   D[i][j] = sum_k 2^(ea[i][k/128] + eb[j][k/128]) A[i][k] B[j][k]   (+ D[i][j])
//
// A and B are rows of e4m3 or e5m2 numbers, contracted along the rows (both K-major).  The scales go to
// the tensor cores as they are: tcgen05.mma.kind::mxf8f6f4 multiplies each row's 32 products of one
// instruction by 2^(ea + eb), so a block of 128 is four instructions that name the same scale byte, and
// scales per row, per 1 x 128 and per 128 x 128 block cost the same.
//
// Large products: two CTAs of a cluster (PAIR) compute a 256 x BN tile with cta_group::2 instructions, each
// holding 128 rows of A and half of B's; a 128 x BN tile of one CTA moves every byte of B into twice as many
// shared memories, and their bandwidth (operands coming in and going to the tensor cores) is what bounds it.
// The even CTA issues; the odd one's copies and scales report to its barriers.
//
// Otherwise one CTA computes 128 x BN output tiles.  Warp 0: one lane issues the TMA copies of the operands (k-blocks
// of 128 bytes per row under the 128-byte swizzle, a ring that runs on across tiles).  Warps 2..5 bring the
// scales: a word holds one row's scales of four k-blocks, and the tensor cores want the words of rows
// i, i + 32, i + 64, i + 96 in lane i of four columns of tensor memory, the same in each quarter of the lanes;
// each warp writes one quarter (tcgen05.st), up to two chunks of eight k-blocks ahead.  (Copies from shared memory
// by the issuing lane, tcgen05.cp, stop the products around them: 850 instead of 450 cycles a k-block.)
// Warp 1: one lane issues the products.  Warps 6..13 read the accumulators back, two sets of which alternate,
// and store.
//
// Accumulation.  tcgen05.mma adds into its FP32 accumulator with truncation, which takes up to an ulp of the sum each
// time: of sums of positive products 4e-6 at K = 8192, 2.4e-5 at 32768, 6e-5 at 65536, 2.8e-4 at 524288.  16-bit results
// take one chain over the whole contraction up to K = 65536, where that is an eighth of FP16's rounding.  Longer ones, and
// FP32 results of any length, cut the chain every eight k-blocks (32 instructions) and add the pieces in registers, rounded
// to nearest: 4096 x 4096 x 4100 is then 1.0e-7 off the exact product, a plain FP32 product 1.0e-7; a 16-bit result at
// K = 524288 3e-7 before its rounding, for 7 % of the time (2048 x 2048: 1644 -> 1766 us).  (Pieces of four k-blocks: the
// reading of tensor memory holds the tensor cores up.)
//
// Few tiles (short A and B, long K): the CTAs of a cluster take a part of the contraction each; the parts
// meet through distributed shared memory and are added in the order of the parts.
//
// Measured: 8192^3 to BF16 391 us in a burst (2810 TFLOP/s), 444 sustained, at 455 of 448 cycles a k-block and the power
// limit; 4096 x 4096 x 4100 with rows 4112 bytes apart 75 us to FP32, 69 to BF16, with rows on 128-byte boundaries 64 and
// 54; 7 x 4096 x 4096 6.5 us.  Results that cannot leave through shared memory are stored from the registers of their row's
// thread, 32 rows at a time, and that time shows: rows of the output off 16-byte boundaries (8192 x 8191 x 1024 to BF16
// 623 us, on boundaries 61; x 8192 848 and 403), accumulation (4096^3 to FP32 131 us, plain 63; to BF16 82 and 53).
//
// Every mbarrier wait is bounded; on expiry the CTA raises a status word (gpd_device_status), drains its
// copies, frees its tensor memory and returns.
#include <cuda.h>

#include <algorithm>

#include "gemm_common.h"
#include "lm_common.h"
#include "tc_common.h"

namespace gpd {

namespace {

using tc::mbar_expect_tx;
using tc::mbar_init;
using tc::mbar_try_wait;
using tc::smem_u32;
using tc::umma_commit;

constexpr int BM = 128, BK = 128, UMMA_K = 32;
constexpr int kSfWarps = 4, kEpiWarps = 8, kThreads = 32 * (2 + kSfWarps + kEpiWarps);
constexpr int kChunk = 8;                              // k-blocks whose scales arrive together; FP32 results: added up in tensor memory
constexpr int kMaxSplits = 8;                          // parts of a split contraction (CTAs of a cluster)
constexpr int kSfSlots = 2;                            // chunks whose scales are in flight
__host__ __device__ constexpr int b_rows(int bn, bool pair) { return pair ? bn / 2 : bn; }
__host__ __device__ constexpr int stage_bytes(int bn, bool pair) { return (BM + b_rows(bn, pair)) * BK; }
__host__ __device__ constexpr int sfb_blocks(int bn) { return bn > 128 ? 2 : 1; }
__host__ __device__ constexpr int sf_cols(int bn) { return 4 * (1 + sfb_blocks(bn)); }   // of tensor memory, per four k-blocks
// SPLIT: half an SM's shared memory and registers per CTA, so that two CTAs share an SM, and room for the other
// parts' shares of this CTA's columns.  Otherwise: room for 32 x 32 results per epilogue warp on their way out
// (elem: bytes of one; 0: results are stored from registers alone).
__host__ __device__ constexpr int extra_bytes(int bn, bool split, int elem) {
    return split ? BM * bn * 4 : kEpiWarps * 32 * 32 * elem;
}
__host__ __device__ constexpr int stages(int bn, bool pair, bool split, int elem) {
    const int n = ((split ? 113664 : 232448) - 1024 - 8192 - extra_bytes(bn, split, elem)) / stage_bytes(bn, pair);
    return n > 10 ? 10 : n;
}
__host__ __device__ constexpr int smem_bytes(int bn, bool pair, bool split, int elem) {
    return 1024 + stages(bn, pair, split, elem) * stage_bytes(bn, pair) + extra_bytes(bn, split, elem);
}
// Bytes of a result where they leave through shared memory and a copy engine (whole lines; stores from the
// registers of a row's thread, 16 bytes of 32 rows at a time, held the copies of the next tile up)
__host__ __device__ constexpr int staged_elem(int bn, bool trans, bool split, int elem) { return !trans && !split && bn >= 64 ? elem : 0; }
__host__ __device__ constexpr int tmem_need(int bn) { return 2 * bn + kSfSlots * 2 * sf_cols(bn); }
__host__ __device__ constexpr int tmem_cols(int bn) {
    return tmem_need(bn) <= 64 ? 64 : tmem_need(bn) <= 128 ? 128 : tmem_need(bn) <= 256 ? 256 : 512;
}

__device__ int g_fp8_status = 0;                       // GPD_ERR_TIMEOUT if a bounded wait expired
__device__ __forceinline__ bool mbar_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    return tc::mbar_wait(bar, parity, abort_flag, &g_fp8_status);
}

// Address of this CTA's `p` in the even CTA of the pair
__device__ __forceinline__ uint32_t in_leader(const void* p) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(0));
    return a;
}
// Arrivals (at a barrier of either CTA of a pair) and waits that order accesses to tensor memory alone, which
// tcgen05.wait and tcgen05.fence before the arrival and tcgen05.fence after the wait take care of: a releasing
// arrival would also wait for the thread's global loads and stores, 1000 cycles and more under load.
__device__ __forceinline__ void mbar_arrive_relaxed(uint32_t addr) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait_relaxed(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.relaxed.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool mbar_wait_relaxed(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    if (mbar_try_wait_relaxed(bar, parity)) return true;
    const long long t0 = clock64();
    while (!mbar_try_wait_relaxed(bar, parity)) {
        if (*abort_flag) return false;
        if (clock64() - t0 > tc::kWaitCycles) {
            *abort_flag = 1;
            atomicExch(&g_fp8_status, (int)GPD_ERR_TIMEOUT);
            return false;
        }
    }
    return true;
}
// bar: shared::cluster address
template <bool PAIR>
__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* map, int c0, int c1, uint32_t bar) {
    if (PAIR)
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4}], [%2];"
            ::"r"(smem_u32(dst)), "l"(map), "r"(bar), "r"(c0), "r"(c1) : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
            ::"r"(smem_u32(dst)), "l"(map), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
// 32 x 32 results from shared memory to (column, row) of the output; what lies beyond it is left out
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];"
                 ::"l"(map), "r"(src), "r"(c0), "r"(c1) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// Whether the phase is over, without waiting
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return ok != 0;
}
// Arrival, at the barrier of every CTA of the tile, once the tensor cores are done with what was issued so far
template <bool PAIR>
__device__ __forceinline__ void commit(uint64_t* bar) {
    if (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(smem_u32(bar)), "h"((unsigned short)3) : "memory");
    else
        umma_commit(bar);
}
// K-major tile with rows of 128 bytes under the 128-byte swizzle: 8-row groups 1024 bytes apart
// (descriptor version 1, layout type 2).
__device__ __forceinline__ uint64_t desc_sw128(uint32_t addr) {
    return (uint64_t)((addr >> 4) & 0x3FFF) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}
// Four columns of this warp's quarter of the lanes
__device__ __forceinline__ void tmem_st4(uint32_t taddr, uint4 v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void umma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                        uint32_t accumulate) {
    if (PAIR)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
// FP32 accumulator, both operands K-major, M = m, N = n, scales e8m0; types 0 = e4m3, 1 = e5m2; `sf` = byte of
// the scale words that this instruction uses
__device__ __forceinline__ uint32_t idesc_mx(int m, int n, int a_type, int b_type, int sf) {
    return ((uint32_t)sf << 4) | ((uint32_t)a_type << 7) | ((uint32_t)b_type << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) |
           ((uint32_t)(m >> 4) << 24) | ((uint32_t)sf << 29);
}
__device__ __forceinline__ void tmem_ld16(uint32_t* r, uint32_t taddr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
}
// True in one lane of the (converged) warp
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, uint32_t rank, float v) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(a), "f"(v) : "memory");
}

struct ScaleRows {
    const uint8_t* p;
    int64_t ld, rows;                                  // rows of the operand
    int shift;                                         // log2 of the operand rows that share a scale row
    bool words;                                        // every row starts on a 4-byte boundary
};
struct Fp8Params {
    ScaleRows sa, sb;
    void* out;
    int64_t ldd, M, N;                                 // rows of A, rows of B
    int kb, a_type, b_type, accumulate;
    bool vec;                                          // 16-byte stores into the rows of out
    bool copy_out;                                     // results leave through shared memory (tmD)
    int tiles_m, tiles_n;
    int part_kb, part_more;                            // SPLIT: k-blocks of a part; the first part_more have one more
};

// Up to four scales of one row as a word.  Rows and k-blocks that do not exist get any valid scale (1): their
// products are zero or not stored.
__device__ __forceinline__ uint32_t scale_bytes(const uint8_t* p, int n) {
    uint32_t w = 0x7f7f7f7fu;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) w = (w & ~(0xffu << (8 * i))) | ((uint32_t)__ldg(p + i) << (8 * i));
    return w;
}

// Tile order: columns of up to 2048 rows, so that the tiles in flight share operands in L2.
template <bool PAIR>
__device__ __forceinline__ void tile_origin(const Fp8Params& p, int tile, int bn, int64_t& m0, int64_t& n0) {
    constexpr int H = PAIR ? 8 : 16;
    const int band = H * p.tiles_n, b = tile / band, r = tile - b * band;
    const int h = min(H, p.tiles_m - H * b);
    m0 = (int64_t)(H * b + r % h) * (PAIR ? 2 * BM : BM);
    n0 = (int64_t)(r / h) * bn;
}

// TRANS: D[i][j] is stored at out[j][i] (the caller swapped the operands); consecutive lanes hold consecutive i.
// SPLIT: gridDim = (parts, tiles), the parts of a tile are a cluster.  PAIR: gridDim = (2, pairs).
// CHUNKED: one chain of additions in tensor memory per chunk, the chunks added up in registers.
template <int BN, typename T, bool TRANS, bool PAIR, bool SPLIT, bool CHUNKED>
__global__ void __launch_bounds__(kThreads, SPLIT ? 2 : 1)
gemm_fp8_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                const __grid_constant__ CUtensorMap tmD, const Fp8Params prm) {
    constexpr int STAGED = staged_elem(BN, TRANS, SPLIT, sizeof(T)), STAGES = stages(BN, PAIR, SPLIT, STAGED), STAGE = stage_bytes(BN, PAIR), SFB = sfb_blocks(BN);
    // columns of an epilogue warp, in units of 32: two warps share a lane quarter, of narrow tiles one does it all
    constexpr int W0 = BN >= 64 ? (BN / 32 + 1) / 2 * 32 : BN, W1 = BN - W0;
    constexpr int COLS = tmem_cols(BN);
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    __shared__ __align__(8) uint64_t full_bar[STAGES], empty_bar[STAGES], sf_full[kSfSlots], sf_empty[kSfSlots],
        acc_full[2], acc_empty[2];
    __shared__ __align__(16) uint4 sf_words[2][2 * (1 + SFB) * 32];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 32) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmA) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmB) : "memory");
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&full_bar[s], 1);
            mbar_init(&empty_bar[s], 1);
        }
        for (int s = 0; s < kSfSlots; ++s) {
            mbar_init(&sf_full[s], PAIR ? 2 * kSfWarps : kSfWarps);
            mbar_init(&sf_empty[s], 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&acc_full[s], 1);
            mbar_init(&acc_empty[s], PAIR ? 2 * kEpiWarps : kEpiWarps);
        }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (PAIR || SPLIT) cluster_sync();                 // the other CTAs of the cluster run, and their barriers exist
    lm::after_previous();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_slot, tmem_sf = tmem + 2 * BN;
    volatile int* abort_p = &abort_flag;

    // this CTA's part of the contraction (whole k-blocks) and its tiles; its place in the pair
    const int S = SPLIT ? (int)gridDim.x : 1, rank = SPLIT ? (int)blockIdx.x : 0, side = PAIR ? (int)blockIdx.x : 0;
    const int kb0 = SPLIT ? rank * prm.part_kb + min(rank, prm.part_more) : 0;
    const int kb1 = SPLIT ? kb0 + prm.part_kb + (rank < prm.part_more) : prm.kb;
    const int tile0 = PAIR || SPLIT ? (int)blockIdx.y : (int)blockIdx.x, tiles = prm.tiles_m * prm.tiles_n;
    const int tile_step = PAIR || SPLIT ? (int)gridDim.y : (int)gridDim.x;

    // Warps 0 and 1 run their loops as a whole, with one elected lane issuing: what the instructions name is then the
    // same for the warp and stays in uniform registers (issued by a lone lane, 4 products with their waits and
    // bookkeeping took 1040 cycles a k-block, more than twice what the tensor cores need for them).
    if (warp == 0) {
        const bool one = elect_one();
        const uint32_t bar0 = PAIR ? in_leader(&full_bar[0]) : smem_u32(&full_bar[0]);
        int s = 0, issued = 0;
        uint32_t phase = 1;                            // of the empty barriers: the first round does not wait
        bool live = true;                              // per lane; the loops run on without issuing when a wait expired
        for (int tile = tile0; tile < tiles; tile += tile_step) {
            int64_t m0, n0;
            tile_origin<PAIR>(prm, tile, BN, m0, n0);
            const int am = (int)m0 + side * BM, bn = (int)n0 + side * b_rows(BN, PAIR);
            for (int kb = kb0; kb < kb1; ++kb) {
                live = live && mbar_wait(&empty_bar[s], phase, abort_p);
                if (one && live) {
                    ++issued;
                    if (side == 0) mbar_expect_tx(&full_bar[s], (PAIR ? 2 : 1) * STAGE);
                    tma_load_2d<PAIR>(smem + s * STAGE, &tmA, kb * BK, am, bar0 + 8 * s);
                    tma_load_2d<PAIR>(smem + s * STAGE + BM * BK, &tmB, kb * BK, bn, bar0 + 8 * s);
                }
                if (++s == STAGES) {
                    s = 0;
                    phase ^= 1;
                }
            }
        }
        if (*abort_p && side == 0 && one) {            // copies still in flight, the pair's too, land before the CTA exits
            for (int j = issued > STAGES ? issued - STAGES : 0; j < issued; ++j) {
                const long long t0 = clock64();
                while (!mbar_try_wait(&full_bar[j % STAGES], (j / STAGES) & 1) && clock64() - t0 < tc::kWaitCycles) {}
            }
        }
    } else if (warp == 1) {
        if (side == 0) {
            const bool one = elect_one();
            const uint64_t desc0 = desc_sw128(smem_u32(smem));
            const uint32_t idesc0 = idesc_mx(PAIR ? 2 * BM : BM, BN, prm.a_type, prm.b_type, 0);
            int s = 0, gs = 0, set = 0;                // stage, scale slot and accumulator set in turn, and their phases
            uint32_t phase = 0, gphase = 0, aphase = 1;
            bool live = true, ready = false;           // ready: the stage's operands are known to be there
            for (int tile = tile0; tile < tiles; tile += tile_step) {
                bool fresh = true;                     // the next product starts a chain
                for (int c = kb0 / kChunk; kChunk * c < kb1; ++c) {
                    if (fresh) live = live && mbar_wait_relaxed(&acc_empty[set], aphase, abort_p);
                    live = live && mbar_wait_relaxed(&sf_full[gs], gphase, abort_p);
                    const uint32_t sf = tmem_sf + gs * 2 * sf_cols(BN), d = tmem + set * BN;
#pragma unroll
                    for (int i = 0; i < kChunk; ++i) {
                        if (kChunk * c + i < kb0 || kChunk * c + i >= kb1) continue;
                        if (!ready) live = live && mbar_wait(&full_bar[s], phase, abort_p);
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint64_t a = desc0 + (uint64_t)((s * STAGE) >> 4), b = a + (uint64_t)((BM * BK) >> 4);
                        // byte i % 4 of the scale words of the chunk's first or second half
                        const uint32_t idesc = idesc0 | (uint32_t)(i & 3) << 4 | (uint32_t)(i & 3) << 29;
                        const uint32_t w = sf + (i >> 2) * sf_cols(BN);
                        uint64_t* done = &empty_bar[s];
                        if (++s == STAGES) {
                            s = 0;
                            phase ^= 1;
                        }
                        ready = mbar_test(&full_bar[s], phase);        // the next stage, looked at while this one is issued
                        if (one && live) {
#pragma unroll
                            for (int k = 0; k < BK / UMMA_K; ++k)
                                umma_mx<PAIR>(d, a + k * (UMMA_K >> 4), b + k * (UMMA_K >> 4), idesc, w, w + 4, !(fresh && k == 0));
                            commit<PAIR>(done);
                        }
                        fresh = false;
                    }
                    const bool end = CHUNKED || kChunk * (c + 1) >= kb1;       // of the chain
                    if (one && live) {
                        commit<PAIR>(&sf_empty[gs]);
                        if (end) commit<PAIR>(&acc_full[set]);
                    }
                    if (++gs == kSfSlots) {
                        gs = 0;
                        gphase ^= 1;
                    }
                    if (end) {
                        fresh = true;
                        if (set) aphase ^= 1;
                        set ^= 1;
                    }
                }
            }
        }
        __syncwarp();
    } else if (warp < 2 + kSfWarps) {
        // Warp q of the four fetches the words of rows 32 q + lane of every block of 128; the warps exchange them
        // through shared memory, and each writes all of them to its quarter.  A chunk's words are fetched two chunks
        // before they are wanted.
        constexpr int NB = 1 + SFB;
        const int q = warp & 3;
        const uint8_t* rows[NB];                       // this lane's scale rows of the tile being fetched; null: none
        int tile = tile0, c = kb0 / kChunk;            // the chunk to be fetched next
        auto find_rows = [&]() {
            int64_t m0, n0;
            tile_origin<PAIR>(prm, tile, BN, m0, n0);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const ScaleRows& s = b == 0 ? prm.sa : prm.sb;
                const int64_t r = (b == 0 ? m0 + side * BM : n0 + 128 * (b - 1)) + 32 * q + lane;
                rows[b] = r < s.rows ? s.p + (r >> s.shift) * s.ld : nullptr;
            }
        };
        auto fetch = [&](uint32_t (&v)[2][NB]) {
            if (tile >= tiles) return;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int kb = kChunk * c + 4 * h;
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    v[h][b] = 0x7f7f7f7fu;
                    if (rows[b] && kb < prm.kb) {
                        if (kb + 4 <= prm.kb && (b == 0 ? prm.sa.words : prm.sb.words)) v[h][b] = __ldg(reinterpret_cast<const uint32_t*>(rows[b] + kb));
                        else v[h][b] = scale_bytes(rows[b] + kb, prm.kb - kb);
                    }
                }
            }
            if (kChunk * (++c) >= kb1) {
                c = kb0 / kChunk;
                tile += tile_step;
                if (tile < tiles) find_rows();
            }
        };
        const int chunks = (kb1 + kChunk - 1) / kChunk - kb0 / kChunk;
        const int total = tile0 < tiles ? chunks * ((tiles - tile0 + tile_step - 1) / tile_step) : 0;
        uint32_t ring[2][2][NB];
        if (total > 0) find_rows();
        fetch(ring[0]);
        fetch(ring[1]);
        const uint32_t sf_full0 = PAIR ? in_leader(&sf_full[0]) : smem_u32(&sf_full[0]);
        bool live = true;
        for (int i0 = 0; i0 < total; i0 += 2) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {              // chunk i0 + i: ring, exchange buffer and slot i
                if (i0 + i >= total) break;
                uint32_t* buf = reinterpret_cast<uint32_t*>(sf_words[i]);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int b = 0; b < NB; ++b) buf[((h * NB + b) * 32 + lane) * 4 + q] = ring[i][h][b];
                fetch(ring[i]);
                asm volatile("bar.sync 1, 128;" ::: "memory");
                live = live && mbar_wait(&sf_empty[i], ((i0 >> 1) & 1) ^ 1, abort_p);
                __syncwarp();
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                for (int b = 0; b < 2 * NB; ++b)
                    tmem_st4(tmem_sf + i * 2 * sf_cols(BN) + 4 * b + ((uint32_t)(q * 32) << 16), sf_words[i][b * 32 + lane]);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0 && live) mbar_arrive_relaxed(sf_full0 + 8 * i);
            }
        }
    } else {
        const int q = warp & 3, half = (warp - 2 - kSfWarps) >> 2;      // tcgen05.ld: a warp reads its quarter of the lanes
        const int c0 = half * W0, width = half ? W1 : W0;
        const uint32_t lane_base = (uint32_t)(q * 32) << 16;
        const uint32_t acc_empty0 = PAIR ? in_leader(&acc_empty[0]) : smem_u32(&acc_empty[0]);
        float acc[CHUNKED ? W0 : 1];                   // CHUNKED: W0 = W1 or W1 = 0
        uint8_t* staging = smem + STAGES * STAGE + (warp - 2 - kSfWarps) * 32 * 32 * STAGED;
        int ac = 0;
        bool ok = true;
        T* out = static_cast<T*>(prm.out);
        const uint32_t parts = smem_u32(smem + STAGES * STAGE);        // SPLIT: [part][column of the share][128]
        const int own = SPLIT ? BN / S : 1;            // columns of a CTA's share
        for (int tile = tile0; tile < tiles && ok; tile += tile_step) {
            int64_t m0, n0;
            tile_origin<PAIR>(prm, tile, BN, m0, n0);
            const int64_t row = m0 + side * BM + q * 32 + lane;
            // w columns from column c of the tile, in f
            auto put = [&](int c, const float* f, int w) {
                if (SPLIT) {
                    for (int j = 0; j < w; ++j) {      // to the CTA that adds up this column
                        const int to = (c + j) / own;
                        st_cluster(parts + 4 * ((rank * own + (c + j) - to * own) * BM + q * 32 + lane), to, f[j]);
                    }
                    return;
                }
                if (row >= prm.M) return;
                if (TRANS) {
#pragma unroll
                    for (int j = 0; j < w; ++j) {
                        if (n0 + c + j >= prm.N) break;
                        T* o = out + (n0 + c + j) * prm.ldd + row;
                        *o = lm::from_f32<T>(prm.accumulate ? f[j] + lm::to_f32(*o) : f[j]);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < w; j += 8) {
                        const int64_t n = prm.N - (n0 + c + j);
                        if (n <= 0) break;
                        T* o = out + row * prm.ldd + n0 + c + j;
                        float v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = f[j + i];
                        if (prm.accumulate) {
                            float old[8];
                            if (prm.vec) lm::unpack8<T>(lm::load8<T, true>(o, n), old);
                            else lm::unpack8<T>(lm::load8<T, false>(o, n), old);
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[i] += old[i];
                        }
                        if (prm.vec) lm::store8<T, true>(o, v, n);
                        else lm::store8<T, false>(o, v, n);
                    }
                }
            };
            // 32 columns from column c of the tile, by way of shared memory
            auto copy_out = [&](int c, const float* f) {
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");      // the last ones have left
                __syncwarp();
                if constexpr (STAGED == 4) {           // rows of 128 bytes under the 128-byte swizzle
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        *reinterpret_cast<float4*>(staging + lane * 128 + ((j ^ (lane & 7)) * 16)) = make_float4(f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3]);
                } else if constexpr (STAGED == 2) {    // rows of 64 bytes under the 64-byte swizzle
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        *reinterpret_cast<uint4*>(staging + lane * 64 + ((j ^ ((lane >> 1) & 3)) * 16)) =
                            make_uint4(lm::pack2(f[8 * j], f[8 * j + 1], T()), lm::pack2(f[8 * j + 2], f[8 * j + 3], T()),
                                       lm::pack2(f[8 * j + 4], f[8 * j + 5], T()), lm::pack2(f[8 * j + 6], f[8 * j + 7], T()));
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                const int64_t r0 = m0 + side * BM + q * 32, col = n0 + c;
                if (lane == 0 && r0 < prm.M && col < prm.N) tma_store_2d(&tmD, smem_u32(staging), (int)col, (int)r0);
            };
            auto emit = [&](int c, const float* f) {
                if constexpr (STAGED != 0) {
                    if (prm.copy_out) {
                        copy_out(c, f);
                        return;
                    }
                }
                put(c, f, BN < 32 ? 16 : 32);
            };
            auto release = [&](int set) {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive_relaxed(acc_empty0 + 8 * set);
            };
            auto ready = [&](int set, int n) {
                const bool r = mbar_wait(&acc_full[set], (n >> 1) & 1, abort_p);
                ok = __all_sync(0xffffffffu, r);       // tcgen05.ld is warp-collective: all lanes or none
                if (ok) asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            };
            constexpr int STEP = BN < 32 ? 16 : 32;    // columns at a time
            auto read = [&](uint32_t taddr, uint32_t (&r)[STEP]) {
                tmem_ld16(r, taddr);
                if constexpr (STEP == 32) tmem_ld16(r + 16, taddr + 16);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
            };
            if constexpr (CHUNKED) {
#pragma unroll
                for (int j = 0; j < W0; ++j) acc[j] = 0.f;
                for (int k = kb0 / kChunk; kChunk * k < kb1 && ok; ++k, ++ac) {
                    ready(ac & 1, ac);
                    if (!ok) break;
                    const uint32_t base = tmem + (ac & 1) * BN + lane_base + c0;
                    if (width) {
#pragma unroll
                        for (int c = 0; c < W0; c += STEP) {
                            uint32_t r[STEP];
                            read(base + c, r);
#pragma unroll
                            for (int j = 0; j < STEP; ++j) acc[c + j] += __uint_as_float(r[j]);
                        }
                    }
                    release(ac & 1);
                }
                if (ok && width) {
#pragma unroll
                    for (int c = 0; c < W0; c += STEP) emit(c0 + c, acc + c);
                }
            } else {
                ready(ac & 1, ac);
                if (!ok) break;
                const uint32_t base = tmem + (ac & 1) * BN + lane_base + c0;
                for (int c = 0; c < width; c += STEP) {
                    uint32_t r[STEP];
                    read(base + c, r);
                    if (c + STEP >= width) release(ac & 1);
                    float f[STEP];
#pragma unroll
                    for (int j = 0; j < STEP; ++j) f[j] = __uint_as_float(r[j]);
                    emit(c0 + c, f);
                }
                if (width == 0) release(ac & 1);
                ++ac;
            }
        }
        if (STAGED && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");     // written before the CTA ends
    }
    __syncwarp();
    if (SPLIT) {
        // one tile per cluster: the parts of this CTA's columns are here once all have arrived, and nothing is
        // written to or read from another CTA after that
        cluster_sync();
        int64_t m0, n0;
        tile_origin<PAIR>(prm, tile0, BN, m0, n0);
        const int own = BN / S;
        const float* part = reinterpret_cast<const float*>(smem + STAGES * STAGE);
        T* out = static_cast<T*>(prm.out);
        if (!abort_flag) {
            for (int e = threadIdx.x; e < own * BM; e += kThreads) {
                const int64_t row = m0 + (e & (BM - 1)), col = n0 + rank * own + e / BM;
                if (row >= prm.M || col >= prm.N) continue;
                float v = 0.f;
                for (int s = 0; s < S; ++s) v += part[s * own * BM + e];
                T* o = TRANS ? out + col * prm.ldd + row : out + row * prm.ldd + col;
                *o = lm::from_f32<T>(prm.accumulate ? v + lm::to_f32(*o) : v);
            }
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (PAIR) cluster_sync();                          // neither CTA's shared or tensor memory goes while the other may use it
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(COLS) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(COLS) : "memory");
    }
}

// ---- host side ---------------------------------------------------------------------------------------
bool make_map_2d(CUtensorMap* map, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
    tc::EncodeTiledFn fn = tc::encode_tiled_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld};
    cuuint32_t box[2] = {BK, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Output of `elem`-byte elements, written in boxes of 32 x 32.
bool make_out_map(CUtensorMap* map, void* base, int64_t rows, int64_t cols, int64_t ld, int elem) {
    tc::EncodeTiledFn fn = tc::encode_tiled_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)(ld * elem)};
    cuuint32_t box[2] = {32, 32};
    cuuint32_t estr[2] = {1, 1};
    return fn(map, elem == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, base, dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, elem == 4 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
              CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Operand {
    const void* q;
    int64_t ld, rows;
    int type;
    ScaleRows s;
};
struct Config { int bn, splits; bool trans, pair; };

template <int BN, typename T, bool TRANS, bool PAIR, bool SPLIT, bool CHUNKED>
gpd_status launch(const Operand& a, const Operand& b, Fp8Params prm, int64_t K, int splits, cudaStream_t st) {
    constexpr int STAGED = staged_elem(BN, TRANS, SPLIT, sizeof(T));
    CUtensorMap tmA, tmB, tmD{};
    prm.copy_out = STAGED != 0 && prm.vec && !prm.accumulate;
    if (prm.copy_out && !make_out_map(&tmD, prm.out, a.rows, b.rows, prm.ldd, sizeof(T))) return GPD_ERR_CUDA;
    if (!make_map_2d(&tmA, a.q, a.rows, K, a.ld, BM) || !make_map_2d(&tmB, b.q, b.rows, K, b.ld, b_rows(BN, PAIR))) return GPD_ERR_CUDA;
    auto kernel = gemm_fp8_kernel<BN, T, TRANS, PAIR, SPLIT, CHUNKED>;
    constexpr int smem = smem_bytes(BN, PAIR, SPLIT, STAGED), rows = PAIR ? 2 * BM : BM;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return GPD_ERR_CUDA;
    prm.sa = a.s;
    prm.sb = b.s;
    prm.M = a.rows;
    prm.N = b.rows;
    prm.a_type = a.type == GPD_DT_E5M2;
    prm.b_type = b.type == GPD_DT_E5M2;
    prm.tiles_m = (int)((a.rows + rows - 1) / rows);
    prm.tiles_n = (int)((b.rows + BN - 1) / BN);
    prm.part_kb = prm.kb / splits;
    prm.part_more = prm.kb % splits;
    const int64_t tiles = (int64_t)prm.tiles_m * prm.tiles_n;
    if (tiles > 0x3fffffff) return GPD_ERR_SHAPE;
    const int cluster = PAIR ? 2 : splits;
    const unsigned n = (unsigned)(SPLIT ? tiles : std::min<int64_t>(tiles, sm_count() / cluster));
    return lm::launch_after(kernel, PAIR || SPLIT ? dim3(cluster, n) : dim3(n), dim3(kThreads), smem, cluster, st, tmA, tmB, tmD, prm);
}

// Tile width, orientation, pairing and split by the smallest estimated time, in cycles.  A k-block of a tile takes the
// tensor cores 2 BN (four dependent instructions: 344 at least) and its copies a cycle per 64 bytes; a tile costs about
// 1500 besides.  A part of a split contraction has half an SM's stages, whose latency shows (about 3300 over their
// number), and 3000 for the meeting of the parts.  Measured over 19 shapes from 1 x 4096 x 4096 to 4096^3 with every
// configuration, outputs on 16-byte boundaries and no accumulation (the others' stores are not in the estimate), the
// choice is within 6 % of the best but for 64 x 8192 x 8192 (18.2 us, in four parts 15.5) and
// 16 x 50000 x 512 in FP32 (9.1, 128 x 16 tiles 8.1).  Examples:
// 7 x 4096 x 4096: 6.7 us in four parts, 8.2 in two; 128 x 8192 x 8192: 17.6 us as 256 x 128 pairs, 30.1 split;
// 512 x 8192 x 8192: 23.5 us as 256 x 224 pairs, 28.9 as 128 x 224 tiles, 30.9 as 256 x 128 pairs.
Config choose(int64_t M, int64_t N, int kb, bool chunked) {
    static const int kWidths[] = {16, 32, 64, 128, 192, 224};
    Config best{128, 1, true, false};
    double best_t = 1e300;
    const int sms = sm_count();
    for (int t = 0; t < 2; ++t) {
        const int64_t rows = t ? N : M, cols = t ? M : N;
        for (int bn : kWidths) {
            if (bn == 224 && chunked) continue;        // a tile's row is kept in registers
            for (int pair = 0; pair <= (bn >= 128 ? 1 : 0); ++pair) {
                const int height = pair ? 2 * BM : BM, slots = pair ? sms / 2 : sms;
                const int64_t tiles = ((rows + height - 1) / height) * ((cols + bn - 1) / bn);
                for (int s = 1; s <= (pair ? 1 : kMaxSplits); s *= 2) {
                    if (s > 1 && (bn > 64 || s > kb || tiles * s > 2 * sms)) continue;
                    // two CTAs of a split product share an SM
                    const double waves = s > 1 ? std::max(1.0, (double)(tiles * s) / sms) : (double)((tiles + slots - 1) / slots);
                    double block = std::max(std::max(2.0 * bn, 344.0), stage_bytes(bn, pair) / 64.0);
                    if (s > 1) block = std::max(block, 3300.0 / stages(bn, false, true, 0));
                    const double time = waves * (((kb + s - 1) / s) * block + (s > 1 ? 3000.0 : 1500.0));
                    if (time < best_t * 0.999) {
                        best_t = time;
                        best = Config{bn, s, t == 1, pair == 1};
                    }
                }
            }
        }
    }
    return best;
}

template <typename T, bool TRANS, bool CHUNKED>
gpd_status launch_bn(const Operand& a, const Operand& b, const Fp8Params& prm, int64_t K, const Config& c, cudaStream_t st) {
    switch (c.pair ? -c.bn : c.bn) {
        case 16: return c.splits > 1 ? launch<16, T, TRANS, false, true, CHUNKED>(a, b, prm, K, c.splits, st) : launch<16, T, TRANS, false, false, CHUNKED>(a, b, prm, K, 1, st);
        case 32: return c.splits > 1 ? launch<32, T, TRANS, false, true, CHUNKED>(a, b, prm, K, c.splits, st) : launch<32, T, TRANS, false, false, CHUNKED>(a, b, prm, K, 1, st);
        case 64: return c.splits > 1 ? launch<64, T, TRANS, false, true, CHUNKED>(a, b, prm, K, c.splits, st) : launch<64, T, TRANS, false, false, CHUNKED>(a, b, prm, K, 1, st);
        case 128: return launch<128, T, TRANS, false, false, CHUNKED>(a, b, prm, K, 1, st);
        case 192: return launch<192, T, TRANS, false, false, CHUNKED>(a, b, prm, K, 1, st);
        case -128: return launch<128, T, TRANS, true, false, CHUNKED>(a, b, prm, K, 1, st);
        case -192: return launch<192, T, TRANS, true, false, CHUNKED>(a, b, prm, K, 1, st);
        default: break;
    }
    if constexpr (!CHUNKED) {
        if (c.pair) return launch<224, T, TRANS, true, false, false>(a, b, prm, K, 1, st);
        return launch<224, T, TRANS, false, false, false>(a, b, prm, K, 1, st);
    }
    return GPD_ERR_UNSUPPORTED;
}
template <typename T, bool CHUNKED>
gpd_status launch_chain(const Operand& a, const Operand& b, Fp8Params prm, int64_t K, cudaStream_t st) {
    const Config c = choose(a.rows, b.rows, prm.kb, CHUNKED);
    prm.vec = lm::rows_aligned(prm.out, prm.ldd, sizeof(T));
    return c.trans ? launch_bn<T, true, CHUNKED>(b, a, prm, K, c, st) : launch_bn<T, false, CHUNKED>(a, b, prm, K, c, st);
}
// K-blocks in one chain of 16-bit results at most (K = 65536)
constexpr int kLongChain = 512;
template <typename T>
gpd_status launch_type(const Operand& a, const Operand& b, const Fp8Params& prm, int64_t K, cudaStream_t st) {
    if constexpr (sizeof(T) == 2) {
        if (prm.kb <= kLongChain) return launch_chain<T, false>(a, b, prm, K, st);
    }
    return launch_chain<T, true>(a, b, prm, K, st);
}

}  // namespace

int fp8_device_status_fetch_and_clear() {
    int v = 0, zero = 0;
    if (cudaMemcpyFromSymbol(&v, g_fp8_status, sizeof(int)) != cudaSuccess) return (int)GPD_ERR_CUDA;
    if (v != 0) cudaMemcpyToSymbol(g_fp8_status, &zero, sizeof(int));
    return v;
}

}  // namespace gpd

using namespace gpd;

extern "C" gpd_status gpd_gemm_fp8(gpd_dtype a_type, const void* A_dev, int64_t lda, const uint8_t* a_scales_dev, int64_t ldsa,
                                   int32_t a_block_rows, gpd_dtype b_type, const void* B_dev, int64_t ldb,
                                   const uint8_t* b_scales_dev, int64_t ldsb, int32_t b_block_rows, gpd_dtype out_type,
                                   void* out_dev, int64_t ldd, int64_t M, int64_t N, int64_t K, int32_t accumulate,
                                   void* stream) {
    if (!lm::is_fp8_type(a_type) || !lm::is_fp8_type(b_type) || !lm::is_float_type(out_type)) return GPD_ERR_ARG;
    if ((a_block_rows != 1 && a_block_rows != lm::kBlock) || (b_block_rows != 1 && b_block_rows != lm::kBlock)) return GPD_ERR_ARG;
    const int64_t limit = 0x7fffffff - 256;            // row and column coordinates of a copy are 32-bit
    if (M < 0 || N < 0 || K < 0 || M > limit || N > limit || K > limit) return GPD_ERR_SHAPE;
    if (M == 0 || N == 0) return GPD_OK;               // empty buffers may have no address
    if (!out_dev) return GPD_ERR_ARG;
    if (ldd < N) return GPD_ERR_SHAPE;
    cudaStream_t st = as_stream(stream);
    if (K == 0) {
        if (accumulate) return GPD_OK;
        const int e = lm::dtype_size(out_type);
        return cuda_ok(cudaMemset2DAsync(out_dev, (size_t)(ldd * e), 0, (size_t)(N * e), (size_t)M, st));
    }
    if (!A_dev || !B_dev || !a_scales_dev || !b_scales_dev) return GPD_ERR_ARG;
    const int64_t kb = (K + BK - 1) / BK;
    if (lda < K || ldb < K || ldsa < kb || ldsb < kb) return GPD_ERR_SHAPE;
    if (!lm::aligned(A_dev, 16) || !lm::aligned(B_dev, 16) || lda % 16 || ldb % 16) return GPD_ERR_ARG;
    auto scale_rows = [&](const uint8_t* p, int64_t ld, int64_t rows, int br) {
        return ScaleRows{p, ld, rows, br == 1 ? 0 : 7, lm::aligned(p, 4) && ld % 4 == 0};
    };
    const Operand a{A_dev, lda, M, a_type, scale_rows(a_scales_dev, ldsa, M, a_block_rows)};
    const Operand b{B_dev, ldb, N, b_type, scale_rows(b_scales_dev, ldsb, N, b_block_rows)};
    Fp8Params prm{};
    prm.out = out_dev;
    prm.ldd = ldd;
    prm.kb = (int)kb;
    prm.accumulate = accumulate != 0;
    if (out_type == GPD_DT_F32) return launch_type<float>(a, b, prm, K, st);
    if (out_type == GPD_DT_BF16) return launch_type<__nv_bfloat16>(a, b, prm, K, st);
    return launch_type<__half>(a, b, prm, K, st);
}
