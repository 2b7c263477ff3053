// Second factor of low-rank adapters: out[t] = base[t] + scale_i W_i h[t] for the rows of every segment, i its adapter.
//
// Bound by reading base and writing out (many rows) or by reading the adapters (one row per segment).  h is FP32 and goes
// through the tensor cores as a sum of 16-bit numbers, its parts: three, which hold all of it, or two of FP16 for FP16 results,
// which lose 2^-23.  FP16 parts are taken of a row over a power of two, so that h may be of any size.  A warp has its 16 rows of
// h as operands in registers, and W comes in chunks of columns through a ring of asynchronous copies; base is read a chunk
// ahead.  The tensor cores leave a lane two neighbouring columns of a tile of eight: the four lanes of a row exchange words, so
// that each reads and writes eight columns, 16 bytes, of it.
//
// Measured (BF16, many rows, base read and out written; the first product is not in these times): 16384 x 8192, rank 32, 104 us
// of 83 at the copy bandwidth (tensor pipe 54 %, DRAM 60 %); 4001 x 6144, rank 64, 40 us cold (tensor pipe 53 %; 33 with two parts):
// the products of three parts, the reads and writes of a tile in shared memory and the copies take turns in a warp.
#include <algorithm>
#include <type_traits>

#include "adapter_rows.h"

namespace gpd {
namespace adapter {

namespace {

constexpr int kThreads = 128, kCols = 64;              // columns of a warp and chunk

template <int KT, int WM, bool TRANS>
struct Shape {
    static constexpr int TM = 16 * WM, RP = 16 * KT, COLS = WM == 4 ? kCols : 4 * kCols, STAGES = WM == 1 && KT >= 4 ? 2 : 3;
    static constexpr int W_ROWS = TRANS ? RP : COLS, W_COLS = TRANS ? COLS : RP, W_PITCH = 2 * W_COLS + 16;
    static constexpr int STAGE = W_ROWS * W_PITCH, SMEM = STAGES * STAGE;
};

// WM = 4: a warp has 16 rows of the tile and all columns.  WM = 1: all warps have the same 16 rows, 64 columns each.
template <typename T, typename O, int KT, int PARTS, int WM, bool TRANS>
__global__ void __launch_bounds__(kThreads) expand_kernel(const __grid_constant__ ExpandArgs a) {
    using S = Shape<KT, WM, TRANS>;
    extern __shared__ __align__(128) unsigned char smem[];
    after_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2;
    const RowTile tile = find_tile<S::TM>(a.seg, (int)blockIdx.x);
    if (tile.rows == 0) return;
    const bool none = tile.id < 0 || tile.id >= a.seg.n;
    if (tile.id < 0 && a.base == a.out) return;
    const T* w = none ? nullptr : static_cast<const T*>(a.w) + (int64_t)tile.id * a.next;
    const int64_t chunks = (a.C + S::COLS - 1) / S::COLS;
    const int64_t from = chunks * blockIdx.y / gridDim.y, to = chunks * (blockIdx.y + 1) / gridDim.y;
    const uint32_t ring = smem_at(smem);
    auto fetch = [&](int64_t k) {
        if (k < to && !none) {
            const uint32_t at = ring + (uint32_t)((k - from) % S::STAGES) * S::STAGE;
            const int64_t c = k * S::COLS;
            if (TRANS) stage_tile<T, S::W_ROWS, S::W_COLS, kThreads>(at, S::W_PITCH, w + c, a.ldw, a.r, a.C - c, a.w_vec);
            else stage_tile<T, S::W_ROWS, S::W_COLS, kThreads>(at, S::W_PITCH, w + c * a.ldw, a.ldw, a.C - c, a.r, a.w_vec);
        }
        copies_end();
    };
    for (int i = 0; i < S::STAGES - 1; ++i) fetch(from + i);

    // the warp's rows of h, as parts
    const int row0 = (WM == 4 ? 16 * warp : 0) + g;
    const bool has[2] = {row0 < tile.rows, row0 + 8 < tile.rows};
    uint32_t ha[PARTS][KT][4];
    float undo[2];
    load_parts<T, KT, PARTS>(a.h + (int64_t)(tile.row + row0) * a.r, none ? 0 : a.r, none || !a.scale ? 1.f : a.scale[tile.id], has, ha, undo);
    const O* base = a.base ? static_cast<const O*>(a.base) + (int64_t)(tile.row + row0) * a.ldb : nullptr;
    O* out = static_cast<O*>(a.out) + (int64_t)(tile.row + row0) * a.ldo;

    Share<O> next;
    auto load_base = [&](int64_t k, Share<O>& s) {
        const int64_t c = k * S::COLS + (WM == 1 ? kCols * warp : 0);
        load_share<O>(s, base ? base + c : nullptr, a.ldb, has, k < to ? (int)min((int64_t)kCols, a.C - c) : 0, a.io_vec);
    };
    load_base(from, next);
    const float nan = __int_as_float(0x7fffffff);
    for (int64_t k = from; k < to; ++k) {
        copies_wait<S::STAGES - 2>();
        __syncthreads();
        fetch(k + S::STAGES - 1);
        const uint32_t ws = ring + (uint32_t)((k - from) % S::STAGES) * S::STAGE;
        const Share<O> share = next;
        load_base(k + 1, next);
        const int wc = WM == 1 ? kCols * warp : 0;     // the warp's first column in the chunk
        float acc[8][4];
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[n][i] = tile.id >= a.seg.n ? nan : 0.f;
        if (!none) {
#pragma unroll
            for (int s = 0; s < KT; ++s)
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    uint32_t b[4];
                    if (TRANS) ldmatrix4<true>(b, ws + (16 * s + (lane & 15)) * S::W_PITCH + 2 * (wc + 16 * p + (lane >> 4) * 8));
                    else ldmatrix4<false>(b, ws + (wc + 16 * p + (lane & 7) + (lane >> 4) * 8) * S::W_PITCH + 2 * (16 * s + (lane >> 3 & 1) * 8));
#pragma unroll
                    for (int i = PARTS - 1; i >= 0; --i) {             // the small parts first
                        mma(acc[2 * p], ha[i][s], b[0], b[1], T());
                        mma(acc[2 * p + 1], ha[i][s], b[2], b[3], T());
                    }
                }
            if (std::is_same<T, __half>::value) {
#pragma unroll
                for (int n = 0; n < 8; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[n][i] *= undo[i >> 1];
            }
        }
        const int64_t c = k * S::COLS + wc;
        store_sum<O>(share, acc, out + c, a.ldo, has, (int)min((int64_t)kCols, a.C - c), a.io_vec, true);
    }
    copies_wait<0>();
}

template <typename T, typename O, int KT, int PARTS, int WM, bool TRANS>
gpd_status launch(const ExpandArgs& a, cudaStream_t st) {
    using S = Shape<KT, WM, TRANS>;
    const int64_t tiles = tiles_of(a.seg, S::TM), chunks = (a.C + S::COLS - 1) / S::COLS;
    if (tiles > 0x7fffffff) return GPD_ERR_SHAPE;
    // about eight CTAs per SM: a CTA loads its rows of h once, so that fewer and longer ones would gain little
    int64_t splits = (8 * sm_count() + tiles - 1) / tiles;
    splits = std::max<int64_t>(1, std::min({splits, chunks, (int64_t)65535}));
    auto kernel = expand_kernel<T, O, KT, PARTS, WM, TRANS>;
    if (S::SMEM > 49152 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) != cudaSuccess) return GPD_ERR_CUDA;
    return launch_after(kernel, dim3((unsigned)tiles, (unsigned)splits), dim3(kThreads), S::SMEM, 1, st, a);
}
// ---- the same with tiles by TMA: many rows, base and out on 16-byte boundaries ---------------------------------
// Tiles of base arrive in shared memory, a lane adds its products to its elements there, and a warp's 16 rows leave from
// there: as one copy if all of them are the segment's, row by row where it ends among them.  A stage is handed back one step
// late, when its copy has left and every load from it has long had its data: a warp ends every step with a group of copies,
// an empty one where it has none, so that all but the newest group are those of the steps before.
__device__ int g_expand_status = 0;                    // GPD_ERR_TIMEOUT if a bounded wait expired

template <typename O, int KT, bool TRANS>
struct TmaShape {
    static constexpr int TM = 64, RP = 16 * KT, STAGES = KT == 8 && sizeof(O) == 4 ? 3 : 4;
    static constexpr int BOX = 128 / sizeof(O), BOXES = kCols / BOX;   // columns of a box of 128 bytes
    using W = WTile<TRANS ? RP : kCols, TRANS ? kCols : RP>;
    static constexpr int BASE = TM * 128 * BOXES, STAGE = BASE + W::BYTES, SMEM = STAGES * STAGE + 1024;
};
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t from, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(from), "r"(c0), "r"(c1), "r"(c2) : "memory");
}

// The CTAs share out the (tile, chunk of columns) pairs in contiguous runs of equal length.  Four warps have 16 rows of a tile
// each, one issues the copies.
template <typename T, typename O, int KT, int PARTS, bool TRANS>
__global__ void __launch_bounds__(kThreads + 32, per_sm(TmaShape<O, KT, TRANS>::SMEM))
expand_tma_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_base, const __grid_constant__ CUtensorMap map_out,
                  const __grid_constant__ ExpandArgs a) {
    using S = TmaShape<O, KT, TRANS>;
    extern __shared__ unsigned char raw[];
    __shared__ Ring<S::STAGES> ring;
    unsigned char* smem = raw + (1024 - (smem_at(raw) & 1023)) % 1024;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) ring.init(a.w_vec ? 1 : 33, 4);
    if (!a.w_vec) {                                    // columns and rows of W that do not exist
        for (int i = threadIdx.x; i < S::STAGES * S::STAGE / 16; i += kThreads + 32) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    // The kernel before this one is the same call's: it began its work, and let this one start, when all before it had
    // completed.  It is the first product, which writes h alone, or that of the factors' gradients, which writes dA and dB, and these
    // overlap nothing else of the call.  So only the warps that read h wait for it; segments, W and base are there.
    bool waited = warp == kThreads / 32;
    const int64_t chunks = (a.C + kCols - 1) / kCols, all = count_tiles<S::TM>(a.seg) * chunks;
    const int64_t last = all * (blockIdx.x + 1) / gridDim.x;
    int k = 0;                                         // stages so far
    for (int64_t at = all * blockIdx.x / gridDim.x, end; at < last; at = end) {
        const int number = (int)(at / chunks);
        end = min(last, (int64_t)(number + 1) * chunks);
        const int first = (int)(at - (int64_t)number * chunks), n = (int)(end - at);
        const RowTile tile = find_tile<S::TM>(a.seg, number);
        const bool none = tile.id < 0 || tile.id >= a.seg.n;
        if (tile.id < 0 && a.base == a.out) continue;
        if (warp == kThreads / 32) {
            const uint32_t bytes = (a.base ? S::BASE : 0) + (none || !a.w_vec ? 0 : S::W::BYTES);
            for (int i = 0; i < n; ++i, ++k) {
                if (!ring.wait_empty(k, &g_expand_status)) break;
                unsigned char *stage = smem + k % S::STAGES * S::STAGE, *ws = stage + S::BASE;
                const int c = (first + i) * kCols;
                uint64_t* bar = &ring.full[k % S::STAGES];
                if (lane == 0) {
                    if (bytes) tc::mbar_expect_tx(bar, bytes);
                    else tc::mbar_arrive(bar);
                    if (a.base)
#pragma unroll
                        for (int j = 0; j < S::BOXES; ++j) tc::tma_load_3d(stage + j * S::TM * 128, &map_base, c + j * S::BOX, (int)tile.row, 0, bar);
                    if (!none && a.w_vec) S::W::load(ws, &map_w, TRANS ? c : 0, TRANS ? 0 : c, (int)tile.id, bar);
                }
                if (!a.w_vec) {
                    if (!none) {
                        const T* w = static_cast<const T*>(a.w) + (int64_t)tile.id * a.next + (TRANS ? c : c * a.ldw);
                        if (TRANS) S::W::template copy<false>(ws, w, a.ldw, a.r, a.C - c, a.r);
                        else S::W::template copy<true>(ws, w, a.ldw, a.C - c, a.r, a.r);
                    }
                    tc::mbar_arrive(bar);
                }
            }
            __syncwarp();
            if (*static_cast<volatile int*>(&ring.abort)) break;
            continue;
        }
        const int g = lane >> 2, q = lane & 3, row0 = 16 * warp + g;
        const bool has[2] = {row0 < tile.rows, row0 + 8 < tile.rows}, whole = 16 * warp + 16 <= tile.rows, any = 16 * warp < tile.rows;
        uint32_t ha[PARTS][KT][4];
        float undo[2];
        if (!waited) after_previous();
        waited = true;
        load_parts<T, KT, PARTS>(a.h + (int64_t)(tile.row + row0) * a.r, none ? 0 : a.r, none || !a.scale ? 1.f : a.scale[tile.id], has, ha, undo);
        for (int i = 0; i < n; ++i, ++k) {
            if (!ring.wait_full(k, &g_expand_status)) break;
            const uint32_t stage = smem_at(smem) + k % S::STAGES * S::STAGE, mine = stage + 16 * warp * 128;
            const uint32_t ws = TRANS ? S::W::lane_at(stage + S::BASE, row_first(), row_first_col())
                                      : S::W::lane_at(stage + S::BASE, col_first_row(), col_first());
            const uint32_t block0 = WTile<S::TM, kCols>::lane_at(mine, row_first(), row_first_col());
            if (any) {
                // the sums begin with base where the result has 16 bits: their chain's steps lose at most 2^-22 of it each, the
                // rounding 2^-8 (adding it behind the chain: 4001 x 4096 -> 6144, rank 64, 58.7 us for both products, so 55.9)
                constexpr bool kOnBase = sizeof(O) == 2 && std::is_same<T, __nv_bfloat16>::value;
#pragma unroll
                for (int half = 0; half < 2; ++half) { // 32 columns: four chains of additions side by side
                    float acc[2][2][4];                // [16 columns][8 columns][row g: 2 q, 2 q + 1; row g + 8]
                    uint32_t b16[2][4];
                    auto block = [&](int i) { return WTile<S::TM, kCols>::on(block0, 0, 32 * half + 16 * i); };
                    if (sizeof(O) == 2) {
#pragma unroll
                        for (int i2 = 0; i2 < 2; ++i2) {
                            b16[i2][0] = b16[i2][1] = b16[i2][2] = b16[i2][3] = 0;
                            if (a.base) ldmatrix4<false>(b16[i2], block(i2));
                        }
                    }
#pragma unroll
                    for (int i2 = 0; i2 < 2; ++i2)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float2 f = make_float2(0.f, 0.f);
                            if (kOnBase) f = unpack2(b16[i2][j], T());
                            acc[i2][j >> 1][2 * (j & 1)] = f.x;
                            acc[i2][j >> 1][2 * (j & 1) + 1] = f.y;
                        }
                    if (!none) {
#pragma unroll
                        for (int s = 0; s < KT; ++s) {
                            uint32_t b[2][4];
#pragma unroll
                            for (int i2 = 0; i2 < 2; ++i2) {
                                if (TRANS) ldmatrix4<true>(b[i2], S::W::on(ws, 16 * s, 32 * half + 16 * i2));
                                else ldmatrix4<false>(b[i2], S::W::on(ws, 32 * half + 16 * i2, 16 * s));
                            }
#pragma unroll
                            for (int j = PARTS - 1; j >= 0; --j)       // the small parts first
#pragma unroll
                                for (int i2 = 0; i2 < 2; ++i2) {
                                    mma(acc[i2][0], ha[j][s], b[i2][0], b[i2][1], T());
                                    mma(acc[i2][1], ha[j][s], b[i2][2], b[i2][3], T());
                                }
                        }
                    } else if (tile.id >= 0) {         // there is no such adapter
#pragma unroll
                        for (int i2 = 0; i2 < 8; ++i2)
#pragma unroll
                            for (int j = 0; j < 2; ++j) acc[i2 >> 2][j][i2 & 3] = __int_as_float(0x7fffffff);
                    }
#pragma unroll
                    for (int i2 = 0; i2 < 2; ++i2) {
                        if constexpr (sizeof(O) == 2) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                float x = acc[i2][j >> 1][2 * (j & 1)], y = acc[i2][j >> 1][2 * (j & 1) + 1];
                                if (!kOnBase) {
                                    const float2 f = unpack2(b16[i2][j], O());
                                    x = fmaf(x, undo[j & 1], f.x);
                                    y = fmaf(y, undo[j & 1], f.y);
                                }
                                b16[i2][j] = pack2(x, y, O());
                            }
                            stmatrix4(b16[i2], block(i2));
                        } else {
#pragma unroll
                            for (int n2 = 0; n2 < 2; ++n2)
#pragma unroll
                                for (int j = 0; j < 2; ++j) {          // row g + 8 j, columns c and c + 1
                                    const int c = 32 * half + 16 * i2 + 8 * n2 + 2 * q;
                                    const uint32_t to = mine + c / S::BOX * S::TM * 128 + swizzled<128>((g + 8 * j) * 128 + c % S::BOX * 4);
                                    float x = 0.f, y = 0.f;
                                    if (a.base) asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(x), "=f"(y) : "r"(to) : "memory");
                                    x = fmaf(acc[i2][n2][2 * j], undo[j], x);
                                    y = fmaf(acc[i2][n2][2 * j + 1], undo[j], y);
                                    asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(x), "f"(y) : "memory");
                                }
                        }
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                const int64_t c0 = (int64_t)(first + i) * kCols;
                if (whole) {
                    if (lane == 0) {
#pragma unroll
                        for (int j = 0; j < S::BOXES; ++j)
                            if (c0 + j * S::BOX < a.C) tma_store_3d(&map_out, mine + j * S::TM * 128, (int)c0 + j * S::BOX, (int)tile.row + 16 * warp, 0);
                    }
                } else {
#pragma unroll
                    for (int b = 0; b < S::BOXES; ++b)
                        for (int j = lane; j < 128; j += 32) {         // a row's pieces of 16 bytes
                            const int r = j >> 3;
                            const int64_t c = c0 + b * S::BOX + (j & 7) * (16 / (int)sizeof(O));
                            if (16 * warp + r >= tile.rows || c >= a.C) continue;
                            uint4 v;
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                                         : "r"(mine + b * S::TM * 128 + swizzled<128>(r * 128 + (j & 7) * 16)) : "memory");
                            O* p = static_cast<O*>(a.out) + (int64_t)(tile.row + 16 * warp + r) * a.ldo + c;
                            if (c + 16 / (int)sizeof(O) <= a.C) {
                                *reinterpret_cast<uint4*>(p) = v;
                            } else {
                                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                                for (int e = 0; e < 16 / (int)sizeof(O); ++e)
                                    if (c + e < a.C) {
                                        if constexpr (sizeof(O) == 4) p[e] = __uint_as_float(w[e]);
                                        else reinterpret_cast<unsigned short*>(p)[e] = (unsigned short)(w[e / 2] >> (16 * (e & 1)));
                                    }
                            }
                        }
                }
            }
            // the stage before this one is free once its copy has left; this step's group, empty or not, may be under way
            if (lane == 0) {
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
            }
            __syncwarp();
            if (lane == 0 && k > 0) tc::mbar_arrive(&ring.empty[(k - 1) % S::STAGES]);
        }
        if (*static_cast<volatile int*>(&ring.abort)) break;
    }
    if (!waited) after_previous();                     // nothing to do here: what comes next still follows h
    if (warp == kThreads / 32) {
        if (lane == 0) ring.drain(k, &g_expand_status);
    } else if (lane == 0) {
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
}

template <typename T, typename O, int KT, int PARTS, bool TRANS>
gpd_status launch_tma(const ExpandArgs& a, cudaStream_t st) {
    using S = TmaShape<O, KT, TRANS>;
    const int64_t tiles = tiles_of(a.seg, S::TM), chunks = (a.C + kCols - 1) / kCols;
    const int64_t ctas = std::min<int64_t>(tiles * chunks, (int64_t)per_sm(S::SMEM) * sm_count());
    CUtensorMap map_w, map_base, map_out;
    if (!make_map(&map_out, a.out, sizeof(O), 1, a.seg.T, a.C, a.ldo, 0, 16, S::BOX)) return GPD_ERR_CUDA;
    map_w = map_base = map_out;                        // where they are not used
    if (a.base && !make_map(&map_base, a.base, sizeof(O), 1, a.seg.T, a.C, a.ldb, 0, S::TM, S::BOX)) return GPD_ERR_CUDA;
    if (a.w_vec && a.seg.n > 0) {
        const bool ok = TRANS ? make_map(&map_w, a.w, 2, a.seg.n, a.r, a.C, a.ldw, a.next, S::RP, kCols)
                              : make_map(&map_w, a.w, 2, a.seg.n, a.C, a.r, a.ldw, a.next, kCols, S::W::PITCH / 2);
        if (!ok) return GPD_ERR_CUDA;
    }
    auto kernel = expand_tma_kernel<T, O, KT, PARTS, TRANS>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) != cudaSuccess) return GPD_ERR_CUDA;
    return launch_after(kernel, dim3((unsigned)ctas), dim3(kThreads + 32), S::SMEM, 1, st, map_w, map_base, map_out, a);
}
template <typename T, typename O, int KT, bool TRANS>
gpd_status launch_rows(const ExpandArgs& a, cudaStream_t st) {
    constexpr int PARTS = kParts<T, O>;
    if (a.seg.T <= 16 * (int64_t)a.seg.S) return launch<T, O, KT, PARTS, 1, TRANS>(a, st);
    return a.tma ? launch_tma<T, O, KT, PARTS, TRANS>(a, st) : launch<T, O, KT, PARTS, 4, TRANS>(a, st);
}
template <typename T, typename O, bool TRANS>
gpd_status launch_rank(const ExpandArgs& a, cudaStream_t st) {
    if (a.r <= 16) return launch_rows<T, O, 1, TRANS>(a, st);
    if (a.r <= 32) return launch_rows<T, O, 2, TRANS>(a, st);
    return a.r <= 64 ? launch_rows<T, O, 4, TRANS>(a, st) : launch_rows<T, O, 8, TRANS>(a, st);
}
template <typename T>
gpd_status launch_type(int out_type, bool transposed, const ExpandArgs& a, cudaStream_t st) {
    if (out_type == GPD_DT_F32) return transposed ? launch_rank<T, float, true>(a, st) : launch_rank<T, float, false>(a, st);
    return transposed ? launch_rank<T, T, true>(a, st) : launch_rank<T, T, false>(a, st);
}

}  // namespace

int expand_status_fetch_and_clear() {
    int v = 0, zero = 0;
    if (cudaMemcpyFromSymbol(&v, g_expand_status, sizeof(int)) != cudaSuccess) return (int)GPD_ERR_CUDA;
    if (v != 0) cudaMemcpyToSymbol(g_expand_status, &zero, sizeof(int));
    return v;
}

gpd_status expand(int type, int out_type, bool transposed, const ExpandArgs& a, cudaStream_t st) {
    return type == GPD_DT_BF16 ? launch_type<__nv_bfloat16>(out_type, transposed, a, st) : launch_type<__half>(out_type, transposed, a, st);
}

}  // namespace adapter
}  // namespace gpd
