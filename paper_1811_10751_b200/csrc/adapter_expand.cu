// Second factor of low-rank adapters: out[t] = base[t] + scale_i W_i h[t] for the rows of every segment, i its adapter.
//
// Bound by reading base and writing out (many rows) or by reading the adapters (one row per segment).  h is FP32 and goes
// through the tensor cores as a sum of two or three 16-bit numbers, its parts: two lose 2^-17 (BF16) or 2^-22 (FP16) of
// it, far below the rounding of a 16-bit result; FP32 results of BF16 adapters take three.  FP16 parts are taken of a row
// over a power of two, so that h may be of any size.  A warp has its 16 rows of h as operands in registers, and W comes in chunks
// of columns through a ring of asynchronous copies; base is read a chunk ahead.  The tensor cores leave a lane two
// neighbouring columns of a tile of eight: the four lanes of a row exchange words, so that each reads and writes eight
// columns, 16 bytes, of it.
#include <algorithm>
#include <type_traits>

#include "adapter_common.h"

namespace gpd {
namespace adapter {

namespace {

constexpr int kThreads = 128, kCols = 64;              // columns of a warp and chunk

template <int KT, int WM, bool TRANS>
struct Shape {
    static constexpr int TM = 16 * WM, RP = 16 * KT, COLS = WM == 4 ? kCols : 4 * kCols, STAGES = WM == 1 && KT == 8 ? 2 : 3;
    static constexpr int W_ROWS = TRANS ? RP : COLS, W_COLS = TRANS ? COLS : RP, W_PITCH = 2 * W_COLS + 16;
    static constexpr int STAGE = W_ROWS * W_PITCH, SMEM = STAGES * STAGE;
};

// Word j of lane t of four becomes word t of lane j.
__device__ __forceinline__ void transpose4(uint32_t (&w)[4]) {
    const int lane = threadIdx.x & 31;
    const bool odd = lane & 1, high = lane & 2;
    uint32_t r0 = __shfl_xor_sync(0xffffffffu, odd ? w[0] : w[1], 1), r1 = __shfl_xor_sync(0xffffffffu, odd ? w[2] : w[3], 1);
    if (odd) {
        w[0] = r0;
        w[2] = r1;
    } else {
        w[1] = r0;
        w[3] = r1;
    }
    r0 = __shfl_xor_sync(0xffffffffu, high ? w[0] : w[2], 2);
    r1 = __shfl_xor_sync(0xffffffffu, high ? w[1] : w[3], 2);
    if (high) {
        w[0] = r0;
        w[1] = r1;
    } else {
        w[2] = r0;
        w[3] = r1;
    }
}

// A thread's share of base in a chunk, as it is in memory
template <typename O> struct Share { uint4 v[2][2]; };                 // [32 columns][row g, g + 8]: eight elements
template <> struct Share<float> { float2 v[8][2]; };                   // [8 columns][row]: two elements

// WM = 4: a warp has 16 rows of the tile and all columns.  WM = 1: all warps have the same 16 rows, 64 columns each.
template <typename T, typename O, int KT, int PARTS, int WM, bool TRANS>
__global__ void __launch_bounds__(kThreads) expand_kernel(const __grid_constant__ ExpandArgs a) {
    using S = Shape<KT, WM, TRANS>;
    extern __shared__ __align__(128) unsigned char smem[];
    after_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
    const RowTile tile = find_tile<S::TM>(a.seg, blockIdx.x);
    if (tile.rows == 0) return;
    const bool none = tile.id < 0 || tile.id >= a.seg.n;
    if (tile.id < 0 && a.base == a.out) return;
    const T* w = none ? nullptr : static_cast<const T*>(a.w) + tile.id * a.next;
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
    float undo[2] = {1.f, 1.f};
    {
        float v[KT][2][4];                             // [16 columns][row][2 q, 2 q + 1, 2 q + 8, 2 q + 9]
        const float scale = none || !a.scale ? 1.f : a.scale[tile.id];
        float most[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float* h = a.h + (tile.row + row0 + 8 * i) * a.r;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = 16 * k + 2 * q + (j & 1) + (j >> 1) * 8;
                    v[k][i][j] = !none && has[i] && c < a.r ? h[c] * scale : 0.f;
                    most[i] = fmaxf(most[i], fabsf(v[k][i][j]));
                }
            }
        if (sizeof(T) == 2 && std::is_same<T, __half>::value) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                most[i] = fmaxf(most[i], __shfl_xor_sync(0xffffffffu, most[i], 1));
                most[i] = fmaxf(most[i], __shfl_xor_sync(0xffffffffu, most[i], 2));
                const int e = exponent_of(most[i]);
                undo[i] = power2(e);
                const float by = power2(-e);
#pragma unroll
                for (int k = 0; k < KT; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[k][i][j] *= by;
            }
        }
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int f = 0; f < 4; ++f) {              // rows g, g + 8, then the same eight columns on
                uint32_t parts[PARTS];
                split2<T, PARTS>(v[k][f & 1][2 * (f >> 1)], v[k][f & 1][2 * (f >> 1) + 1], parts);
#pragma unroll
                for (int p = 0; p < PARTS; ++p) ha[p][k][f] = parts[p];
            }
    }
    const O* base = a.base ? static_cast<const O*>(a.base) + (tile.row + row0) * a.ldb : nullptr;
    O* out = static_cast<O*>(a.out) + (tile.row + row0) * a.ldo;

    Share<O> next;
    auto load_base = [&](int64_t k, Share<O>& s) {
        const int64_t c0 = k * S::COLS + (WM == 1 ? kCols * warp : 0);
        if constexpr (sizeof(O) == 4) {
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int64_t c = c0 + 8 * n + 2 * q;
                    s.v[n][i] = make_float2(0.f, 0.f);
                    if (!base || !has[i] || k >= to || c >= a.C) continue;
                    const float* p = base + 8 * i * a.ldb + c;
                    if (a.io_vec && c + 2 <= a.C) s.v[n][i] = *reinterpret_cast<const float2*>(p);
                    else s.v[n][i] = make_float2(p[0], c + 1 < a.C ? p[1] : 0.f);
                }
        } else {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int64_t c = c0 + 32 * n + 8 * q;
                    s.v[n][i] = make_uint4(0, 0, 0, 0);
                    if (!base || !has[i] || k >= to || c >= a.C) continue;
                    const O* p = base + 8 * i * a.ldb + c;
                    s.v[n][i] = a.io_vec ? load8<O, true>(p, (int)min((int64_t)8, a.C - c)).v : load8<O, false>(p, (int)min((int64_t)8, a.C - c)).v;
                }
        }
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
        const int64_t c0 = k * S::COLS + wc;
        if constexpr (sizeof(O) == 4) {
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int64_t c = c0 + 8 * n + 2 * q;
                    if (!has[i] || c >= a.C) continue;
                    float* p = out + 8 * i * a.ldo + c;
                    const float2 v = make_float2(share.v[n][i].x + acc[n][2 * i], share.v[n][i].y + acc[n][2 * i + 1]);
                    if (a.io_vec && c + 2 <= a.C) {
                        *reinterpret_cast<float2*>(p) = v;
                    } else {
                        p[0] = v.x;
                        if (c + 1 < a.C) p[1] = v.y;
                    }
                }
        } else {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t b[4] = {share.v[n][i].x, share.v[n][i].y, share.v[n][i].z, share.v[n][i].w};
                    transpose4(b);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 f = unpack2(b[j], O());
                        b[j] = pack2(f.x + acc[4 * n + j][2 * i], f.y + acc[4 * n + j][2 * i + 1], O());
                    }
                    transpose4(b);
                    const int64_t c = c0 + 32 * n + 8 * q;
                    if (!has[i] || c >= a.C) continue;
                    O* p = out + 8 * i * a.ldo + c;
                    if (a.io_vec && c + 8 <= a.C) {
                        *reinterpret_cast<uint4*>(p) = make_uint4(b[0], b[1], b[2], b[3]);
                    } else {
                        unsigned short* s = reinterpret_cast<unsigned short*>(p);
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (c + j < a.C) s[j] = (unsigned short)(b[j / 2] >> (16 * (j & 1)));
                    }
                }
        }
    }
    copies_wait<0>();
}

template <typename T, typename O, int KT, int PARTS, int WM, bool TRANS>
gpd_status launch(const ExpandArgs& a, cudaStream_t st) {
    using S = Shape<KT, WM, TRANS>;
    const int64_t tiles = tiles_of(a.seg, S::TM), chunks = (a.C + S::COLS - 1) / S::COLS;
    if (tiles > 0x7fffffff) return GPD_ERR_SHAPE;
    // eight CTAs per SM, of eight chunks at least where there are enough of them
    int64_t splits = (8 * sm_count() + tiles - 1) / tiles;
    splits = std::max<int64_t>(1, std::min({splits, chunks, (int64_t)65535}));
    auto kernel = expand_kernel<T, O, KT, PARTS, WM, TRANS>;
    if (S::SMEM > 49152 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) != cudaSuccess) return GPD_ERR_CUDA;
    return launch_after(kernel, dim3((unsigned)tiles, (unsigned)splits), dim3(kThreads), S::SMEM, 1, st, a);
}
template <typename T, typename O, int KT, bool TRANS>
gpd_status launch_rows(const ExpandArgs& a, cudaStream_t st) {
    constexpr int PARTS = sizeof(O) == 4 && std::is_same<T, __nv_bfloat16>::value ? 3 : 2;
    return a.seg.T <= 16 * (int64_t)a.seg.S ? launch<T, O, KT, PARTS, 1, TRANS>(a, st) : launch<T, O, KT, PARTS, 4, TRANS>(a, st);
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

gpd_status expand(int type, int out_type, bool transposed, const ExpandArgs& a, cudaStream_t st) {
    return type == GPD_DT_BF16 ? launch_type<__nv_bfloat16>(out_type, transposed, a, st) : launch_type<__half>(out_type, transposed, a, st);
}

}  // namespace adapter
}  // namespace gpd
