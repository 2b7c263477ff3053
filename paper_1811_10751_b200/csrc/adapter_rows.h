// Pieces that the kernels of adapters' second product share: rows of h as operands, and reading base and writing out where
// a lane holds two neighbouring columns of a tile of eight.
#pragma once

#include <type_traits>

#include "adapter_common.h"

namespace gpd {
namespace adapter {

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

// A thread's share of base in 64 columns, as it is in memory: of rows g and g + 8
template <typename O> struct Share { uint4 v[2][2]; };                 // [32 columns][row]: eight elements
template <> struct Share<float> { float2 v[8][2]; };                   // [8 columns][row]: two elements
// base: row g, from column c0 - of which `cols` exist (<= 0: none); null: zeros.  vec: 16-byte (FP32: 8-byte) boundaries.
template <typename O>
__device__ __forceinline__ void load_share(Share<O>& s, const O* base, int64_t ld, const bool (&has)[2], int cols, bool vec) {
    const int q = threadIdx.x & 3;
    if constexpr (sizeof(O) == 4) {
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int c = 8 * n + 2 * q;
                s.v[n][i] = make_float2(0.f, 0.f);
                if (!base || !has[i] || c >= cols) continue;
                const float* p = base + 8 * i * ld + c;
                if (vec && c + 2 <= cols) s.v[n][i] = *reinterpret_cast<const float2*>(p);
                else s.v[n][i] = make_float2(p[0], c + 1 < cols ? p[1] : 0.f);
            }
    } else {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int c = 32 * n + 8 * q;
                s.v[n][i] = make_uint4(0, 0, 0, 0);
                if (!base || !has[i] || c >= cols) continue;
                const O* p = base + 8 * i * ld + c;
                s.v[n][i] = vec ? load8<O, true>(p, cols - c).v : load8<O, false>(p, cols - c).v;
            }
    }
}
// out = share + acc, acc[n]: columns 8 n + 2 q and the next of row g, and of row g + 8 (`both`: any lane has one).  All lanes
// call it.
template <typename O>
__device__ __forceinline__ void store_sum(const Share<O>& s, const float (&acc)[8][4], O* out, int64_t ld, const bool (&has)[2], int cols, bool vec,
                                          bool both) {
    const int q = threadIdx.x & 3;
    if constexpr (sizeof(O) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (i == 1 && !both) break;
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                const int c = 8 * n + 2 * q;
                if (!has[i] || c >= cols) continue;
                float* p = out + 8 * i * ld + c;
                const float2 v = make_float2(s.v[n][i].x + acc[n][2 * i], s.v[n][i].y + acc[n][2 * i + 1]);
                if (vec && c + 2 <= cols) {
                    *reinterpret_cast<float2*>(p) = v;
                } else {
                    p[0] = v.x;
                    if (c + 1 < cols) p[1] = v.y;
                }
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (i == 1 && !both) break;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                uint32_t b[4] = {s.v[n][i].x, s.v[n][i].y, s.v[n][i].z, s.v[n][i].w};
                transpose4(b);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 f = unpack2(b[j], O());
                    b[j] = pack2(f.x + acc[4 * n + j][2 * i], f.y + acc[4 * n + j][2 * i + 1], O());
                }
                transpose4(b);
                const int c = 32 * n + 8 * q;
                if (!has[i] || c >= cols) continue;
                O* p = out + 8 * i * ld + c;
                if (vec && c + 8 <= cols) {
                    *reinterpret_cast<uint4*>(p) = make_uint4(b[0], b[1], b[2], b[3]);
                } else {
                    unsigned short* to = reinterpret_cast<unsigned short*>(p);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (c + j < cols) to[j] = (unsigned short)(b[j / 2] >> (16 * (j & 1)));
                }
            }
        }
    }
}

// The warp's rows of h (those that there are) times scale, as operands of the tensor cores; undo[i]: what FP16 parts of
// row g + 8 i have to be multiplied with.
template <typename T, int KT, int PARTS>
__device__ __forceinline__ void load_parts(const float* h, int r, float scale, const bool (&has)[2], uint32_t (&ha)[PARTS][KT][4], float (&undo)[2]) {
    const int q = threadIdx.x & 3;
    float v[KT][2][4];                                 // [16 columns][row][2 q, 2 q + 1, 2 q + 8, 2 q + 9]
    float most[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KT; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = 16 * k + 2 * q + (j & 1) + (j >> 1) * 8;
                v[k][i][j] = has[i] && c < r ? h[(int64_t)8 * i * r + c] * scale : 0.f;
                most[i] = fmaxf(most[i], fabsf(v[k][i][j]));
            }
    undo[0] = undo[1] = 1.f;
    if (std::is_same<T, __half>::value) {
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
        for (int f = 0; f < 4; ++f) {                  // rows g, g + 8, then the same eight columns on
            uint32_t parts[PARTS];
            split2<T, PARTS>(v[k][f & 1][2 * (f >> 1)], v[k][f & 1][2 * (f >> 1) + 1], parts);
#pragma unroll
            for (int p = 0; p < PARTS; ++p) ha[p][k][f] = parts[p];
        }
}

}  // namespace adapter
}  // namespace gpd
