// Shared by the low-precision layer operators (rmsnorm.cu, quantize.cu, gemm_fp8.cu, logits.cu):
// loads and stores of eight neighbouring elements of any of the storage types, the 8-bit conversions and
// the power-of-two block scale.
//
// A block's scale is 2^e with the smallest e for which the block's largest magnitude is at most
// top * 2^e, top = 448 (e4m3) or 57344 (e5m2), both 0.875 times a power of two.  A power of two makes the
// division by the scale exact (one rounding per element, the conversion's), costs at most one step of an
// 8-bit type's exponent range, and is the form the tensor cores apply by themselves; it is stored as its
// biased exponent in one byte (e8m0).  A block of zeros has scale 1; a block holding a NaN or an infinity
// has the scale byte 255, which stands for NaN, so that nothing computed from it looks like a number.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "gpd_internal.h"

namespace gpd {
namespace lm {

constexpr int kBlock = 128;                            // elements that share a scale

template <typename T> struct Raw8 { uint4 v; };        // eight 16-bit elements
template <> struct Raw8<float> { uint4 v, w; };

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi, __nv_bfloat16) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __half) {
    const __half2 p = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ float2 unpack2(uint32_t u, __nv_bfloat16) {
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
__device__ __forceinline__ float2 unpack2(uint32_t u, __half) {
    return __half22float2(*reinterpret_cast<const __half2*>(&u));
}

// Pairs of FP32 numbers, one instruction for both
typedef unsigned long long F2;
__device__ __forceinline__ F2 f2(float lo, float hi) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 f2(F2 a) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a));
    return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// Eight elements at p, of which n (may be <= 0 or >= 8) exist; the others read as zero.  VEC: p is
// 16-byte aligned (the caller has checked base and row stride).
template <typename T, bool VEC>
__device__ __forceinline__ Raw8<T> load8(const T* p, int n) {
    Raw8<T> r;
    if constexpr (sizeof(T) == 4) {
        if (VEC && n >= 8) {
            r.v = reinterpret_cast<const uint4*>(p)[0];
            r.w = reinterpret_cast<const uint4*>(p)[1];
        } else {
            uint32_t u[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = i < n ? __float_as_uint(p[i]) : 0u;
            r.v = make_uint4(u[0], u[1], u[2], u[3]);
            r.w = make_uint4(u[4], u[5], u[6], u[7]);
        }
    } else {
        if (VEC && n >= 8) {
            r.v = *reinterpret_cast<const uint4*>(p);
        } else {
            const unsigned short* s = reinterpret_cast<const unsigned short*>(p);
            uint32_t u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = 2 * i < n ? s[2 * i] : 0u, hi = 2 * i + 1 < n ? s[2 * i + 1] : 0u;
                u[i] = lo | (hi << 16);
            }
            r.v = make_uint4(u[0], u[1], u[2], u[3]);
        }
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void unpack8(const Raw8<T>& r, float (&f)[8]) {
    if constexpr (sizeof(T) == 4) {
        f[0] = __uint_as_float(r.v.x); f[1] = __uint_as_float(r.v.y); f[2] = __uint_as_float(r.v.z); f[3] = __uint_as_float(r.v.w);
        f[4] = __uint_as_float(r.w.x); f[5] = __uint_as_float(r.w.y); f[6] = __uint_as_float(r.w.z); f[7] = __uint_as_float(r.w.w);
    } else {
        const float2 a = unpack2(r.v.x, T()), b = unpack2(r.v.y, T()), c = unpack2(r.v.z, T()), d = unpack2(r.v.w, T());
        f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y; f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
    }
}
// Eight elements as four pairs and back, and all of eight elements at a 16-byte boundary.
template <typename T>
__device__ __forceinline__ void pairs8(const Raw8<T>& r, F2 (&p)[4]) {
    if constexpr (sizeof(T) == 4) {
        p[0] = f2(__uint_as_float(r.v.x), __uint_as_float(r.v.y));
        p[1] = f2(__uint_as_float(r.v.z), __uint_as_float(r.v.w));
        p[2] = f2(__uint_as_float(r.w.x), __uint_as_float(r.w.y));
        p[3] = f2(__uint_as_float(r.w.z), __uint_as_float(r.w.w));
    } else {
        const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack2(w[i], T());
            p[i] = f2(f.x, f.y);
        }
    }
}
__device__ __forceinline__ void floats8(const F2 (&p)[4], float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 x = f2(p[i]);
        f[2 * i] = x.x;
        f[2 * i + 1] = x.y;
    }
}
template <typename T>
__device__ __forceinline__ Raw8<T> load8_all(const T* p) {
    Raw8<T> r;
    r.v = reinterpret_cast<const uint4*>(p)[0];
    if constexpr (sizeof(T) == 4) r.w = reinterpret_cast<const uint4*>(p)[1];
    return r;
}
// Elements 2 i and 2 i + 1 of eight.
template <typename T>
__device__ __forceinline__ float2 pair_of(const Raw8<T>& r, int i) {
    if constexpr (sizeof(T) == 4) {
        const uint4& h = i < 2 ? r.v : r.w;
        return i & 1 ? make_float2(__uint_as_float(h.z), __uint_as_float(h.w)) : make_float2(__uint_as_float(h.x), __uint_as_float(h.y));
    } else {
        return unpack2(i == 0 ? r.v.x : i == 1 ? r.v.y : i == 2 ? r.v.z : r.v.w, T());
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* p, const float (&f)[8], int n) {
    if (VEC && n >= 8) {
        if constexpr (sizeof(T) == 4) {
            reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
            reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
        } else {
            *reinterpret_cast<uint4*>(p) = make_uint4(pack2(f[0], f[1], T()), pack2(f[2], f[3], T()),
                                                      pack2(f[4], f[5], T()), pack2(f[6], f[7], T()));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = from_f32<T>(f[i]);
    }
}

// ---- rows that do not start on 16-byte boundaries ----------------------------------------------------------
// Four words from the `n` words w, starting `s` elements in.
template <typename T, int N>
__device__ __forceinline__ void shifted4(const uint32_t (&w)[N], int s, uint32_t (&o)[4]) {
    constexpr int per = 4 / sizeof(T);                 // elements of a word
    const int ws = s / per;
    uint32_t a[6], b[5];
#pragma unroll
    for (int i = 0; i < 6; ++i) a[i] = i + 2 < N ? (ws & 2 ? w[i + 2] : w[i]) : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) b[i] = ws & 1 ? a[i + 1] : a[i];
    const uint32_t sel = per == 2 && (s & 1) ? 0x5432u : 0x3210u;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = per == 2 ? __byte_perm(b[i], b[i + 1], sel) : b[i];
}
// Eight elements at p, anywhere, by 16-byte loads of what surrounds them.  [begin, end): the tensor; what would reach
// beyond it is loaded element by element.
template <typename T>
__device__ __forceinline__ Raw8<T> load8_near(const T* p, const T* begin, const T* end) {
    constexpr int N = 16 / sizeof(T);
    const int mis = (int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
    if (mis == 0) return load8_all<T>(p);
    const T* q = p - mis;
    if (q < begin || q + 8 + N > end) return load8<T, false>(p, 8);
    const uint4* v = reinterpret_cast<const uint4*>(q);
    const uint4 x = v[0], y = v[1];
    uint32_t o[4];
    Raw8<T> r;
    if constexpr (sizeof(T) == 2) {
        const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        shifted4<T>(w, mis, o);
        r.v = make_uint4(o[0], o[1], o[2], o[3]);
    } else {
        const uint4 z = v[2];
        const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w}, u[8] = {y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
        shifted4<T>(w, mis, o);
        r.v = make_uint4(o[0], o[1], o[2], o[3]);
        shifted4<T>(u, mis, o);
        r.w = make_uint4(o[0], o[1], o[2], o[3]);
    }
    return r;
}
// The n (<= 8, possibly none) elements f to p, where the lanes of the warp hold consecutive eights of one row: a lane
// stores the 16-byte piece that begins among its elements and ends among the next lane's.  All lanes call it.
template <typename T>
__device__ __forceinline__ void store8_near(T* p, const float (&f)[8], int n) {
    constexpr int N = 16 / sizeof(T), W = 8 / (4 / sizeof(T));         // elements of a piece, words of eight elements
    const int lane = threadIdx.x & 31, mis = (int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
    if (mis == 0) {                                    // the same for all lanes of the warp
        store8<T, true>(p, f, n);
        return;
    }
    uint32_t w[W], next[W];
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack2(f[2 * i], f[2 * i + 1], T());
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(f[i]);
    }
#pragma unroll
    for (int i = 0; i < W; ++i) next[i] = __shfl_down_sync(0xffffffffu, w[i], 1);
    const uint32_t full = __ballot_sync(0xffffffffu, n >= 8);
    const bool before = lane > 0 && full >> (lane - 1) & 1, after = lane < 31 && full >> (lane + 1) & 1;
    const int head = N - mis, tail = 8 - mis;          // the first whole piece starts at `head`, the last one begun at `tail`
    if (n >= 8) {
        uint32_t o[4];
        if constexpr (sizeof(T) == 4) {
            const uint32_t own[8] = {w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]};
            shifted4<T>(own, head, o);
            *reinterpret_cast<uint4*>(p + head) = make_uint4(o[0], o[1], o[2], o[3]);
        }
        if (after) {
            const uint32_t both[8] = {w[W - 4], w[W - 3], w[W - 2], w[W - 1], next[0], next[1], next[2], next[3]};
            shifted4<T>(both, head, o);
            *reinterpret_cast<uint4*>(p + tail) = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)                        // what no piece covers
        if (i < n && (n < 8 || (i < head && !before) || (i >= tail && !after))) p[i] = from_f32<T>(f[i]);
}

// ---- 8-bit blocks ----------------------------------------------------------------------------------
// top = 0.875 * 2^kTopExp
template <int Q> struct Fp8;
template <> struct Fp8<GPD_DT_E4M3> { static constexpr int kTopExp = 9; };
template <> struct Fp8<GPD_DT_E5M2> { static constexpr int kTopExp = 16; };

// Scale byte of a block whose largest magnitude has these bits.  Magnitudes are compared as bit patterns: NaN is then the
// largest and cannot be lost in a maximum.
template <int Q>
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
    if (amax == 0u) return 127u;
    if (amax >= 0x7f800000u) return 255u;
    const int e = (int)(amax >> 23) + 1 - Fp8<Q>::kTopExp + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)max(e, 0);
}
// 1 / scale = 2^(127 - byte); for the byte 255 any number will do.
__device__ __forceinline__ float scale_inverse(uint32_t byte) { return __uint_as_float((254u - min(byte, 253u)) << 23); }

template <int Q>
__device__ __forceinline__ uint32_t cvt_fp8x4(float a, float b, float c, float d) {
    uint32_t r;
    if constexpr (Q == GPD_DT_E4M3)
        asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\tmov.b32 %0, {lo, hi};\n\t}"
            : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
    else
        asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e5m2x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e5m2x2.f32 hi, %4, %3;\n\tmov.b32 %0, {lo, hi};\n\t}"
            : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}
// Eight bytes at p, anywhere, of which n exist
__device__ __forceinline__ void store8_bytes(uint8_t* p, uint2 b, int n) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = (uint8_t)((i < 4 ? b.x >> (8 * i) : b.y >> (8 * (i - 4))) & 0xffu);
}

// Bits of the largest magnitude of eight numbers, a NaN above all
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint32_t amax8(const float (&f)[8]) {
    float m = max_nan(fabsf(f[0]), fabsf(f[1]));
#pragma unroll
    for (int i = 2; i < 8; ++i) m = max_nan(m, fabsf(f[i]));
    return __float_as_uint(m);
}
// Eight numbers times `inv`, in 8 bits
template <int Q>
__device__ __forceinline__ uint2 to_fp8x8(const float (&f)[8], float inv) {
    return make_uint2(cvt_fp8x4<Q>(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv),
                      cvt_fp8x4<Q>(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv));
}

// Scale bytes of N (1, 2, 4 or 8) blocks, each spread over the sixteen lanes of a half-warp: amax[i] holds the bits of
// this lane's largest magnitude in block i, `bits` turns the block's maximum into FP32 bits.  The lanes halve the blocks
// among them while they exchange maxima, so that a lane ends with one block (`mine`, the same in 16 / N lanes) and its
// byte is worked out once; then they hand the bytes back.  Every lane gets all N, packed; `first` in one lane per block.
struct BlockScales { uint32_t lo, hi, byte; int mine; bool first; };
__device__ __forceinline__ uint32_t packed_byte(const BlockScales& b, int i) { return (i < 4 ? b.lo >> (8 * i) : b.hi >> (8 * (i - 4))) & 0xffu; }
template <int Q, int N, typename F>
__device__ __forceinline__ BlockScales block_scales(const uint32_t (&amax)[N], F bits) {
    const int cg = threadIdx.x & 15;
    uint32_t r[N];
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = amax[i];
    BlockScales b{0, 0, 0, 0, false};
#pragma unroll
    for (int n = N, o = 8; o > 0; n >>= 1, o >>= 1) {
        if (n > 1) {
            const bool up = cg & o;
            b.mine = 2 * b.mine + up;
#pragma unroll
            for (int i = 0; i < n / 2; ++i) {
                const uint32_t keep = up ? r[i + n / 2] : r[i], send = up ? r[i] : r[i + n / 2];
                r[i] = max(keep, __shfl_xor_sync(0xffffffffu, send, o));
            }
        } else {
            r[0] = max(r[0], __shfl_xor_sync(0xffffffffu, r[0], o));
        }
    }
    b.byte = scale_byte<Q>(bits(r[0]));
    b.first = (cg & (16 / N - 1)) == 0;
    b.lo = b.byte;
#pragma unroll
    for (int have = 1, o = 16 / N; have < N; have *= 2, o *= 2) {
        const uint32_t other = __shfl_xor_sync(0xffffffffu, b.lo, o);
        const bool up = cg & o;
        const uint32_t low = up ? other : b.lo, high = up ? b.lo : other;
        if (have < 4) {
            b.lo = low | high << (8 * have);
        } else {
            b.lo = low;
            b.hi = high;
        }
    }
    return b;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// ---- launches ------------------------------------------------------------------------------------------
// The operators' kernels are launched so that a kernel's start-up (its launch, barriers, tensor memory) overlaps
// the end of the kernel before it in the stream: each calls `after_previous` before it touches memory, which waits
// for that kernel's completion, and thereby lets the next one start.
__device__ __forceinline__ void after_previous() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
// cluster: CTAs per cluster along x (1: none)
template <typename... P, typename... A>
gpd_status launch_after(void (*kernel)(P...), dim3 grid, dim3 block, int smem, int cluster, cudaStream_t st, const A&... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cuda_ok(cudaLaunchKernelEx(&cfg, kernel, args...));
}

// ---- host side: argument checks ---------------------------------------------------------------------
inline int dtype_size(int t) { return t == GPD_DT_F32 ? 4 : (t == GPD_DT_BF16 || t == GPD_DT_F16) ? 2 : 1; }
inline bool is_float_type(int t) { return t == GPD_DT_F32 || t == GPD_DT_BF16 || t == GPD_DT_F16; }
inline bool is_fp8_type(int t) { return t == GPD_DT_E4M3 || t == GPD_DT_E5M2; }
inline bool aligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
// A matrix of `elem`-byte elements can be read in 16-byte pieces of every row (absent matrices can).
inline bool rows_aligned(const void* p, int64_t ld, int elem, int bytes = 16) {
    return !p || (aligned(p, bytes) && (ld * elem) % bytes == 0);
}

}  // namespace lm
}  // namespace gpd
