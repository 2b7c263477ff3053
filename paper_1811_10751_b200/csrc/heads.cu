// Norms of queries and keys for each head with the rotation by position in the same pass, and their gradient.
//
//   s = (mean_d x^2 + eps)^(-1/2),   z = x s w,   y = R z          (FP32 throughout, y rounded once)
//   (a, b) -> (a cos - b sin, b cos + a sin) for the pairs of the first R columns, the others stay
//   g = R^T dy,   dw_d = sum g x s,   dx = s (g w - x s^2 mean_d(g w x))
//
// Every element is read once and written once, with a handful of operations: HBM bounds both directions.  A head of D
// columns is cut into units of V pairs: the two vectors of V elements that hold them, so that a pair's halves are in one
// thread's registers in either pairing and loads are 16 bytes (or 8) per lane.  G lanes hold a head, 32 / G heads are in a
// warp; the norm is a butterfly over the G lanes, no shared memory and no barrier.  A piece of work is one token, whose
// angles are loaded once, and up to U * 32 / G of its heads; warps walk over the pieces, and load the next one before they
// work on the present one.  Arithmetic is on pairs of numbers.
//
// Measured: 16384 tokens x 72 heads of 128 BF16 115 us of 95 at the copy bandwidth (issue 54 %, two thirds of it conversions, the norm's butterfly
// and the turn); 8 tokens 3.4 us; the gradient of 4096 x 40 heads 33 us of 20 (issue 48 %), 4 of them the sum of the
// weights' gradients.
#include <algorithm>
#include <numeric>

#include "gemm_common.h"
#include "lm_common.h"
#include "tc_common.h"

namespace gpd {

namespace {

using namespace lm;

constexpr int kWarps = 4, kWalkPerSm = 4;              // warps of a CTA; CTAs of the forward pass on an SM
constexpr int kMaxHead = GPD_HEAD_MAX_DIM;

// Queries or keys
struct Part {
    const void* x; int64_t ldx;
    const void* dy; int64_t lddy;                      // gradient only
    void* out; int64_t ldo;
    const void* w;                                     // null: no norm
    int heads, chunks;                                 // a token's work: chunks of U * 32 / G heads
};
struct HeadArgs {
    Part part[2];
    unsigned split;                                    // CTAs of the first part
    const float* table; int64_t ldt, P;
    const void* pos; int64_t ldp;
    const uint8_t* axes;
    float* parts;                                      // gradient: [gridDim.x][D]
    int64_t T;
    int D, R, A, lanes;                                // lanes: G
    float eps, inv_d;                                  // 1 / D
    bool wide_pos, w_f32, neighbours, inverse, table_vec;
};

template <typename T, int V> struct Vec;               // V neighbouring elements
template <> struct Vec<float, 4> { uint4 r; };
template <> struct Vec<__nv_bfloat16, 8> { uint4 r; };
template <> struct Vec<__half, 8> { uint4 r; };
template <> struct Vec<__nv_bfloat16, 4> { uint2 r; };
template <> struct Vec<__half, 4> { uint2 r; };
template <typename T> struct Vec<T, 1> { T r; };

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load_vec(const T* p) { return *reinterpret_cast<const Vec<T, V>*>(p); }
template <typename T, int V>
__device__ __forceinline__ void unpack(const Vec<T, V>& v, float (&f)[V]) {
    if constexpr (V == 1) {
        f[0] = to_f32(v.r);
    } else if constexpr (sizeof(T) == 4) {
        f[0] = __uint_as_float(v.r.x); f[1] = __uint_as_float(v.r.y); f[2] = __uint_as_float(v.r.z); f[3] = __uint_as_float(v.r.w);
    } else {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(&v.r);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const float2 x = unpack2(w[i], T());
            f[2 * i] = x.x;
            f[2 * i + 1] = x.y;
        }
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_vec(T* p, const float (&f)[V]) {
    Vec<T, V> v;
    if constexpr (V == 1) {
        v.r = from_f32<T>(f[0]);
    } else if constexpr (sizeof(T) == 4) {
        v.r = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    } else {
        uint32_t* w = reinterpret_cast<uint32_t*>(&v.r);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) w[i] = pack2(f[2 * i], f[2 * i + 1], T());
    }
    *reinterpret_cast<Vec<T, V>*>(p) = v;
}

// Unit u of a head: columns c1 .. c1 + V - 1 and c2 .. c2 + V - 1; turned or not.
template <int V>
struct Unit {
    int c1, c2;
    bool there, turned;
    __device__ __forceinline__ Unit(int u, const HeadArgs& a) {
        const int nr = a.R / (2 * V);
        there = u < a.D / (2 * V);
        turned = u < nr;
        if (a.neighbours) {
            c1 = 2 * V * u;
            c2 = c1 + V;
        } else {
            const int i = turned ? u : u - nr, from = turned ? 0 : a.R;
            c1 = from + V * i;
            c2 = c1 + (turned ? a.R : a.D - a.R) / 2;
        }
    }
};
// The two vectors of a unit as first and second halves of its pairs, and back.
template <int V>
__device__ __forceinline__ void to_pairs(const float (&x)[V], const float (&y)[V], bool neighbours, float (&a)[V], float (&b)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (V == 1) {
            a[i] = x[i];
            b[i] = y[i];
        } else {
            const float ea = 2 * i < V ? x[2 * i % V] : y[2 * i % V], eb = 2 * i < V ? x[(2 * i + 1) % V] : y[(2 * i + 1) % V];
            a[i] = neighbours ? ea : x[i];
            b[i] = neighbours ? eb : y[i];
        }
    }
}
template <int V>
__device__ __forceinline__ void from_pairs(const float (&a)[V], const float (&b)[V], bool neighbours, float (&x)[V], float (&y)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (V == 1) {
            x[i] = a[i];
            y[i] = b[i];
        } else {
            const int lo = i / 2, hi = V / 2 + i / 2;
            x[i] = neighbours ? (i & 1 ? b[lo] : a[lo]) : a[i];
            y[i] = neighbours ? (i & 1 ? b[hi] : a[hi]) : b[i];
        }
    }
}

// V floats at p; vec: on a 16-byte boundary
template <int V>
__device__ __forceinline__ void load_floats(const float* p, bool vec, float (&f)[V]) {
    if (V % 4 == 0 && vec) {
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            const float4 v = __ldg(reinterpret_cast<const float4*>(p) + i);
            f[4 * i] = v.x; f[4 * i + 1 < V ? 4 * i + 1 : 0] = v.y; f[4 * i + 2 < V ? 4 * i + 2 : 0] = v.z; f[4 * i + 3 < V ? 4 * i + 3 : 0] = v.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = __ldg(p + i);
    }
}

// Cosines and sines of unit u at the rows `pos` of the table, one for each axis.  Several axes: every pair takes its own
// from its axis's row, all loads at once.  Positions outside the table (-1), and axes that there are none of, give NaN.
template <int V>
__device__ __forceinline__ void angles(const HeadArgs& a, const int (&pos)[GPD_HEAD_MAX_AXES], int u, float (&cs)[V], float (&sn)[V]) {
    const float* first = a.table + V * u;
    if (!a.axes) {
#pragma unroll
        for (int i = 0; i < V; ++i) cs[i] = sn[i] = __int_as_float(0x7fffffff);
        if (pos[0] < 0) return;
        load_floats<V>(first + pos[0] * a.ldt, a.table_vec, cs);
        load_floats<V>(first + pos[0] * a.ldt + a.R / 2, a.table_vec, sn);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int x = __ldg(a.axes + V * u + i);
            const int row = x >= a.A ? -1 : x == 0 ? pos[0] : x == 1 ? pos[1] : x == 2 ? pos[2] : pos[3];
            cs[i] = sn[i] = __int_as_float(0x7fffffff);
            if (row >= 0) {
                const float* p = first + row * a.ldt + i;
                cs[i] = __ldg(p);
                sn[i] = __ldg(p + a.R / 2);
            }
        }
    }
    if (a.inverse) {
#pragma unroll
        for (int i = 0; i < V; ++i) sn[i] = -sn[i];
    }
}
// Rows of the table for token t, one for each axis; -1: none
__device__ __forceinline__ void positions(const HeadArgs& a, int64_t t, int (&at)[GPD_HEAD_MAX_AXES]) {
#pragma unroll
    for (int x = 0; x < GPD_HEAD_MAX_AXES; ++x) {
        if (x >= a.A || a.R == 0) continue;
        const int64_t v = a.wide_pos ? static_cast<const int64_t*>(a.pos)[t * a.ldp + x] : static_cast<const int32_t*>(a.pos)[t * a.ldp + x];
        at[x] = v < 0 || v >= a.P ? -1 : (int)v;
    }
}
template <typename T, int V>
__device__ __forceinline__ void weights(const HeadArgs& a, const void* w, const Unit<V>& u, float (&wa)[V], float (&wb)[V]) {
    float x[V], y[V];
    if (a.w_f32) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            x[i] = static_cast<const float*>(w)[u.c1 + i];
            y[i] = static_cast<const float*>(w)[u.c2 + i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            x[i] = to_f32(static_cast<const T*>(w)[u.c1 + i]);
            y[i] = to_f32(static_cast<const T*>(w)[u.c2 + i]);
        }
    }
    to_pairs<V>(x, y, a.neighbours, wa, wb);
}
// Sum over the G lanes of a head
__device__ __forceinline__ float lanes_sum(float v, int G) {
    if (G == 8) {                                      // 128 columns of 16 bits
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    } else {
        for (int o = G >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    }
    return v;
}

// Rows that no vector fits: element by element, N units per lane.
template <typename T, int N>
__global__ void __launch_bounds__(32 * kWarps) heads_kernel(const __grid_constant__ HeadArgs a) {
    constexpr int V = 1, U = 1;
    after_previous();
    const bool second = blockIdx.x >= a.split;
    const Part& p = a.part[second];
    const int64_t work = (int64_t)(blockIdx.x - (second ? a.split : 0)) * kWarps + (threadIdx.x >> 5);
    const int64_t t = work / p.chunks;
    if (t >= a.T) return;                              // whole warps
    const int lane = threadIdx.x & 31, G = a.lanes, per = 32 / G;
    const int h0 = (int)(work - t * p.chunks) * per * U + lane / G;
    const T* x = static_cast<const T*>(p.x) + t * p.ldx;
    T* y = static_cast<T*>(p.out) + t * p.ldo;

    Vec<T, V> r1[U][N], r2[U][N];
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const Unit<V> u(lane % G + n * G, a);
            const int h = h0 + i * per;
            r1[i][n] = r2[i][n] = Vec<T, V>{};
            if (u.there && h < p.heads) {
                r1[i][n] = load_vec<T, V>(x + (int64_t)h * a.D + u.c1);
                r2[i][n] = load_vec<T, V>(x + (int64_t)h * a.D + u.c2);
            }
        }
    int at[GPD_HEAD_MAX_AXES];
    positions(a, t, at);
    float cs[N][V], sn[N][V], wa[N][V], wb[N][V];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const Unit<V> u(lane % G + n * G, a);
        if (u.there && u.turned) angles<V>(a, at, lane % G + n * G, cs[n], sn[n]);
        if (u.there && p.w) weights<T, V>(a, p.w, u, wa[n], wb[n]);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int h = h0 + i * per;
        float fa[N][V], fb[N][V];
        float sum = 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float f[V], g[V];
            unpack<T, V>(r1[i][n], f);
            unpack<T, V>(r2[i][n], g);
            to_pairs<V>(f, g, a.neighbours, fa[n], fb[n]);
#pragma unroll
            for (int j = 0; j < V; ++j) sum = fmaf(fa[n][j], fa[n][j], fmaf(fb[n][j], fb[n][j], sum));
        }
        const float s = p.w ? rsqrtf(lanes_sum(sum, G) * a.inv_d + a.eps) : 1.f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const Unit<V> u(lane % G + n * G, a);
            if (!u.there || h >= p.heads) continue;
            if (p.w) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    fa[n][j] = fa[n][j] * s * wa[n][j];
                    fb[n][j] = fb[n][j] * s * wb[n][j];
                }
            }
            if (u.turned) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float c = fa[n][j], d = fb[n][j];
                    fa[n][j] = c * cs[n][j] - d * sn[n][j];
                    fb[n][j] = d * cs[n][j] + c * sn[n][j];
                }
            }
            float f[V], g[V];
            from_pairs<V>(fa[n], fb[n], a.neighbours, f, g);
            store_vec<T, V>(y + (int64_t)h * a.D + u.c1, f);
            store_vec<T, V>(y + (int64_t)h * a.D + u.c2, g);
        }
    }
}

// Gradient with norm: warps walk over the tokens and add up their lanes' share of dw in registers.
template <typename T, int N>
__global__ void __launch_bounds__(32 * kWarps) heads_backward_kernel(const __grid_constant__ HeadArgs a) {
    constexpr int V = 1, U = 1;
    __shared__ float shares[kWarps][kMaxHead];
    after_previous();
    const bool second = blockIdx.x >= a.split;
    const Part& p = a.part[second];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, G = a.lanes, per = 32 / G;
    const int64_t ctas = second ? gridDim.x - a.split : a.split, all = a.T * p.chunks;
    float wa[N][V], wb[N][V], da[N][V], db[N][V];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const Unit<V> u(lane % G + n * G, a);
#pragma unroll
        for (int j = 0; j < V; ++j) wa[n][j] = wb[n][j] = da[n][j] = db[n][j] = 0.f;
        if (u.there) weights<T, V>(a, p.w, u, wa[n], wb[n]);
    }
    for (int64_t work = (int64_t)(blockIdx.x - (second ? a.split : 0)) * kWarps + warp; work < all; work += ctas * kWarps) {
        const int64_t t = work / p.chunks;
        const int h0 = (int)(work - t * p.chunks) * per * U + lane / G;
        const T* x = static_cast<const T*>(p.x) + t * p.ldx;
        const T* dy = static_cast<const T*>(p.dy) + t * p.lddy;
        T* dx = static_cast<T*>(p.out) + t * p.ldo;
        Vec<T, V> x1[U][N], x2[U][N], y1[U][N], y2[U][N];
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const Unit<V> u(lane % G + n * G, a);
                const int h = h0 + i * per;
                x1[i][n] = x2[i][n] = y1[i][n] = y2[i][n] = Vec<T, V>{};
                if (u.there && h < p.heads) {
                    const int64_t at = (int64_t)h * a.D;
                    x1[i][n] = load_vec<T, V>(x + at + u.c1);
                    x2[i][n] = load_vec<T, V>(x + at + u.c2);
                    y1[i][n] = load_vec<T, V>(dy + at + u.c1);
                    y2[i][n] = load_vec<T, V>(dy + at + u.c2);
                }
            }
        int where[GPD_HEAD_MAX_AXES];
        positions(a, t, where);
        float cs[N][V], sn[N][V];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const Unit<V> u(lane % G + n * G, a);
            if (u.there && u.turned) angles<V>(a, where, lane % G + n * G, cs[n], sn[n]);
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int h = h0 + i * per;
            float xa[N][V], xb[N][V], ga[N][V], gb[N][V];
            float squares = 0.f, dot = 0.f;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const Unit<V> u(lane % G + n * G, a);
                float f[V], g[V];
                unpack<T, V>(x1[i][n], f);
                unpack<T, V>(x2[i][n], g);
                to_pairs<V>(f, g, a.neighbours, xa[n], xb[n]);
                unpack<T, V>(y1[i][n], f);
                unpack<T, V>(y2[i][n], g);
                to_pairs<V>(f, g, a.neighbours, ga[n], gb[n]);
                // heads and units that do not exist are zeros and stay so
                if (u.there && u.turned && h < p.heads) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {      // a.inverse: the sines are negated
                        const float c = ga[n][j], d = gb[n][j];
                        ga[n][j] = c * cs[n][j] - d * sn[n][j];
                        gb[n][j] = d * cs[n][j] + c * sn[n][j];
                    }
                }
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    squares = fmaf(xa[n][j], xa[n][j], fmaf(xb[n][j], xb[n][j], squares));
                    dot = fmaf(ga[n][j] * wa[n][j], xa[n][j], fmaf(gb[n][j] * wb[n][j], xb[n][j], dot));
                }
            }
            const float s = rsqrtf(lanes_sum(squares, G) * a.inv_d + a.eps);
            const float k = s * s * (lanes_sum(dot, G) * a.inv_d);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const Unit<V> u(lane % G + n * G, a);
                if (!u.there || h >= p.heads) continue;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    da[n][j] = fmaf(ga[n][j] * s, xa[n][j], da[n][j]);
                    db[n][j] = fmaf(gb[n][j] * s, xb[n][j], db[n][j]);
                    ga[n][j] = s * fmaf(xa[n][j], -k, ga[n][j] * wa[n][j]);
                    gb[n][j] = s * fmaf(xb[n][j], -k, gb[n][j] * wb[n][j]);
                }
                float f[V], g[V];
                from_pairs<V>(ga[n], gb[n], a.neighbours, f, g);
                store_vec<T, V>(dx + (int64_t)h * a.D + u.c1, f);
                store_vec<T, V>(dx + (int64_t)h * a.D + u.c2, g);
            }
        }
    }
    // the warp's heads, then the CTA's warps, in a fixed order
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const Unit<V> u(lane % G + n * G, a);
        for (int o = G; o < 32; o <<= 1) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                da[n][j] += __shfl_xor_sync(0xffffffffu, da[n][j], o);
                db[n][j] += __shfl_xor_sync(0xffffffffu, db[n][j], o);
            }
        }
        if (u.there && lane < G) {
            float f[V], g[V];
            from_pairs<V>(da[n], db[n], a.neighbours, f, g);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                shares[warp][u.c1 + j] = f[j];
                shares[warp][u.c2 + j] = g[j];
            }
        }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.D; c += 32 * kWarps) {
        float v = shares[0][c];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) v += shares[w][c];
        a.parts[(int64_t)blockIdx.x * a.D + c] = v;
    }
}

// Both weights' gradients: sums over their CTAs' rows in a fixed order, 32 threads per column, then theirs.
__global__ void __launch_bounds__(1024) heads_dweight_kernel(const float* parts, int split, int n, int D, float* dqw, float* dkw) {
    __shared__ float s[32][33];
    after_previous();
    const int c = blockIdx.x * 32 + threadIdx.x, from = blockIdx.y ? split : 0, to = blockIdx.y ? n : split;
    float* dw = blockIdx.y ? dkw : dqw;
    float v = 0.f;
    if (c < D)
#pragma unroll 8
        for (int p = from + threadIdx.y; p < to; p += 32) v += parts[(int64_t)p * D + c];
    s[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    // a warp per column now, the same tree for every column
    v = warp_sum(s[threadIdx.x][threadIdx.y]);
    const int mine = blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x == 0 && mine < D && dw) dw[mine] = v;
}

// ---- the same with whole vectors: warps walk over the work, the next piece's loads under way --------------------------
template <typename T, int V>
__device__ __forceinline__ void write_vec(uint32_t to, const float (&f)[V]) {
    uint32_t w[V * sizeof(T) / 4];
#pragma unroll
    for (int i = 0; i < (int)(V * sizeof(T) / 4); ++i) {
        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(f[i]);
        else w[i] = pack2(f[2 * i], f[2 * i + 1], T());
    }
    if constexpr (V * sizeof(T) == 16) asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    else asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(to), "r"(w[0]), "r"(w[1]) : "memory");
}
// Halves of a unit's pairs, two at a time
template <typename T, int V, bool NEAR>
__device__ __forceinline__ void pairs(const Vec<T, V>& r1, const Vec<T, V>& r2, F2 (&a)[V / 2], F2 (&b)[V / 2]) {
    float2 w[V];                                       // neighbours in memory
    const uint32_t *u1 = reinterpret_cast<const uint32_t*>(&r1.r), *u2 = reinterpret_cast<const uint32_t*>(&r2.r);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        if constexpr (sizeof(T) == 4) {
            w[i] = make_float2(__uint_as_float(u1[2 * i]), __uint_as_float(u1[2 * i + 1]));
            w[V / 2 + i] = make_float2(__uint_as_float(u2[2 * i]), __uint_as_float(u2[2 * i + 1]));
        } else {
            w[i] = unpack2(u1[i], T());
            w[V / 2 + i] = unpack2(u2[i], T());
        }
    }
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        a[i] = NEAR ? f2(w[2 * i].x, w[2 * i + 1].x) : f2(w[i].x, w[i].y);
        b[i] = NEAR ? f2(w[2 * i].y, w[2 * i + 1].y) : f2(w[V / 2 + i].x, w[V / 2 + i].y);
    }
}
template <int V, bool NEAR>
__device__ __forceinline__ void from_pairs2(const F2 (&a)[V / 2], const F2 (&b)[V / 2], float (&x)[V], float (&y)[V]) {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        const float2 u = f2(a[i]), v = f2(b[i]);
        if (NEAR) {
            float* q = i < V / 4 ? x : y;
            const int at = 4 * i % V;
            q[at] = u.x;
            q[at + 1] = v.x;
            q[at + 2] = u.y;
            q[at + 3] = v.y;
        } else {
            x[2 * i] = u.x;
            x[2 * i + 1] = u.y;
            y[2 * i] = v.x;
            y[2 * i + 1] = v.y;
        }
    }
}
template <typename T, int V, bool NEAR>
__device__ __forceinline__ void store_pairs(T* p1, T* p2, const F2 (&a)[V / 2], const F2 (&b)[V / 2]) {
    float x[V], y[V];
    from_pairs2<V, NEAR>(a, b, x, y);
    store_vec<T, V>(p1, x);
    store_vec<T, V>(p2, y);
}
template <typename T, int V, bool NEAR>
__device__ __forceinline__ void write_pairs(uint32_t p1, uint32_t p2, const F2 (&a)[V / 2], const F2 (&b)[V / 2]) {
    float x[V], y[V];
    from_pairs2<V, NEAR>(a, b, x, y);
    write_vec<T, V>(p1, x);
    write_vec<T, V>(p2, y);
}
template <int V>
__device__ __forceinline__ void two_by_two(const float (&f)[V], F2 (&o)[V / 2]) {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) o[i] = f2(f[2 * i], f[2 * i + 1]);
}
// (a, b) turned
template <int N>
__device__ __forceinline__ void turn(F2 (&a)[N], F2 (&b)[N], const F2 (&c)[N], const F2 (&s)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const F2 x = a[i];
        a[i] = fma2(b[i] ^ 0x8000000080000000ull, s[i], mul2(x, c[i]));
        b[i] = fma2(x, s[i], mul2(b[i], c[i]));
    }
}
__device__ __forceinline__ float both(F2 v) {
    const float2 f = f2(v);
    return f.x + f.y;
}

// One warp's walk over the tokens t, t + step, ... with the heads h0, h0 + per, ...: U of a lane in one piece of work.
template <typename T, int V, int U, bool NEAR>
__device__ __forceinline__ void walk(const HeadArgs& a, const Part& p, int t, int step, int h0, int per) {
    constexpr int P = V / 2;
    const int lane = threadIdx.x & 31, G = a.lanes, T_all = (int)a.T;
    const Unit<V> u(lane % G, a);
    const bool turned = u.there && u.turned;
    F2 wa[P], wb[P];
    if (p.w && u.there) {
        float x[V], y[V];
        weights<T, V>(a, p.w, u, x, y);
        two_by_two<V>(x, wa);
        two_by_two<V>(y, wb);
    } else {
#pragma unroll
        for (int i = 0; i < P; ++i) wa[i] = wb[i] = f2(0.f, 0.f);
    }
    Vec<T, V> x1[U], x2[U];                            // the next piece, as it comes
    int at[GPD_HEAD_MAX_AXES];                     // its positions
    auto fetch = [&](int t) {
        const T* x = static_cast<const T*>(p.x) + t * p.ldx + h0 * a.D;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const bool here = u.there && h0 + i * per < p.heads;
            const int d = i * per * a.D;
            x1[i] = x2[i] = Vec<T, V>{};
            if (here) {
                x1[i] = load_vec<T, V>(x + d + u.c1);
                x2[i] = load_vec<T, V>(x + d + u.c2);
            }
        }
        positions(a, t, at);
    };
    if (t < T_all) fetch(t);
    for (; t < T_all; t += step) {
        F2 c[P], s[P];
        if (turned) {
            float cs[V], sn[V];
            angles<V>(a, at, lane % G, cs, sn);
            two_by_two<V>(cs, c);
            two_by_two<V>(sn, s);
        }
        Vec<T, V> r1[U], r2[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            r1[i] = x1[i];
            r2[i] = x2[i];
        }
        if (t < T_all - step) fetch(t + step);
        T* out = static_cast<T*>(p.out) + t * p.ldo + h0 * a.D;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const bool here = u.there && h0 + i * per < p.heads;
            T* o = out + i * per * a.D;
            F2 xa[P], xb[P];
            pairs<T, V, NEAR>(r1[i], r2[i], xa, xb);
            if (p.w) {
                F2 squares = f2(0.f, 0.f);
#pragma unroll
                for (int j = 0; j < P; ++j) squares = fma2(xa[j], xa[j], fma2(xb[j], xb[j], squares));
                const float f = rsqrtf(lanes_sum(both(squares), G) * a.inv_d + a.eps);
                const F2 f_2 = f2(f, f);
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    xa[j] = mul2(mul2(xa[j], f_2), wa[j]);
                    xb[j] = mul2(mul2(xb[j], f_2), wb[j]);
                }
            }
            if (turned) turn<P>(xa, xb, c, s);
            if (here) store_pairs<T, V, NEAR>(o + u.c1, o + u.c2, xa, xb);
        }
    }
}
// The forward pass, or the gradient without norm.  U: heads of a lane in one piece of work, if there are so many; pieces with
// half of them and less do not pay for the absent ones (15504 tokens x 5 + 1 heads of 128 BF16: 37 -> 25 us, 8490 x 8 + 2 of 64: 20 -> 11).
template <typename T, int V, int U, bool NEAR>
__global__ void __launch_bounds__(32 * kWarps, kWalkPerSm) heads_walk_kernel(const __grid_constant__ HeadArgs a) {
    after_previous();
    const bool second = blockIdx.x >= a.split;
    const Part& p = a.part[second];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = 32 / a.lanes;
    // a warp keeps to one chunk of heads and walks over the tokens: the part's warps are a multiple of its chunks
    const int warps = (int)(second ? gridDim.x - a.split : a.split) * kWarps, index = (int)(blockIdx.x - (second ? a.split : 0)) * kWarps + warp;
    const int step = warps / p.chunks, t = index / p.chunks, from = index % p.chunks * per * U, left = p.heads - from, h0 = from + lane / a.lanes;
    if (U >= 2 && left <= per) walk<T, V, 1, NEAR>(a, p, t, step, h0, per);
    else if (U > 2 && left <= 2 * per) walk<T, V, 2, NEAR>(a, p, t, step, h0, per);
    else walk<T, V, U, NEAR>(a, p, t, step, h0, per);
}

// ---- gradient with norm, rows and heads on 16-byte boundaries ------------------------------------------------------
// Pieces, which are whole stretches of a row, come into a ring in shared memory by bulk copies of the warp's own, with the
// table's row where one is enough, and leave from there: what two inputs and the sums of dw need in registers leaves no room
// to load ahead (4096 x 40 heads of 128 BF16: 33 us, loading ahead into registers 38; the forward pass gains nothing, 120
// and 118 us at 16384 x 72 heads).
__device__ int g_heads_status = 0;                     // GPD_ERR_TIMEOUT if a bounded wait expired

constexpr int kBackHeads = 2, kBackStages = 3, kBackPerSm = 3;         // heads of a lane in a piece; stages; CTAs per SM
struct Stage {
    static constexpr int X = kBackHeads * 1024, BYTES = 2 * X + kMaxHead * 4;          // inputs, gradients, angles
};
__device__ __forceinline__ void bulk_load(uint32_t to, const void* from, int bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(to), "l"(from), "r"(bytes), "r"(tc::smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void bulk_store(void* to, uint32_t from, int bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(to), "r"(from), "r"(bytes) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
template <typename T, int V>
__device__ __forceinline__ Vec<T, V> read_vec(uint32_t at) {
    Vec<T, V> v;
    if constexpr (V * sizeof(T) == 16) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.r.x), "=r"(v.r.y), "=r"(v.r.z), "=r"(v.r.w) : "r"(at) : "memory");
    else asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.r.x), "=r"(v.r.y) : "r"(at) : "memory");
    return v;
}

template <typename T, int V, bool NEAR>
__global__ void __launch_bounds__(32 * kWarps, kBackPerSm) heads_back_kernel(const __grid_constant__ HeadArgs a) {
    constexpr int P = V / 2, U = kBackHeads, STAGES = kBackStages;
    using S = Stage;
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ float shares[kWarps][kMaxHead];
    __shared__ uint64_t full[kWarps][STAGES];
    __shared__ int row_of[kWarps][STAGES], abort;      // the table's row; -1: none
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane == 0) {
        for (int i = 0; i < STAGES; ++i) tc::mbar_init(&full[warp][i], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 0) abort = 0;
    __syncthreads();
    after_previous();
    const bool second = blockIdx.x >= a.split;
    const Part& p = a.part[second];
    const int G = a.lanes, per = 32 / G;
    // a warp keeps to one chunk of heads and walks over the tokens: the part's warps are a multiple of its chunks
    const int warps = (int)(second ? gridDim.x - a.split : a.split) * kWarps, index = (int)(blockIdx.x - (second ? a.split : 0)) * kWarps + warp;
    const int step = warps / p.chunks, h0 = index % p.chunks * per * U, T_all = (int)a.T, first = index / p.chunks;
    const int here = min(per * U, p.heads - h0), bytes = here * a.D * (int)sizeof(T);  // heads of the chunk
    const Unit<V> u(lane % G, a);
    const bool turned = u.there && u.turned, by_row = a.R > 0 && a.A == 1 && a.table_vec && a.R % 4 == 0;
    F2 wa[P], wb[P], da[P], db[P];
#pragma unroll
    for (int i = 0; i < P; ++i) wa[i] = wb[i] = da[i] = db[i] = f2(0.f, 0.f);
    if (u.there) {
        float x[V], y[V];
        weights<T, V>(a, p.w, u, x, y);
        two_by_two<V>(x, wa);
        two_by_two<V>(y, wb);
    }
    const uint32_t mine = tc::smem_u32(ring) + warp * (STAGES * S::BYTES);
    const T *x_at = static_cast<const T*>(p.x) + (int64_t)first * p.ldx + h0 * a.D, *dy_at = static_cast<const T*>(p.dy) + (int64_t)first * p.lddy + h0 * a.D;
    T* out_at = static_cast<T*>(p.out) + (int64_t)first * p.ldo + h0 * a.D;
    const int64_t x_step = step * p.ldx, dy_step = step * p.lddy, out_step = step * p.ldo;
    int at[GPD_HEAD_MAX_AXES] = {-1, -1, -1, -1};      // rows of the table for the token that is asked for next (one row), or worked on next
    // asks for a token's piece; lane 0
    auto fetch = [&](int stage) {
        uint64_t* bar = &full[warp][stage];
        const uint32_t to = mine + stage * S::BYTES;
        const bool row = by_row && at[0] >= 0;
        row_of[warp][stage] = at[0];
        tc::mbar_expect_tx(bar, bytes * 2 + (row ? a.R * 4 : 0));
        bulk_load(to, x_at, bytes, bar);
        bulk_load(to + S::X, dy_at, bytes, bar);
        if (row) bulk_load(to + S::BYTES - kMaxHead * 4, a.table + at[0] * a.ldt, a.R * 4, bar);
        x_at += x_step;
        dy_at += dy_step;
    };
    auto later = [&](int t, int n) { return t < T_all - n * (int64_t)step; };          // whether there is a token n on
    int asked = 0;
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
        if (later(first, i)) {
            if (by_row) positions(a, first + i * step, at);
            if (lane == 0) fetch(i);
            ++asked;
        }
    if (by_row && later(first, STAGES - 1)) positions(a, first + (STAGES - 1) * step, at);
    if (!by_row && a.R > 0 && first < T_all) positions(a, first, at);
    int k = 0, done = 0;
    uint32_t phase = 0;
    for (int t = first; t < T_all; t += step, ++done) {
        float cs[V], sn[V];
        if (!by_row && turned) angles<V>(a, at, lane % G, cs, sn);     // under way while the piece is awaited
        const bool live = tc::mbar_wait(&full[warp][k], phase, &abort, &g_heads_status);
        if (!__all_sync(0xffffffffu, live)) break;
        const uint32_t piece = mine + k * S::BYTES + lane / G * a.D * (int)sizeof(T);
        F2 c[P], s[P];
        if (turned) {
            if (by_row) {
                const uint32_t row = mine + k * S::BYTES + S::BYTES - kMaxHead * 4 + V * (lane % G) * 4;
                const bool there = row_of[warp][k] >= 0;
#pragma unroll
                for (int i = 0; i < V / 4; ++i) {
                    const Vec<float, 4> x = read_vec<float, 4>(row + 16 * i), y = read_vec<float, 4>(row + a.R * 2 + 16 * i);
                    c[2 * i] = f2(__uint_as_float(x.r.x), __uint_as_float(x.r.y));
                    c[2 * i + 1] = f2(__uint_as_float(x.r.z), __uint_as_float(x.r.w));
                    s[2 * i] = f2(__uint_as_float(y.r.x), __uint_as_float(y.r.y));
                    s[2 * i + 1] = f2(__uint_as_float(y.r.z), __uint_as_float(y.r.w));
                }
                const float nan = __int_as_float(0x7fffffff);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    s[i] ^= 0x8000000080000000ull;     // back
                    if (!there) c[i] = s[i] = f2(nan, nan);
                }
            } else {
                two_by_two<V>(cs, c);
                two_by_two<V>(sn, s);
            }
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (i * per >= here) break;                // the same for the warp
            const bool mine_too = u.there && i * per + lane / G < here;
            const uint32_t from = piece + i * per * a.D * (int)sizeof(T), at1 = from + u.c1 * (int)sizeof(T), at2 = from + u.c2 * (int)sizeof(T);
            Vec<T, V> r1{}, r2{};
            if (mine_too) {
                r1 = read_vec<T, V>(at1);
                r2 = read_vec<T, V>(at2);
            }
            F2 xa[P], xb[P];
            pairs<T, V, NEAR>(r1, r2, xa, xb);
            Vec<T, V> g1{}, g2{};
            if (mine_too) {
                g1 = read_vec<T, V>(at1 + S::X);
                g2 = read_vec<T, V>(at2 + S::X);
            }
            F2 ga[P], gb[P];
            pairs<T, V, NEAR>(g1, g2, ga, gb);
            if (turned && mine_too) turn<P>(ga, gb, c, s);         // heads and units that do not exist are zeros and stay so
            F2 squares = f2(0.f, 0.f), dot = f2(0.f, 0.f), ta[P], tb[P];
#pragma unroll
            for (int j = 0; j < P; ++j) {
                squares = fma2(xa[j], xa[j], fma2(xb[j], xb[j], squares));
                ta[j] = mul2(ga[j], xa[j]);
                tb[j] = mul2(gb[j], xb[j]);
                dot = fma2(ta[j], wa[j], fma2(tb[j], wb[j], dot));
            }
            const float sq = lanes_sum(both(squares), G), dt = lanes_sum(both(dot), G);
            // each product is about one of the terms below, so that none leaves FP32 where they do not (f^3 would for x of 1e13)
            // Heads that do not exist are zeros, whose root is an infinity without eps: they get 0.
            const float f = mine_too ? rsqrtf(sq * a.inv_d + a.eps) : 0.f, q = f * (dt * a.inv_d) * f * f;
            const F2 f_2 = f2(f, f), q_2 = f2(-q, -q);
#pragma unroll
            for (int j = 0; j < P; ++j) {
                da[j] = fma2(ta[j], f_2, da[j]);
                db[j] = fma2(tb[j], f_2, db[j]);
                ga[j] = fma2(xa[j], q_2, mul2(mul2(ga[j], wa[j]), f_2));
                gb[j] = fma2(xb[j], q_2, mul2(mul2(gb[j], wb[j]), f_2));
            }
            if (mine_too) write_pairs<T, V, NEAR>(at1, at2, ga, gb);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            bulk_store(out_at, mine + k * S::BYTES, bytes);
            // the stage before this one has left: it takes the token that is asked for next
            asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
            if (later(t, STAGES - 1)) fetch(k == 0 ? STAGES - 1 : k - 1);
        }
        asked += later(t, STAGES - 1);
        if (by_row && later(t, STAGES)) positions(a, t + STAGES * step, at);
        if (!by_row && a.R > 0 && later(t, 1)) positions(a, t + step, at);
        out_at += out_step;
        if (++k == STAGES) {
            k = 0;
            phase ^= 1;
        }
    }
    if (lane == 0) {
        int never = 0;                                 // given up: copies in flight land before the CTA ends
        if (*static_cast<volatile int*>(&abort))
            for (int i = done; i < asked; ++i) tc::mbar_wait(&full[warp][i % STAGES], i / STAGES & 1, &never, &g_heads_status);
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    // the warp's heads, then the CTA's warps, in a fixed order
    float fa[V], fb[V];
#pragma unroll
    for (int j = 0; j < P; ++j) {
        const float2 v = f2(da[j]), w = f2(db[j]);
        fa[2 * j] = v.x;
        fa[2 * j + 1] = v.y;
        fb[2 * j] = w.x;
        fb[2 * j + 1] = w.y;
    }
    for (int o = G; o < 32; o <<= 1) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            fa[j] += __shfl_xor_sync(0xffffffffu, fa[j], o);
            fb[j] += __shfl_xor_sync(0xffffffffu, fb[j], o);
        }
    }
    if (u.there && lane < G) {
        float f[V], h[V];
        from_pairs<V>(fa, fb, NEAR, f, h);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            shares[warp][u.c1 + j] = f[j];
            shares[warp][u.c2 + j] = h[j];
        }
    }
    __syncthreads();
    for (int d = threadIdx.x; d < a.D; d += 32 * kWarps) {
        float v = shares[0][d];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) v += shares[w][d];
        a.parts[(int64_t)blockIdx.x * a.D + d] = v;
    }
}

// ---- host side ---------------------------------------------------------------------------------------
// Largest vector that the layout allows: whole units (turned and not), and every row on a boundary of it, or of 16 bytes where
// bulk copies take whole heads; else 1.
int vector_width(const HeadArgs& a, int elem, bool bulk) {
    if (bulk && a.D * elem % 16 != 0) return 1;
    for (int V = 16 / elem; V >= 4; V /= 2) {
        bool ok = a.D % (2 * V) == 0 && a.R % (2 * V) == 0;
        const int bytes = bulk ? 16 : V * elem;
        for (const Part& p : a.part)
            if (p.heads > 0)
                ok = ok && rows_aligned(p.x, p.ldx, elem, bytes) && rows_aligned(p.dy, p.lddy, elem, bytes) && rows_aligned(p.out, p.ldo, elem, bytes);
        if (ok) return V;
    }
    return 1;
}
int pow2_lanes(int units) {
    int g = 1;
    while (g < units && g < 32) g *= 2;
    return g;
}

// Gives each part its chunks and CTAs: as many as there is work, about `most` at most in all, shared out by the amount of it:
// pieces, or (walk) heads of a lane and two more for what a token costs in each piece.
// fixed: so many that their warps are a multiple of the chunks.
int share_out(HeadArgs& a, int U, int64_t most, bool fixed, bool walk) {
    const int per = 32 / a.lanes, step = per * U;
    int64_t work[2], cost[2], n[2], unit[2];
    for (int i = 0; i < 2; ++i) {
        const int chunks = std::max(1, (a.part[i].heads + step - 1) / step);
        a.part[i].chunks = chunks;
        work[i] = a.part[i].heads > 0 ? (a.T * chunks + kWarps - 1) / kWarps : 0;
        cost[i] = a.part[i].heads > 0 ? chunks + (walk ? chunks + (a.part[i].heads + per - 1) / per : 0) : 0;
        unit[i] = fixed ? chunks / std::gcd(chunks, kWarps) : 1;       // CTAs
    }
    for (int i = 0; i < 2; ++i) {
        const int64_t share = work[0] + work[1] > most ? most * cost[i] / (cost[0] + cost[1]) : work[i];
        n[i] = work[i] == 0 ? 0 : std::max<int64_t>(1, std::min((work[i] + unit[i] - 1) / unit[i], share / unit[i])) * unit[i];
    }
    a.split = (unsigned)n[0];
    return (int)(n[0] + n[1]);
}
template <typename T, int V, int U>
gpd_status launch_walk(HeadArgs a, cudaStream_t st) {
    const int ctas = share_out(a, U, kWalkPerSm * sm_count(), true, true);
    auto kernel = a.neighbours ? heads_walk_kernel<T, V, U, true> : heads_walk_kernel<T, V, U, false>;
    return launch_after(kernel, dim3((unsigned)ctas), dim3(32 * kWarps), 0, 1, st, a);
}
template <typename T, int V>
gpd_status launch_back(const HeadArgs& a, int ctas, cudaStream_t st) {
    constexpr int smem = kWarps * kBackStages * Stage::BYTES;
    static_assert(kBackPerSm * (smem + kWarps * kMaxHead * 4 + 2048) <= 227 * 1024, "the CTAs of an SM find room");
    auto kernel = a.neighbours ? heads_back_kernel<T, V, true> : heads_back_kernel<T, V, false>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return GPD_ERR_CUDA;
    return launch_after(kernel, dim3((unsigned)ctas), dim3(32 * kWarps), smem, 1, st, a);
}
template <typename T, int V>
gpd_status launch_forward(HeadArgs a, cudaStream_t st) {
    a.lanes = pow2_lanes(a.D / (2 * V));
    // Few tokens: one head per lane and piece, so that the heads are spread over the SMs.
    const int64_t steps = a.T * ((a.part[0].heads + a.part[1].heads) / (32 / a.lanes) + 1);
    return steps < 8 * (int64_t)sm_count() * kWarps ? launch_walk<T, V, 1>(a, st) : launch_walk<T, V, 4>(a, st);
}
template <typename T>
gpd_status launch_heads(HeadArgs a, cudaStream_t st) {
    switch (vector_width(a, sizeof(T), false)) {
        case sizeof(T) == 2 ? 8 : -1: return launch_forward<T, 16 / sizeof(T)>(a, st);
        case 4: return launch_forward<T, 4>(a, st);
    }
    a.lanes = pow2_lanes(a.D / 2);
    const int ctas = share_out(a, 1, INT32_MAX, false, false);
    return launch_after(heads_kernel<T, kMaxHead / 64>, dim3((unsigned)ctas), dim3(32 * kWarps), 0, 1, st, a);
}

template <typename T>
gpd_status launch_heads_backward(HeadArgs a, float* dqw, float* dkw, cudaStream_t st) {
    const int V = vector_width(a, sizeof(T), true);
    a.lanes = pow2_lanes(a.D / (2 * V));
    const int ctas = share_out(a, V == 1 ? 1 : kBackHeads, kBackPerSm * sm_count(), V > 1, false);
    if (ctas > 0) {
        gpd_status rc;
        if (V == 1) rc = launch_after(heads_backward_kernel<T, kMaxHead / 64>, dim3((unsigned)ctas), dim3(32 * kWarps), 0, 1, st, a);
        else rc = V == 4 ? launch_back<T, 4>(a, ctas, st) : launch_back<T, 16 / sizeof(T)>(a, ctas, st);
        if (rc != GPD_OK) return rc;
    }
    const float* parts = a.parts;
    const int split = (int)a.split;
    return launch_after(heads_dweight_kernel, dim3((unsigned)((a.D + 31) / 32), 2), dim3(32, 32), 0, 1, st, parts, split, ctas, a.D, dqw, dkw);
}

// What both directions check.  GPD_OK with a.T = 0: nothing to do.
gpd_status check_heads(int type, int weight_type, const HeadArgs& a, int index_bytes, bool norm) {
    if (!is_float_type(type) || (norm && weight_type != type && weight_type != GPD_DT_F32)) return GPD_ERR_ARG;
    if (a.T < 0 || a.T > GPD_LM_MAX_ROWS || a.D <= 0 || a.D % 2 || a.D > kMaxHead || a.R < 0 || a.R % 2 || a.R > a.D) return GPD_ERR_SHAPE;
    if (!norm && a.R == 0) return GPD_ERR_ARG;
    const Part *q = &a.part[0], *k = &a.part[1];
    if (q->heads < 0 || k->heads < 0 || q->heads > GPD_HEAD_MAX_HEADS || k->heads > GPD_HEAD_MAX_HEADS) return GPD_ERR_SHAPE;
    if (a.R > 0) {
        if (a.A < 1 || a.A > GPD_HEAD_MAX_AXES || a.P < 0 || a.P > 0x7fffffff || (a.P > 1 && a.ldt < a.R) || (a.T > 1 && a.ldp < a.A)) return GPD_ERR_SHAPE;
        if ((index_bytes != 4 && index_bytes != 8) || (a.A > 1 && !a.axes)) return GPD_ERR_ARG;
        if ((a.P > 0 && !a.table) || (a.T > 0 && !a.pos)) return GPD_ERR_ARG;
    }
    for (const Part& p : a.part) {
        if (p.heads == 0 || a.T == 0) continue;
        const int64_t row = (int64_t)p.heads * a.D;
        if (p.ldx < row || p.ldo < row) return GPD_ERR_SHAPE;
        if (!p.out) return GPD_ERR_ARG;
    }
    return GPD_OK;
}

}  // namespace

int heads_status_fetch_and_clear() {
    int v = 0, zero = 0;
    if (cudaMemcpyFromSymbol(&v, g_heads_status, sizeof(int)) != cudaSuccess) return (int)GPD_ERR_CUDA;
    if (v != 0) cudaMemcpyToSymbol(g_heads_status, &zero, sizeof(int));
    return v;
}

}  // namespace gpd

using namespace gpd;

extern "C" gpd_status gpd_head_norm_rope(gpd_dtype type, const void* q_dev, int64_t ldq, int32_t q_heads, const void* k_dev,
                                         int64_t ldk, int32_t k_heads, int32_t head_dim, gpd_dtype weight_type,
                                         const void* q_weight_dev, const void* k_weight_dev, float eps,
                                         const float* table_dev, int64_t ldt, int64_t positions, int32_t rotated,
                                         int32_t neighbours, int32_t index_bytes, const void* pos_dev, int64_t ldp,
                                         int32_t n_axes, const uint8_t* axes_dev, void* q_out_dev, int64_t ldqo, void* k_out_dev,
                                         int64_t ldko, int64_t T, void* stream) {
    HeadArgs a{{{q_dev, ldq, nullptr, 0, q_out_dev, ldqo, q_weight_dev, q_heads, 0}, {k_dev, ldk, nullptr, 0, k_out_dev, ldko, k_weight_dev, k_heads, 0}},
               0, table_dev, ldt, positions, pos_dev, ldp, n_axes > 1 ? axes_dev : nullptr, nullptr, T, head_dim, rotated, n_axes, 0, eps, head_dim > 0 ? 1.f / (float)head_dim : 0.f,
               index_bytes == 8, weight_type == GPD_DT_F32, neighbours != 0, false, lm::rows_aligned(table_dev, ldt, 4)};
    const bool norm = q_weight_dev || k_weight_dev;
    const gpd_status rc = check_heads(type, weight_type, a, index_bytes, norm);
    if (rc != GPD_OK) return rc;
    if (T == 0 || q_heads + k_heads == 0) return GPD_OK;   // empty buffers may have no address
    for (const Part& p : a.part)
        if (p.heads > 0 && (!p.x || (norm && !p.w))) return GPD_ERR_ARG;
    cudaStream_t st = as_stream(stream);
    if (type == GPD_DT_F32) return launch_heads<float>(a, st);
    return type == GPD_DT_BF16 ? launch_heads<__nv_bfloat16>(a, st) : launch_heads<__half>(a, st);
}

extern "C" gpd_status gpd_head_norm_rope_backward(gpd_dtype type, const void* dq_dev, int64_t lddq, const void* dk_dev, int64_t lddk,
                                                  const void* q_dev, int64_t ldq, int32_t q_heads, const void* k_dev, int64_t ldk,
                                                  int32_t k_heads, int32_t head_dim, gpd_dtype weight_type,
                                                  const void* q_weight_dev, const void* k_weight_dev, float eps,
                                                  const float* table_dev, int64_t ldt, int64_t positions, int32_t rotated,
                                                  int32_t neighbours, int32_t index_bytes, const void* pos_dev, int64_t ldp,
                                                  int32_t n_axes, const uint8_t* axes_dev, void* dq_in_dev, int64_t lddqi,
                                                  void* dk_in_dev, int64_t lddki, float* dq_weight_dev, float* dk_weight_dev,
                                                  int64_t T, void* workspace_dev, int64_t workspace_bytes, void* stream) {
    const bool norm = q_weight_dev || k_weight_dev;
    // without norm the gradient is the forward pass of dy with the angles negated
    const void *xq = norm ? q_dev : dq_dev, *xk = norm ? k_dev : dk_dev;
    HeadArgs a{{{xq, norm ? ldq : lddq, norm ? dq_dev : nullptr, lddq, dq_in_dev, lddqi, q_weight_dev, q_heads, 0},
                {xk, norm ? ldk : lddk, norm ? dk_dev : nullptr, lddk, dk_in_dev, lddki, k_weight_dev, k_heads, 0}},
               0, table_dev, ldt, positions, pos_dev, ldp, n_axes > 1 ? axes_dev : nullptr, static_cast<float*>(workspace_dev), T, head_dim,
               rotated, n_axes, 0, eps, head_dim > 0 ? 1.f / (float)head_dim : 0.f, index_bytes == 8, weight_type == GPD_DT_F32, neighbours != 0, true,
               lm::rows_aligned(table_dev, ldt, 4)};
    const gpd_status rc = check_heads(type, weight_type, a, index_bytes, norm);
    if (rc != GPD_OK) return rc;
    cudaStream_t st = as_stream(stream);
    if (!norm) {
        if (T == 0 || q_heads + k_heads == 0) return GPD_OK;
        for (const Part& p : a.part)
            if (p.heads > 0 && !p.x) return GPD_ERR_ARG;
        if (type == GPD_DT_F32) return launch_heads<float>(a, st);
        return type == GPD_DT_BF16 ? launch_heads<__nv_bfloat16>(a, st) : launch_heads<__half>(a, st);
    }
    if (T > 0) {
        for (const Part& p : a.part)
            if (p.heads > 0 && (!p.x || !p.dy || !p.w || p.lddy < (int64_t)p.heads * head_dim)) return p.x && p.dy && p.w ? GPD_ERR_SHAPE : GPD_ERR_ARG;
        if (q_heads + k_heads > 0 && (!workspace_dev || workspace_bytes < 2 * GPD_HEAD_NORM_MAX_PARTS * (int64_t)head_dim * 4 || !lm::aligned(workspace_dev, 4)))
            return GPD_ERR_WORKSPACE;
    }
    if ((q_heads > 0 && !dq_weight_dev) || (k_heads > 0 && !dk_weight_dev)) return GPD_ERR_ARG;
    if (type == GPD_DT_F32) return launch_heads_backward<float>(a, dq_weight_dev, dk_weight_dev, st);
    return type == GPD_DT_BF16 ? launch_heads_backward<__nv_bfloat16>(a, dq_weight_dev, dk_weight_dev, st)
                               : launch_heads_backward<__half>(a, dq_weight_dev, dk_weight_dev, st);
}
