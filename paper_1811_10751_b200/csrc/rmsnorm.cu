// Root-mean-square norm with the residual's addition and an 8-bit output, and its gradient.
//
//   h = x + r,   s = (mean_c h^2 + eps)^(-1/2),   y = h s w      (FP32 throughout; h is rounded once, when stored)
//   q, scale = y cut into blocks of 128 columns (lm_common.h)
//   dx = s (g - h s^2 mean_c(g h)) + dh  with g = dy w,   dw_c = sum_t dy h s
//
// Both directions move each element once and do a few operations on it, so HBM bounds them.  A row stays
// in registers between the sum over its columns and its use: thread i of the row's G threads holds the
// vectors i, i + G, ... of eight neighbouring elements, so that loads and stores are 16 bytes per lane and
// the sixteen vectors of a scale block lie in sixteen adjacent lanes.
// Measured: forward 8192 x 8192 BF16 with residual 78-84 us, up to 0.92 of the copy bandwidth; gradient 4096 x 4096 BF16
// 31.5 us, 0.65 (instructions and the latency of a row's two steps; dw's partial rows are summed in a kernel of 4 us).
// Rows too long for registers are read twice and their share of dw goes through memory: gradient of 2048 x 16384 205 us
// BF16 (0.20), 276 us FP32 (0.30).
#include <algorithm>

#include "lm_common.h"

namespace gpd {

namespace {

using namespace lm;

struct NormArgs {
    const void* x; int64_t ldx;
    const void* residual; int64_t ldr;
    const void* weight;
    void* h; int64_t ldh;
    void* y; int64_t ldy;
    uint8_t* q; int64_t ldq;
    uint8_t* scales; int64_t lds;
    float* rstd;
    int64_t T, H;
    float eps;
    bool q_vec;                                        // rows of q start on 8-byte boundaries
};

// Eight weights from column c < H (VEC: all there, on a 16-byte boundary)
template <typename W, bool VEC>
__device__ __forceinline__ Raw8<W> weight_at(const W* w, int c, int H) {
    if (VEC || (c + 8 <= H && (reinterpret_cast<uintptr_t>(w) & 15) == 0)) return load8_all<W>(w + c);
    return load8<W, false>(w + c, H - c);
}

// Sum over the G threads of a row (a multiple of 32, threadIdx.x); every thread gets it.  G = 32: a warp of its
// own, no barrier.  Otherwise row `g` of the CTA has named barrier g + 1 and two sets of 32 floats in
// `scratch`, used in turn, so that one barrier per sum is enough.
__device__ __forceinline__ float row_sum(float v, int G, int g, float* scratch) {
    v = warp_sum(v);
    if (G == 32) return v;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = G >> 5;
    if (lane == 0) scratch[warp] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(g + 1), "r"(G) : "memory");
    return warp_sum(lane < n ? scratch[lane] : 0.f);
}

// VPT vectors per thread are kept in registers; VPT = 0: rows too long for that are read twice.
// blockDim = (G, rows per CTA), rows per CTA > 1 only with G = 32.  VEC: every vector is whole and on a 16-byte boundary.
template <typename T, typename W, int Q, int VPT, bool VEC>
__global__ void __launch_bounds__(VPT > 0 ? 512 : 1024) rmsnorm_kernel(const NormArgs a) {
    __shared__ float scratch[32];
    after_previous();
    const int G = blockDim.x, H = (int)a.H;
    const int64_t t = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    if (t >= a.T) return;                              // a whole warp (G = 32) or, with one row per CTA, never
    const T* x = static_cast<const T*>(a.x) + t * a.ldx;
    const T* res = a.residual ? static_cast<const T*>(a.residual) + t * a.ldr : nullptr;
    const W* wt = static_cast<const W*>(a.weight);
    T* hout = a.h ? static_cast<T*>(a.h) + t * a.ldh : nullptr;
    T* yout = a.y ? static_cast<T*>(a.y) + t * a.ldy : nullptr;
    uint8_t* qout = a.q ? a.q + t * a.ldq : nullptr;
    uint8_t* sout = a.q ? a.scales + t * a.lds : nullptr;

    auto load = [&](const T* p, int c, const void* base, int64_t ld) {
        if (VEC) return c < H ? load8_all<T>(p + c) : Raw8<T>{};
        const T* begin = static_cast<const T*>(base);
        return c + 8 <= H ? load8_near<T>(p + c, begin, begin + (a.T - 1) * ld + H) : c < H ? load8<T, false>(p + c, H - c) : Raw8<T>{};
    };
    auto store = [&](T* p, int c, const float (&f)[8]) {               // every lane of the warp calls it
        if (!VEC) store8_near<T>(p + c, f, H - c);
        else if (c < H) store8<T, true>(p + c, f, 8);
    };
    auto add = [&](const Raw8<T>& rx, const Raw8<T>& rr, F2 (&h)[4]) {
        pairs8<T>(rx, h);
        if (res) {
            F2 r[4];
            pairs8<T>(rr, r);
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = add2(h[i], r[i]);
        }
    };
    // y of one vector, from h; h and y are stored where they are wanted
    auto normed = [&](int c, const F2 (&h)[4], float s, float (&y)[8]) {
        if (hout) {
            floats8(h, y);
            store(hout, c, y);
        }
        F2 w[4] = {0, 0, 0, 0};                        // columns that do not exist: y = 0
        if (c < H) pairs8<W>(weight_at<W, VEC>(wt, c, H), w);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = mul2(mul2(h[i], f2(s, s)), w[i]);
        floats8(w, y);
        if (c >= H) {                                  // whatever s is
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = 0.f;
        }
        if (yout) store(yout, c, y);
    };
    // N vectors of this thread, G vectors apart, in 8 bits; every lane of a warp gets here together
    auto finish = [&](int c0, const auto& h, float s) {
        constexpr int N = sizeof(h) / sizeof(h[0]);
        float y[N][8];
        uint32_t m[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            normed(c0 + 8 * i * G, h[i], s, y[i]);
            m[i] = amax8(y[i]);
        }
        if (!qout) return;
        const BlockScales b = block_scales<Q, N>(m, [](uint32_t x) { return x; });
        const int mine = (c0 + 8 * b.mine * G) / kBlock;
        if (b.first && mine * kBlock < H) sout[mine] = (uint8_t)b.byte;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = c0 + 8 * i * G, n = H - c;
            if (n > 0) {
                const uint2 v = to_fp8x8<Q>(y[i], scale_inverse(packed_byte(b, i)));
                if (VEC || (a.q_vec && n >= 8)) *reinterpret_cast<uint2*>(qout + c) = v;
                else store8_bytes(qout + c, v, n);
            }
        }
    };
    auto square = [](const F2 (&h)[4], F2 sum) {
#pragma unroll
        for (int i = 0; i < 4; ++i) sum = fma2(h[i], h[i], sum);
        return sum;
    };
    auto inverse_root = [&](F2 squares) {
        const float2 p = f2(squares);
        const float s = rsqrtf(row_sum(p.x + p.y, G, 0, scratch) / (float)H + a.eps);
        if (a.rstd && threadIdx.x == 0) a.rstd[t] = s;
        return s;
    };

    F2 sum = f2(0.f, 0.f);
    if constexpr (VPT > 0) {
        F2 h[VPT][4];
        Raw8<T> rx[VPT], rr[VPT];                      // all loads before the first use
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = 8 * (threadIdx.x + i * G);
            rx[i] = load(x, c, a.x, a.ldx);
            rr[i] = res ? load(res, c, a.residual, a.ldr) : Raw8<T>{};
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            add(rx[i], rr[i], h[i]);
            sum = square(h[i], sum);
        }
        const float s = inverse_root(sum);
        // four vectors at a time: more would not fit in registers beside their y
        constexpr int N = VPT < 4 ? VPT : 4;
#pragma unroll
        for (int i = 0; i < VPT; i += N) finish(8 * (threadIdx.x + i * G), *reinterpret_cast<F2(*)[N][4]>(&h[i]), s);
    } else {
        // h may be stored over x or r: nothing is written before the second reading, and each element
        // is read and written by the same thread
        const int step = 8 * G, rounds = (H + step - 1) / step;
        F2 h[1][4];
        for (int i = 0; i < rounds; ++i) {
            const int c = 8 * threadIdx.x + i * step;
            add(load(x, c, a.x, a.ldx), res ? load(res, c, a.residual, a.ldr) : Raw8<T>{}, h[0]);
            sum = square(h[0], sum);
        }
        const float s = inverse_root(sum);
        for (int i = 0; i < rounds; ++i) {
            const int c = 8 * threadIdx.x + i * step;
            add(load(x, c, a.x, a.ldx), res ? load(res, c, a.residual, a.ldr) : Raw8<T>{}, h[0]);
            finish(c, h, s);
        }
    }
}

template <typename T, typename W, int Q, bool VEC>
gpd_status launch_norm(const NormArgs& a, cudaStream_t st) {
    const int64_t vecs = (a.H + 7) / 8;
    if (vecs <= 128) {                                 // a warp per row, four rows per CTA: no barrier
        const dim3 block(32, 4);
        const unsigned grid = (unsigned)((a.T + 3) / 4);
        if (vecs <= 32) return launch_after(rmsnorm_kernel<T, W, Q, 1, VEC>, dim3(grid), block, 0, 1, st, a);
        if (vecs <= 64) return launch_after(rmsnorm_kernel<T, W, Q, 2, VEC>, dim3(grid), block, 0, 1, st, a);
        return launch_after(rmsnorm_kernel<T, W, Q, 4, VEC>, dim3(grid), block, 0, 1, st, a);
    }
    // Many rows: four vectors per thread, which leaves several rows in flight on an SM (8192 x 8192 BF16 with residual:
    // 80 us; two vectors 85, eight 107).  Few rows: two, for the latency of one row.
    constexpr int kMost = sizeof(T) == 4 ? 4 : 8;
    const int vpt = vecs > 512 * kMost ? 0 : vecs > 2048 ? kMost : a.T >= 4 * sm_count() || vecs > 1024 ? 4 : 2;
    const int threads = vpt ? (int)(((vecs + vpt - 1) / vpt + 31) / 32 * 32) : 1024;
    switch (vpt) {
        case 2: return launch_after(rmsnorm_kernel<T, W, Q, 2, VEC>, dim3((unsigned)a.T), dim3(threads), 0, 1, st, a);
        case 4: return launch_after(rmsnorm_kernel<T, W, Q, 4, VEC>, dim3((unsigned)a.T), dim3(threads), 0, 1, st, a);
        case kMost == 8 ? 8 : -1: return launch_after(rmsnorm_kernel<T, W, Q, kMost, VEC>, dim3((unsigned)a.T), dim3(threads), 0, 1, st, a);
        default: return launch_after(rmsnorm_kernel<T, W, Q, 0, VEC>, dim3((unsigned)a.T), dim3(threads), 0, 1, st, a);
    }
}
template <typename T, typename W, int Q>
gpd_status launch_norm_q(const NormArgs& a, cudaStream_t st) {
    const int e = sizeof(T);
    const bool vec = a.H % 8 == 0 && rows_aligned(a.x, a.ldx, e) && rows_aligned(a.residual, a.ldr, e) && rows_aligned(a.h, a.ldh, e) &&
                     rows_aligned(a.y, a.ldy, e) && rows_aligned(a.q, a.ldq, 1, 8) && aligned(a.weight, 16);
    return vec ? launch_norm<T, W, Q, true>(a, st) : launch_norm<T, W, Q, false>(a, st);
}
template <typename T, typename W>
gpd_status launch_norm_w(const NormArgs& a, int q_type, cudaStream_t st) {
    return q_type == GPD_DT_E5M2 ? launch_norm_q<T, W, GPD_DT_E5M2>(a, st) : launch_norm_q<T, W, GPD_DT_E4M3>(a, st);
}

// ---- gradient ----------------------------------------------------------------------------------------
struct NormBwdArgs {
    const void* dy; int64_t lddy;
    const void* h; int64_t ldh;
    const void* dh; int64_t lddh;
    const void* weight;
    const float* rstd;
    void* dx; int64_t lddx;
    float* parts;                                      // [gridDim.x][H]
    int64_t T, H;
};

constexpr int kBwdThreads = 512;

// blockDim = (G, R): R rows of the CTA at a time, G threads each.  A thread adds up its columns' share of dw over
// its rows: in registers, met in shared memory at the end, one partial row per CTA; or (VPT = 0, long rows, R = 1)
// in the CTA's row of `parts`, element by element by the thread that owns the column.
// PIECES: the rows' 16-byte pieces are the threads' vectors.  A row that starts `shift` elements after a boundary has
// its first vector begin that much before it; the tensors share their shifts, and a thread's rows are so many
// apart that they have the same one, so that its columns stay its own.
// AHEAD: the next row is loaded while the present one's sum is awaited and its results are written.
template <typename T, typename W, int VPT, bool PIECES, bool AHEAD>
__global__ void __launch_bounds__(VPT > 0 ? kBwdThreads : 1024) rmsnorm_backward_kernel(const NormBwdArgs a) {
    __shared__ float scratch[16][2][32];
    extern __shared__ __align__(16) float dw_rows[];   // the threads' weights; at the end [R][H], the rows' shares of dw
    after_previous();
    const int G = blockDim.x, g = threadIdx.y, H = (int)a.H, step = 8 * G;
    const W* wt = static_cast<const W*>(a.weight);
    float* part = a.parts + (int64_t)blockIdx.x * a.H;
    constexpr int N = VPT > 0 ? VPT : 1;
    const int64_t stride = (int64_t)gridDim.x * blockDim.y, first = (int64_t)blockIdx.x * blockDim.y + g;
    const int shift = PIECES ? (int)((first * a.ldh) & (16 / sizeof(T) - 1)) : 0;
    const int c0 = 8 * threadIdx.x - shift;            // first column of the thread's first vector
    F2 dw[N][4];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) dw[i][j] = f2(0.f, 0.f);
    int turn = 0;
    // eight columns from c, some of which may lie outside the row
    auto whole = [&](int c) { return c >= 0 && c + 8 <= H; };
    auto edge = [&](const auto* p, int c, float (&f)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = c + j >= 0 && c + j < H ? to_f32(p[c + j]) : 0.f;
    };
    auto load = [&](const T* p, int c, const void* base, int64_t ld) {
        if (whole(c)) {
            if (PIECES) return load8_all<T>(p + c);
            const T* begin = static_cast<const T*>(base);
            return load8_near<T>(p + c, begin, begin + (a.T - 1) * ld + H);
        }
        Raw8<T> r{};
        if (c > -8 && c < H) {
            float f[8];
            edge(p, c, f);
            if constexpr (sizeof(T) == 4) {
                r.v = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
                r.w = make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
            } else {
                r.v = make_uint4(pack2(f[0], f[1], T()), pack2(f[2], f[3], T()), pack2(f[4], f[5], T()), pack2(f[6], f[7], T()));
            }
        }
        return r;
    };
    // the thread's weights, FP32, in places of its own in shared memory; long rows read them anew
    float4* own_w = reinterpret_cast<float4*>(dw_rows) + (size_t)g * 2 * N * G + threadIdx.x;
    if (VPT > 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float f[8];
            edge(wt, c0 + i * step, f);
            own_w[(2 * i) * G] = make_float4(f[0], f[1], f[2], f[3]);
            own_w[(2 * i + 1) * G] = make_float4(f[4], f[5], f[6], f[7]);
        }
    }
    auto weights = [&](int i, F2 (&w)[4]) {
        float f[8];
        if (VPT > 0) {
            const float4 lo = own_w[(2 * i) * G], hi = own_w[(2 * i + 1) * G];
            w[0] = f2(lo.x, lo.y);
            w[1] = f2(lo.z, lo.w);
            w[2] = f2(hi.x, hi.y);
            w[3] = f2(hi.z, hi.w);
            return;
        }
        const int c = c0 + i * step;
        if (whole(c) && ((reinterpret_cast<uintptr_t>(wt + c)) & 15) == 0) {
            pairs8<W>(load8_all<W>(wt + c), w);
            return;
        }
        edge(wt, c, f);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = f2(f[2 * j], f[2 * j + 1]);
    };
    Raw8<T> rdy[N], rh[N], rdh[N];
    auto fetch = [&](int64_t t) {
        const T* dy = static_cast<const T*>(a.dy) + t * a.lddy;
        const T* h = static_cast<const T*>(a.h) + t * a.ldh;
        const T* dh = a.dh ? static_cast<const T*>(a.dh) + t * a.lddh : nullptr;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = c0 + i * step;
            rdy[i] = load(dy, c, a.dy, a.lddy);
            rh[i] = load(h, c, a.h, a.ldh);
            rdh[i] = dh ? load(dh, c, a.dh, a.lddh) : Raw8<T>{};
        }
    };
    if (AHEAD && first < a.T) fetch(first);
    for (int64_t t = first; t < a.T; t += stride, turn ^= 1) {
        const T* dy = static_cast<const T*>(a.dy) + t * a.lddy;
        const T* h = static_cast<const T*>(a.h) + t * a.ldh;
        const T* dh = a.dh ? static_cast<const T*>(a.dh) + t * a.lddh : nullptr;
        T* dx = static_cast<T*>(a.dx) + t * a.lddx;
        const float s = a.rstd[t];
        auto dot8 = [&](int i, const Raw8<T>& qdy, const Raw8<T>& qh, F2 sum) {
            F2 fy[4], fh[4], w[4];
            pairs8<T>(qdy, fy);
            pairs8<T>(qh, fh);
            weights(i, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) sum = fma2(mul2(fy[j], w[j]), fh[j], sum);
            return sum;
        };
        // every lane of the warp gets here
        auto write = [&](int i, const Raw8<T>& qdy, const Raw8<T>& qh, const Raw8<T>& qdh, float k, F2 (&acc)[4]) {
            const int c = c0 + i * step;
            F2 fy[4], fh[4], fd[4], w[4];
            pairs8<T>(qdy, fy);
            pairs8<T>(qh, fh);
            pairs8<T>(qdh, fd);
            weights(i, w);
            const F2 ss = f2(s, s), mk = f2(-k, -k);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                acc[j] = fma2(mul2(fy[j], ss), fh[j], acc[j]);
                fd[j] = fma2(ss, fma2(fh[j], mk, mul2(fy[j], w[j])), fd[j]);
            }
            float o[8];
            floats8(fd, o);
            if (!PIECES) {
                store8_near<T>(dx + c, o, H - c);
            } else if (whole(c)) {
                store8<T, true>(dx + c, o, 8);
            } else if (c > -8 && c < H) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j >= 0 && c + j < H) dx[c + j] = from_f32<T>(o[j]);
            }
        };
        F2 sum = f2(0.f, 0.f);
        if constexpr (VPT > 0) {
            if (!AHEAD) fetch(t);
            Raw8<T> cdy[VPT], ch[VPT], cdh[VPT];
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                cdy[i] = rdy[i];
                ch[i] = rh[i];
                cdh[i] = rdh[i];
            }
#pragma unroll
            for (int i = 0; i < VPT; ++i) sum = dot8(i, cdy[i], ch[i], sum);
            if (AHEAD && t + stride < a.T) fetch(t + stride);
            const float2 p = f2(sum);
            const float k = s * s * (row_sum(p.x + p.y, G, g, scratch[g][turn]) / (float)H);
#pragma unroll
            for (int i = 0; i < VPT; ++i) write(i, cdy[i], ch[i], cdh[i], k, dw[i]);
        } else {
            const int rounds = (H + shift + step - 1) / step;
            for (int i = 0; i < rounds; ++i) {
                const int c = c0 + i * step;
                sum = dot8(i, load(dy, c, a.dy, a.lddy), load(h, c, a.h, a.ldh), sum);
            }
            const float2 p = f2(sum);
            const float k = s * s * (row_sum(p.x + p.y, G, g, scratch[g][turn]) / (float)H);
            for (int i = 0; i < rounds; ++i) {
                const int c = c0 + i * step;
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = c + j >= 0 && c + j < H && t != first ? part[c + j] : 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) dw[0][j] = f2(f[2 * j], f[2 * j + 1]);
                write(i, load(dy, c, a.dy, a.lddy), load(h, c, a.h, a.ldh), dh ? load(dh, c, a.dh, a.lddh) : Raw8<T>{}, k, dw[0]);
                floats8(dw[0], f);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j >= 0 && c + j < H) part[c + j] = f[j];
            }
        }
    }
    if constexpr (VPT > 0) {
        // the R rows' shares in the order of the rows; their shifts may differ, so each has all H columns
        __syncthreads();                               // the weights have been read
        float* mine = dw_rows + (int64_t)g * H;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = c0 + i * step;
            float f[8];
            floats8(dw[i], f);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j >= 0 && c + j < H) mine[c + j] = f[j];
        }
        __syncthreads();
        for (int c = g * G + threadIdx.x; c < H; c += G * blockDim.y) {
            float v = dw_rows[c];
            for (int r = 1; r < (int)blockDim.y; ++r) v += dw_rows[(int64_t)r * H + c];
            part[c] = v;
        }
    }
}

// dw_c = sum over the partial rows, in a fixed order: sixteen threads per column, then their sums.
__global__ void __launch_bounds__(512) rmsnorm_dweight_kernel(const float* parts, int n, int64_t H, float* dw) {
    __shared__ float s[16][33];
    after_previous();
    const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x;
    float v = 0.f;
    if (c < H)
#pragma unroll 8
        for (int p = threadIdx.y; p < n; p += 16) v += parts[(int64_t)p * H + c];
    s[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.y == 0 && c < H) {
        for (int i = 1; i < 16; ++i) v += s[i][threadIdx.x];
        dw[c] = v;
    }
}

template <typename T, typename W>
gpd_status launch_bwd(const NormBwdArgs& a, float* dweight, cudaStream_t st) {
    constexpr int e = sizeof(T), per16 = 16 / e, V = e == 4 ? 2 : 3, A = 2;   // vectors per thread that fit in registers, with the next row's (16-bit)
    // whether the tensors' rows start equally far from 16-byte boundaries, and whether that differs from row to row
    auto like_h = [&](const void* p, int64_t ld) { return !p || (aligned(p, 16) && (ld - a.ldh) % per16 == 0); };
    const bool pieces = like_h(a.dy, a.lddy) && like_h(a.h, a.ldh) && like_h(a.dh, a.lddh) && like_h(a.dx, a.lddx);
    const bool shifts = pieces && a.ldh % per16 != 0;
    const int64_t vecs = (a.H + 7 + (shifts ? per16 - 1 : 0)) / 8;
    // two vectors per thread leave room for the next row (4096 x 4096 BF16: 32 us, without it 37 from four vectors);
    // FP32 rows do not gain from it (one vector 49.8 us, two without the next row 48.5)
    // nor do rows for which it would leave more than a quarter of the CTA's 512 threads out
    auto group = [&](int per) { return (int)(((vecs + per - 1) / per + 31) / 32 * 32); };
    const bool ahead = e == 2 && pieces && vecs <= kBwdThreads * A && kBwdThreads / group(A) * group(A) >= kBwdThreads * 3 / 4;
    const bool loop = !ahead && vecs > kBwdThreads * V;
    const int per = ahead ? A : V, G = loop ? 1024 : group(per);
    // one CTA per SM: R rows of G threads at a time, as many as it takes for T rows; named barriers 1 .. 15
    int R = loop ? 1 : std::max(1, std::min(kBwdThreads / G, 15));
    R = (int)std::max<int64_t>(1, std::min<int64_t>(R, (a.T + sm_count() - 1) / sm_count()));
    int parts = (int)std::min<int64_t>(std::min<int64_t>((a.T + R - 1) / R, sm_count()), GPD_RMSNORM_MAX_PARTS);
    // a thread's rows are a multiple of per16 apart where the shifts differ, unless it has one row only
    if (shifts && (int64_t)parts * R < a.T) {
        while (R > 1 && R % 2) --R;
        while ((int64_t)parts * R % per16 != 0) --parts;
    }
    if (parts > 0) {
        auto kernel = loop    ? (pieces ? rmsnorm_backward_kernel<T, W, 0, true, false> : rmsnorm_backward_kernel<T, W, 0, false, false>)
                      : ahead ? rmsnorm_backward_kernel<T, W, A, true, e == 2>
                              : (pieces ? rmsnorm_backward_kernel<T, W, V, true, false> : rmsnorm_backward_kernel<T, W, V, false, false>);
        const int smem = loop ? 0 : R * G * per * 32;  // at most 64 KB; H <= 8 per G
        if (smem > 40960 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
            return GPD_ERR_CUDA;
        const gpd_status rc = launch_after(kernel, dim3(parts), dim3(G, R), smem, 1, st, a);
        if (rc != GPD_OK) return rc;
    }
    const float* partial = a.parts;
    return launch_after(rmsnorm_dweight_kernel, dim3((unsigned)((a.H + 31) / 32)), dim3(32, 16), 0, 1, st, partial, parts, a.H, dweight);
}

}  // namespace

}  // namespace gpd

using namespace gpd;

extern "C" gpd_status gpd_rmsnorm_quant(gpd_dtype type, const void* x_dev, int64_t ldx, const void* residual_dev,
                                        int64_t ldr, gpd_dtype weight_type, const void* weight_dev, float eps,
                                        void* residual_out_dev, int64_t ldh, void* y_dev, int64_t ldy, gpd_dtype q_type,
                                        void* q_dev, int64_t ldq, uint8_t* scales_dev, int64_t lds, float* rstd_dev,
                                        int64_t T, int64_t H, void* stream) {
    if (!is_float_type(type) || (weight_type != type && weight_type != GPD_DT_F32)) return GPD_ERR_ARG;
    if (T < 0 || H <= 0 || T > 0x7fffffff || H > 0x7ffffff0 / 2) return GPD_ERR_SHAPE;
    if (T == 0) return GPD_OK;                         // empty buffers may have no address
    if (!x_dev || !weight_dev || (q_dev && (!scales_dev || !is_fp8_type(q_type)))) return GPD_ERR_ARG;
    if (ldx < H || (residual_dev && ldr < H) || (residual_out_dev && ldh < H) || (y_dev && ldy < H) ||
        (q_dev && (ldq < H || lds < (H + lm::kBlock - 1) / lm::kBlock)))
        return GPD_ERR_SHAPE;
    const NormArgs a{x_dev, ldx, residual_dev, ldr, weight_dev, residual_out_dev, ldh, y_dev, ldy, static_cast<uint8_t*>(q_dev),
                     ldq, scales_dev, lds, rstd_dev, T, H, eps, lm::rows_aligned(q_dev, ldq, 1, 8)};
    cudaStream_t st = as_stream(stream);
    if (type == GPD_DT_F32) return launch_norm_w<float, float>(a, q_type, st);
    if (type == GPD_DT_BF16)
        return weight_type == GPD_DT_F32 ? launch_norm_w<__nv_bfloat16, float>(a, q_type, st)
                                         : launch_norm_w<__nv_bfloat16, __nv_bfloat16>(a, q_type, st);
    return weight_type == GPD_DT_F32 ? launch_norm_w<__half, float>(a, q_type, st) : launch_norm_w<__half, __half>(a, q_type, st);
}

extern "C" gpd_status gpd_rmsnorm_backward(gpd_dtype type, const void* dy_dev, int64_t lddy, const void* h_dev, int64_t ldh,
                                           gpd_dtype weight_type, const void* weight_dev, const float* rstd_dev,
                                           const void* dresidual_dev, int64_t lddh, void* dx_dev, int64_t lddx,
                                           float* dweight_dev, int64_t T, int64_t H, void* workspace_dev,
                                           int64_t workspace_bytes, void* stream) {
    if (!is_float_type(type) || (weight_type != type && weight_type != GPD_DT_F32)) return GPD_ERR_ARG;
    if (T < 0 || H <= 0 || H > 0x7ffffff0 / 2) return GPD_ERR_SHAPE;
    if (!dweight_dev || (T > 0 && (!dy_dev || !h_dev || !weight_dev || !rstd_dev || !dx_dev))) return GPD_ERR_ARG;
    if (T > 0 && (lddy < H || ldh < H || (dresidual_dev && lddh < H) || lddx < H)) return GPD_ERR_SHAPE;
    if (T > 0 && (!workspace_dev || workspace_bytes < std::min<int64_t>(T, GPD_RMSNORM_MAX_PARTS) * H * (int64_t)sizeof(float) ||
                  !aligned(workspace_dev, 4)))
        return GPD_ERR_WORKSPACE;
    const NormBwdArgs a{dy_dev, lddy, h_dev, ldh, dresidual_dev, lddh, weight_dev, rstd_dev, dx_dev, lddx,
                        static_cast<float*>(workspace_dev), T, H};
    cudaStream_t st = as_stream(stream);
    if (type == GPD_DT_F32) return launch_bwd<float, float>(a, dweight_dev, st);
    if (type == GPD_DT_BF16)
        return weight_type == GPD_DT_F32 ? launch_bwd<__nv_bfloat16, float>(a, dweight_dev, st)
                                         : launch_bwd<__nv_bfloat16, __nv_bfloat16>(a, dweight_dev, st);
    return weight_type == GPD_DT_F32 ? launch_bwd<__half, float>(a, dweight_dev, st)
                                     : launch_bwd<__half, __half>(a, dweight_dev, st);
}
