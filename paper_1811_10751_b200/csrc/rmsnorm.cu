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
// Measured: forward 8192 x 8192 BF16 with residual 78 us, 0.92 of the copy bandwidth.
#include <algorithm>

#include "gemm_common.h"
#include "lm_common.h"
#include "tc_common.h"

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
                else store8_bytes<false>(qout + c, v, n);
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
template <typename T, typename W, int VPT, bool VEC>
__global__ void __launch_bounds__(VPT > 0 ? kBwdThreads : 1024) rmsnorm_backward_kernel(const NormBwdArgs a) {
    __shared__ float scratch[16][2][32];
    extern __shared__ float dw_rows[];                 // [R - 1][8 VPT G]
    after_previous();
    const int G = blockDim.x, g = threadIdx.y;
    const W* wt = static_cast<const W*>(a.weight);
    float* part = a.parts + (int64_t)blockIdx.x * a.H;
    constexpr int N = VPT > 0 ? VPT : 1;
    F2 dw[N][4];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) dw[i][j] = f2(0.f, 0.f);
    const int H = (int)a.H, step = 8 * G;
    const int64_t first = (int64_t)blockIdx.x * blockDim.y + g;
    int turn = 0;
    auto load = [&](const T* p, int c, const void* base, int64_t ld) {
        if (VEC) return c < H ? load8_all<T>(p + c) : Raw8<T>{};
        const T* begin = static_cast<const T*>(base);
        return c + 8 <= H ? load8_near<T>(p + c, begin, begin + (a.T - 1) * ld + H) : c < H ? load8<T, false>(p + c, H - c) : Raw8<T>{};
    };
    auto weights = [&](int c, F2 (&w)[4]) {
        if (VEC || c < H) pairs8<W>(weight_at<W, VEC>(wt, c, H), w);
        else w[0] = w[1] = w[2] = w[3] = 0;
    };

    for (int64_t t = first; t < a.T; t += (int64_t)gridDim.x * blockDim.y, turn ^= 1) {
        const T* dy = static_cast<const T*>(a.dy) + t * a.lddy;
        const T* h = static_cast<const T*>(a.h) + t * a.ldh;
        const T* dh = a.dh ? static_cast<const T*>(a.dh) + t * a.lddh : nullptr;
        T* dx = static_cast<T*>(a.dx) + t * a.lddx;
        const float s = a.rstd[t];
        auto dot8 = [&](int c, const Raw8<T>& rdy, const Raw8<T>& rh, F2 sum) {
            F2 fy[4], fh[4], w[4];
            pairs8<T>(rdy, fy);
            pairs8<T>(rh, fh);
            weights(c, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) sum = fma2(mul2(fy[j], w[j]), fh[j], sum);
            return sum;
        };
        auto write = [&](int c, const Raw8<T>& rdy, const Raw8<T>& rh, const Raw8<T>& rdh, float k, F2 (&acc)[4]) {
            F2 fy[4], fh[4], fd[4], w[4];
            pairs8<T>(rdy, fy);
            pairs8<T>(rh, fh);
            pairs8<T>(rdh, fd);
            weights(c, w);
            const F2 ss = f2(s, s), mk = f2(-k, -k);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                acc[j] = fma2(mul2(fy[j], ss), fh[j], acc[j]);
                fd[j] = fma2(ss, fma2(fh[j], mk, mul2(fy[j], w[j])), fd[j]);
            }
            float o[8];
            floats8(fd, o);
            if (!VEC) store8_near<T>(dx + c, o, H - c);        // every lane of the warp gets here
            else store8<T, true>(dx + c, o, 8);
        };
        F2 sum = f2(0.f, 0.f);
        if constexpr (VPT > 0) {
            Raw8<T> rdy[VPT], rh[VPT], rdh[VPT];
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int c = 8 * (threadIdx.x + i * G);
                rdy[i] = load(dy, c, a.dy, a.lddy);
                rh[i] = load(h, c, a.h, a.ldh);
                rdh[i] = dh ? load(dh, c, a.dh, a.lddh) : Raw8<T>{};
            }
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int c = 8 * (threadIdx.x + i * G);
                if (!VEC || c < H) sum = dot8(c, rdy[i], rh[i], sum);
            }
            const float2 p = f2(sum);
            const float k = s * s * (row_sum(p.x + p.y, G, g, scratch[g][turn]) / (float)H);
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int c = 8 * (threadIdx.x + i * G);
                if (!VEC || c < H) write(c, rdy[i], rh[i], rdh[i], k, dw[i]);
            }
        } else {
            const int rounds = (H + step - 1) / step;
            for (int i = 0; i < rounds; ++i) {
                const int c = 8 * threadIdx.x + i * step;
                if (!VEC || c < H) sum = dot8(c, load(dy, c, a.dy, a.lddy), load(h, c, a.h, a.ldh), sum);
            }
            const float2 p = f2(sum);
            const float k = s * s * (row_sum(p.x + p.y, G, g, scratch[g][turn]) / (float)H);
            for (int i = 0; i < rounds; ++i) {
                const int c = 8 * threadIdx.x + i * step;
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = c + j < H && t != first ? part[c + j] : 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) dw[0][j] = f2(f[2 * j], f[2 * j + 1]);
                if (!VEC || c < H) write(c, load(dy, c, a.dy, a.lddy), load(h, c, a.h, a.ldh), dh ? load(dh, c, a.dh, a.lddh) : Raw8<T>{}, k, dw[0]);
                floats8(dw[0], f);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < H) part[c + j] = f[j];
            }
        }
    }
    if constexpr (VPT > 0) {
        // the R rows' shares in the order of the rows; [j][thread] keeps neighbouring threads in neighbouring banks
        float f[VPT][8];
#pragma unroll
        for (int i = 0; i < VPT; ++i) floats8(dw[i], f[i]);
        if (g > 0) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) dw_rows[((g - 1) * 8 * VPT + 8 * i + j) * G + threadIdx.x] = f[i][j];
        }
        __syncthreads();
        if (g > 0) return;
        for (int r = 1; r < (int)blockDim.y; ++r)
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) f[i][j] += dw_rows[((r - 1) * 8 * VPT + 8 * i + j) * G + threadIdx.x];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = 8 * (threadIdx.x + i * G);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j < H) part[c + j] = f[i][j];
        }
    }
}

// The same for rows off 16-byte boundaries, brought to shared memory by bulk copies, two rows ahead for each of the R rows
// at a time.  A row is copied in whole
// 16-byte pieces, from the boundary before its start to the one after its end, so its place may be any multiple of
// an element; every tensor starts on a boundary, a row has 64 bytes or more (so that only the last row's last piece can
// reach beyond the tensor), and what that piece would bring is loaded element by element.
// The bounded waits raise a status word (gpd_device_status) and skip what is left.
constexpr int kRing = 2, kRingThreads = 1024;
__device__ int g_norm_status = 0;
// room for a row from a boundary on, and for the last piece that a thread reads around its elements
__host__ __device__ constexpr int span_bytes(int64_t H, int e) { return (int)((H * e + 15) / 16 + (e == 4 ? 2 : 1)) * 16; }

template <typename T, typename W, int VPT>
__global__ void __launch_bounds__(kRingThreads) rmsnorm_backward_ring_kernel(const NormBwdArgs a) {
    __shared__ float scratch[16][2][32];
    __shared__ __align__(8) uint64_t full[16][kRing];
    __shared__ int abort_flag;
    extern __shared__ __align__(16) uint8_t ring[];    // [R][kRing][3][span]; afterwards the rows' shares of dw
    const int G = blockDim.x, g = threadIdx.y, H = (int)a.H, span = span_bytes(H, sizeof(T));
    const W* wt = static_cast<const W*>(a.weight);
    const int64_t stride = (int64_t)gridDim.x * blockDim.y, first = (int64_t)blockIdx.x * blockDim.y + g;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kRing; ++i) tc::mbar_init(&full[g][i], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 0 && g == 0) abort_flag = 0;
    __syncthreads();
    after_previous();

    auto tensor = [&](int k) { return k == 0 ? a.dy : k == 1 ? a.h : a.dh; };
    auto ld_of = [&](int k) { return k == 0 ? a.lddy : k == 1 ? a.ldh : a.lddh; };
    auto buffer = [&](int i, int k) { return ring + ((size_t)((g * kRing + i) * 3 + k)) * span; };
    // first byte of a row, and the bytes that whole pieces bring from the boundary before it
    auto place = [&](int k, int64_t t, int& mis, int& bytes, bool& cut) {
        const int64_t at = t * ld_of(k) * (int64_t)sizeof(T);
        mis = (int)(at & 15);
        bytes = (mis + H * (int)sizeof(T) + 15) & ~15;
        cut = t == a.T - 1 && ((mis + H * (int)sizeof(T)) & 15) != 0;      // the last piece ends beyond the tensor
        if (cut) bytes -= 16;
        return static_cast<const uint8_t*>(tensor(k)) + at - mis;
    };
    auto send = [&](int64_t t, int i) {                // thread 0 of the row
        int mis, bytes, sum = 0;
        bool cut;
        for (int k = 0; k < (a.dh ? 3 : 2); ++k) {
            place(k, t, mis, bytes, cut);
            sum += bytes;
        }
        tc::mbar_expect_tx(&full[g][i], sum);
        for (int k = 0; k < (a.dh ? 3 : 2); ++k) {
            const uint8_t* src = place(k, t, mis, bytes, cut);
            if (bytes > 0)
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                             ::"r"(tc::smem_u32(buffer(i, k))), "l"(src), "r"(bytes), "r"(tc::smem_u32(&full[g][i])) : "memory");
        }
    };
    if (threadIdx.x == 0)
        for (int i = 0; i < kRing; ++i)
            if (first + i * stride < a.T) send(first + i * stride, i);

    F2 dw[VPT][4];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) dw[i][j] = f2(0.f, 0.f);
    auto group_sync = [&]() {
        if (G > 32) asm volatile("bar.sync %0, %1;" ::"r"(g + 1), "r"(G) : "memory");
        else __syncwarp();
    };
    int turn = 0, slot = 0;
    uint32_t phase = 0;
    bool live = true;
    int rows = 0, lost = 0;                            // rows so far; the one whose copies did not come
    for (int64_t t = first; t < a.T; t += stride, turn ^= 1, ++rows) {
        if (live && !tc::mbar_wait(&full[g][slot], phase, &abort_flag, &g_norm_status)) {
            live = false;
            lost = rows;
        }
        const T* at[3];                                // the row's first elements
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            int mis = 0, bytes = 0;
            bool cut = false;
            const uint8_t* src = k < 2 || a.dh ? place(k, t, mis, bytes, cut) : nullptr;
            at[k] = reinterpret_cast<const T*>(buffer(slot, k) + mis);
            if (cut) {                                 // what is left of the row, by the elements
                const int from = (bytes - mis) / (int)sizeof(T) > 0 ? (bytes - mis) / (int)sizeof(T) : 0;
                const T* row = reinterpret_cast<const T*>(src + mis);
                T* to = reinterpret_cast<T*>(buffer(slot, k) + mis);
                for (int j = from + threadIdx.x; j < H; j += G) to[j] = row[j];
            }
        }
        if (t == a.T - 1) group_sync();
        const float s = a.rstd[t];
        T* dx = static_cast<T*>(a.dx) + t * a.lddx;
        // eight elements from column c of a row in shared memory; pieces that surround them are inside the ring
        auto near = [&](const T* p, int c, F2 (&f)[4]) {
            const int mis = (int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
            if (mis == 0) {
                pairs8<T>(load8_all<T>(p + c), f);
            } else {
                const uint4* v = reinterpret_cast<const uint4*>(p + c - mis);
                const uint4 x = v[0], y = v[1];
                const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
                uint32_t o[4];
                Raw8<T> r;
                shifted4<T>(w, mis, o);
                r.v = make_uint4(o[0], o[1], o[2], o[3]);
                if constexpr (sizeof(T) == 4) {
                    const uint4 z = v[2];
                    const uint32_t u[8] = {y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
                    shifted4<T>(u, mis, o);
                    r.w = make_uint4(o[0], o[1], o[2], o[3]);
                }
                pairs8<T>(r, f);
            }
            if (c + 8 > H) {                           // columns beyond the row
                float q[8];
                floats8(f, q);
#pragma unroll
                for (int j = 0; j < 8; ++j) q[j] = c + j < H ? q[j] : 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) f[j] = f2(q[2 * j], q[2 * j + 1]);
            }
        };
        F2 sum = f2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = 8 * (threadIdx.x + i * G);
            if (c < H) {
                F2 fy[4], fh[4], w[4];
                near(at[0], c, fy);
                near(at[1], c, fh);
                pairs8<W>(weight_at<W, false>(wt, c, H), w);
#pragma unroll
                for (int j = 0; j < 4; ++j) sum = fma2(mul2(fy[j], w[j]), fh[j], sum);
            }
        }
        const float2 p = f2(sum);
        const float k = s * s * (row_sum(p.x + p.y, G, g, scratch[g][turn]) / (float)H);
        const F2 ss = f2(s, s), mk = f2(-k, -k);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = 8 * (threadIdx.x + i * G);
            float o[8];
            if (c < H) {
                F2 fy[4], fh[4], fd[4], w[4];
                near(at[0], c, fy);
                near(at[1], c, fh);
                if (a.dh) near(at[2], c, fd);
                else fd[0] = fd[1] = fd[2] = fd[3] = f2(0.f, 0.f);
                pairs8<W>(weight_at<W, false>(wt, c, H), w);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    dw[i][j] = fma2(mul2(fy[j], ss), fh[j], dw[i][j]);
                    fd[j] = fma2(ss, fma2(fh[j], mk, mul2(fy[j], w[j])), fd[j]);
                }
                floats8(fd, o);
            }
            store8_near<T>(dx + c, o, H - c);          // every lane of the warp
        }
        group_sync();                                  // the slot has been read
        if (threadIdx.x == 0 && live && t + kRing * stride < a.T) send(t + kRing * stride, slot);
        if (++slot == kRing) {
            slot = 0;
            phase ^= 1;
        }
    }
    if (!live && threadIdx.x == 0) {                   // copies still under way land before the CTA goes on, or time runs out
        for (int i = lost; i < lost + kRing && first + i * stride < a.T; ++i) {
            const long long t0 = clock64();
            while (!tc::mbar_try_wait(&full[g][i % kRing], (i / kRing) & 1) && clock64() - t0 < tc::kWaitCycles) {}
        }
    }
    // the R rows' shares in the order of the rows; [j][thread] keeps neighbouring threads in neighbouring banks
    float f[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i) floats8(dw[i], f[i]);
    __syncthreads();                                   // every copy that was sent for has been waited for by its row
    float* dw_rows = reinterpret_cast<float*>(ring);   // [R - 1][8 VPT G]
    if (g > 0) {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) dw_rows[((g - 1) * 8 * VPT + 8 * i + j) * G + threadIdx.x] = f[i][j];
    }
    __syncthreads();
    if (g > 0) return;
    float* part = a.parts + (int64_t)blockIdx.x * a.H;
    for (int r = 1; r < (int)blockDim.y; ++r)
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) f[i][j] += dw_rows[((r - 1) * 8 * VPT + 8 * i + j) * G + threadIdx.x];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int c = 8 * (threadIdx.x + i * G);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < H) part[c + j] = f[i][j];
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
    constexpr int e = sizeof(T), V = e == 4 ? 2 : 4;   // vectors per thread that fit in registers
    const int64_t vecs = (a.H + 7) / 8;
    constexpr int RV = V / 2;                          // of the ring kernel: twice the threads
    const bool bases = aligned(a.dy, 16) && aligned(a.h, 16) && aligned(a.dh, 16);
    // one CTA per SM: R rows of G threads at a time, as many as it takes for T rows
    const int room = 220 * 1024 / (3 * kRing * span_bytes(std::min<int64_t>(a.H, 1 << 20), e));
    const bool vec = a.H % 8 == 0 && rows_aligned(a.dy, a.lddy, e) && rows_aligned(a.h, a.ldh, e) && rows_aligned(a.dh, a.lddh, e) &&
                     rows_aligned(a.dx, a.lddx, e) && aligned(a.weight, 16);
    // rows on boundaries: registers (4000 x 4096 BF16: 37 us, through the ring 51); off them: the ring (4000 x 4133: 69 us,
    // from registers 114), where it has room and is allowed; long rows: read twice
    const bool ring = !vec && bases && a.H * e >= 64 && vecs <= kRingThreads * RV && room > 0, loop = !ring && vecs > kBwdThreads * V;
    const int per = ring ? RV : V, G = loop ? 1024 : (int)(((vecs + per - 1) / per + 31) / 32 * 32);
    int R = loop ? 1 : std::max(1, std::min((ring ? kRingThreads : kBwdThreads) / G, 15));      // named barriers 1 .. 15
    if (ring) R = std::min(R, room);
    R = (int)std::max<int64_t>(1, std::min<int64_t>(R, (a.T + sm_count() - 1) / sm_count()));
    const int parts = (int)std::min<int64_t>(std::min<int64_t>((a.T + R - 1) / R, sm_count()), GPD_RMSNORM_MAX_PARTS);
    if (parts > 0) {
        const int shares = (R - 1) * 8 * per * G * (int)sizeof(float);  // at most 64 KB
        gpd_status rc;
        if (loop) {
            rc = launch_after(vec ? rmsnorm_backward_kernel<T, W, 0, true> : rmsnorm_backward_kernel<T, W, 0, false>, dim3(parts),
                              dim3(1024), 0, 1, st, a);
        } else {
            const int smem = ring ? std::max(shares, R * 3 * kRing * span_bytes(a.H, e)) : shares;
            auto kernel = ring ? rmsnorm_backward_ring_kernel<T, W, RV>
                          : vec ? rmsnorm_backward_kernel<T, W, V, true> : rmsnorm_backward_kernel<T, W, V, false>;
            if (smem > 40960 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
                return GPD_ERR_CUDA;
            rc = launch_after(kernel, dim3(parts), dim3(G, R), smem, 1, st, a);
        }
        if (rc != GPD_OK) return rc;
    }
    const float* partial = a.parts;
    return launch_after(rmsnorm_dweight_kernel, dim3((unsigned)((a.H + 31) / 32)), dim3(32, 16), 0, 1, st, partial, parts, a.H, dweight);
}

}  // namespace

int norm_device_status_fetch_and_clear() {
    int v = 0, zero = 0;
    if (cudaMemcpyFromSymbol(&v, g_norm_status, sizeof(int)) != cudaSuccess) return (int)GPD_ERR_CUDA;
    if (v != 0) cudaMemcpyToSymbol(g_norm_status, &zero, sizeof(int));
    return v;
}

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
