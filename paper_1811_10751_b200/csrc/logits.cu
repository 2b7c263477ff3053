// Operators on rows of logits (T tokens, V entries): log probabilities of given tokens with entropy and top
// alternatives, their gradient, and distillation from a teacher's top logits (loss and gradient).
//
// With z = x / tau, m = max x, k = log2(e) / tau:
//   S = sum_v 2^(k (x_v - m)),   U = sum_v 2^(k (x_v - m)) (x_v - m)
//   lse = m / tau + ln S,  log p_v = (x_v - m) / tau - ln S,  entropy = ln S - U / (S tau)
// in one pass that keeps the running maximum and rescales S and U when it rises (FP32).  Partial results of
// threads, warps and CTAs are merged by the same rule in a fixed order.
//
// HBM's 2 or 4 bytes per entry and the issue of instructions are close to each other, so FP32 arithmetic is done on
// pairs (add / mul / fma.f32x2), maxima of 16-bit entries are taken two at a time and a thread rescales its sums
// once per 64 bytes at most: about four instructions per entry, one of them a 2^x.  A row is
// read by one CTA, or, when there are too few rows to fill the GPU, by the CTAs of a cluster, whose partial
// results meet in distributed shared memory: one launch and no workspace either way.
//
// Measured: distillation step of 4096 x 128000 BF16 448-468 us (reads and writes at 0.70 of the copy bandwidth; passes
// over a row alternate between reading HBM and writing it), log probabilities and gradient of 2048 x 50257 BF16
// 129-135 us, of that the forward pass 54 us with the entropy asked for or not, 16 x 128000 FP32 with 20 alternatives
// 11.8 us (latency; 54 us where only ten entries of a row are not masked, as every entry is then a candidate),
// 61 x 32000 BF16 loss 5.5 us.
//
// Special values.  -inf is an ordinary mask (probability 0); a row of -inf alone has lse -inf, entropy 0,
// log probabilities -inf, distillation loss inf and gradient 0.  A NaN or +inf makes its row's lse, log probabilities, entropy,
// loss and gradient NaN.
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "lm_common.h"

namespace gpd {

namespace {

using namespace lm;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxTop = GPD_LOGPROBS_MAX_TOP, kMaxTokens = GPD_LOGPROBS_MAX_TOKENS, kMaxTeacher = GPD_DISTILL_MAX_TOP;
constexpr int kCand = 512;                             // candidates for the top entries kept by a CTA
constexpr int kMaxThreads = 512;

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ F2 ex2_pair(F2 a) {
    const float2 x = f2(a);
    return f2(ex2(x.x), ex2(x.y));
}

// Sixteen bytes of a row: its N entries as pairs, their extremes, and what stands for no entry
template <typename T> struct Piece {
    static constexpr int N = 8;
    static __device__ __forceinline__ uint32_t word(const uint4& r, int i) { return i == 0 ? r.x : i == 1 ? r.y : i == 2 ? r.z : r.w; }
    static __device__ __forceinline__ F2 pair(const uint4& r, int i) {
        const float2 f = unpack2(word(r, i), T());
        return f2(f.x, f.y);
    }
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b);
    static __device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b);
    static __device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b);
    static constexpr uint32_t kNone = std::is_same<T, __half>::value ? 0xfc00fc00u : 0xff80ff80u;      // -inf, -inf
};
#define GPD_PAIR_OP(T, T2, name, op)                                                                            \
    template <> __device__ __forceinline__ uint32_t Piece<T>::name(uint32_t a, uint32_t b) {                    \
        const T2 r = op(*reinterpret_cast<const T2*>(&a), *reinterpret_cast<const T2*>(&b));                    \
        return *reinterpret_cast<const uint32_t*>(&r);                                                          \
    }
GPD_PAIR_OP(__nv_bfloat16, __nv_bfloat162, max2, __hmax2)
GPD_PAIR_OP(__nv_bfloat16, __nv_bfloat162, max2_nan, __hmax2_nan)
GPD_PAIR_OP(__nv_bfloat16, __nv_bfloat162, min2, __hmin2)
GPD_PAIR_OP(__half, __half2, max2, __hmax2)
GPD_PAIR_OP(__half, __half2, max2_nan, __hmax2_nan)
GPD_PAIR_OP(__half, __half2, min2, __hmin2)
#undef GPD_PAIR_OP
template <> struct Piece<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ uint32_t word(const uint4& r, int i) { return i == 0 ? r.x : i == 1 ? r.y : i == 2 ? r.z : r.w; }
    static __device__ __forceinline__ F2 pair(const uint4& r, int i) {
        return i == 0 ? f2(__uint_as_float(r.x), __uint_as_float(r.y)) : f2(__uint_as_float(r.z), __uint_as_float(r.w));
    }
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
    static __device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
        float r;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)));
        return __float_as_uint(r);
    }
    static __device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) { return __float_as_uint(fminf(__uint_as_float(a), __uint_as_float(b))); }
    static constexpr uint32_t kNone = 0xff800000u;
};
// The value in the two halves of a word (16-bit entries), or the word's own
template <typename T> __device__ __forceinline__ float2 halves(uint32_t w) { return unpack2(w, T()); }
template <> __device__ __forceinline__ float2 halves<float>(uint32_t w) { return make_float2(__uint_as_float(w), __uint_as_float(w)); }
template <typename T, int U> __device__ __forceinline__ float top_of(const uint4 (&r)[U]) {
    uint32_t m = Piece<T>::kNone;
#pragma unroll
    for (int j = 0; j < U; ++j) m = Piece<T>::max2(m, Piece<T>::max2(Piece<T>::max2(r[j].x, r[j].y), Piece<T>::max2(r[j].z, r[j].w)));
    const float2 f = halves<T>(m);
    return fmaxf(f.x, f.y);
}
template <typename T, int U> __device__ __forceinline__ float bottom_of(const uint4 (&r)[U]) {
    uint32_t m = r[0].x;
#pragma unroll
    for (int j = 0; j < U; ++j) m = Piece<T>::min2(m, Piece<T>::min2(Piece<T>::min2(r[j].x, r[j].y), Piece<T>::min2(r[j].z, r[j].w)));
    const float2 f = halves<T>(m);
    return fminf(f.x, f.y);
}

struct Stats { float m, s, u; };
__device__ __forceinline__ Stats no_stats() { return Stats{-FLT_MAX, 0.f, 0.f}; }
__device__ __forceinline__ Stats merge(const Stats& a, const Stats& b, float k) {
    Stats r;
    r.m = fmaxf(a.m, b.m);
    const float da = a.m - r.m, db = b.m - r.m, fa = ex2(k * da), fb = ex2(k * db);   // 1 for the larger one
    r.s = a.s * fa + b.s * fb;
    r.u = (fa > 0.f ? fa * fmaf(da, a.s, a.u) : 0.f) + (fb > 0.f ? fb * fmaf(db, b.s, b.u) : 0.f);
    return r;
}

// The entries [v0, v1) of a row in 16-byte pieces, the first and last ones short where the row is not aligned.
// `start` sends for the first U pieces of every thread, so that they arrive during other work.  `run` calls
// batch(index of the first entry, entries between pieces, pieces there, raw[U]) for U pieces at a time, the next ones
// on their way, and some(index, raw, n) for the n entries of a short piece; what is not there reads as -inf.
// LAST: the entries are not read again.
template <typename T, int U>
struct Pieces {
    static constexpr int N = Piece<T>::N;
    const T* row = nullptr;
    int v0 = 0, v1 = 0, a0 = 0, pieces = 0;
    uint4 next[U];

    template <bool LAST>
    __device__ __forceinline__ void send(int i) {
        constexpr uint32_t none = Piece<T>::kNone;
        const uint4* p = reinterpret_cast<const uint4*>(row + a0) + i;
        const int step = blockDim.x;
        if (i + (U - 1) * step < pieces) {
#pragma unroll
            for (int j = 0; j < U; ++j) next[j] = LAST ? __ldcs(p + j * step) : p[j * step];
        } else {
#pragma unroll
            for (int j = 0; j < U; ++j) {
                next[j] = make_uint4(none, none, none, none);
                if (i + j * step < pieces) next[j] = LAST ? __ldcs(p + j * step) : p[j * step];
            }
        }
    }
    template <bool LAST>
    __device__ __forceinline__ void start(const T* r, int from, int to) {
        row = r;
        v0 = from;
        v1 = to;
        const int mis = (int)((reinterpret_cast<uintptr_t>(row + v0) & 15) / sizeof(T));
        a0 = min(v1, mis ? v0 + N - mis : v0);
        pieces = (v1 - a0) / N;
        send<LAST>(threadIdx.x);
    }
    template <bool LAST, typename B, typename S>
    __device__ __forceinline__ void run(B batch, S some) {
        constexpr uint32_t none = Piece<T>::kNone;
        const int a1 = a0 + pieces * N, step = blockDim.x;
        auto shorter = [&](int b, int n) {             // fewer than N entries
            uint32_t w[4] = {none, none, none, none};
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (j < n) {
                    if constexpr (sizeof(T) == 4) {
                        w[j] = __float_as_uint(row[b + j]);
                    } else {
                        const uint32_t v = reinterpret_cast<const unsigned short*>(row)[b + j];
                        w[j >> 1] = j & 1 ? (w[j >> 1] & 0xffffu) | v << 16 : (w[j >> 1] & 0xffff0000u) | v;
                    }
                }
            some(b, make_uint4(w[0], w[1], w[2], w[3]), n);
        };
        if (threadIdx.x == 0 && a0 > v0) shorter(v0, a0 - v0);
        if (threadIdx.x == blockDim.x - 1 && v1 > a1) shorter(a1, v1 - a1);
        for (int i = threadIdx.x; i < pieces; i += U * step) {
            uint4 r[U];
#pragma unroll
            for (int j = 0; j < U; ++j) r[j] = next[j];
            if (i + U * step < pieces) send<LAST>(i + U * step);
            batch(a0 + i * N, step * N, (pieces - i + step - 1) / step, r);
        }
    }
};

// Sixteen bytes that are not read again soon
template <typename T>
__device__ __forceinline__ void store_piece(T* p, const float (&o)[8]) {
    if constexpr (sizeof(T) == 4) __stcs(reinterpret_cast<float4*>(p), make_float4(o[0], o[1], o[2], o[3]));
    else __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack2(o[0], o[1], T()), pack2(o[2], o[3], T()), pack2(o[4], o[5], T()), pack2(o[6], o[7], T())));
}

// Gradient of a row or a part of it: value(pair of entries), stored where the pair stands in d.
template <typename T, int U, typename V>
__device__ __forceinline__ void write_gradient(Pieces<T, U>& in, T* d, V value) {
    constexpr int N = Piece<T>::N;
    const bool same = ((reinterpret_cast<uintptr_t>(in.row + in.v0) ^ reinterpret_cast<uintptr_t>(d + in.v0)) & 15) == 0;
    auto store = [&](const uint4& r, int b, int n) {
        float o[8];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const float2 f = f2(value(Piece<T>::pair(r, i)));
            o[2 * i] = f.x;
            o[2 * i + 1] = f.y;
        }
        if (n == N && same) {
            store_piece<T>(d + b, o);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (j < n) d[b + j] = from_f32<T>(o[j]);
        }
    };
    in.template run<true>(
        [&](int b, int step, int n, const uint4 (&r)[U]) {
#pragma unroll
            for (int j = 0; j < U; ++j)
                if (j < n) store(r[j], b + j * step, N);
        },
        [&](int b, const uint4& r, int n) { store(r, b, n); });
}

template <typename T, bool ENTROPY, bool LAST, int U>
__device__ __forceinline__ Stats thread_stats(Pieces<T, U>& in, float k) {
    float m = -FLT_MAX;
    F2 s = f2(0.f, 0.f), u = f2(0.f, 0.f);
    const F2 kk = f2(k, k);
    auto take = [&](const auto& r) {
        const float top = top_of<T>(r);
        if (top > m) {
            const float d = m - top, f = ex2(k * d);
            if (ENTROPY) u = f > 0.f ? mul2(f2(f, f), fma2(f2(d, d), s, u)) : f2(0.f, 0.f);
            s = mul2(f2(f, f), s);
            m = top;
        }
        // k (x - m), not k x - k m, which is infinity less infinity for large logits
        const F2 mm = f2(-m, -m);
        const bool masked = ENTROPY && bottom_of<T>(r) - m == -INFINITY;       // -inf, or too far below m for FP32
#pragma unroll
        for (int j = 0; j < (int)(sizeof(r) / sizeof(r[0])); ++j)
#pragma unroll
            for (int i = 0; i < Piece<T>::N / 2; ++i) {
                F2 d = add2(Piece<T>::pair(r[j], i), mm);
                const F2 e = ex2_pair(mul2(d, kk));
                s = add2(s, e);
                if (ENTROPY) {
                    if (masked) {                      // 0 * -inf is not wanted
                        const float2 x = f2(d);
                        d = f2(fmaxf(x.x, -FLT_MAX), fmaxf(x.y, -FLT_MAX));
                    }
                    u = fma2(e, d, u);
                }
            }
    };
    in.template run<LAST>([&](int, int, int, const uint4 (&r)[U]) { take(r); },
                          [&](int, const uint4& p, int) {
                              const uint4 r[1] = {p};
                              take(r);
                          });
    const float2 fs = f2(s), fu = f2(u);
    return Stats{m, fs.x + fs.y, fu.x + fu.y};
}

__device__ __forceinline__ Stats warp_merge(Stats st, float k) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const Stats b{__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o), __shfl_xor_sync(0xffffffffu, st.u, o)};
        st = merge(st, b, k);
    }
    return st;
}
// Over the CTA; every thread gets the result.  `scratch`: a Stats per warp.
__device__ __forceinline__ Stats block_merge(Stats st, float k, Stats* scratch) {
    st = warp_merge(st, k);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = blockDim.x >> 5;
    if (lane == 0) scratch[warp] = st;
    __syncthreads();
    st = warp_merge(lane < n ? scratch[lane] : no_stats(), k);
    __syncthreads();
    return st;
}

// ---- clusters ------------------------------------------------------------------------------------------
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_here() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_all_here() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t peer_addr(const void* p, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ void to_peer(float* p, uint32_t rank, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(peer_addr(p, rank)), "f"(v) : "memory");
}
__device__ __forceinline__ void to_peer(uint64_t* p, uint32_t rank, uint64_t v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(peer_addr(p, rank)), "l"(v) : "memory");
}
// Results of the C CTAs of a row meet: each writes its own into the others' shared memory, slot by rank, so that one
// barrier is enough and nobody's shared memory is touched after it.  Before that all of them have to run: they arrive
// at a barrier when they start and wait for it when the first pass is over.
constexpr int kMaxSplit = 8;
__device__ __forceinline__ void to_peers(Stats* slots, int C, int rank, const Stats& st) {
    if ((int)threadIdx.x < C) {
        to_peer(&slots[rank].m, threadIdx.x, st.m);
        to_peer(&slots[rank].s, threadIdx.x, st.s);
        to_peer(&slots[rank].u, threadIdx.x, st.u);
    }
}
__device__ __forceinline__ Stats from_peers(const Stats* slots, int C, float k) {
    const int lane = threadIdx.x & 31;
    return warp_merge(lane < C ? slots[lane] : no_stats(), k);
}
// Part `rank` of C of a row, cut at multiples of eight entries.
__device__ __forceinline__ void slice(int V, int C, int rank, int& v0, int& v1) {
    const int n = ((V + C - 1) / C + 7) & ~7;
    v0 = min(V, rank * n);
    v1 = min(V, v0 + n);
}

__device__ __forceinline__ int64_t index_at(const void* p, int bytes, int64_t i) {
    return bytes == 8 ? static_cast<const int64_t*>(p)[i] : (int64_t) static_cast<const int32_t*>(p)[i];
}

// Log probability of an entry x; -inf where nothing is left.  From its distance to the maximum and not from lse, whose
// rounding goes by the size of the logits (3e-5 at 1000) and not of the result.
__device__ __forceinline__ float logp_of(const Stats& st, float x, float inv_tau, float log_s) {
    return st.s == 0.f ? -INFINITY : fmaf(x - st.m, inv_tau, -log_s);
}

// ---- top entries ---------------------------------------------------------------------------------------
// A key orders entries by value (NaN first), equal ones by their index: larger keys come first.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0xffffffffu;
    const uint32_t b = __float_as_uint(x + 0.f);       // one zero
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
    return o == 0xffffffffu ? __uint_as_float(0x7fc00000u) : __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint64_t key_of(float x, int v) { return (uint64_t)order_of(x) << 32 | (0xffffffffu - (uint32_t)v); }

struct __align__(16) TopShared {
    uint64_t cand[kCand];
    uint64_t top[kMaxTop];
    uint64_t from[kMaxSplit * kMaxTop];                // the lists of a row's CTAs
    int larger[kMaxSplit * kMaxTop];
    float maxima[32];
    uint32_t threshold;
    int count;
};

// The K largest of n <= kCand keys, in order, to sh.top (0: none); all threads.  A warp counts, for one key
// after another, how many are larger.
__device__ __forceinline__ void rank_top(TopShared& sh, const uint64_t* keys, int n, int K) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    if (threadIdx.x < K) sh.top[threadIdx.x] = 0;
    __syncthreads();
    const int rounds = (n + 31) >> 5;
    for (int i = warp; i < n; i += warps) {
        const uint64_t key = keys[i];
        int larger = 0;
#pragma unroll 2
        for (int j = 0; j < rounds; ++j) larger += 32 * j + lane < n && keys[32 * j + lane] > key;
        larger = __reduce_add_sync(0xffffffffu, larger);
        if (lane == 0 && larger < K && key) sh.top[larger] = key;
    }
    __syncthreads();
}

// The K largest of C ordered lists of K keys in sh.from (0: no key), in order, to sh.top; all threads.  A thread looks
// for one key's place in one list.
__device__ __forceinline__ void merge_top(TopShared& sh, int C, int K) {
    const int n = C * K;
    for (int i = threadIdx.x; i < n; i += blockDim.x) sh.larger[i] = 0;
    if (threadIdx.x < K) sh.top[threadIdx.x] = 0;
    __syncthreads();
    for (int task = threadIdx.x; task < n * C; task += blockDim.x) {
        const int i = task / C;
        const uint64_t key = sh.from[i], *list = sh.from + (task - i * C) * K;
        int lo = 0, hi = K;                            // the first entry that is not larger
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (list[mid] > key) lo = mid + 1;
            else hi = mid;
        }
        atomicAdd(&sh.larger[i], lo);                  // a count: any order will do
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x)
        if (sh.from[i] && sh.larger[i] < K) sh.top[sh.larger[i]] = sh.from[i];
    __syncthreads();
}

// The K largest entries of [v0, v1), in order, to sh.top.  `mine`: this thread's largest entry (-FLT_MAX: none).
// K entries are at least as large as the K-th largest of any set of entries, so the K-th largest among the
// largest 32 / warps thread maxima of every warp bounds the answer from below; what reaches the bound is
// gathered and ranked.  Where more reaches it than there is room for (many equal entries), each warp keeps
// a sorted list of 32 instead.
// `in` has been through the slice once; where its first pieces were all of them, they are still in registers.
template <typename T, int U>
__device__ void block_top(Pieces<T, U>& in, float mine, int K, TopShared& sh) {
    const T* row = in.row;
    const int v0 = in.v0, v1 = in.v1;
    constexpr int N = 16 / sizeof(T);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5, per = 32 / warps;
    float v = mine;                                    // sorted over the warp, largest first
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
        for (int o = size >> 1; o > 0; o >>= 1) {
            const float w = __shfl_xor_sync(0xffffffffu, v, o);
            const bool larger = ((lane & o) == 0) == ((lane & size) == 0 || size == 32);
            v = larger ? fmaxf(v, w) : fminf(v, w);
        }
    if (lane < per) sh.maxima[warp * per + lane] = v;
    if (threadIdx.x == 0) {
        sh.count = 0;
        sh.threshold = 0;
    }
    __syncthreads();
    if (warp == 0) {                                   // K <= 32 of 32
        const float x = sh.maxima[lane];
        int r = 0;
#pragma unroll 8
        for (int j = 0; j < 32; ++j) {
            const float y = __shfl_sync(0xffffffffu, x, j);
            r += y > x || (y == x && j < lane);
        }
        if (r == K - 1 && x > -FLT_MAX) sh.threshold = order_of(x);
    }
    __syncthreads();
    const float bound = sh.threshold ? value_of(sh.threshold) : -INFINITY;       // a NaN is not below it
    auto keep = [&](const uint4& r, int b, int n) {
        const float2 top = halves<T>(Piece<T>::max2_nan(Piece<T>::max2_nan(r.x, r.y), Piece<T>::max2_nan(r.z, r.w)));
        if (top.x < bound && top.y < bound) return;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float2 f = f2(Piece<T>::pair(r, j >> 1));
            const float x = j & 1 ? f.y : f.x;
            if (j < n && !(x < bound)) {
                const int at = atomicAdd(&sh.count, 1);        // any order: the ranks decide
                if (at < kCand) sh.cand[at] = key_of(x, b + j);
            }
        }
    };
    if (in.pieces > U * (int)blockDim.x) in.template start<true>(row, v0, v1);
    in.template run<true>(
        [&](int b, int step, int n, const uint4 (&r)[U]) {
#pragma unroll
            for (int j = 0; j < U; ++j)
                if (j < n) keep(r[j], b + j * step, N);
        },
        [&](int b, const uint4& r, int n) { keep(r, b, n); });
    __syncthreads();
    int n = sh.count;
    if (n > kCand) {
        uint64_t best = 0;                             // the warp's list, lane 0 the largest
        const int per_warp = (v1 - v0 + warps - 1) / warps, w0 = v0 + warp * per_warp, w1 = min(v1, w0 + per_warp);
        for (int b = w0; b < w1; b += 32) {
            const uint64_t key = b + lane < w1 ? key_of(to_f32(row[b + lane]), b + lane) : 0;
            uint32_t todo = __ballot_sync(0xffffffffu, key > __shfl_sync(0xffffffffu, best, 31));
            while (todo) {
                const uint64_t x = __shfl_sync(0xffffffffu, key, __ffs(todo) - 1);
                todo &= todo - 1;
                const int at = __popc(__ballot_sync(0xffffffffu, best > x));
                const uint64_t up = __shfl_up_sync(0xffffffffu, best, 1);
                best = lane < at ? best : lane == at ? x : up;
            }
        }
        sh.cand[threadIdx.x] = best;
        n = blockDim.x;
        __syncthreads();
    }
    rank_top(sh, sh.cand, n, K);
}

// ---- log probabilities -----------------------------------------------------------------------------------
struct LogprobArgs {
    const void* logits; int64_t ld;
    const void* tokens; int index_bytes;
    float *logprobs, *lse, *entropy;
    int32_t* top_ids; float* top_logprobs;
    int64_t T;
    int V, G, K;
    float inv_tau;
};

// C CTAs per row (gridDim.x = C, a cluster); the rows blockIdx.y, blockIdx.y + gridDim.y, ...
template <typename T, bool TOP>
__global__ void __launch_bounds__(kMaxThreads, 2) logprobs_kernel(const LogprobArgs a) {
    __shared__ Stats scratch[32], slots[kMaxSplit];
    __shared__ typename std::conditional<TOP, TopShared, int>::type top;
    after_previous();
    const int C = gridDim.x, rank = blockIdx.x;
    const float k = kLog2e * a.inv_tau;
    int v0, v1;
    slice(a.V, C, rank, v0, v1);
    Pieces<T, 4> in;
    for (int64_t t = blockIdx.y; t < a.T; t += gridDim.y) {
        const T* row = static_cast<const T*>(a.logits) + t * a.ld;
        in.template start<!TOP>(row, v0, v1);
        if (C > 1) cluster_here();                     // one row per cluster then
        // this thread's token and its logit arrive during the pass
        int64_t token = -1;
        float x_token = 0.f;
        if (rank == 0 && (int)threadIdx.x < a.G) {
            token = index_at(a.tokens, a.index_bytes, t * a.G + threadIdx.x);
            if (token >= 0 && token < a.V) x_token = to_f32(row[token]);
        }
        Stats st = thread_stats<T, true, !TOP>(in, k);
        const float mine = st.m;
        st = block_merge(st, k, scratch);
        if constexpr (TOP) block_top(in, mine, a.K, top);
        if (C > 1) {
            cluster_all_here();
            to_peers(slots, C, rank, st);
            if constexpr (TOP) {
                if ((int)threadIdx.x < a.K) to_peer(&top.from[rank * a.K + threadIdx.x], 0, top.top[threadIdx.x]);
            }
            cluster_sync_all();
            if (rank != 0) return;
            st = from_peers(slots, C, k);
            if constexpr (TOP) merge_top(top, C, a.K);
        }
        const float log_s = logf(st.s);
        if (threadIdx.x == 0) {
            a.lse[t] = st.s == 0.f ? -INFINITY : fmaf(st.m, a.inv_tau, log_s);
            if (a.entropy) a.entropy[t] = st.s == 0.f ? 0.f : log_s - st.u / st.s * a.inv_tau;
        }
        if ((int)threadIdx.x < a.G) {                  // at most 64, fewer than there are threads
            float lp = 0.f;
            if (token >= a.V) lp = __uint_as_float(0x7fc00000u);
            else if (token >= 0) lp = logp_of(st, x_token, a.inv_tau, log_s);
            a.logprobs[t * a.G + threadIdx.x] = lp;
        }
        if constexpr (TOP) {
            if (threadIdx.x < a.K) {
                const uint64_t key = top.top[threadIdx.x];
                a.top_ids[t * a.K + threadIdx.x] = (int32_t)(0xffffffffu - (uint32_t)key);
                if (a.top_logprobs)
                    a.top_logprobs[t * a.K + threadIdx.x] = logp_of(st, value_of((uint32_t)(key >> 32)), a.inv_tau, log_s);
            }
        }
        if (TOP) __syncthreads();                      // `top` is taken up again
    }
}

// d[v] = (1/tau) [ p_v (c - gH (log p_v + H)) + sum_{i: token_i = v} g_i ],  c = -sum_i g_i
struct LogprobBwdArgs {
    const void* logits; int64_t ld;
    const void* tokens; int index_bytes;
    const float *lse, *entropy, *dlogprobs, *dentropy;
    void* d; int64_t ldd;
    int V, G, parts;
    float inv_tau;
};

// Log probabilities below this one are taken for it: 2^x of them is 0, and p (log p + H) g has to be 0 there for every g
// in use, so log p g may not overflow (a masked entry's log p is -inf, or -3e38 under a mask of the lowest value).
constexpr float kLeastLogp = -1024.f;

template <typename T>
__global__ void __launch_bounds__(kMaxThreads, 2) logprobs_backward_kernel(const LogprobBwdArgs a) {
    __shared__ float g[kMaxTokens], x_at[kMaxTokens];
    __shared__ int at[kMaxTokens];
    after_previous();
    const int64_t t = blockIdx.x / a.parts;
    const T* row = static_cast<const T*>(a.logits) + t * a.ld;
    T* d = static_cast<T*>(a.d) + t * a.ldd;
    int v0, v1;
    slice(a.V, a.parts, (int)(blockIdx.x % a.parts), v0, v1);
    Pieces<T, 4> in;
    in.template start<true>(row, v0, v1);
    // the logits at the tokens first: d may be the logits' own buffer
    for (int i = threadIdx.x; i < a.G; i += blockDim.x) {
        const int64_t v = index_at(a.tokens, a.index_bytes, t * a.G + i);
        const bool ok = v >= 0 && v < a.V;
        at[i] = ok ? (int)v : -1;
        g[i] = ok && a.dlogprobs ? a.dlogprobs[t * a.G + i] : 0.f;
        x_at[i] = ok && v >= v0 && v < v1 ? to_f32(row[v]) : 0.f;
    }
    __syncthreads();
    const float lse = a.lse[t], gh = a.dentropy ? a.dentropy[t] : 0.f;
    float c = 0.f;
    for (int i = 0; i < a.G; ++i) c -= g[i];
    if (a.dentropy) c -= gh * a.entropy[t];
    const bool none = lse == -INFINITY;
    auto dp = [&](float x) {                           // at a token, without its own term
        const float logp = fmaf(x, a.inv_tau, -lse), p = ex2(logp * kLog2e);
        return none ? 0.f : p * fmaf(-gh, fmaxf(logp, kLeastLogp), c) * a.inv_tau;
    };
    const F2 it = f2(a.inv_tau, a.inv_tau), ml = f2(-lse, -lse), l2e = f2(kLog2e, kLog2e), mg = f2(-gh * a.inv_tau, -gh * a.inv_tau),
             cc = f2(c * a.inv_tau, c * a.inv_tau);
    if (none) {
        write_gradient(in, d, [&](F2) { return f2(0.f, 0.f); });
    } else if (a.dentropy) {
        write_gradient(in, d, [&](F2 x) {
            const F2 logp = fma2(x, it, ml);
            const float2 l = f2(logp);
            return mul2(ex2_pair(mul2(logp, l2e)), fma2(mg, f2(fmaxf(l.x, kLeastLogp), fmaxf(l.y, kLeastLogp)), cc));
        });
    } else {
        write_gradient(in, d, [&](F2 x) { return mul2(ex2_pair(mul2(fma2(x, it, ml), l2e)), cc); });
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.G; i += blockDim.x) {
        if (at[i] < v0 || at[i] >= v1) continue;
        float s = 0.f;                                 // a token named twice: its first holder writes the sum
        int first = i;
        for (int j = a.G - 1; j >= 0; --j)
            if (at[j] == at[i]) {
                s += g[j];
                first = j;
            }
        if (first == i) d[at[i]] = from_f32<T>(none ? 0.f : fmaf(s, a.inv_tau, dp(x_at[i])));
    }
}

// ---- distillation ------------------------------------------------------------------------------------------
struct DistillArgs {
    const void* logits; int64_t ld;
    const void* ids; int index_bytes; int64_t ldi;
    const void* teacher; int64_t ldt; int teacher_type;
    const float* weights;
    float* loss;
    void* d; int64_t ldd;
    int64_t T;
    int V, K;
    float tau;
};

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float teacher_at(const DistillArgs& a, int64_t t, int i) {
    const int64_t j = t * a.ldt + i;
    return a.teacher_type == GPD_DT_F32    ? static_cast<const float*>(a.teacher)[j]
           : a.teacher_type == GPD_DT_BF16 ? to_f32(static_cast<const __nv_bfloat16*>(a.teacher)[j])
                                           : to_f32(static_cast<const __half*>(a.teacher)[j]);
}

// A row's list in shared memory: the teacher's logits (-inf: does not count), the student's there, and the
// entries (kAbsent: none, kBeyond: an id >= V); filled up to a multiple of four.
constexpr int kAbsent = -1, kBeyond = -2;
struct __align__(16) TeacherList {
    int at[kMaxTeacher];
    float t[kMaxTeacher], x[kMaxTeacher];
};

// C CTAs per row (gridDim.x = C, a cluster); the rows blockIdx.y, blockIdx.y + gridDim.y, ...  A row passes from HBM
// to the first pass and from L2 to the second, which writes the gradient.
template <typename T>
__global__ void __launch_bounds__(kMaxThreads, 2) distill_kernel(const DistillArgs a) {
    __shared__ Stats scratch[32], slots[kMaxSplit];
    // In turn, so that a row's last readers need no barrier: the next row that fills a list takes the other one and passes
    // block_merge, which all threads reach only after them.  Rows without weight pass no barrier and take no turn.
    __shared__ TeacherList lists[2];
    after_previous();
    const int C = gridDim.x, rank = blockIdx.x, lane = threadIdx.x & 31;
    const float inv_tau = 1.f / a.tau, k = kLog2e * inv_tau;
    int v0, v1;
    slice(a.V, C, rank, v0, v1);
    Pieces<T, 4> in;
    int turn = 0;
    for (int64_t t = blockIdx.y; t < a.T; t += gridDim.y) {
        const T* row = static_cast<const T*>(a.logits) + t * a.ld;
        T* d = a.d ? static_cast<T*>(a.d) + t * a.ldd : nullptr;
        in.template start<false>(row, v0, v1);
        if (C > 1) cluster_here();                     // one row per cluster then
        const float wt = a.weights ? a.weights[t] : 1.f;
        // this thread's entry of the list arrives during the first pass
        int64_t id = 0;
        float te = 0.f;
        if (threadIdx.x < a.K) {
            id = index_at(a.ids, a.index_bytes, t * a.ldi + threadIdx.x);
            te = teacher_at(a, t, threadIdx.x);
        }
        TeacherList& list = lists[turn];
        auto nothing = [&]() {                         // loss and gradient 0
            if (rank == 0 && threadIdx.x == 0) a.loss[t] = 0.f;
            if (d)
                for (int v = v0 + threadIdx.x; v < v1; v += blockDim.x) d[v] = from_f32<T>(0.f);
        };
        if (wt == 0.f) {                               // the same in all parts
            if (C > 1) cluster_all_here();
            nothing();
            continue;
        }
        Stats st = thread_stats<T, false, false>(in, k);
        if (d) in.template start<true>(row, v0, v1);
        const int K4 = (a.K + 3) & ~3;
        for (int i = threadIdx.x; i < K4; i += blockDim.x) {
            const bool there = i < a.K;
            const int64_t v = !there ? -1 : i == threadIdx.x ? id : index_at(a.ids, a.index_bytes, t * a.ldi + i);
            const float x = !there ? 0.f : i == threadIdx.x ? te : teacher_at(a, t, i);
            const bool ok = v >= 0 && v < a.V;
            list.at[i] = ok ? (int)v : v < 0 ? kAbsent : kBeyond;
            list.t[i] = ok ? x : -INFINITY;
            list.x[i] = ok ? to_f32(row[v]) : 0.f;     // before d, perhaps the same buffer, is written
        }
        st = block_merge(st, k, scratch);              // its barriers publish the list
        turn ^= 1;
        if (C > 1) {
            cluster_all_here();
            to_peers(slots, C, rank, st);
            cluster_sync_all();
            st = from_peers(slots, C, k);
        }
        // the teacher's distribution, in every warp
        float tmax = -INFINITY, qs = 0.f;
        bool bad = false, beyond = false;              // a NaN, +inf or an id beyond the row: no distribution; such an id
        for (int i = lane; i < a.K; i += 32) {
            const float x = list.t[i];
            beyond = beyond || list.at[i] == kBeyond;
            bad = bad || !(x < INFINITY) || beyond;
            tmax = fmaxf(tmax, x);
        }
        bad = __any_sync(0xffffffffu, bad);
        beyond = __any_sync(0xffffffffu, beyond);
        tmax = warp_max(tmax);
        if (tmax == -INFINITY && !bad) {               // nothing in the list
            nothing();
            continue;
        }
        for (int i = lane; i < a.K; i += 32) qs += list.t[i] == -INFINITY ? 0.f : ex2(k * (list.t[i] - tmax));
        qs = warp_sum(qs);
        const bool none = st.s == 0.f && !bad;         // every logit of the row is masked
        if (rank == 0 && threadIdx.x < 32) {
            const float log_s = logf(st.s), log_qs = logf(qs);
            float l = 0.f;
            for (int i = lane; i < a.K; i += 32) {
                const float lq = (list.t[i] - tmax) * inv_tau - log_qs, q = list.t[i] == -INFINITY ? 0.f : ex2(lq * kLog2e);
                if (q > 0.f) l = fmaf(q, lq - ((list.x[i] - st.m) * inv_tau - log_s), l);
            }
            l = warp_sum(l);
            if (lane == 0) a.loss[t] = bad ? __uint_as_float(0x7fc00000u) : none ? INFINITY : wt * a.tau * a.tau * l;
        }
        if (d) {
            // the share of an id beyond the row has no place in d: all of it is NaN, like the loss
            const float scale = none ? 0.f : beyond ? __uint_as_float(0x7fc00000u) : wt * a.tau / st.s, m = st.m;
            const F2 mm = f2(-m, -m), kk = f2(k, k), sc = f2(scale, scale);
            write_gradient(in, d, [&](F2 x) { return mul2(sc, ex2_pair(mul2(add2(x, mm), kk))); });
            __syncthreads();
            for (int i = threadIdx.x; i < a.K; i += blockDim.x) {
                const int v = list.at[i];
                if (v < v0 || v >= v1) continue;
                float s = 0.f;                         // an entry named twice: its first holder writes the sum
                int first_at = i;
                for (int j = a.K - 1 & ~3; j >= 0; j -= 4) {
                    const int4 o = *reinterpret_cast<const int4*>(list.at + j);
                    const int four[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                    for (int u = 3; u >= 0; --u)
                        if (four[u] == v) {
                            s += list.t[j + u] == -INFINITY ? 0.f : ex2(k * (list.t[j + u] - tmax));
                            first_at = j + u;
                        }
                }
                if (first_at == i) d[v] = from_f32<T>(none ? 0.f : scale * ex2((list.x[i] - m) * k) - wt * a.tau * (s / qs));
            }
        }
    }
}

// ---- host side ---------------------------------------------------------------------------------------------
// CTAs per row: as many (up to 8) as the GPU has SMs for, while each still has 4096 entries to read.
int row_split(int64_t T, int64_t V) {
    int c = 1;
    while (c < kMaxSplit && T * c * 2 <= 2 * sm_count() && V / (2 * c) >= 4096) c *= 2;
    return c;
}
unsigned row_threads(int64_t entries) { return entries >= 8192 ? 512 : entries >= 4096 ? 256 : 128; }

// C CTAs for each of the rows.  (CTAs that stay and take row after row, their first pieces sent for in advance, were
// measured: 553 instead of 452 us for 4096 x 128000 BF16 with gradient, all SMs then read and write in step.)
template <typename... P, typename A>
gpd_status launch_rows(void (*kernel)(P...), const A& a, int64_t rows, int C, unsigned threads, cudaStream_t st) {
    return launch_after(kernel, dim3((unsigned)C, (unsigned)std::min<int64_t>(rows, 65535)), dim3(threads), 0, C, st, a);
}
template <typename T>
gpd_status launch_logprobs(const LogprobArgs& a, cudaStream_t st) {
    const int C = row_split(a.T, a.V);
    return launch_rows(a.K ? logprobs_kernel<T, true> : logprobs_kernel<T, false>, a, a.T, C, row_threads(a.V / C), st);
}
template <typename T>
gpd_status launch_logprobs_backward(LogprobBwdArgs a, int64_t rows, cudaStream_t st) {
    // no sums over the row, so any cut will do: enough CTAs for the GPU, each with 8192 entries or more
    const int64_t wanted = (4 * sm_count() + rows - 1) / rows;
    a.parts = (int)std::max<int64_t>(1, std::min<int64_t>((a.V + 8191) / 8192, wanted));
    if (rows * a.parts > 0x7fffffff) return GPD_ERR_SHAPE;
    return launch_after(logprobs_backward_kernel<T>, dim3((unsigned)(rows * a.parts)), dim3(row_threads(a.V / a.parts)), 0, 1, st, a);
}
template <typename T>
gpd_status launch_distill(const DistillArgs& a, cudaStream_t st) {
    const int C = row_split(a.T, a.V);
    return launch_rows(distill_kernel<T>, a, a.T, C, row_threads(a.V / C), st);
}

// log2(e) / tau multiplies differences of logits, 0 among them, so it has to be a number.
bool bad_temperature(float t) { return !(t > 0.f) || isinf(t) || isinf(kLog2e * (1.f / t)); }
bool bad_rows(int64_t T, int64_t V) { return T < 0 || V <= 0 || V > 0x40000000; }

}  // namespace

}  // namespace gpd

using namespace gpd;

extern "C" gpd_status gpd_token_logprobs(gpd_dtype type, const void* logits_dev, int64_t ld, int32_t index_bytes,
                                         const void* tokens_dev, int32_t G, float temperature, float* logprobs_dev,
                                         float* lse_dev, float* entropy_dev, int32_t K, int32_t* top_ids_dev,
                                         float* top_logprobs_dev, int64_t T, int64_t V, void* stream) {
    if (!is_float_type(type) || bad_temperature(temperature)) return GPD_ERR_ARG;
    if (bad_rows(T, V) || G < 0 || G > kMaxTokens || K < 0 || K > kMaxTop || K > V) return GPD_ERR_SHAPE;
    if (T == 0) return GPD_OK;                         // empty buffers may have no address
    if (!logits_dev || !lse_dev || (G > 0 && (!tokens_dev || !logprobs_dev || (index_bytes != 4 && index_bytes != 8))) ||
        (K > 0 && !top_ids_dev))
        return GPD_ERR_ARG;
    if (ld < V) return GPD_ERR_SHAPE;
    const LogprobArgs a{logits_dev, ld, tokens_dev, index_bytes, logprobs_dev, lse_dev, entropy_dev, top_ids_dev,
                        top_logprobs_dev, T, (int)V, G, K, 1.f / temperature};
    cudaStream_t st = as_stream(stream);
    if (type == GPD_DT_F32) return launch_logprobs<float>(a, st);
    if (type == GPD_DT_BF16) return launch_logprobs<__nv_bfloat16>(a, st);
    return launch_logprobs<__half>(a, st);
}

extern "C" gpd_status gpd_token_logprobs_backward(gpd_dtype type, const void* logits_dev, int64_t ld, int32_t index_bytes,
                                                  const void* tokens_dev, int32_t G, float temperature, const float* lse_dev,
                                                  const float* entropy_dev, const float* dlogprobs_dev,
                                                  const float* dentropy_dev, void* dlogits_dev, int64_t ldd, int64_t T,
                                                  int64_t V, void* stream) {
    if (!is_float_type(type) || bad_temperature(temperature)) return GPD_ERR_ARG;
    if (bad_rows(T, V) || G < 0 || G > kMaxTokens) return GPD_ERR_SHAPE;
    if (T == 0) return GPD_OK;
    if (!logits_dev || !lse_dev || !dlogits_dev || (dentropy_dev && !entropy_dev) ||
        (G > 0 && (!tokens_dev || (index_bytes != 4 && index_bytes != 8))))
        return GPD_ERR_ARG;
    if (ld < V || ldd < V) return GPD_ERR_SHAPE;
    const LogprobBwdArgs a{logits_dev, ld, tokens_dev, index_bytes, lse_dev, entropy_dev, dlogprobs_dev, dentropy_dev,
                           dlogits_dev, ldd, (int)V, G, 1, 1.f / temperature};
    cudaStream_t st = as_stream(stream);
    if (type == GPD_DT_F32) return launch_logprobs_backward<float>(a, T, st);
    if (type == GPD_DT_BF16) return launch_logprobs_backward<__nv_bfloat16>(a, T, st);
    return launch_logprobs_backward<__half>(a, T, st);
}

extern "C" gpd_status gpd_distill_topk(gpd_dtype type, const void* logits_dev, int64_t ld, int32_t index_bytes,
                                       const void* teacher_ids_dev, int64_t ldi, gpd_dtype teacher_type,
                                       const void* teacher_logits_dev, int64_t ldt, int32_t K, const float* weights_dev,
                                       float temperature, float* loss_dev, void* dlogits_dev, int64_t ldd, int64_t T,
                                       int64_t V, void* stream) {
    if (!is_float_type(type) || !is_float_type(teacher_type) || bad_temperature(temperature)) return GPD_ERR_ARG;
    if (bad_rows(T, V) || K < 0 || K > kMaxTeacher) return GPD_ERR_SHAPE;
    if (T == 0) return GPD_OK;
    if (!logits_dev || !loss_dev || (K > 0 && (!teacher_ids_dev || !teacher_logits_dev || (index_bytes != 4 && index_bytes != 8))))
        return GPD_ERR_ARG;
    if (ld < V || ldi < K || ldt < K || (dlogits_dev && ldd < V)) return GPD_ERR_SHAPE;
    const DistillArgs a{logits_dev, ld, teacher_ids_dev, index_bytes, ldi, teacher_logits_dev, ldt, teacher_type, weights_dev,
                        loss_dev, dlogits_dev, ldd, T, (int)V, K, temperature};
    cudaStream_t st = as_stream(stream);
    if (type == GPD_DT_F32) return launch_distill<float>(a, st);
    if (type == GPD_DT_BF16) return launch_distill<__nv_bfloat16>(a, st);
    return launch_distill<__half>(a, st);
}
