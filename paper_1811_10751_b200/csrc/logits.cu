// Operators on rows of logits (T tokens, V entries): log probabilities of given tokens with entropy and top
// alternatives, their gradient, and distillation from a teacher's top logits (loss and gradient).
//
// With z = x / tau, m = max x, k = log2(e) / tau:
//   S = sum_v 2^(k (x_v - m)),   U = sum_v 2^(k (x_v - m)) (x_v - m)
//   lse = m / tau + ln S,  log p_v = x_v / tau - lse,  entropy = ln S - U / (S tau)
// in one pass that keeps the running maximum and rescales S and U when it rises (FP32).  Partial results of
// threads, warps and CTAs are merged by the same rule in a fixed order.
//
// HBM bounds all of them: 2 or 4 bytes per entry against about six instructions, one of them a 2^x.  A row is
// read by one CTA, or, when there are too few rows to fill the GPU, by the CTAs of a cluster, whose partial
// results meet in distributed shared memory: one launch and no workspace either way.
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

// The entries [v0, v1) of a row in 16-byte pieces: `each(index, values, n)` with n entries, the first and
// last pieces short where the row is not aligned.
template <typename T, int UNROLL, typename F>
__device__ __forceinline__ void for_pieces(const T* row, int v0, int v1, F each) {
    constexpr int N = 16 / sizeof(T);
    const int mis = (int)((reinterpret_cast<uintptr_t>(row + v0) & 15) / sizeof(T));
    const int a0 = min(v1, mis ? v0 + N - mis : v0), pieces = (v1 - a0) / N, a1 = a0 + pieces * N;
    auto unpack = [&](const uint4& r, float (&f)[N]) {
        if constexpr (N == 4) {
            f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
        } else {
            unpack8<T>(Raw8<T>{r}, f);
        }
    };
    auto some = [&](int b, int n) {                    // fewer than N entries
        float f[N];
#pragma unroll
        for (int j = 0; j < N; ++j) f[j] = j < n ? to_f32(row[b + j]) : -INFINITY;
        each(b, f, n);
    };
    if (threadIdx.x == 0 && a0 > v0) some(v0, a0 - v0);
    if (threadIdx.x == blockDim.x - 1 && v1 > a1) some(a1, v1 - a1);
    // the next UNROLL pieces are on their way while the present ones are worked on
    const uint4* p = reinterpret_cast<const uint4*>(row + a0);
    const int step = blockDim.x;
    uint4 next[UNROLL];
    int i = threadIdx.x;
#pragma unroll
    for (int j = 0; j < UNROLL; ++j)
        if (i + j * step < pieces) next[j] = p[i + j * step];
    while (i < pieces) {
        uint4 r[UNROLL];
#pragma unroll
        for (int j = 0; j < UNROLL; ++j) r[j] = next[j];
        const int n = i + UNROLL * step;
#pragma unroll
        for (int j = 0; j < UNROLL; ++j)
            if (n + j * step < pieces) next[j] = p[n + j * step];
#pragma unroll
        for (int j = 0; j < UNROLL; ++j)
            if (i + j * step < pieces) {
                float f[N];
                unpack(r[j], f);
                each(a0 + (i + j * step) * N, f, N);
            }
        i = n;
    }
}

template <typename T, bool ENTROPY>
__device__ __forceinline__ Stats thread_stats(const T* row, int v0, int v1, float k) {
    constexpr int N = 16 / sizeof(T);
    Stats st = no_stats();
    for_pieces<T, 4>(row, v0, v1, [&](int, const float (&f)[N], int) {
        float top = f[0];
#pragma unroll
        for (int j = 1; j < N; ++j) top = fmaxf(top, f[j]);
        if (top > st.m) {
            st = merge(st, Stats{top, 0.f, 0.f}, k);
        }
        // k (x - m), not k x - k m: differences stay finite for logits of any size
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float d = f[j] - st.m, e = ex2(d * k);
            st.s += e;
            if (ENTROPY) st.u = fmaf(e, fmaxf(d, -FLT_MAX), st.u);         // 0 * -inf is not wanted
        }
    });
    return st;
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
__device__ __forceinline__ uint32_t peer_addr(const void* p, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ float peer_f32(const void* p, uint32_t rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(peer_addr(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ uint64_t peer_u64(const void* p, uint32_t rank) {
    uint64_t v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(peer_addr(p, rank)) : "memory");
    return v;
}
// Stats of the row from those of the cluster's CTAs (each in its own `mine`); a barrier comes first.
__device__ __forceinline__ Stats cluster_merge(const Stats* mine, int C, float k) {
    cluster_sync_all();
    Stats st = no_stats();
    for (int r = 0; r < C; ++r) {
        const Stats b{peer_f32(&mine->m, r), peer_f32(&mine->s, r), peer_f32(&mine->u, r)};
        st = merge(st, b, k);
    }
    return st;
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

// lse in units of z; -inf where nothing is left
__device__ __forceinline__ float lse_of(const Stats& st, float inv_tau) {
    return st.s == 0.f ? -INFINITY : fmaf(st.m, inv_tau, logf(st.s));
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

struct TopShared {
    uint64_t cand[kCand];
    uint64_t top[kMaxTop];
    float maxima[64];
    uint32_t threshold;
    int count;
};

// cand[0 .. n) -> the K largest in order in top (0: none); all threads.
__device__ __forceinline__ void rank_top(TopShared& sh, int n, int K) {
    if (threadIdx.x < K) sh.top[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const uint64_t key = sh.cand[i];
        int r = 0;
        for (int j = 0; j < n; ++j) r += sh.cand[j] > key;
        if (r < K && key) sh.top[r] = key;
    }
    __syncthreads();
}

// The K largest entries of [v0, v1), in order, to sh.top.  `mine`: this thread's largest entry (-FLT_MAX: none).
// K entries are at least as large as the K-th largest of any set of entries, so the K-th largest among the
// largest 64 / warps thread maxima of every warp bounds the answer from below; what reaches the bound is
// gathered and ranked.  Where more reaches it than there is room for (many equal entries), each warp keeps
// a sorted list of 32 instead.
template <typename T>
__device__ void block_top(const T* row, int v0, int v1, float mine, int K, TopShared& sh) {
    constexpr int N = 16 / sizeof(T);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5, per = 64 / warps;
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
    if (threadIdx.x < warps * per) {
        const float x = sh.maxima[threadIdx.x];
        int r = 0;
        for (int j = 0; j < warps * per; ++j) r += sh.maxima[j] > x || (sh.maxima[j] == x && j < (int)threadIdx.x);
        if (r == K - 1 && x > -FLT_MAX) sh.threshold = order_of(x);
    }
    __syncthreads();
    const uint32_t bound = sh.threshold;
    for_pieces<T, 4>(row, v0, v1, [&](int b, const float (&f)[N], int n) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < n && order_of(f[j]) >= bound) {
                const int at = atomicAdd(&sh.count, 1);        // any order: the ranks decide
                if (at < kCand) sh.cand[at] = key_of(f[j], b + j);
            }
    });
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
    rank_top(sh, n, K);
}

// ---- log probabilities -----------------------------------------------------------------------------------
struct LogprobArgs {
    const void* logits; int64_t ld;
    const void* tokens; int index_bytes;
    float *logprobs, *lse, *entropy;
    int32_t* top_ids; float* top_logprobs;
    int V, G, K, C;
    float inv_tau;
};

template <typename T, bool TOP>
__global__ void __launch_bounds__(kMaxThreads, 2) logprobs_kernel(const LogprobArgs a) {
    __shared__ Stats scratch[32];
    __shared__ Stats part;
    __shared__ typename std::conditional<TOP, TopShared, int>::type top;
    after_previous();
    const int C = a.C, rank = C > 1 ? blockIdx.x % C : 0;
    const int64_t t = blockIdx.x / C;
    const T* row = static_cast<const T*>(a.logits) + t * a.ld;
    const float k = kLog2e * a.inv_tau;
    int v0, v1;
    slice(a.V, C, rank, v0, v1);
    Stats st = thread_stats<T, true>(row, v0, v1, k);
    const float mine = st.m;
    st = block_merge(st, k, scratch);
    if constexpr (TOP) block_top<T>(row, v0, v1, mine, a.K, top);
    if (C > 1) {
        if (threadIdx.x == 0) part = st;
        st = cluster_merge(&part, C, k);
        if constexpr (TOP) {
            if (rank == 0) {
                for (int i = threadIdx.x; i < C * a.K; i += blockDim.x) top.cand[i] = peer_u64(&top.top[i % a.K], i / a.K);
                __syncthreads();
                rank_top(top, C * a.K, a.K);           // overwrites this CTA's own list, which has been copied
            }
        }
    }
    if (rank == 0) {
        const float lse = lse_of(st, a.inv_tau);
        if (threadIdx.x == 0) {
            a.lse[t] = lse;
            if (a.entropy) a.entropy[t] = st.s == 0.f ? 0.f : logf(st.s) - st.u / st.s * a.inv_tau;
        }
        for (int i = threadIdx.x; i < a.G; i += blockDim.x) {
            const int64_t v = index_at(a.tokens, a.index_bytes, t * a.G + i);
            float lp = 0.f;
            if (v >= a.V) lp = __uint_as_float(0x7fc00000u);
            else if (v >= 0) lp = st.s == 0.f ? -INFINITY : fmaf(to_f32(row[v]), a.inv_tau, -lse);
            a.logprobs[t * a.G + i] = lp;
        }
        if constexpr (TOP) {
            if (threadIdx.x < a.K) {
                const uint64_t key = top.top[threadIdx.x];
                a.top_ids[t * a.K + threadIdx.x] = (int32_t)(0xffffffffu - (uint32_t)key);
                if (a.top_logprobs)
                    a.top_logprobs[t * a.K + threadIdx.x] =
                        st.s == 0.f ? -INFINITY : fmaf(value_of((uint32_t)(key >> 32)), a.inv_tau, -lse);
            }
        }
    }
    if (C > 1) cluster_sync_all();                     // shared memory of all parts stays until it has been read
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

template <typename T>
__global__ void __launch_bounds__(kMaxThreads, 2) logprobs_backward_kernel(const LogprobBwdArgs a) {
    __shared__ float g[kMaxTokens], x_at[kMaxTokens];
    __shared__ int at[kMaxTokens];
    constexpr int N = 16 / sizeof(T);
    after_previous();
    const int64_t t = blockIdx.x / a.parts;
    const T* row = static_cast<const T*>(a.logits) + t * a.ld;
    T* d = static_cast<T*>(a.d) + t * a.ldd;
    int v0, v1;
    slice(a.V, a.parts, (int)(blockIdx.x % a.parts), v0, v1);
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
    auto dp = [&](float x) {                           // without the tokens' own term
        const float logp = fmaf(x, a.inv_tau, -lse), p = ex2(logp * kLog2e);
        return none ? 0.f : p * fmaf(-gh, fmaxf(logp, -FLT_MAX), c) * a.inv_tau;
    };
    const bool same = ((reinterpret_cast<uintptr_t>(row + v0) ^ reinterpret_cast<uintptr_t>(d + v0)) & 15) == 0;
    for_pieces<T, 4>(row, v0, v1, [&](int b, const float (&f)[N], int n) {
        float o[8];
#pragma unroll
        for (int j = 0; j < N; ++j) o[j] = dp(f[j]);
        if (n == N && same) {
            if constexpr (N == 4) *reinterpret_cast<float4*>(d + b) = make_float4(o[0], o[1], o[2], o[3]);
            else store8<T, true>(d + b, o, 8);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (j < n) d[b + j] = from_f32<T>(o[j]);
        }
    });
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
    int V, K, C;
    float tau;
};

__device__ __forceinline__ float block_reduce(float v, bool maximum, float* scratch) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = blockDim.x >> 5;
    auto reduce = [&](float x) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const float y = __shfl_xor_sync(0xffffffffu, x, o);
            x = maximum ? fmaxf(x, y) : x + y;
        }
        return x;
    };
    v = reduce(v);
    if (lane == 0) scratch[warp] = v;
    __syncthreads();
    v = reduce(lane < n ? scratch[lane] : (maximum ? -INFINITY : 0.f));
    __syncthreads();
    return v;
}

template <typename T>
__global__ void __launch_bounds__(kMaxThreads, 2) distill_kernel(const DistillArgs a) {
    __shared__ Stats scratch[32];
    __shared__ Stats part;
    __shared__ float q[kMaxTeacher], x_at[kMaxTeacher], red[32];
    __shared__ int at[kMaxTeacher];
    constexpr int N = 16 / sizeof(T);
    after_previous();
    const int C = a.C, rank = C > 1 ? blockIdx.x % C : 0;
    const int64_t t = blockIdx.x / C;
    const T* row = static_cast<const T*>(a.logits) + t * a.ld;
    T* d = a.d ? static_cast<T*>(a.d) + t * a.ldd : nullptr;
    const float inv_tau = 1.f / a.tau, k = kLog2e * inv_tau, w = a.weights ? a.weights[t] : 1.f;
    int v0, v1;
    slice(a.V, C, rank, v0, v1);

    // the teacher's distribution over its list, and the student's logits there (before d overwrites them)
    float tmax = -INFINITY;
    bool bad = false;
    for (int i = threadIdx.x; i < a.K; i += blockDim.x) {
        const int64_t v = index_at(a.ids, a.index_bytes, t * a.ldi + i);
        const int64_t j = t * a.ldt + i;
        float x = a.teacher_type == GPD_DT_F32 ? static_cast<const float*>(a.teacher)[j]
                  : a.teacher_type == GPD_DT_BF16 ? to_f32(static_cast<const __nv_bfloat16*>(a.teacher)[j])
                                                  : to_f32(static_cast<const __half*>(a.teacher)[j]);
        const bool ok = v >= 0 && v < a.V;
        bad = bad || v >= a.V;
        x = ok ? x : -INFINITY;
        at[i] = ok ? (int)v : -1;
        q[i] = x;
        x_at[i] = ok && w != 0.f ? to_f32(row[v]) : 0.f;
        tmax = x != x ? x : fmaxf(tmax, x);
    }
    bad = __syncthreads_or(bad || tmax != tmax);       // an index beyond the row, a NaN
    tmax = block_reduce(tmax, true, red);
    if (w == 0.f || (tmax == -INFINITY && !bad)) {     // no weight, or nothing in the list: the same in all parts
        if (rank == 0 && threadIdx.x == 0) a.loss[t] = 0.f;
        if (d)
            for (int v = v0 + threadIdx.x; v < v1; v += blockDim.x) d[v] = from_f32<T>(0.f);
        return;
    }
    float qs = 0.f;
    for (int i = threadIdx.x; i < a.K; i += blockDim.x) qs += q[i] == -INFINITY ? 0.f : ex2(k * (q[i] - tmax));
    qs = block_reduce(qs, false, red);

    Stats st = block_merge(thread_stats<T, false>(row, v0, v1, k), k, scratch);
    if (C > 1) {
        if (threadIdx.x == 0) part = st;
        st = cluster_merge(&part, C, k);
    }
    const float log_s = logf(st.s), log_qs = logf(qs);
    float l = 0.f;
    for (int i = threadIdx.x; i < a.K; i += blockDim.x) {
        const float lq = (q[i] - tmax) * inv_tau - log_qs, p = q[i] == -INFINITY ? 0.f : ex2(lq * kLog2e);
        if (p > 0.f) l = fmaf(p, lq - ((x_at[i] - st.m) * inv_tau - log_s), l);
        q[i] = p;
    }
    l = block_reduce(l, false, red);                   // its barriers also publish q
    const bool none = st.s == 0.f;                     // every logit of the row is masked
    if (rank == 0 && threadIdx.x == 0)
        a.loss[t] = bad ? __uint_as_float(0x7fc00000u) : none ? INFINITY : w * a.tau * a.tau * l;
    if (d) {
        const float scale = none ? 0.f : w * a.tau / st.s;
        const bool same = ((reinterpret_cast<uintptr_t>(row + v0) ^ reinterpret_cast<uintptr_t>(d + v0)) & 15) == 0;
        for_pieces<T, 4>(row, v0, v1, [&](int b, const float (&f)[N], int n) {
            float o[8];
#pragma unroll
            for (int j = 0; j < N; ++j) o[j] = scale * ex2((f[j] - st.m) * k);
            if (n == N && same) {
                if constexpr (N == 4) *reinterpret_cast<float4*>(d + b) = make_float4(o[0], o[1], o[2], o[3]);
                else store8<T, true>(d + b, o, 8);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (j < n) d[b + j] = from_f32<T>(o[j]);
            }
        });
        __syncthreads();
        for (int i = threadIdx.x; i < a.K; i += blockDim.x) {
            if (at[i] < v0 || at[i] >= v1) continue;
            float s = 0.f;                             // an entry named twice: its first holder writes the sum
            int first = i;
            for (int j = a.K - 1; j >= 0; --j)
                if (at[j] == at[i]) {
                    s += q[j];
                    first = j;
                }
            if (first == i) d[at[i]] = from_f32<T>(none ? 0.f : scale * ex2((x_at[i] - st.m) * k) - w * a.tau * s);
        }
    }
    if (C > 1) cluster_sync_all();                     // `part` stays until all have read it
}

// ---- host side ---------------------------------------------------------------------------------------------
// CTAs per row: as many (up to 8) as the GPU has SMs for, while each still has 4096 entries to read.
int row_split(int64_t T, int64_t V) {
    int c = 1;
    while (c < 8 && T * c * 2 <= 2 * sm_count() && V / (2 * c) >= 4096) c *= 2;
    return c;
}
unsigned row_threads(int64_t entries) { return entries >= 8192 ? 512 : entries >= 4096 ? 256 : 128; }

template <typename... P, typename A>
gpd_status launch_rows(void (*kernel)(P...), const A& a, int64_t T, int C, unsigned threads, cudaStream_t st) {
    if (T * C > 0x7fffffff) return GPD_ERR_SHAPE;
    return launch_after(kernel, dim3((unsigned)(T * C)), dim3(threads), 0, C, st, a);
}
template <typename T>
gpd_status launch_logprobs(LogprobArgs a, int64_t rows, cudaStream_t st) {
    a.C = row_split(rows, a.V);
    const unsigned threads = row_threads(a.V / a.C);
    return a.K ? launch_rows(logprobs_kernel<T, true>, a, rows, a.C, threads, st)
               : launch_rows(logprobs_kernel<T, false>, a, rows, a.C, threads, st);
}
template <typename T>
gpd_status launch_logprobs_backward(LogprobBwdArgs a, int64_t rows, cudaStream_t st) {
    // no sums over the row, so any cut will do: enough CTAs for the GPU, each with 8192 entries or more
    const int64_t wanted = (4 * sm_count() + rows - 1) / rows;
    a.parts = (int)std::max<int64_t>(1, std::min<int64_t>((a.V + 8191) / 8192, wanted));
    return launch_rows(logprobs_backward_kernel<T>, a, rows * a.parts, 1, row_threads(a.V / a.parts), st);
}
template <typename T>
gpd_status launch_distill(DistillArgs a, int64_t rows, cudaStream_t st) {
    a.C = row_split(rows, a.V);
    return launch_rows(distill_kernel<T>, a, rows, a.C, row_threads(a.V / a.C), st);
}

bool bad_rows(int64_t T, int64_t V) { return T < 0 || V <= 0 || V > 0x7fffff00; }

}  // namespace

}  // namespace gpd

using namespace gpd;

extern "C" gpd_status gpd_token_logprobs(gpd_dtype type, const void* logits_dev, int64_t ld, int32_t index_bytes,
                                         const void* tokens_dev, int32_t G, float temperature, float* logprobs_dev,
                                         float* lse_dev, float* entropy_dev, int32_t K, int32_t* top_ids_dev,
                                         float* top_logprobs_dev, int64_t T, int64_t V, void* stream) {
    if (!is_float_type(type) || !(temperature > 0.f) || isinf(temperature)) return GPD_ERR_ARG;
    if (bad_rows(T, V) || G < 0 || G > kMaxTokens || K < 0 || K > kMaxTop || K > V) return GPD_ERR_SHAPE;
    if (T == 0) return GPD_OK;                         // empty buffers may have no address
    if (!logits_dev || !lse_dev || (G > 0 && (!tokens_dev || !logprobs_dev || (index_bytes != 4 && index_bytes != 8))) ||
        (K > 0 && !top_ids_dev))
        return GPD_ERR_ARG;
    if (ld < V) return GPD_ERR_SHAPE;
    const LogprobArgs a{logits_dev, ld, tokens_dev, index_bytes, logprobs_dev, lse_dev, entropy_dev, top_ids_dev,
                        top_logprobs_dev, (int)V, G, K, 1, 1.f / temperature};
    cudaStream_t st = as_stream(stream);
    if (type == GPD_DT_F32) return launch_logprobs<float>(a, T, st);
    if (type == GPD_DT_BF16) return launch_logprobs<__nv_bfloat16>(a, T, st);
    return launch_logprobs<__half>(a, T, st);
}

extern "C" gpd_status gpd_token_logprobs_backward(gpd_dtype type, const void* logits_dev, int64_t ld, int32_t index_bytes,
                                                  const void* tokens_dev, int32_t G, float temperature, const float* lse_dev,
                                                  const float* entropy_dev, const float* dlogprobs_dev,
                                                  const float* dentropy_dev, void* dlogits_dev, int64_t ldd, int64_t T,
                                                  int64_t V, void* stream) {
    if (!is_float_type(type) || !(temperature > 0.f) || isinf(temperature)) return GPD_ERR_ARG;
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
    if (!is_float_type(type) || !is_float_type(teacher_type) || !(temperature > 0.f) || isinf(temperature)) return GPD_ERR_ARG;
    if (bad_rows(T, V) || K < 0 || K > kMaxTeacher) return GPD_ERR_SHAPE;
    if (T == 0) return GPD_OK;
    if (!logits_dev || !loss_dev || (K > 0 && (!teacher_ids_dev || !teacher_logits_dev || (index_bytes != 4 && index_bytes != 8))))
        return GPD_ERR_ARG;
    if (ld < V || ldi < K || ldt < K || (dlogits_dev && ldd < V)) return GPD_ERR_SHAPE;
    const DistillArgs a{logits_dev, ld, teacher_ids_dev, index_bytes, ldi, teacher_logits_dev, ldt, teacher_type, weights_dev,
                        loss_dev, dlogits_dev, ldd, (int)V, K, 1, temperature};
    cudaStream_t st = as_stream(stream);
    if (type == GPD_DT_F32) return launch_distill<float>(a, T, st);
    if (type == GPD_DT_BF16) return launch_distill<__nv_bfloat16>(a, T, st);
    return launch_distill<__half>(a, T, st);
}
