// Norm over many gradients together, and clipping by it.
//
//   norm = (sum over all elements of all tensors of g^2)^(1/2),   out = g min(1, max_norm / norm)
//
// One pass reads every element, the other reads and writes it: HBM bounds both, and many small tensors the launches.  So
// one launch covers up to 640 tensors of any sizes and types: their addresses travel with the launch (constant memory),
// and the tensors are cut into chunks of 8192 elements, of which every CTA has a contiguous range; only its first chunk's
// tensor is searched for.  Clipping walks from the end of each range to its beginning: what the norm's pass read last
// is then still in L2.
//
// Squares are summed in FP32 within a thread's 16 elements of a chunk and in FP64 from there on, in a fixed order.  Sums
// of squares that leave FP32's safe range are taken again in FP64 from the registers, so that gradients of any
// magnitude have their norm.
//
// Measured: 400 million BF16 gradients in 290 tensors, norm and clipping, 404 us (2.4 GB at 5.9 TB/s); 56 small ones 11 us, which is the
// three launches (9 in a graph).
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "lm_common.h"

namespace gpd {

namespace {

using namespace lm;

constexpr int kThreads = 512, kUnits = 2, kChunk = kThreads * kUnits * 8;   // a unit: eight elements of one thread
constexpr int kMost = 640, kFew = 64;                  // tensors of a launch; few: their table is a tenth as long
constexpr int kCtasPerSm = 4, kMostCtas = GPD_GRAD_NORM_WORKSPACE / 8;

struct Tensor {
    const void* in;
    void* out;                                         // clipping only
    int64_t count, first;                              // elements; number of its first chunk
    int in_type, out_type;
};
template <int N>
struct Tensors {
    Tensor t[N];
    int n;
    int64_t chunks;
};

// Elements of a tensor before the first 16-byte boundary belong to a unit that begins before the tensor.
__device__ __forceinline__ int misaligned(const void* p, int type) {
    return (int)(reinterpret_cast<uintptr_t>(p) & 15) >> (type == GPD_DT_F32 ? 2 : 1);
}

// f(tensor, number of the chunk in it) for the chunks of this CTA; DOWN: the last first
template <int N, bool DOWN, typename F>
__device__ __forceinline__ void for_chunks(const Tensors<N>& a, F f) {
    const int64_t from = a.chunks * blockIdx.x / gridDim.x, to = a.chunks * (blockIdx.x + 1) / gridDim.x;
    if (from >= to) return;
    const int64_t start = DOWN ? to - 1 : from;
    int lo = 0, hi = a.n - 1;                          // the last tensor whose first chunk is <= start
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (a.t[mid].first <= start) lo = mid;
        else hi = mid - 1;
    }
    if (DOWN) {
        for (int64_t c = start; c >= from; --c) {
            while (a.t[lo].first > c) --lo;
            f(a.t[lo], c - a.t[lo].first);
        }
    } else {
        for (int64_t c = start; c < to; ++c) {
            while (lo + 1 < a.n && a.t[lo + 1].first <= c) ++lo;
            f(a.t[lo], c - a.t[lo].first);
        }
    }
}

// The thread's units of a chunk: units stand `mis` elements before multiples of eight; missing elements are zero.
template <typename T>
__device__ __forceinline__ void load_units(const T* p, int64_t count, int mis, int64_t chunk, Raw8<T> (&r)[kUnits]) {
    const int64_t base = chunk * kChunk + 8 * threadIdx.x - mis;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const int64_t e = base + (int64_t)i * kThreads * 8;
        if (e >= 0 && e + 8 <= count) {
            r[i] = load8_all<T>(p + e);
        } else {
            r[i] = Raw8<T>{};
            if (e > -8 && e < count) {
                uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (e + j >= 0 && e + j < count) {
                        if constexpr (sizeof(T) == 4) w[j] = __float_as_uint(p[e + j]);
                        else w[j / 2] |= (uint32_t)reinterpret_cast<const unsigned short*>(p)[e + j] << (16 * (j & 1));
                    }
                r[i].v = make_uint4(w[0], w[1], w[2], w[3]);
                if constexpr (sizeof(T) == 4) r[i].w = make_uint4(w[4], w[5], w[6], w[7]);
            }
        }
    }
}

template <typename T>
__device__ __forceinline__ double squares(const Tensor& t, int64_t chunk) {
    Raw8<T> r[kUnits];
    load_units<T>(static_cast<const T*>(t.in), t.count, misaligned(t.in, t.in_type), chunk, r);
    F2 sum = f2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        F2 p[4];
        pairs8<T>(r[i], p);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum = fma2(p[j], p[j], sum);
    }
    const float2 s = f2(sum);
    const float both = s.x + s.y;
    if (both < 1.3e36f && both > 7.9e-31f) return (double)both;        // 2^120, 2^-100: no overflow, and what underflowed is nothing beside it
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        float f[8];
        unpack8<T>(r[i], f);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (f[j] != 0.f) d = fma((double)f[j], (double)f[j], d);
    }
    return d;
}

// Sum over the CTA in a fixed order; thread 0 has it.
__device__ __forceinline__ double cta_sum(double v) {
    __shared__ double s[kThreads / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
    if (threadIdx.x == 0)
        for (int i = 0; i < kThreads / 32; ++i) v += s[i];
    return v;
}

// parts[CTA]: its sum of squares, added to what an earlier launch left there where `more`
template <int N>
__global__ void __launch_bounds__(kThreads) grad_squares_kernel(const __grid_constant__ Tensors<N> a, double* parts, bool more) {
    after_previous();
    double sum = 0.0;
    for_chunks<N, false>(a, [&](const Tensor& t, int64_t chunk) {
        sum += t.in_type == GPD_DT_F32    ? squares<float>(t, chunk)
               : t.in_type == GPD_DT_BF16 ? squares<__nv_bfloat16>(t, chunk)
                                          : squares<__half>(t, chunk);
    });
    sum = cta_sum(sum);
    if (threadIdx.x == 0) parts[blockIdx.x] = more ? parts[blockIdx.x] + sum : sum;
}
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const double* parts, int n, float* norm) {
    after_previous();
    double v = 0.0;
    for (int i = threadIdx.x; i < n; i += kThreads) v += parts[i];
    v = cta_sum(v);
    if (threadIdx.x == 0) *norm = (float)sqrt(v);
}

template <typename T, typename O>
__device__ __forceinline__ void scale_chunk(const Tensor& t, int64_t chunk, float by) {
    const T* in = static_cast<const T*>(t.in);
    O* out = static_cast<O*>(t.out);
    const int mis = misaligned(in, t.in_type);
    Raw8<T> r[kUnits];
    load_units<T>(in, t.count, mis, chunk, r);
    const bool vec = ((reinterpret_cast<uintptr_t>(out) - (uintptr_t)mis * sizeof(O)) & 15) == 0;
    const int64_t base = chunk * kChunk + 8 * threadIdx.x - mis;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const int64_t e = base + (int64_t)i * kThreads * 8;
        float f[8];
        unpack8<T>(r[i], f);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] *= by;
        if (vec && e >= 0 && e + 8 <= t.count) {
            store8<O, true>(out + e, f, 8);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (e + j >= 0 && e + j < t.count) out[e + j] = from_f32<O>(f[j]);
        }
    }
}
template <typename T>
__device__ __forceinline__ void scale_to(const Tensor& t, int64_t chunk, float by) {
    if (t.out_type == GPD_DT_F32) scale_chunk<T, float>(t, chunk, by);
    else if (t.out_type == GPD_DT_BF16) scale_chunk<T, __nv_bfloat16>(t, chunk, by);
    else scale_chunk<T, __half>(t, chunk, by);
}
// A factor below 2^-100, of which FP32 may hold less than 24 bits, in two steps: 2^-64 first, which is exact wherever the result is not
// zero (a gradient below 2^-62 would be scaled to less than 2^-162).  Element by element: it is rare, and within the registers
// of the other form.
constexpr float kFirst = 5.421010862427522e-20f, kFar = 7.9e-31f;      // 2^-64, 2^-100
__device__ __forceinline__ void scale_far(const Tensor& t, int64_t chunk, float by) {
    const int64_t from = chunk * kChunk - misaligned(t.in, t.in_type);
#pragma unroll 1
    for (int i = threadIdx.x; i < kChunk; i += kThreads) {
        const int64_t e = from + i;
        if (e < 0 || e >= t.count) continue;
        const float f = t.in_type == GPD_DT_F32    ? static_cast<const float*>(t.in)[e]
                        : t.in_type == GPD_DT_BF16 ? to_f32(static_cast<const __nv_bfloat16*>(t.in)[e])
                                                   : to_f32(static_cast<const __half*>(t.in)[e]);
        const float v = f * kFirst * by;
        if (t.out_type == GPD_DT_F32) static_cast<float*>(t.out)[e] = v;
        else if (t.out_type == GPD_DT_BF16) static_cast<__nv_bfloat16*>(t.out)[e] = from_f32<__nv_bfloat16>(v);
        else static_cast<__half*>(t.out)[e] = from_f32<__half>(v);
    }
}
// in_place: every tensor's output is itself; nothing to do where the norm is within the bound
template <int N>
__global__ void __launch_bounds__(kThreads) clip_kernel(const __grid_constant__ Tensors<N> a, const float* norm, float max_norm, bool in_place) {
    after_previous();
    const float n = *norm;
    if (in_place && n <= max_norm) return;
    const float by = n <= max_norm ? 1.f : max_norm / n;               // NaN: NaN
    if (by < kFar && n <= 3.4e38f) {
        const float rest = max_norm / (n * kFirst);
        for_chunks<N, true>(a, [&](const Tensor& t, int64_t chunk) { scale_far(t, chunk, rest); });
        return;
    }
    for_chunks<N, true>(a, [&](const Tensor& t, int64_t chunk) {
        if (t.in_type == GPD_DT_F32) scale_to<float>(t, chunk, by);
        else if (t.in_type == GPD_DT_BF16) scale_to<__nv_bfloat16>(t, chunk, by);
        else scale_to<__half>(t, chunk, by);
    });
}

// ---- host side ---------------------------------------------------------------------------------------
int64_t chunks_of(const void* p, int type, int64_t count) {
    const int64_t mis = (int64_t)(reinterpret_cast<uintptr_t>(p) & 15) / dtype_size(type);
    return (count + mis + kChunk - 1) / kChunk;
}

// Calls launch(table) for every group of tensors, empty ones left out; returns the first status that is not GPD_OK.
template <int N, typename F>
gpd_status for_groups(int32_t n, const int32_t* types, const void* const* in, const int32_t* out_types, void* const* out,
                      const int64_t* counts, F launch) {
    Tensors<N> a;
    a.n = 0;
    a.chunks = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (counts[i] > 0) {
            a.t[a.n++] = Tensor{in[i], out ? out[i] : nullptr, counts[i], a.chunks, types[i], out_types ? out_types[i] : types[i]};
            a.chunks += chunks_of(in[i], types[i], counts[i]);
        }
        if (a.n > 0 && (a.n == N || i == n - 1)) {
            const gpd_status rc = launch(a);
            if (rc != GPD_OK) return rc;
            a.n = 0;
            a.chunks = 0;
        }
    }
    return GPD_OK;
}

gpd_status check_tensors(int32_t n, const int32_t* types, const void* const* in, const int64_t* counts) {
    if (n < 0) return GPD_ERR_SHAPE;
    if (n > 0 && (!types || !in || !counts)) return GPD_ERR_ARG;
    int64_t sum = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (!is_float_type(types[i])) return GPD_ERR_ARG;
        if (counts[i] < 0 || counts[i] > (int64_t)1 << 45 || (sum += counts[i]) > (int64_t)1 << 45) return GPD_ERR_SHAPE;
        if (counts[i] > 0 && (!in[i] || !aligned(in[i], dtype_size(types[i])))) return GPD_ERR_ARG;
    }
    return GPD_OK;
}

template <int N>
gpd_status launch_norm(int32_t n, const int32_t* types, const void* const* grads, const int64_t* counts, float* norm, double* parts,
                       cudaStream_t st) {
    int used = 0;
    const gpd_status rc = for_groups<N>(n, types, grads, nullptr, nullptr, counts, [&](const Tensors<N>& a) {
        // a later group adds to the parts that the first has written, so it has at most as many CTAs
        const int most = used ? used : std::min(kCtasPerSm * sm_count(), kMostCtas);
        const int ctas = (int)std::min<int64_t>(a.chunks, most);
        const bool more = used > 0;
        if (!used) used = ctas;
        return launch_after(grad_squares_kernel<N>, dim3((unsigned)ctas), dim3(kThreads), 0, 1, st, a, parts, more);
    });
    if (rc != GPD_OK) return rc;
    const double* p = parts;
    return launch_after(grad_norm_kernel, dim3(1), dim3(kThreads), 0, 1, st, p, used, norm);
}
template <int N>
gpd_status launch_clip(int32_t n, const int32_t* types, const void* const* grads, const int32_t* out_types, void* const* out,
                       const int64_t* counts, const float* norm, float max_norm, bool in_place, cudaStream_t st) {
    return for_groups<N>(n, types, grads, out_types, out, counts, [&](const Tensors<N>& a) {
        const int ctas = (int)std::min<int64_t>(a.chunks, kCtasPerSm * sm_count());
        return launch_after(clip_kernel<N>, dim3((unsigned)ctas), dim3(kThreads), 0, 1, st, a, norm, max_norm, in_place);
    });
}

// Whether an output shares memory with another output, with another tensor's input or with the norm.
struct Range {
    uintptr_t from, to;
    bool written;
};
bool overlapping(int32_t n, const int32_t* types, const void* const* in, const int32_t* out_types, void* const* out, const int64_t* counts,
                 const float* norm) {
    std::vector<Range> r;
    r.reserve(2 * (size_t)n + 1);
    auto add = [&](const void* p, int64_t count, int type, bool written) {
        const auto from = reinterpret_cast<uintptr_t>(p);
        r.push_back({from, from + (uintptr_t)count * dtype_size(type), written});
    };
    for (int32_t i = 0; i < n; ++i)
        if (counts[i] > 0) add(out[i], counts[i], out_types[i], true);
    const auto outs = (std::ptrdiff_t)r.size();
    for (int32_t i = 0; i < n; ++i)
        if (counts[i] > 0 && out[i] != in[i]) add(in[i], counts[i], types[i], false);
    add(norm, 1, GPD_DT_F32, false);
    // most often each half is in order: then one merging pass
    auto before = [](const Range& a, const Range& b) { return a.from < b.from; };
    const auto middle = r.begin() + outs;
    if (!std::is_sorted(r.begin(), middle, before)) std::sort(r.begin(), middle, before);
    if (!std::is_sorted(middle, r.end(), before)) std::sort(middle, r.end(), before);
    std::inplace_merge(r.begin(), middle, r.end(), before);
    uintptr_t end = 0, written_end = 0;
    for (const Range& x : r) {
        if (x.from < written_end || (x.written && x.from < end)) return true;
        end = std::max(end, x.to);
        if (x.written) written_end = std::max(written_end, x.to);
    }
    return false;
}

}  // namespace

}  // namespace gpd

using namespace gpd;

extern "C" gpd_status gpd_grad_norm(int32_t n, const int32_t* types_host, const void* const* grads_host, const int64_t* counts_host,
                                    float* norm_dev, void* workspace_dev, int64_t workspace_bytes, void* stream) {
    const gpd_status rc = check_tensors(n, types_host, grads_host, counts_host);
    if (rc != GPD_OK) return rc;
    if (!norm_dev) return GPD_ERR_ARG;
    if (!workspace_dev || workspace_bytes < GPD_GRAD_NORM_WORKSPACE || !lm::aligned(workspace_dev, 8)) return GPD_ERR_WORKSPACE;
    cudaStream_t st = as_stream(stream);
    double* parts = static_cast<double*>(workspace_dev);
    return n <= kFew ? launch_norm<kFew>(n, types_host, grads_host, counts_host, norm_dev, parts, st)
                     : launch_norm<kMost>(n, types_host, grads_host, counts_host, norm_dev, parts, st);
}

extern "C" gpd_status gpd_clip_grads(int32_t n, const int32_t* types_host, const void* const* grads_host, const int32_t* out_types_host,
                                     void* const* out_host, const int64_t* counts_host, const float* norm_dev, float max_norm,
                                     void* stream) {
    gpd_status rc = check_tensors(n, types_host, grads_host, counts_host);
    if (rc != GPD_OK) return rc;
    if (!norm_dev || !(max_norm > 0.f)) return GPD_ERR_ARG;
    if (n == 0) return GPD_OK;
    if (!out_types_host || !out_host) return GPD_ERR_ARG;
    rc = check_tensors(n, out_types_host, out_host, counts_host);
    if (rc != GPD_OK) return rc;
    bool in_place = true;
    for (int32_t i = 0; i < n; ++i) {
        const bool same = out_host[i] == grads_host[i];
        if (same && out_types_host[i] != types_host[i] && counts_host[i] > 0) return GPD_ERR_ARG;
        in_place = in_place && (same || counts_host[i] == 0);
    }
    try {
        if (overlapping(n, types_host, grads_host, out_types_host, out_host, counts_host, norm_dev)) return GPD_ERR_ARG;
    } catch (const std::bad_alloc&) {
        return GPD_ERR_SHAPE;
    }
    cudaStream_t st = as_stream(stream);
    return n <= kFew ? launch_clip<kFew>(n, types_host, grads_host, out_types_host, out_host, counts_host, norm_dev, max_norm, in_place, st)
                     : launch_clip<kMost>(n, types_host, grads_host, out_types_host, out_host, counts_host, norm_dev, max_norm, in_place, st);
}
