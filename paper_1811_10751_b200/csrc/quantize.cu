// Cutting a matrix into 8-bit blocks with power-of-two scales, straight and transposed in one pass.
//
//   straight:    blocks of 1 x 128 (or 128 x 128) elements of src, q[r][c], scale[r / br][c / 128]
//   transposed:  the same of src^T, qT[c][r], scaleT[c / br][r / 128]: the operand of a product that
//                contracts over src's rows
//
// One CTA takes a 128 x 128 tile, which holds whole blocks of either kind, so the source is read once for
// both: HBM bounds it (source bytes + one byte per element and output).  Thread (rg, cg) holds the 8 x 8
// patch at rows 8 rg, columns 8 cg.  A row's sixteen column groups sit in sixteen adjacent lanes (maximum
// by shuffles); the column maxima meet in shared memory.  A patch's column is eight bytes of a transposed
// row, so the transposed tile goes through shared memory in 8-byte pieces and leaves in 16-byte ones.
//
// Measured: 4096 x 8192 BF16 both ways 29.6 us, 0.70 of the copy bandwidth (issue slots 57 % busy: two conversions and
// the maxima per element); 1000 x 4096 FP32 in 128 x 128 blocks 5.3 us.  A CTA per tile, three on an SM: tiles of other
// shapes would hold parts of blocks of one kind or the other.
#include "lm_common.h"

namespace gpd {

namespace {

using namespace lm;

struct CutArgs {
    const void* src; int64_t ld;
    uint8_t* q; int64_t ldq;
    uint8_t* s; int64_t lds;
    uint8_t* qT; int64_t ldqT;
    uint8_t* sT; int64_t ldsT;
    int64_t M, K;
    bool q_vec, qT_vec;                                // rows of q (qT) start on 8-byte (16-byte) boundaries
};

// Byte offset of the 8-byte chunk `chunk` of transposed row `col` in shared memory.  The chunks of a row are
// permuted by the row's column group, so that the sixteen lanes that write one chunk column, 1024 bytes
// apart, fall on all banks.
__device__ __forceinline__ int chunk_at(int col, int chunk) { return col * kBlock + ((chunk ^ (col >> 3)) & 15) * 8; }

// Maxima of 16-bit magnitudes are taken two at a time (a NaN is above all), and only the final ones become FP32 bits.
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b, __nv_bfloat16) {
    const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b, __half) {
    const __half2 r = __hmax2_nan(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
template <typename T>
struct Maxima {
    uint32_t w[4];                                     // columns 2 i (low half) and 2 i + 1
    __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = 0; }
    __device__ __forceinline__ uint32_t take(const Raw8<T>& r) {       // returns the row's maximum
        const uint32_t a[4] = {r.v.x & 0x7fff7fffu, r.v.y & 0x7fff7fffu, r.v.z & 0x7fff7fffu, r.v.w & 0x7fff7fffu};
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = max_pair(w[i], a[i], T());
        const uint32_t m = max_pair(max_pair(a[0], a[1], T()), max_pair(a[2], a[3], T()), T());
        return max(m & 0xffffu, m >> 16);
    }
    __device__ __forceinline__ uint32_t column(int j) const { return j & 1 ? w[j >> 1] >> 16 : w[j >> 1] & 0xffffu; }
};
template <>
struct Maxima<float> {
    uint32_t w[8];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 0;
    }
    __device__ __forceinline__ uint32_t take(const Raw8<float>& r) {
        const uint32_t a[8] = {r.v.x, r.v.y, r.v.z, r.v.w, r.w.x, r.w.y, r.w.z, r.w.w};
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t b = a[i] & 0x7fffffffu;
            w[i] = max(w[i], b);
            m = max(m, b);
        }
        return m;
    }
    __device__ __forceinline__ uint32_t column(int j) const { return w[j]; }
};
// FP32 bits of a magnitude given by its own bits
template <typename T> __device__ __forceinline__ uint32_t magnitude(uint32_t b);
template <> __device__ __forceinline__ uint32_t magnitude<float>(uint32_t b) { return b; }
template <> __device__ __forceinline__ uint32_t magnitude<__nv_bfloat16>(uint32_t b) { return b << 16; }
template <> __device__ __forceinline__ uint32_t magnitude<__half>(uint32_t b) {
    return __float_as_uint(__half2float(__ushort_as_half((unsigned short)b)));
}

template <typename T, int Q, bool SQUARE, bool VEC>
__global__ void __launch_bounds__(256, sizeof(T) == 4 ? 2 : 3) cut_kernel(const CutArgs a, int tiles_k) {
    __shared__ __align__(16) uint8_t tile[kBlock * kBlock];
    __shared__ uint32_t colmax[16][kBlock];
    after_previous();
    const int rg = threadIdx.x >> 4, cg = threadIdx.x & 15;
    const int64_t bm = blockIdx.x / tiles_k, bk = blockIdx.x % tiles_k;
    const int64_t r0 = bm * kBlock + 8 * rg, c0 = bk * kBlock + 8 * cg;
    const int nc = (int)min(a.K - c0, (int64_t)8), nr = (int)min(a.M - r0, (int64_t)8);      // of the patch, possibly <= 0
    const T *begin = static_cast<const T*>(a.src), *end = begin + (a.M - 1) * a.ld + a.K, *src = begin + r0 * a.ld + c0;

    Raw8<T> raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        raw[i] = i < nr && nc > 0 ? (nc < 8 ? load8<T, false>(src + i * a.ld, nc) : VEC ? load8_all<T>(src + i * a.ld) : load8_near<T>(src + i * a.ld, begin, end)) : Raw8<T>{};

    Maxima<T> cm;                                      // of the patch's columns
    uint32_t rmax[8];                                  // of its rows
    cm.clear();
#pragma unroll
    for (int i = 0; i < 8; ++i) rmax[i] = cm.take(raw[i]);
    uint32_t byte = 0;                                 // SQUARE: the tile's scale
    if (SQUARE) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, rmax[i]);
        m = __reduce_max_sync(0xffffffffu, magnitude<T>(m));
        if ((threadIdx.x & 31) == 0) colmax[0][threadIdx.x >> 5] = m;
        __syncthreads();
        m = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) m = max(m, colmax[0][w]);
        byte = scale_byte<Q>(m);
        if (threadIdx.x == 0) {
            if (a.q) a.s[bm * a.lds + bk] = (uint8_t)byte;
            if (a.qT) a.sT[bk * a.ldsT + bm] = (uint8_t)byte;
        }
    } else if (a.qT) {
#pragma unroll
        for (int j = 0; j < 8; ++j) colmax[rg][8 * cg + j] = cm.column(j);
        __syncthreads();
        if (threadIdx.x < kBlock) {                    // thread = column
            uint32_t m = 0;
#pragma unroll
            for (int g = 0; g < 16; ++g) m = max(m, colmax[g][threadIdx.x]);
            const uint32_t b = scale_byte<Q>(magnitude<T>(m));
            colmax[0][threadIdx.x] = b;                // only this thread reads row 0 of its column
            const int64_t c = bk * kBlock + threadIdx.x;
            if (c < a.K) a.sT[c * a.ldsT + bm] = (uint8_t)b;
        }
        __syncthreads();
    }

    if (a.q) {
        uint8_t* q = a.q + r0 * a.ldq + c0;
        uint8_t* sc = a.s + r0 * a.lds + bk;
        BlockScales rows{};
        if (!SQUARE) {
            rows = block_scales<Q, 8>(rmax, [](uint32_t m) { return magnitude<T>(m); });
            if (rows.first && rows.mine < nr) sc[rows.mine * a.lds] = (uint8_t)rows.byte;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t b = SQUARE ? byte : packed_byte(rows, i);
            if (i < nr && nc > 0) {
                const float inv = scale_inverse(b);
                F2 p[4];
                pairs8<T>(raw[i], p);
#pragma unroll
                for (int j = 0; j < 4; ++j) p[j] = mul2(p[j], f2(inv, inv));
                float f[8];
                floats8(p, f);
                const uint2 v = make_uint2(cvt_fp8x4<Q>(f[0], f[1], f[2], f[3]), cvt_fp8x4<Q>(f[4], f[5], f[6], f[7]));
                if (a.q_vec && nc == 8) *reinterpret_cast<uint2*>(q + i * a.ldq) = v;
                else store8_bytes(q + i * a.ldq, v, nc);
            }
        }
    }
    if (a.qT) {
        float inv[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) inv[j] = scale_inverse(SQUARE ? byte : colmax[0][8 * cg + j]);
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            float lo[8], hi[8];                        // columns j and j + 1 of the patch
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 x = pair_of<T>(raw[i], j >> 1), f = f2(mul2(f2(x.x, x.y), f2(inv[j], inv[j + 1])));
                lo[i] = f.x;
                hi[i] = f.y;
            }
            *reinterpret_cast<uint2*>(tile + chunk_at(8 * cg + j, rg)) =
                make_uint2(cvt_fp8x4<Q>(lo[0], lo[1], lo[2], lo[3]), cvt_fp8x4<Q>(lo[4], lo[5], lo[6], lo[7]));
            *reinterpret_cast<uint2*>(tile + chunk_at(8 * cg + j + 1, rg)) =
                make_uint2(cvt_fp8x4<Q>(hi[0], hi[1], hi[2], hi[3]), cvt_fp8x4<Q>(hi[4], hi[5], hi[6], hi[7]));
        }
        __syncthreads();
#pragma unroll
        for (int p = 0; p < 4; ++p) {                  // 32 transposed rows per pass, 8 lanes of 16 bytes each
            const int col = 32 * p + (threadIdx.x >> 3), piece = threadIdx.x & 7;
            const int64_t c = bk * kBlock + col, r = bm * kBlock + 16 * piece;
            const int n = (int)min(a.M - r, (int64_t)16);
            if (c >= a.K || n <= 0) continue;
            // chunks 2 piece and 2 piece + 1 stay neighbours, in exchanged order for odd column groups
            uint4 v = *reinterpret_cast<const uint4*>(tile + (chunk_at(col, 2 * piece) & ~15));
            if ((col >> 3) & 1) v = make_uint4(v.z, v.w, v.x, v.y);
            uint8_t* dst = a.qT + c * a.ldqT + r;
            if (a.qT_vec && n >= 16) {
                *reinterpret_cast<uint4*>(dst) = v;
            } else {
                store8_bytes(dst, make_uint2(v.x, v.y), n);
                store8_bytes(dst + 8, make_uint2(v.z, v.w), n - 8);
            }
        }
    }
}

template <typename T, int Q>
gpd_status launch_cut(const CutArgs& a, bool square, cudaStream_t st) {
    const int64_t tk = (a.K + kBlock - 1) / kBlock, tm = (a.M + kBlock - 1) / kBlock;
    if (tk * tm > 0x7fffffff) return GPD_ERR_SHAPE;
    const unsigned grid = (unsigned)(tk * tm);
    const bool vec = rows_aligned(a.src, a.ld, sizeof(T));
    auto kernel = square ? (vec ? cut_kernel<T, Q, true, true> : cut_kernel<T, Q, true, false>)
                         : (vec ? cut_kernel<T, Q, false, true> : cut_kernel<T, Q, false, false>);
    return launch_after(kernel, dim3(grid), dim3(256), 0, 1, st, a, (int)tk);
}
template <typename T>
gpd_status launch_cut_q(const CutArgs& a, int q_type, bool square, cudaStream_t st) {
    return q_type == GPD_DT_E4M3 ? launch_cut<T, GPD_DT_E4M3>(a, square, st) : launch_cut<T, GPD_DT_E5M2>(a, square, st);
}

}  // namespace

}  // namespace gpd

using namespace gpd;

extern "C" gpd_status gpd_quantize_blocks(gpd_dtype type, const void* src_dev, int64_t ld, gpd_dtype q_type, int32_t block_rows,
                                          void* q_dev, int64_t ldq, uint8_t* scales_dev, int64_t lds, void* qT_dev,
                                          int64_t ldqT, uint8_t* scalesT_dev, int64_t ldsT, int64_t M, int64_t K, void* stream) {
    if (!is_float_type(type) || !is_fp8_type(q_type) || (block_rows != 1 && block_rows != lm::kBlock)) return GPD_ERR_ARG;
    if (M < 0 || K < 0) return GPD_ERR_SHAPE;
    if (M == 0 || K == 0) return GPD_OK;               // empty buffers may have no address
    if (!src_dev || (!q_dev && !qT_dev) || (q_dev && !scales_dev) || (qT_dev && !scalesT_dev)) return GPD_ERR_ARG;
    const int64_t kb = (K + lm::kBlock - 1) / lm::kBlock, mb = (M + lm::kBlock - 1) / lm::kBlock;
    if (ld < K || (q_dev && (ldq < K || lds < kb)) || (qT_dev && (ldqT < M || ldsT < mb))) return GPD_ERR_SHAPE;
    const CutArgs a{src_dev, ld, static_cast<uint8_t*>(q_dev), ldq, scales_dev, lds, static_cast<uint8_t*>(qT_dev), ldqT,
                    scalesT_dev, ldsT, M, K, lm::rows_aligned(q_dev, ldq, 1, 8), lm::rows_aligned(qT_dev, ldqT, 1)};
    const bool square = block_rows != 1;
    cudaStream_t st = as_stream(stream);
    if (type == GPD_DT_F32) return launch_cut_q<float>(a, q_type, square, st);
    if (type == GPD_DT_BF16) return launch_cut_q<__nv_bfloat16>(a, q_type, square, st);
    return launch_cut_q<__half>(a, q_type, square, st);
}
