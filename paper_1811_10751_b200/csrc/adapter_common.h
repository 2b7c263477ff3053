// Shared by the kernels of low-rank adapters (adapter_shrink.cu, adapter_expand.cu, adapter_grad.cu).
//
// The rows of a batch are cut into segments; segment s covers the rows offsets[s] .. offsets[s + 1] - 1 and has the
// adapter index[s].  Products run on the tensor cores as 16 x 8 x 16 steps with FP32 sums; what they accumulate in one
// chain is cut every few steps and added to nearest, because the chain itself truncates.
#pragma once

#include <type_traits>

#include "lm_common.h"
#include "tc_common.h"

namespace gpd {
namespace adapter {

using namespace lm;

constexpr int kMaxRank = GPD_ADAPTER_MAX_RANK;

struct Segments {
    const void *offsets, *index;
    int64_t T;
    int S, n;                                          // segments, adapters
    bool wide;                                         // 8-byte numbers
};
// A row tile: rows of one segment.  rows 0: none.  adapter -1: the segment has none; n: there is no such adapter.  Rows and
// adapters are below 2^31.
struct RowTile {
    int row, rows, id;
};
__device__ __forceinline__ int64_t number(const void* p, int64_t i, bool wide) {
    return wide ? static_cast<const int64_t*>(p)[i] : static_cast<const int32_t*>(p)[i];
}
__device__ __forceinline__ int offset_at(const Segments& s, int64_t i) {
    const int64_t v = number(s.offsets, i, s.wide);
    return (int)(v < 0 ? 0 : v > s.T ? s.T : v);       // whatever stands there, rows stay inside the batch
}
__device__ __forceinline__ int adapter_at(const Segments& s, int64_t i) {
    const int64_t v = number(s.index, i, s.wide);
    return v < 0 ? -1 : v >= s.n ? s.n : (int)v;
}
// How many tiles of TM rows the segments have.  Every warp works it out by itself.
template <int TM>
__device__ __forceinline__ int64_t count_tiles(const Segments& s) {
    int n = 0;
#pragma unroll 4
    for (int i = threadIdx.x & 31; i < s.S; i += 32) {
        const int rows = offset_at(s, i + 1) - offset_at(s, i);
        if (rows > 0) n += (rows + TM - 1) / TM;
    }
    return __reduce_add_sync(0xffffffffu, n);
}
// Tile number `tile` of the segments' tiles of TM rows.  Every warp works it out by itself: 128 segments per round.
template <int TM>
__device__ __forceinline__ RowTile find_tile(const Segments& s, int tile) {
    const int lane = threadIdx.x & 31;
    RowTile r{0, 0, -1};
    for (int base = 0; base < s.S; base += 128) {
        int at[5], id[4], n[4], sum = 0;
#pragma unroll
        for (int j = 0; j < 5; ++j) {
            const int i = base + lane * 4 + j;
            at[j] = offset_at(s, min(i, s.S));
            if (j < 4) id[j] = i < s.S ? adapter_at(s, i) : -1;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            n[j] = at[j + 1] > at[j] ? (at[j + 1] - at[j] + TM - 1) / TM : 0;
            sum += n[j];
        }
        int scan = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += v;
        }
        const uint32_t has = __ballot_sync(0xffffffffu, tile < scan);
        if (has) {
            int from = scan - sum;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (tile >= from && tile < from + n[j]) {
                    r.row = at[j] + (tile - from) * TM;
                    r.rows = min(TM, at[j + 1] - r.row);
                    r.id = id[j];
                }
                from += n[j];
            }
            const int who = __ffs(has) - 1;            // the first lane whose segments reach the tile
            r.row = __shfl_sync(0xffffffffu, r.row, who);
            r.rows = __shfl_sync(0xffffffffu, r.rows, who);
            r.id = __shfl_sync(0xffffffffu, r.id, who);
            return r;
        }
        tile -= __shfl_sync(0xffffffffu, scan, 31);
    }
    return r;
}

// ---- tensor core steps ---------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
template <bool TRANS>
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t at) {
    if constexpr (TRANS)
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
    else
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void stmatrix4(const uint32_t (&r)[4], uint32_t at) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// ---- asynchronous copies ---------------------------------------------------------------------------------
__device__ __forceinline__ void copy16(uint32_t to, const void* from, int bytes) {     // what is missing is zero
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Eight 16-bit elements on a boundary of their own size, of which n (may be <= 0) exist: three words and two elements beside them
// where all do, so that nothing else is read.
__device__ __forceinline__ void any8(const unsigned short* s, int n, uint32_t (&w)[4]) {
    w[0] = w[1] = w[2] = w[3] = 0;
    if (n >= 8) {
        const bool odd = reinterpret_cast<uintptr_t>(s) & 2;
        const uint32_t* m = reinterpret_cast<const uint32_t*>(s + (odd ? 1 : 2));
        const uint32_t a = s[0], b = s[odd ? 7 : 1], m0 = m[0], m1 = m[1], m2 = m[2];
        w[0] = a | (odd ? m0 : b) << 16;
        w[1] = odd ? __byte_perm(m0, m1, 0x5432) : m0;
        w[2] = odd ? __byte_perm(m1, m2, 0x5432) : m1;
        w[3] = odd ? m2 >> 16 | b << 16 : m2;
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) w[i / 2] |= (uint32_t)s[i] << (16 * (i & 1));
    }
}
__device__ __forceinline__ void put8(uint32_t to, const uint32_t (&w)[4]) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
}
// Eight 16-bit elements to shared memory, of which n (may be <= 0) exist; vec: from is on a 16-byte boundary (and
// an address of the tensor, whether or not anything is there).
template <typename T>
__device__ __forceinline__ void stage8(uint32_t to, const T* from, int n, bool vec) {
    if (vec) {
        copy16(to, from, n <= 0 ? 0 : n >= 8 ? 16 : 2 * n);
    } else {
        uint32_t w[4];
        any8(reinterpret_cast<const unsigned short*>(from), n, w);
        put8(to, w);
    }
}
// ROWS x COLS elements (COLS a multiple of 8) from p, of which rows x cols exist; rows are `pitch` bytes apart in shared memory.
// Off 16-byte boundaries all loads of four pieces come before their stores (2246 rows x 8535, rank 128: 281 us, piece by piece 297).
template <typename T, int ROWS, int COLS, int THREADS>
__device__ __forceinline__ void stage_tile(uint32_t to, int pitch, const T* p, int64_t ld, int64_t rows, int64_t cols, bool vec) {
    constexpr int per = COLS / 8, N = 4;
    auto left = [&](int r, int c) { return r < rows ? (int)min((int64_t)8, cols - c) : 0; };
    if (vec) {
#pragma unroll 4
        for (int i = threadIdx.x; i < ROWS * per; i += THREADS) {
            const int r = i / per, c = i % per * 8, n = left(r, c);
            copy16(to + r * pitch + 2 * c, n > 0 ? p + (int64_t)r * ld + c : p, n <= 0 ? 0 : n >= 8 ? 16 : 2 * n);
        }
        return;
    }
#pragma unroll 1
    for (int first = threadIdx.x; first < ROWS * per; first += N * THREADS) {
        uint32_t w[N][4];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = first + j * THREADS, r = i / per, c = i % per * 8;
            any8(reinterpret_cast<const unsigned short*>(p + (int64_t)r * ld + c), i < ROWS * per ? left(r, c) : 0, w[j]);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = first + j * THREADS;
            if (i < ROWS * per) put8(to + i / per * pitch + i % per * 16, w[j]);
        }
    }
}

// ---- tiles by TMA ------------------------------------------------------------------------------------------
// A ring of stages that one warp fills and four empty.  Waits are bounded: on expiry the CTA gives up and raises the
// kernel's status word (gpd_device_status).
template <int STAGES>
struct Ring {
    uint64_t full[STAGES], empty[STAGES];
    int abort;
    // one thread; arrivals that fill a stage (beside the copies' bytes) and that empty it
    __device__ __forceinline__ void init(int fills, int empties) {
        for (int i = 0; i < STAGES; ++i) {
            tc::mbar_init(&full[i], fills);
            tc::mbar_init(&empty[i], empties);
        }
        abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __device__ __forceinline__ bool wait_full(int k, int* status) { return tc::mbar_wait(&full[k % STAGES], (k / STAGES) & 1, &abort, status); }
    __device__ __forceinline__ bool wait_empty(int k, int* status) { return tc::mbar_wait(&empty[k % STAGES], ((k / STAGES) & 1) ^ 1, &abort, status); }
    // After giving up: copies in flight land before the CTA's memory is another's.  `issued` stages were begun.
    __device__ __forceinline__ void drain(int issued, int* status) {
        int never = 0;
        if (*static_cast<volatile int*>(&abort))
            for (int k = issued > STAGES ? issued - STAGES : 0; k < issued; ++k)
                tc::mbar_wait(&full[k % STAGES], (k / STAGES) & 1, &never, status);
    }
};
// A lane's row and column in the 16 x 16 block that four matrices of a load make up: rows first (the two halves of an operand's
// depth in neighbouring registers where the block is transposed), or columns first.
__device__ __forceinline__ int row_first() { return threadIdx.x & 15; }
__device__ __forceinline__ int row_first_col() { return (threadIdx.x >> 4 & 1) * 8; }
__device__ __forceinline__ int col_first_row() { return (threadIdx.x & 7) + (threadIdx.x >> 4 & 1) * 8; }
__device__ __forceinline__ int col_first() { return (threadIdx.x >> 3 & 1) * 8; }
constexpr int per_sm(int smem) { return 227 * 1024 / (smem + 1536) < 5 ? 227 * 1024 / (smem + 1536) : 5; }     // CTAs that shared memory has room for
// Byte of a tile whose rows are PITCH (32, 64 or 128) bytes, as TMA's swizzle of that width places it (the tile starts on a
// 1024-byte boundary): eight rows' pieces of 16 bytes at one column lie in different banks.
template <int PITCH>
__device__ __forceinline__ uint32_t swizzled(uint32_t byte) { return byte ^ ((byte >> 7 & (PITCH / 16 - 1)) << 4); }
// Factors' tiles of ROWS x COLS elements: columns in parts of 64 (128 bytes), one behind the other.
template <int ROWS, int COLS>
struct WTile {
    static constexpr int PITCH = COLS >= 64 ? 128 : 2 * COLS, PARTS = COLS > 64 ? COLS / 64 : 1, BYTES = ROWS * COLS * 2;
    static __device__ __forceinline__ uint32_t at(int row, int col) {
        return (uint32_t)(col / 64 * ROWS * 128) + swizzled<PITCH>((uint32_t)(row * PITCH + col % 64 * 2));
    }
    // The same in two steps, for addresses of matrix loads: a lane's place (row below 16, column 0 or 8) in the tile at `tile`,
    // and from there, by one operation, the place `row` (a multiple of 8) rows and `col` (a multiple of 16) columns on.
    static __device__ __forceinline__ uint32_t lane_at(uint32_t tile, int row, int col) { return tile + swizzled<PITCH>((uint32_t)(row * PITCH + col * 2)); }
    static __device__ __forceinline__ uint32_t on(uint32_t lane, int row, int col) {
        return (lane ^ (uint32_t)(col % 64 * 2)) + (uint32_t)(row * PITCH + col / 64 * ROWS * 128);
    }
    static __device__ __forceinline__ void load(unsigned char* to, const CUtensorMap* map, int col, int row, int id, uint64_t* bar) {
#pragma unroll
        for (int i = 0; i < PARTS; ++i) tc::tma_load_3d(to + i * ROWS * 128, map, col + 64 * i, row, id, bar);
    }
    // Element by element, by one warp: rows off 16-byte boundaries.  What lies outside is zero already, or is written so.
    // BY_ROW: a lane has two of the 64 rows, and `rank` columns of them are used; otherwise two of the 64 columns, and `rank`
    // rows.  All loads of eight of these before the first store.
    template <bool BY_ROW, typename T>
    static __device__ __forceinline__ void copy(unsigned char* to, const T* p, int64_t ld, int64_t rows, int64_t cols, int rank) {
        const int lane = threadIdx.x & 31;
        constexpr int N = 8;
        for (int first = 0; first < rank; first += N) {
            T v[N][2];
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int r = BY_ROW ? lane + 32 * i : first + j, c = BY_ROW ? first + j : lane + 32 * i;
                    v[j][i] = from_f32<T>(0.f);
                    if (first + j < rank && r < rows && c < cols) v[j][i] = p[r * ld + c];
                }
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (first + j < rank) *reinterpret_cast<T*>(to + (BY_ROW ? at(lane + 32 * i, first + j) : at(first + j, lane + 32 * i))) = v[j][i];
        }
    }
};

// ---- numbers of FP32 as sums of 16-bit ones ----------------------------------------------------------------
// x = parts[0] + parts[1] + parts[2] up to 2^-25 of it in BF16, two at a time.  An infinity or a NaN
// is its first part, the others are then zero.  FP16: 2^-23 (two parts) or 2^-34 of it, or 2^-25 where that is more: its
// smallest numbers are 2^-24 apart.
template <typename T, int PARTS>
__device__ __forceinline__ void split2(float x, float y, uint32_t (&parts)[PARTS]) {
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        parts[i] = pack2(x, y, T());
        const float2 f = unpack2(parts[i], T());
        x = fabsf(f.x) <= 3.4e38f ? x - f.x : 0.f;
        y = fabsf(f.y) <= 3.4e38f ? y - f.y : 0.f;
    }
}
// e with m * 2^-e below 2^15 (FP16 parts of numbers of any size) and both 2^e and 2^-e normal; 0 for zeros, infinities and NaN.
// So near the top of FP16's range that three parts hold all 24 bits of what is down to 2^-14 of m, and 2^-39 of m of the rest.
__device__ __forceinline__ int exponent_of(float m) {
    const int e = (int)(__float_as_uint(m) >> 23 & 0xff);
    return e == 0xff || m == 0.f ? 0 : max(e - 127 - 14, -126);
}
// Parts that an FP32 factor is cut into.  Three lose nothing of its 24 bits.  Two of FP16, 22 bits, are enough for results of FP16;
// two of BF16 would be 16 bits, which 16-bit results hide only until terms cancel (and flip one rounding in 400 where they do not).
template <typename T, typename O> constexpr int kParts = sizeof(O) == 4 || std::is_same<T, __nv_bfloat16>::value ? 3 : 2;
__device__ __forceinline__ float power2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // |e| <= 126

// ---- launches (host) -----------------------------------------------------------------------------------
struct ShrinkArgs {                                    // h[t] = scale_i W_i x[t]
    Segments seg;
    const void* x; int64_t ldx;
    const void* w; int64_t ldw, next;                  // rows of W, adapters apart; transposed: W_i is [C][r]
    const float* scale;
    float* h;                                          // [T][r]
    int64_t C;                                         // columns of x
    int r;
    bool x_vec, w_vec;
};
struct ExpandArgs {                                    // out[t] = base[t] + scale_i W_i h[t]
    Segments seg;
    const float* h;
    const void* w; int64_t ldw, next;                  // W_i is [C][r]; transposed: [r][C]
    const float* scale;
    const void* base; int64_t ldb;
    void* out; int64_t ldo;
    int64_t C;                                         // columns of out
    int r;
    bool w_vec, io_vec, tma;                           // W on 16-byte boundaries; base and out: pairs or eights; both on 16 bytes
};
struct GradArgs {                                      // dW_i[c][k] = scale_i sum_t y[t][c] h[t][k], over the rows of adapter i
    const void* y; int64_t ldy;
    const float* h;
    const float* scale;
    void* dw; int64_t ldw, next;                       // [C][r]; transposed: [r][C]
    int64_t C;
    bool y_vec, transposed;
};
gpd_status shrink(int type, bool transposed, const ShrinkArgs& a, cudaStream_t st);
gpd_status expand(int type, int out_type, bool transposed, const ExpandArgs& a, cudaStream_t st);
gpd_status short_segments(int type, int out_type, const ShrinkArgs& down, const ExpandArgs& above, bool* taken, cudaStream_t st);
int64_t grad_workspace(int64_t T, int64_t n, int64_t r, int64_t K, int64_t N);
bool gradients_fit(const Segments& seg, const GradArgs (&two)[2]);
gpd_status gradients(int type, int grad_type, bool accumulate, const Segments& seg, int r, const GradArgs (&two)[2], void* workspace,
                     cudaStream_t st);

int shrink_status_fetch_and_clear();                   // synchronous reads of the kernels' status words
int expand_status_fetch_and_clear();
int short_status_fetch_and_clear();
int grad_status_fetch_and_clear();

// n matrices of rows x cols (rows ld apart, matrices next) in boxes of box_rows x box_cols; rows of a box are swizzled over
// their whole width; elements outside read as zero and are not written.
inline bool make_map(CUtensorMap* map, const void* base, int elem, int64_t n, int64_t rows, int64_t cols, int64_t ld, int64_t next, int box_rows,
                     int box_cols) {
    tc::EncodeTiledFn fn = tc::encode_tiled_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)n};
    cuuint64_t strides[2] = {(cuuint64_t)(ld * elem), (cuuint64_t)((n > 1 ? next : ld) * elem)};
    cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    const int width = box_cols * elem;
    return fn(map, elem == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, const_cast<void*>(base), dims, strides, box,
              estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              width == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : width == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

inline int64_t tiles_of(const Segments& s, int TM) { return s.T / TM + (s.S < s.T ? s.S : s.T); }

}  // namespace adapter
}  // namespace gpd
