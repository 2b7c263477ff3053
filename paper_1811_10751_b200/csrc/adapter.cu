// Entry points of low-rank adapters beside a shared projection: argument checks, and the order of the kernels.
#include "adapter_common.h"
#include "gemm_common.h"

using namespace gpd;
using namespace gpd::adapter;

namespace {

// Rows, segments and adapters are counted in 32 bits: there is room for the steps of the loops over them.
constexpr int32_t kMost = 1 << 30;
bool sizes_fit(int64_t T, int64_t K, int64_t N, int32_t n, int32_t r) {
    return T >= 0 && T <= GPD_LM_MAX_ROWS && K > 0 && N > 0 && K <= GPD_LM_MAX_ROWS && N <= GPD_LM_MAX_ROWS && n >= 0 && n <= kMost && r > 0 && r <= kMaxRank;
}
gpd_status check_adapters(int type, int64_t T, int64_t K, int64_t N, int32_t n, int32_t r, const void* A, int64_t lda, int64_t next_a,
                          const void* B, int64_t ldb, int64_t next_b, int32_t index_bytes, const void* offsets, const void* index, int32_t S) {
    if (type != GPD_DT_BF16 && type != GPD_DT_F16) return GPD_ERR_ARG;
    if (!sizes_fit(T, K, N, n, r) || S < 0 || S > kMost) return GPD_ERR_SHAPE;
    if (lda < K || ldb < r || (n > 1 && (next_a < lda * (r - 1) + K || next_b < ldb * (N - 1) + r))) return GPD_ERR_SHAPE;
    if (index_bytes != 4 && index_bytes != 8) return GPD_ERR_ARG;
    if (n > 0 && (!A || !B)) return GPD_ERR_ARG;
    if (S > 0 && (!offsets || !index)) return GPD_ERR_ARG;
    return GPD_OK;
}
bool weights_aligned(const void* w, int64_t ld, int64_t next) { return lm::rows_aligned(w, ld, 2) && next % 8 == 0; }
int64_t up(int64_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace

int gpd::adapter_status_fetch_and_clear() {
    const int a = shrink_status_fetch_and_clear(), b = expand_status_fetch_and_clear(), c = grad_status_fetch_and_clear(), d = short_status_fetch_and_clear();
    return a != 0 ? a : b != 0 ? b : c != 0 ? c : d;
}

extern "C" gpd_status gpd_adapter(gpd_dtype type, const void* x_dev, int64_t ldx, int32_t n, int32_t r, const void* A_dev, int64_t lda,
                                  int64_t next_a, const void* B_dev, int64_t ldb, int64_t next_b, const float* scale_dev,
                                  int32_t index_bytes, const void* offsets_dev, const void* index_dev, int32_t S, float* h_dev,
                                  gpd_dtype out_type, const void* base_dev, int64_t ldbase, void* out_dev, int64_t ldo, int64_t T,
                                  int64_t K, int64_t N, void* stream) {
    const gpd_status rc = check_adapters(type, T, K, N, n, r, A_dev, lda, next_a, B_dev, ldb, next_b, index_bytes, offsets_dev, index_dev, S);
    if (rc != GPD_OK) return rc;
    if (out_type != type && out_type != GPD_DT_F32) return GPD_ERR_ARG;
    if (T == 0 || S == 0) return GPD_OK;               // no rows: nothing is written
    if (!x_dev || !h_dev || !out_dev) return GPD_ERR_ARG;
    if (ldx < K || ldo < N || (base_dev && ldbase < N)) return GPD_ERR_SHAPE;
    const Segments seg{offsets_dev, index_dev, T, S, n, index_bytes == 8};
    const int e = lm::dtype_size(out_type), wide = e == 4 ? 8 : 16;
    cudaStream_t st = as_stream(stream);
    const ShrinkArgs down{seg, x_dev, ldx, A_dev, lda, next_a, nullptr, h_dev, K, r, lm::rows_aligned(x_dev, ldx, 2),
                          weights_aligned(A_dev, lda, next_a)};
    const ExpandArgs above{seg, h_dev, B_dev, ldb, next_b, scale_dev, base_dev, ldbase, out_dev, ldo, N, r, weights_aligned(B_dev, ldb, next_b),
                           lm::rows_aligned(base_dev, ldbase, e, wide) && lm::rows_aligned(out_dev, ldo, e, wide),
                           lm::rows_aligned(base_dev, ldbase, e) && lm::rows_aligned(out_dev, ldo, e)};
    bool taken = false;
    const gpd_status both = short_segments(type, out_type, down, above, &taken, st);
    if (both != GPD_OK || taken) return both;
    const gpd_status first = shrink(type, false, down, st);
    return first != GPD_OK ? first : expand(type, out_type, false, above, st);
}

extern "C" gpd_status gpd_adapter_backward_workspace(int64_t T, int64_t K, int64_t N, int32_t n, int32_t r, int64_t* bytes_host) {
    if (!bytes_host) return GPD_ERR_ARG;
    if (!sizes_fit(T, K, N, n, r)) return GPD_ERR_SHAPE;
    *bytes_host = up(4 * T * r) + grad_workspace(T, n, r, K, N);
    return GPD_OK;
}

extern "C" gpd_status gpd_adapter_backward(gpd_dtype type, const void* dout_dev, int64_t lddo, const void* x_dev, int64_t ldx, int32_t n,
                                           int32_t r, const void* A_dev, int64_t lda, int64_t next_a, const void* B_dev, int64_t ldb,
                                           int64_t next_b, const float* scale_dev, const float* h_dev, int32_t index_bytes,
                                           const void* offsets_dev, const void* index_dev, int32_t S, gpd_dtype dx_type,
                                           const void* dbase_dev, int64_t lddb, void* dx_dev, int64_t lddx, gpd_dtype grad_type,
                                           void* dA_dev, int64_t ldda, int64_t next_da, void* dB_dev, int64_t lddB, int64_t next_db,
                                           int32_t accumulate, int64_t T, int64_t K, int64_t N, void* workspace_dev,
                                           int64_t workspace_bytes, void* stream) {
    const gpd_status rc = check_adapters(type, T, K, N, n, r, A_dev, lda, next_a, B_dev, ldb, next_b, index_bytes, offsets_dev, index_dev, S);
    if (rc != GPD_OK) return rc;
    if ((!dA_dev) != (!dB_dev) && n > 0) return GPD_ERR_ARG;
    const bool grads = dA_dev && n > 0, rows = T > 0 && S > 0;
    if (dx_dev && dx_type != type && dx_type != GPD_DT_F32) return GPD_ERR_ARG;
    if (grads && grad_type != type && grad_type != GPD_DT_F32) return GPD_ERR_ARG;
    if (grads && (ldda < K || lddB < r || (n > 1 && (next_da < ldda * (r - 1) + K || next_db < lddB * (N - 1) + r)))) return GPD_ERR_SHAPE;
    if (!dx_dev && !grads) return GPD_OK;
    if (rows) {
        if (!dout_dev || (grads && (!x_dev || !h_dev))) return GPD_ERR_ARG;
        if (lddo < N || (grads && ldx < K) || (dx_dev && (lddx < K || (dbase_dev && lddb < K)))) return GPD_ERR_SHAPE;
    }
    if (!rows && !grads) return GPD_OK;
    const int64_t own = up(4 * T * r);
    if (!workspace_dev || workspace_bytes < own + grad_workspace(T, n, r, K, N) || !lm::aligned(workspace_dev, 16)) return GPD_ERR_WORKSPACE;
    const Segments seg{offsets_dev, index_dev, T, rows ? S : 0, n, index_bytes == 8};
    cudaStream_t st = as_stream(stream);
    float* u = static_cast<float*>(workspace_dev);     // scale_i B_i^T dout, [T][r]
    // dB first: dout may still be in L2
    const GradArgs two[2] = {{dout_dev, lddo, h_dev, scale_dev, dB_dev, lddB, next_db, N, lm::rows_aligned(dout_dev, lddo, 2), false},
                             {x_dev, ldx, u, nullptr, dA_dev, ldda, next_da, K, lm::rows_aligned(x_dev, ldx, 2), true}};
    if (grads && !gradients_fit(seg, two)) return GPD_ERR_SHAPE;
    if (rows) {
        const ShrinkArgs down{seg, dout_dev, lddo, B_dev, ldb, next_b, scale_dev, u, N, r, lm::rows_aligned(dout_dev, lddo, 2),
                              weights_aligned(B_dev, ldb, next_b)};
        const gpd_status s = shrink(type, true, down, st);
        if (s != GPD_OK) return s;
    }
    if (grads) {                                       // before dx
        const gpd_status s = gradients(type, grad_type, accumulate != 0, seg, r, two, static_cast<unsigned char*>(workspace_dev) + own, st);
        if (s != GPD_OK) return s;
    }
    if (!rows || !dx_dev) return GPD_OK;
    const int e = lm::dtype_size(dx_type), wide = e == 4 ? 8 : 16;
    const ExpandArgs above{seg, u, A_dev, lda, next_a, nullptr, dbase_dev, lddb, dx_dev, lddx, K, r, weights_aligned(A_dev, lda, next_a),
                           lm::rows_aligned(dbase_dev, lddb, e, wide) && lm::rows_aligned(dx_dev, lddx, e, wide),
                           lm::rows_aligned(dbase_dev, lddb, e) && lm::rows_aligned(dx_dev, lddx, e)};
    return expand(type, dx_type, true, above, st);
}
