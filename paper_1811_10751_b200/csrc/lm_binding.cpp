// Python calls of the low-precision layer and output-head operators (lm.py) into libgpd.so.  The smallest of
// them run for two or three microseconds on the GPU, so the checks of their ten to twenty arguments are made
// here, in well under a microsecond each, instead of in Python.  Every function takes its arguments by
// position, raises ValueError for wrong devices, types, shapes or strides, and returns the library's status.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdarg>
#include <cstdio>
#include <stdexcept>
#include <string>
#include <vector>

#include "gpd.h"

namespace {

using at::ScalarType;

constexpr int64_t kBlock = 128;
inline int64_t blocks(int64_t n, int64_t per = kBlock) { return (n + per - 1) / per; }

// Sets of element types
enum : unsigned { kF32 = 1, kBF16 = 2, kF16 = 4, kE4M3 = 8, kE5M2 = 16, kE8M0 = 32, kU8 = 64, kI32 = 128, kI64 = 256, kOther = 0 };
constexpr unsigned kFloats = kF32 | kBF16 | kF16, kFp8 = kE4M3 | kE5M2, kScales = kE8M0 | kU8, kIndex = kI32 | kI64;
unsigned type_bit(ScalarType t) {
    switch (t) {
        case ScalarType::Float: return kF32;
        case ScalarType::BFloat16: return kBF16;
        case ScalarType::Half: return kF16;
        case ScalarType::Float8_e4m3fn: return kE4M3;
        case ScalarType::Float8_e5m2: return kE5M2;
        case ScalarType::Float8_e8m0fnu: return kE8M0;
        case ScalarType::Byte: return kU8;
        case ScalarType::Int: return kI32;
        case ScalarType::Long: return kI64;
        default: return kOther;
    }
}
gpd_dtype gpd_type(unsigned bit) {
    return bit == kF32 ? GPD_DT_F32 : bit == kBF16 ? GPD_DT_BF16 : bit == kF16 ? GPD_DT_F16 : bit == kE4M3 ? GPD_DT_E4M3 : GPD_DT_E5M2;
}
std::string type_names(unsigned set) {
    static const char* names[] = {"float32", "bfloat16", "float16", "float8_e4m3fn", "float8_e5m2", "float8_e8m0fnu", "uint8", "int32", "int64"};
    std::string s;
    for (int i = 0; i < 9; ++i)
        if (set >> i & 1) s += (s.empty() ? "" : " or ") + std::string(names[i]);
    return s;
}

struct Refusal : std::invalid_argument { using std::invalid_argument::invalid_argument; };
[[noreturn]] void refuse(const char* name, const std::string& why) { throw Refusal(std::string(name) + ": " + why); }
struct PythonError {};                                 // the interpreter's error is set already

std::string shape_text(const at::Tensor& t) {
    std::string s = "(";
    for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
    return s + ")";
}

// The device and stream of a call, and its arguments.
class Call {
public:
    Call(PyObject* const* args, Py_ssize_t n, Py_ssize_t want) : args_(args) {
        if (n != want) throw Refusal("wrong number of arguments");
    }
    bool absent(int i) const { return args_[i] == Py_None; }
    const at::Tensor& tensor(const char* name, int i) const {
        if (!THPVariable_Check(args_[i])) refuse(name, "tensor expected");
        return THPVariable_Unpack(args_[i]);
    }
    double number(int i) const {
        const double v = PyFloat_AsDouble(args_[i]);
        if (v == -1.0 && PyErr_Occurred()) throw PythonError();
        return v;
    }
    int64_t integer(int i) const {
        const long long v = PyLong_AsLongLong(args_[i]);
        if (v == -1 && PyErr_Occurred()) throw PythonError();
        return v;
    }
    // The leading tensor: fixes the device (the current one) and the shape.
    const at::Tensor& lead(const char* name, int i, unsigned types, int dims = 2) {
        const at::Tensor& t = tensor(name, i);
        if (!t.is_cuda()) refuse(name, "device tensor expected");
        device_ = t.device();
        const int current = c10::cuda::current_device();
        if (device_.index() != current)
            refuse(name, "tensor is on cuda:" + std::to_string(device_.index()) + ", the current device is cuda:" + std::to_string(current));
        if (t.dim() != dims) refuse(name, std::string(dims == 2 ? "matrix" : "vector") + " expected, got shape " + shape_text(t));
        check_type(name, t, types);
        return t;
    }
    unsigned check_type(const char* name, const at::Tensor& t, unsigned types) const {
        const unsigned b = type_bit(t.scalar_type());
        if (!(b & types)) refuse(name, type_names(types) + " expected, got " + c10::toString(t.scalar_type()));
        return b;
    }
    struct Mat { void* p = nullptr; int64_t ld = 0; unsigned type = 0; };
    // [rows, cols] with adjacent columns; none: null
    Mat mat(const char* name, int i, unsigned types, int64_t rows, int64_t cols) const {
        Mat m;
        if (absent(i)) return m;
        const at::Tensor& t = tensor(name, i);
        m.type = check_type(name, t, types);
        check_device(name, t);
        if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols)
            refuse(name, "shape (" + std::to_string(rows) + ", " + std::to_string(cols) + ") expected, got " + shape_text(t));
        m.ld = t.stride(0);
        if (cols > 1 && t.stride(1) != 1) refuse(name, "columns have to be adjacent");
        if (m.ld < cols) {
            if (rows > 1) refuse(name, "rows overlap");
            m.ld = cols;
        }
        m.p = t.data_ptr();
        return m;
    }
    Mat need_mat(const char* name, int i, unsigned types, int64_t rows, int64_t cols) const {
        if (absent(i)) refuse(name, "needed");
        return mat(name, i, types, rows, cols);
    }
    // contiguous, `n` elements, [n] or, with G >= 0, [T] (G = 1) or [T, G]
    void* vec(const char* name, int i, unsigned types, int64_t n, unsigned* type = nullptr) const {
        if (absent(i)) return nullptr;
        const at::Tensor& t = tensor(name, i);
        const unsigned b = check_type(name, t, types);
        if (type) *type = b;
        check_device(name, t);
        if (t.dim() != 1 || t.size(0) != n || (n > 1 && t.stride(0) != 1))
            refuse(name, "contiguous vector of " + std::to_string(n) + " expected, got shape " + shape_text(t));
        return t.data_ptr();
    }
    void* need_vec(const char* name, int i, unsigned types, int64_t n, unsigned* type = nullptr) const {
        if (absent(i)) refuse(name, "needed");
        return vec(name, i, types, n, type);
    }
    void* per_row(const char* name, int i, unsigned types, int64_t T, int64_t G) const {
        if (absent(i)) return nullptr;
        const at::Tensor& t = tensor(name, i);
        check_type(name, t, types);
        check_device(name, t);
        const bool shape = t.dim() == 2 ? t.size(0) == T && t.size(1) == G : t.dim() == 1 && G == 1 && t.size(0) == T;
        if (!shape || !t.is_contiguous())
            refuse(name, "contiguous (" + std::to_string(T) + ", " + std::to_string(G) + ") tensor expected, got shape " + shape_text(t));
        return t.data_ptr();
    }
    // contiguous, of any type
    void* buffer(const char* name, int i, int64_t* bytes) const {
        if (absent(i)) refuse(name, "needed");
        const at::Tensor& t = tensor(name, i);
        check_device(name, t);
        if (!t.is_contiguous()) refuse(name, "contiguous buffer expected");
        *bytes = t.numel() * (int64_t)t.element_size();
        return t.data_ptr();
    }
    void check_device(const char* name, const at::Tensor& t) const {
        if (t.device() != device_) refuse(name, "tensor on cuda:" + std::to_string(device_.index()) + " expected, got " + t.device().str());
    }
    // None: the current stream; else an object with `cuda_stream`, or a handle
    void* stream(int i) const {
        PyObject* o = args_[i];
        if (o == Py_None) return c10::cuda::getCurrentCUDAStream(device_.index()).stream();
        PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
        if (!h) {
            PyErr_Clear();
            h = Py_NewRef(o);
        }
        void* p = PyLong_AsVoidPtr(h);
        Py_DECREF(h);
        if (!p && PyErr_Occurred()) throw PythonError();
        return p;
    }

private:
    PyObject* const* args_;
    at::Device device_{at::kCPU};
};

gpd_status rmsnorm_quant(PyObject* const* args, Py_ssize_t n) {
    // x, weight, eps, residual, residual_out, y, q, scales, rstd, stream
    Call c(args, n, 10);
    const at::Tensor& x = c.lead("x", 0, kFloats);
    const int64_t T = x.size(0), H = x.size(1);
    const unsigned same = type_bit(x.scalar_type());
    const auto mx = c.mat("x", 0, same, T, H), mr = c.mat("residual", 3, same, T, H);
    unsigned wt = 0;
    void* w = c.need_vec("weight", 1, same | kF32, H, &wt);
    const auto mh = c.mat("residual_out", 4, same, T, H), my = c.mat("y", 5, same, T, H), mq = c.mat("q", 6, kFp8, T, H);
    if (c.absent(6) != c.absent(7)) throw Refusal("8-bit values and their scales go together");
    const auto ms = c.mat("scales", 7, kScales, T, blocks(H));
    float* rstd = static_cast<float*>(c.vec("rstd", 8, kF32, T));
    return gpd_rmsnorm_quant(gpd_type(same), mx.p, mx.ld, mr.p, mr.ld, gpd_type(wt), w, (float)c.number(2), mh.p, mh.ld, my.p, my.ld,
                             mq.type ? gpd_type(mq.type) : GPD_DT_E4M3, mq.p, mq.ld, static_cast<uint8_t*>(ms.p), ms.ld, rstd, T, H,
                             c.stream(9));
}

gpd_status rmsnorm_backward(PyObject* const* args, Py_ssize_t n) {
    // dy, h, weight, rstd, dx, dweight, workspace, dresidual, stream
    Call c(args, n, 9);
    const at::Tensor& h = c.lead("h", 1, kFloats);
    const int64_t T = h.size(0), H = h.size(1);
    const unsigned same = type_bit(h.scalar_type());
    const auto mdy = c.need_mat("dy", 0, same, T, H), mh = c.mat("h", 1, same, T, H), md = c.mat("dresidual", 7, same, T, H),
               mx = c.need_mat("dx", 4, same, T, H);
    unsigned wt = 0;
    void* w = c.need_vec("weight", 2, same | kF32, H, &wt);
    float* rstd = static_cast<float*>(c.need_vec("rstd", 3, kF32, T));
    float* dw = static_cast<float*>(c.need_vec("dweight", 5, kF32, H));
    const at::Tensor& ws = c.tensor("workspace", 6);
    c.check_device("workspace", ws);
    if (!ws.is_contiguous()) refuse("workspace", "contiguous buffer expected");
    return gpd_rmsnorm_backward(gpd_type(same), mdy.p, mdy.ld, mh.p, mh.ld, gpd_type(wt), w, rstd, md.p, md.ld, mx.p, mx.ld, dw, T, H,
                                ws.data_ptr(), ws.numel() * (int64_t)ws.element_size(), c.stream(8));
}

gpd_status quantize_blocks(PyObject* const* args, Py_ssize_t n) {
    // src, q, scales, qT, scalesT, block_rows, stream
    Call c(args, n, 7);
    const at::Tensor& src = c.lead("src", 0, kFloats);
    const int64_t M = src.size(0), K = src.size(1), br = c.integer(5);
    if (br != 1 && br != kBlock) refuse("block_rows", "1 or 128");
    if (c.absent(1) && c.absent(3)) throw Refusal("q or qT: one of them is needed");
    if (c.absent(1) != c.absent(2) || c.absent(3) != c.absent(4)) throw Refusal("8-bit values and their scales go together");
    const auto ms = c.mat("src", 0, kFloats, M, K), mq = c.mat("q", 1, kFp8, M, K), mqs = c.mat("scales", 2, kScales, blocks(M, br), blocks(K)),
               mt = c.mat("qT", 3, kFp8, K, M), mts = c.mat("scalesT", 4, kScales, blocks(K, br), blocks(M));
    if (mq.type && mt.type && mq.type != mt.type) throw Refusal("q and qT: one 8-bit type expected");
    return gpd_quantize_blocks(gpd_type(ms.type), ms.p, ms.ld, gpd_type(mq.type ? mq.type : mt.type), (int32_t)br, mq.p, mq.ld,
                               static_cast<uint8_t*>(mqs.p), mqs.ld, mt.p, mt.ld, static_cast<uint8_t*>(mts.p), mts.ld, M, K, c.stream(6));
}

gpd_status gemm_fp8(PyObject* const* args, Py_ssize_t n) {
    // A, a_scales, B, b_scales, out, accumulate, stream
    Call c(args, n, 7);
    const at::Tensor& A = c.lead("A", 0, kFp8);
    const at::Tensor& B = c.tensor("B", 2);
    if (B.dim() != 2) refuse("B", "matrix expected, got shape " + shape_text(B));
    const int64_t M = A.size(0), K = A.size(1), N = B.size(0), kb = blocks(K);
    // one scale row per operand row, or per 128 of them
    auto scales = [&](const char* name, int i, int64_t rows, int32_t& br) {
        const at::Tensor& s = c.tensor(name, i);
        const int64_t r = s.dim() == 2 ? s.size(0) : -1;
        if (r != rows && r != blocks(rows))
            refuse(name, std::to_string(rows) + " or " + std::to_string(blocks(rows)) + " rows of scales expected, got shape " + shape_text(s));
        br = r == rows ? 1 : (int32_t)kBlock;
        return c.mat(name, i, kScales, r, kb);
    };
    auto ma = c.mat("A", 0, kFp8, M, K), mb = c.need_mat("B", 2, kFp8, N, K);
    int32_t ra = 1, rb = 1;
    const auto msa = scales("a_scales", 1, M, ra), msb = scales("b_scales", 3, N, rb);
    const auto mo = c.need_mat("out", 4, kFloats, M, N);
    if (M == 1) ma.ld = blocks(ma.ld, 16) * 16;        // a single row has no stride
    if (N == 1) mb.ld = blocks(mb.ld, 16) * 16;
    const int acc = PyObject_IsTrue(args[5]);
    if (acc < 0) throw PythonError();
    return gpd_gemm_fp8(gpd_type(ma.type), ma.p, ma.ld, static_cast<uint8_t*>(msa.p), msa.ld, ra, gpd_type(mb.type), mb.p, mb.ld,
                        static_cast<uint8_t*>(msb.p), msb.ld, rb, gpd_type(mo.type), mo.p, mo.ld, M, N, K, acc, c.stream(6));
}

int64_t tokens_per_row(const at::Tensor& t) {
    if (t.dim() == 1) return 1;
    if (t.dim() == 2 && t.size(1) <= 0x7fffffff) return t.size(1);
    refuse("tokens", "[T] or [T, G] expected, got shape " + shape_text(t));
}

gpd_status token_logprobs(PyObject* const* args, Py_ssize_t n) {
    // logits, tokens, logprobs, lse, entropy, top_ids, top_logprobs, temperature, stream
    Call c(args, n, 9);
    const at::Tensor& x = c.lead("logits", 0, kFloats);
    const int64_t T = x.size(0), V = x.size(1);
    const auto mx = c.mat("logits", 0, kFloats, T, V);
    const at::Tensor& tok = c.tensor("tokens", 1);
    const int64_t G = tokens_per_row(tok);
    int64_t K = 0;
    if (!c.absent(5)) {
        const at::Tensor& ids = c.tensor("top_ids", 5);
        if (ids.dim() != 2 || ids.size(1) > 0x7fffffff) refuse("top_ids", "matrix expected, got shape " + shape_text(ids));
        K = ids.size(1);
    } else if (!c.absent(6)) {
        throw Refusal("top_ids: needed with top_logprobs");
    }
    void* pt = c.per_row("tokens", 1, kIndex, T, G);
    float* lp = static_cast<float*>(c.per_row("logprobs", 2, kF32, T, G));
    float* lse = static_cast<float*>(c.need_vec("lse", 3, kF32, T));
    float* H = static_cast<float*>(c.vec("entropy", 4, kF32, T));
    int32_t* ids = static_cast<int32_t*>(c.per_row("top_ids", 5, kI32, T, K));
    float* tlp = static_cast<float*>(c.per_row("top_logprobs", 6, kF32, T, K));
    return gpd_token_logprobs(gpd_type(mx.type), mx.p, mx.ld, (int32_t)tok.element_size(), pt, (int32_t)G, (float)c.number(7), lp, lse, H,
                              (int32_t)K, ids, tlp, T, V, c.stream(8));
}

gpd_status token_logprobs_backward(PyObject* const* args, Py_ssize_t n) {
    // logits, tokens, lse, entropy, dlogprobs, dentropy, dlogits, temperature, stream
    Call c(args, n, 9);
    const at::Tensor& x = c.lead("logits", 0, kFloats);
    const int64_t T = x.size(0), V = x.size(1);
    const auto mx = c.mat("logits", 0, kFloats, T, V), md = c.need_mat("dlogits", 6, type_bit(x.scalar_type()), T, V);
    const at::Tensor& tok = c.tensor("tokens", 1);
    const int64_t G = tokens_per_row(tok);
    void* pt = c.per_row("tokens", 1, kIndex, T, G);
    const float* lse = static_cast<float*>(c.need_vec("lse", 2, kF32, T));
    const float* H = static_cast<float*>(c.vec("entropy", 3, kF32, T));
    const float* gl = static_cast<float*>(c.per_row("dlogprobs", 4, kF32, T, G));
    const float* gh = static_cast<float*>(c.vec("dentropy", 5, kF32, T));
    return gpd_token_logprobs_backward(gpd_type(mx.type), mx.p, mx.ld, (int32_t)tok.element_size(), pt, (int32_t)G, (float)c.number(7), lse,
                                       H, gl, gh, md.p, md.ld, T, V, c.stream(8));
}

gpd_status distill_topk(PyObject* const* args, Py_ssize_t n) {
    // logits, teacher_ids, teacher_logits, weights, loss, dlogits, temperature, stream
    Call c(args, n, 8);
    const at::Tensor& x = c.lead("logits", 0, kFloats);
    const int64_t T = x.size(0), V = x.size(1);
    const at::Tensor& ids = c.tensor("teacher_ids", 1);
    if (ids.dim() != 2 || ids.size(1) > 0x7fffffff) refuse("teacher_ids", "matrix expected, got shape " + shape_text(ids));
    const int64_t K = ids.size(1);
    const auto mx = c.mat("logits", 0, kFloats, T, V), mi = c.mat("teacher_ids", 1, kIndex, T, K),
               mt = c.need_mat("teacher_logits", 2, kFloats, T, K), md = c.mat("dlogits", 5, type_bit(x.scalar_type()), T, V);
    const float* w = static_cast<float*>(c.vec("weights", 3, kF32, T));
    float* loss = static_cast<float*>(c.need_vec("loss", 4, kF32, T));
    return gpd_distill_topk(gpd_type(mx.type), mx.p, mx.ld, (int32_t)ids.element_size(), mi.p, mi.ld, gpd_type(mt.type), mt.p, mt.ld,
                            (int32_t)K, w, (float)c.number(6), loss, md.p, md.ld, T, V, c.stream(7));
}

// Queries or keys and their head count: [T, heads * D], None for no heads.
int32_t heads_of(const Call& c, const char* name, int i, int64_t T, int64_t D) {
    if (c.absent(i)) return 0;
    const at::Tensor& t = c.tensor(name, i);
    if (t.dim() != 2 || t.size(0) != T || t.size(1) % D || t.size(1) / D > GPD_HEAD_MAX_HEADS)
        refuse(name, "(" + std::to_string(T) + ", heads * " + std::to_string(D) + ") expected, got shape " + shape_text(t));
    return (int32_t)(t.size(1) / D);
}
// Table of angles, positions and axes from argument `at` on (table, positions, axes).
struct Angles {
    const float* table = nullptr;
    int64_t ldt = 0, P = 0, ldp = 0;
    int32_t R = 0, index_bytes = 4, n = 1;
    const void* pos = nullptr;
    const uint8_t* axes = nullptr;
    Angles(const Call& c, int at, int64_t T) {
        if (c.absent(at)) {
            if (!c.absent(at + 1) || !c.absent(at + 2)) throw Refusal("table: needed with positions or axes");
            return;
        }
        const at::Tensor& t = c.tensor("table", at);
        if (t.dim() != 2 || t.size(1) > GPD_HEAD_MAX_DIM || t.size(1) % 2) refuse("table", "[positions, columns] expected, got shape " + shape_text(t));
        const auto m = c.mat("table", at, kF32, t.size(0), t.size(1));
        table = static_cast<const float*>(m.p);
        ldt = m.ld;
        P = t.size(0);
        R = (int32_t)t.size(1);
        if (c.absent(at + 1)) refuse("positions", "needed");
        const at::Tensor& p = c.tensor("positions", at + 1);
        index_bytes = (int32_t)p.element_size();
        if (p.dim() == 1) {
            pos = c.vec("positions", at + 1, kIndex, T);
            ldp = 1;
        } else {
            if (p.dim() != 2 || p.size(1) < 1 || p.size(1) > GPD_HEAD_MAX_AXES)
                refuse("positions", "[T] or [T, axes] expected, got shape " + shape_text(p));
            n = (int32_t)p.size(1);
            const auto mp = c.mat("positions", at + 1, kIndex, T, n);
            pos = mp.p;
            ldp = mp.ld;
        }
        if (n > 1 && c.absent(at + 2)) refuse("axes", "needed with positions of several axes");
        axes = static_cast<const uint8_t*>(c.vec("axes", at + 2, kU8, R / 2));
    }
};

gpd_status head_norm_rope(PyObject* const* args, Py_ssize_t n) {
    // q, k, table, positions, axes, q_out, k_out, head_dim, q_weight, k_weight, eps, neighbours, stream
    Call c(args, n, 13);
    const int first = c.absent(0) ? 1 : 0;
    const at::Tensor& x = c.lead(first ? "k" : "q", first, kFloats);
    const int64_t T = x.size(0), D = c.integer(7);
    if (D <= 0 || D > GPD_HEAD_MAX_DIM) refuse("head_dim", "1 .. " + std::to_string(GPD_HEAD_MAX_DIM));
    const unsigned same = type_bit(x.scalar_type());
    const int32_t Hq = heads_of(c, "q", 0, T, D), Hk = heads_of(c, "k", 1, T, D);
    const auto mq = c.mat("q", 0, same, T, Hq * D), mk = c.mat("k", 1, same, T, Hk * D);
    const Angles an(c, 2, T);
    if (c.absent(0) != c.absent(5)) throw Refusal("q and q_out go together");
    if (c.absent(1) != c.absent(6)) throw Refusal("k and k_out go together");
    const auto oq = c.mat("q_out", 5, same, T, Hq * D), ok = c.mat("k_out", 6, same, T, Hk * D);
    unsigned wq = 0, wk = 0;
    void *pq = c.vec("q_weight", 8, same | kF32, D, &wq), *pk = c.vec("k_weight", 9, same | kF32, D, &wk);
    if (wq && wk && wq != wk) throw Refusal("q_weight and k_weight: one type expected");
    const int near = PyObject_IsTrue(args[11]);
    if (near < 0) throw PythonError();
    return gpd_head_norm_rope(gpd_type(same), mq.p, mq.ld, Hq, mk.p, mk.ld, Hk, (int32_t)D, gpd_type(wq ? wq : wk ? wk : same), pq, pk,
                              (float)c.number(10), an.table, an.ldt, an.P, an.R, near, an.index_bytes, an.pos, an.ldp, an.n, an.axes, oq.p,
                              oq.ld, ok.p, ok.ld, T, c.stream(12));
}

gpd_status head_norm_rope_backward(PyObject* const* args, Py_ssize_t n) {
    // dq, dk, table, positions, axes, q, k, dq_in, dk_in, head_dim, q_weight, k_weight, dq_weight, dk_weight, workspace, eps,
    // neighbours, stream
    Call c(args, n, 18);
    const int first = c.absent(0) ? 1 : 0;
    const at::Tensor& x = c.lead(first ? "dk" : "dq", first, kFloats);
    const int64_t T = x.size(0), D = c.integer(9);
    if (D <= 0 || D > GPD_HEAD_MAX_DIM) refuse("head_dim", "1 .. " + std::to_string(GPD_HEAD_MAX_DIM));
    const unsigned same = type_bit(x.scalar_type());
    const int32_t Hq = heads_of(c, "dq", 0, T, D), Hk = heads_of(c, "dk", 1, T, D);
    const auto gq = c.mat("dq", 0, same, T, Hq * D), gk = c.mat("dk", 1, same, T, Hk * D);
    const Angles an(c, 2, T);
    if (c.absent(0) != c.absent(7)) throw Refusal("dq and dq_in go together");
    if (c.absent(1) != c.absent(8)) throw Refusal("dk and dk_in go together");
    const auto mq = c.mat("q", 5, same, T, Hq * D), mk = c.mat("k", 6, same, T, Hk * D), oq = c.mat("dq_in", 7, same, T, Hq * D),
               ok = c.mat("dk_in", 8, same, T, Hk * D);
    unsigned wq = 0, wk = 0;
    void *pq = c.vec("q_weight", 10, same | kF32, D, &wq), *pk = c.vec("k_weight", 11, same | kF32, D, &wk);
    if (wq && wk && wq != wk) throw Refusal("q_weight and k_weight: one type expected");
    float *dwq = static_cast<float*>(c.vec("dq_weight", 12, kF32, D)), *dwk = static_cast<float*>(c.vec("dk_weight", 13, kF32, D));
    void* ws = nullptr;
    int64_t ws_bytes = 0;
    if (!c.absent(14)) ws = c.buffer("workspace", 14, &ws_bytes);
    const int near = PyObject_IsTrue(args[16]);
    if (near < 0) throw PythonError();
    return gpd_head_norm_rope_backward(gpd_type(same), gq.p, gq.ld, gk.p, gk.ld, mq.p, mq.ld, Hq, mk.p, mk.ld, Hk, (int32_t)D,
                                       gpd_type(wq ? wq : wk ? wk : same), pq, pk, (float)c.number(15), an.table, an.ldt, an.P, an.R, near,
                                       an.index_bytes, an.pos, an.ldp, an.n, an.axes, oq.p, oq.ld, ok.p, ok.ld, dwq, dwk, T, ws, ws_bytes,
                                       c.stream(17));
}

// n matrices of rows x cols
struct Cube {
    void* p = nullptr;
    int64_t ld = 0, next = 0;
    unsigned type = 0;
};
Cube cube(const Call& c, const char* name, int i, unsigned types, int64_t n, int64_t rows, int64_t cols) {
    Cube m;
    if (c.absent(i)) return m;
    const at::Tensor& t = c.tensor(name, i);
    m.type = c.check_type(name, t, types);
    c.check_device(name, t);
    if (t.dim() != 3 || t.size(0) != n || t.size(1) != rows || t.size(2) != cols)
        refuse(name, "shape (" + std::to_string(n) + ", " + std::to_string(rows) + ", " + std::to_string(cols) + ") expected, got " + shape_text(t));
    if (cols > 1 && t.stride(2) != 1) refuse(name, "columns have to be adjacent");
    m.ld = rows > 1 ? t.stride(1) : cols;
    if (m.ld < cols) refuse(name, "rows overlap");
    const int64_t size = m.ld * (rows - 1) + cols;
    m.next = n > 1 ? t.stride(0) : size;
    if (m.next < size) refuse(name, "matrices overlap");
    m.p = t.data_ptr();
    return m;
}
// The segments of a batch: offsets [S + 1] and index [S], of one type.
struct Parts {
    const void *offsets, *index;
    int32_t S, index_bytes;
    Parts(const Call& c, int at) {
        const at::Tensor &o = c.tensor("offsets", at), &i = c.tensor("index", at + 1);
        if (i.dim() != 1 || i.size(0) >= 0x7fffffff) refuse("index", "vector expected, got shape " + shape_text(i));
        S = (int32_t)i.size(0);
        offsets = c.vec("offsets", at, kIndex, (int64_t)S + 1);
        index = c.vec("index", at + 1, kIndex, S);
        if (o.scalar_type() != i.scalar_type()) throw Refusal("offsets and index: one type expected");
        index_bytes = (int32_t)o.element_size();
    }
};
// Sizes that A [n, r, K] and B [n, N, r] give.
struct Factors {
    int64_t n, r, N;
    Cube A, B;
    Factors(const Call& c, int at, unsigned type, int64_t K) {
        const at::Tensor &a = c.tensor("A", at), &b = c.tensor("B", at + 1);
        if (a.dim() != 3 || a.size(0) > 0x7fffffff || a.size(1) < 1 || a.size(1) > GPD_ADAPTER_MAX_RANK)
            refuse("A", "[adapters, rank of at most " + std::to_string(GPD_ADAPTER_MAX_RANK) + ", K] expected, got shape " + shape_text(a));
        if (b.dim() != 3) refuse("B", "[adapters, N, rank] expected, got shape " + shape_text(b));
        n = a.size(0);
        r = a.size(1);
        N = b.size(1);
        if (K < 1 || N < 1) throw Refusal("A, B: K and N of at least 1 expected");
        A = cube(c, "A", at, type, n, r, K);
        B = cube(c, "B", at + 1, type, n, N, r);
    }
};

gpd_status adapter(PyObject* const* args, Py_ssize_t n) {
    // x, A, B, offsets, index, out, h, base, scale, stream
    Call c(args, n, 10);
    const at::Tensor& x = c.lead("x", 0, kBF16 | kF16);
    const int64_t T = x.size(0), K = x.size(1);
    const unsigned same = type_bit(x.scalar_type());
    const auto mx = c.mat("x", 0, same, T, K);
    const Factors f(c, 1, same, K);
    const Parts p(c, 3);
    const auto mo = c.need_mat("out", 5, same | kF32, T, f.N);
    const auto mb = c.mat("base", 7, mo.type, T, f.N);
    if (c.absent(6)) refuse("h", "needed");
    float* h = static_cast<float*>(c.per_row("h", 6, kF32, T, f.r));
    const float* scale = static_cast<float*>(c.vec("scale", 8, kF32, f.n));
    return gpd_adapter(gpd_type(same), mx.p, mx.ld, (int32_t)f.n, (int32_t)f.r, f.A.p, f.A.ld, f.A.next, f.B.p, f.B.ld, f.B.next, scale,
                       p.index_bytes, p.offsets, p.index, p.S, h, gpd_type(mo.type), mb.p, mb.ld, mo.p, mo.ld, T, K, f.N, c.stream(9));
}

gpd_status adapter_backward(PyObject* const* args, Py_ssize_t n) {
    // dout, x, A, B, h, offsets, index, dx, dA, dB, workspace, dbase, scale, accumulate, stream
    Call c(args, n, 15);
    const at::Tensor& x = c.lead("x", 1, kBF16 | kF16);
    const int64_t T = x.size(0), K = x.size(1);
    const unsigned same = type_bit(x.scalar_type());
    const auto mx = c.mat("x", 1, same, T, K);
    const Factors f(c, 2, same, K);
    const auto md = c.need_mat("dout", 0, same, T, f.N);
    const Parts p(c, 5);
    if (c.absent(4)) refuse("h", "needed");
    const float* h = static_cast<float*>(c.per_row("h", 4, kF32, T, f.r));
    const auto mdx = c.mat("dx", 7, same | kF32, T, K);
    if (!mdx.type && !c.absent(11)) throw Refusal("dbase: dx is needed with it");
    const auto mdb = c.mat("dbase", 11, mdx.type, T, K);
    if (c.absent(8) != c.absent(9)) throw Refusal("dA and dB go together");
    const Cube dA = cube(c, "dA", 8, same | kF32, f.n, f.r, K), dB = cube(c, "dB", 9, same | kF32, f.n, f.N, f.r);
    if (dA.type != dB.type) throw Refusal("dA and dB: one type expected");
    int64_t ws_bytes = 0;
    void* ws = c.buffer("workspace", 10, &ws_bytes);
    const float* scale = static_cast<float*>(c.vec("scale", 12, kF32, f.n));
    const int acc = PyObject_IsTrue(args[13]);
    if (acc < 0) throw PythonError();
    return gpd_adapter_backward(gpd_type(same), md.p, md.ld, mx.p, mx.ld, (int32_t)f.n, (int32_t)f.r, f.A.p, f.A.ld, f.A.next, f.B.p, f.B.ld,
                                f.B.next, scale, h, p.index_bytes, p.offsets, p.index, p.S, mdx.type ? gpd_type(mdx.type) : GPD_DT_F32, mdb.p,
                                mdb.ld, mdx.p, mdx.ld, dA.type ? gpd_type(dA.type) : GPD_DT_F32, dA.p, dA.ld, dA.next, dB.p, dB.ld, dB.next,
                                acc, T, K, f.N, ws, ws_bytes, c.stream(14));
}

// Tensors of a list or tuple: floating types, on the call's device, dense (in any order of their dimensions).
struct TensorList {
    PyObject* items = nullptr;                         // keeps the tensors
    int32_t n = 0;
    std::vector<int64_t> counts;
    std::vector<void*> at;
    std::vector<int32_t> types;
    TensorList(const Call& c, const char* name, PyObject* list) {
        if (THPVariable_Check(list)) refuse(name, "list of tensors expected");
        items = PySequence_Fast(list, "list of tensors expected");
        if (!items) {
            PyErr_Clear();
            refuse(name, "list of tensors expected");
        }
        try {
            fill(c, name);
        } catch (...) {
            Py_DECREF(items);
            throw;
        }
    }
    ~TensorList() { Py_DECREF(items); }
    TensorList(const TensorList&) = delete;
    TensorList& operator=(const TensorList&) = delete;
    const at::Tensor& tensor(int32_t i) const { return THPVariable_Unpack(PySequence_Fast_GET_ITEM(items, i)); }

private:
    void fill(const Call& c, const char* name) {
        const Py_ssize_t size = PySequence_Fast_GET_SIZE(items);
        if (size > 0x7fffffff) refuse(name, "too many tensors");
        n = (int32_t)size;
        counts.resize(n);
        at.resize(n);
        types.resize(n);
        for (int32_t i = 0; i < n; ++i) {
            PyObject* o = PySequence_Fast_GET_ITEM(items, i);
            if (!THPVariable_Check(o)) refuse(name, "list of tensors expected");
            const at::Tensor& t = THPVariable_Unpack(o);
            types[i] = gpd_type(c.check_type(name, t, kFloats));
            c.check_device(name, t);
            if (!t.is_non_overlapping_and_dense()) refuse(name, "dense tensors expected, item " + std::to_string(i) + " is not");
            counts[i] = t.numel();
            at[i] = counts[i] ? t.data_ptr() : nullptr;
        }
    }
};

// Whether two dense tensors of one shape have their elements in the same order; dimensions of one element have no order.
bool same_order(const at::Tensor& a, const at::Tensor& b) {
    if (a.numel() == 0) return true;
    for (int64_t i = 0; i < a.dim(); ++i)
        if (a.size(i) > 1 && a.stride(i) != b.stride(i)) return false;
    return true;
}

gpd_status grad_norm(PyObject* const* args, Py_ssize_t n) {
    // grads, norm, workspace, stream
    Call c(args, n, 4);
    c.lead("norm", 1, kF32, 1);
    float* norm = static_cast<float*>(c.need_vec("norm", 1, kF32, 1));
    const TensorList g(c, "grads", args[0]);
    int64_t ws_bytes = 0;
    void* ws = c.buffer("workspace", 2, &ws_bytes);
    return gpd_grad_norm(g.n, g.types.data(), g.at.data(), g.counts.data(), norm, ws, ws_bytes, c.stream(3));
}

gpd_status clip_grads(PyObject* const* args, Py_ssize_t n) {
    // grads, norm, max_norm, out, stream
    Call c(args, n, 5);
    c.lead("norm", 1, kF32, 1);
    const float* norm = static_cast<float*>(c.need_vec("norm", 1, kF32, 1));
    const TensorList g(c, "grads", args[0]);
    const float max_norm = (float)c.number(2);
    if (c.absent(3))
        return gpd_clip_grads(g.n, g.types.data(), g.at.data(), g.types.data(), g.at.data(), g.counts.data(), norm, max_norm,
                              c.stream(4));
    const TensorList o(c, "out", args[3]);
    if (o.n != g.n) refuse("out", std::to_string(g.n) + " tensors expected, got " + std::to_string(o.n));
    for (int32_t i = 0; i < g.n; ++i) {
        const at::Tensor &a = g.tensor(i), &b = o.tensor(i);
        if (a.sizes() != b.sizes()) refuse("out", "item " + std::to_string(i) + " has shape " + shape_text(b) + " for a gradient of shape " + shape_text(a));
        if (!same_order(a, b))
            refuse("out", "item " + std::to_string(i) + " has its dimensions in another order than its gradient");
    }
    return gpd_clip_grads(g.n, g.types.data(), g.at.data(), o.types.data(), o.at.data(), g.counts.data(), norm, max_norm,
                          c.stream(4));
}

// No C++ exception leaves for the interpreter.
template <gpd_status (*F)(PyObject* const*, Py_ssize_t)>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        return PyLong_FromLong((long)F(args, n));
    } catch (const PythonError&) {
    } catch (const Refusal& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

#define ENTRY(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<name>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(rmsnorm_quant), ENTRY(rmsnorm_backward), ENTRY(quantize_blocks), ENTRY(gemm_fp8), ENTRY(token_logprobs),
                         ENTRY(token_logprobs_backward), ENTRY(distill_topk), ENTRY(head_norm_rope), ENTRY(head_norm_rope_backward),
                         ENTRY(grad_norm), ENTRY(clip_grads), ENTRY(adapter), ENTRY(adapter_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lm", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lm() { return PyModule_Create(&module); }
