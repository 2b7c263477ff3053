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
    const at::Tensor& lead(const char* name, int i, unsigned types) {
        const at::Tensor& t = tensor(name, i);
        if (!t.is_cuda()) refuse(name, "device tensor expected");
        device_ = t.device();
        const int current = c10::cuda::current_device();
        if (device_.index() != current)
            refuse(name, "tensor is on cuda:" + std::to_string(device_.index()) + ", the current device is cuda:" + std::to_string(current));
        if (t.dim() != 2) refuse(name, "matrix expected, got shape " + shape_text(t));
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
                         ENTRY(token_logprobs_backward), ENTRY(distill_topk), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lm", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lm() { return PyModule_Create(&module); }
