// The per-step calls of binding.py as native code: read the tensors, allocate the outputs, take the current stream and
// call the C ABI (include/loka.h).  Nothing is computed here.
//
// Why native: a small layer is two launches of a few microseconds of GPU time, and the same marshalling through ctypes
// (a Python-level allocation per output, a stream object, five to ten boxed pointers per call) took 12 - 14 us of
// host time per call, so the GPU waited for the host.  Positional arguments only; binding.py's wrappers carry the
// keyword interface.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/loka.h"

namespace {

PyObject* g_error = nullptr;       // binding.LokaError

// (status, what) becomes LokaError(status, what)
PyObject* fail(loka_status st, const char* what) {
    PyObject* args = Py_BuildValue("(is)", static_cast<int>(st), what);
    if (args) {
        PyErr_SetObject(g_error ? g_error : PyExc_RuntimeError, args);
        Py_DECREF(args);
    }
    return nullptr;
}

const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) throw std::invalid_argument("expected a tensor");
    return THPVariable_Unpack(o);
}
void* ptr(const at::Tensor& t) { return t.data_ptr(); }
void* ptr_or_null(PyObject* o) { return o == Py_None ? nullptr : tensor(o).data_ptr(); }

at::Tensor empty(at::IntArrayRef size, at::ScalarType type, const at::Device& dev) {
    return at::Tensor(at::detail::empty_cuda(size, type, dev, std::nullopt));
}
// the caller's tensor, or a new one
at::Tensor given_or(PyObject* o, at::IntArrayRef size, at::ScalarType type, const at::Device& dev) {
    return o == Py_None ? empty(size, type, dev) : tensor(o);
}
at::Tensor scratch(size_t bytes, const at::Device& dev) {
    return bytes ? empty({static_cast<int64_t>(bytes)}, at::kByte, dev) : at::Tensor();
}
void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

loka_gemm_desc desc_of(PyObject* o) {      // a ctypes structure: its bytes are the descriptor
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) {
        PyErr_Clear();
        throw std::invalid_argument("expected a GemmDesc");
    }
    loka_gemm_desc d;
    const bool ok = b.len == static_cast<Py_ssize_t>(sizeof(d));
    if (ok) memcpy(&d, b.buf, sizeof(d));
    PyBuffer_Release(&b);
    if (!ok) throw std::invalid_argument("expected a GemmDesc");
    return d;
}

// the library call without the interpreter lock (a launch can block while the hardware queue is full); a tensor without
// storage throws where its pointer is taken, and the lock has to be back before that becomes a Python exception
struct LockReleased {
    PyThreadState* const state = PyEval_SaveThread();
    ~LockReleased() { PyEval_RestoreThread(state); }
};
template <class F>
loka_status unlocked(F&& f) {
    const LockReleased released;
    return f();
}

PyObject* wrap(const at::Tensor& t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
PyObject* pack(std::initializer_list<at::Tensor> ts) {
    PyObject* r = PyTuple_New(static_cast<Py_ssize_t>(ts.size()));
    if (!r) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor& t : ts) {
        PyObject* o = wrap(t);
        if (!o) { Py_DECREF(r); return nullptr; }
        PyTuple_SET_ITEM(r, i++, o);
    }
    return r;
}
bool need_args(Py_ssize_t n, Py_ssize_t want) {
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
    return false;
}

// quantize(x, mode, transpose_out) -> (codes, scales)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 3)) return nullptr;
    const at::Tensor& x = tensor(a[0]);
    const long mode_l = PyLong_AsLong(a[1]);
    const int tr = PyObject_IsTrue(a[2]);
    if ((mode_l == -1 && PyErr_Occurred()) || tr < 0) return nullptr;
    if (x.scalar_type() != at::kBFloat16 || x.dim() != 2 || x.stride(1) != 1) {
        PyErr_SetString(PyExc_AssertionError, "x: bf16 [rows, cols] with contiguous rows");
        return nullptr;
    }
    const loka_scale_mode mode = static_cast<loka_scale_mode>(mode_l);
    const int64_t rows = x.size(0), cols = x.size(1), groups = loka_scale_count(mode, rows, cols);
    if (groups < 0) return fail(LOKA_ERR_SHAPE, "loka_scale_count");
    const at::Device dev = x.device();
    at::Tensor q = tr ? empty({cols, rows}, at::kByte, dev) : empty({rows, cols}, at::kByte, dev);
    at::Tensor s = empty({groups}, at::kFloat, dev);
    const size_t bytes = loka_quantize_workspace(mode, rows, cols, tr);
    at::Tensor ws = scratch(bytes, dev);
    void* st_ = stream();
    const loka_status st = unlocked([&] {
        return loka_quantize(ptr(x), rows, cols, x.stride(0), mode, tr, static_cast<uint8_t*>(ptr(q)),
                             static_cast<float*>(ptr(s)), bytes ? ptr(ws) : nullptr, bytes, st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_quantize");
    return pack({q, s});
    END_HANDLE_TH_ERRORS
}

// gemm_norm(desc, xq, sx, wq, sw, gamma, beta, want_y, out, y, workspace) -> (out, y or None)
PyObject* gemm_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 11)) return nullptr;
    const loka_gemm_desc d = desc_of(a[0]);
    const at::Device dev = tensor(a[1]).device();
    const int64_t rows = d.batch * d.M;
    const int want_y = PyObject_IsTrue(a[7]);
    if (want_y < 0) return nullptr;
    at::Tensor out = given_or(a[8], {rows, d.N}, at::kBFloat16, dev);
    at::Tensor y = (want_y || a[9] != Py_None) ? given_or(a[9], {rows, d.N}, at::kFloat, dev) : at::Tensor();
    at::Tensor ws = a[10] == Py_None ? scratch(loka_fp8_gemm_norm_workspace(&d), dev) : tensor(a[10]);
    void* const p[6] = {ptr_or_null(a[1]), ptr_or_null(a[2]), ptr_or_null(a[3]), ptr_or_null(a[4]), ptr_or_null(a[5]), ptr_or_null(a[6])};
    void* st_ = stream();
    const loka_status st = unlocked([&] {
        return loka_fp8_gemm_norm(&d, static_cast<uint8_t*>(p[0]), static_cast<float*>(p[1]), static_cast<uint8_t*>(p[2]),
                                  static_cast<float*>(p[3]), p[4], p[5], ptr(out), y.defined() ? static_cast<float*>(ptr(y)) : nullptr,
                                  ws.defined() ? ptr(ws) : nullptr, ws.defined() ? static_cast<size_t>(ws.numel()) : 0, st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_fp8_gemm_norm");
    return pack({out, y});
    END_HANDLE_TH_ERRORS
}

// gemm_norm_fp8out(desc, xq, sx, wq, sw, gamma, beta, want_y, oq, so, y, workspace) -> (codes, row scales, y or None)
PyObject* gemm_norm_fp8out(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 12)) return nullptr;
    const loka_gemm_desc d = desc_of(a[0]);
    const at::Device dev = tensor(a[1]).device();
    const int64_t rows = d.batch * d.M;
    const int want_y = PyObject_IsTrue(a[7]);
    if (want_y < 0) return nullptr;
    at::Tensor oq = given_or(a[8], {rows, d.N}, at::kByte, dev);
    at::Tensor so = given_or(a[9], {rows}, at::kFloat, dev);
    at::Tensor y = (want_y || a[10] != Py_None) ? given_or(a[10], {rows, d.N}, at::kFloat, dev) : at::Tensor();
    at::Tensor ws = a[11] == Py_None ? scratch(loka_fp8_gemm_norm_fp8out_workspace(&d), dev) : tensor(a[11]);
    void* const p[6] = {ptr_or_null(a[1]), ptr_or_null(a[2]), ptr_or_null(a[3]), ptr_or_null(a[4]), ptr_or_null(a[5]), ptr_or_null(a[6])};
    void* st_ = stream();
    const loka_status st = unlocked([&] {
        return loka_fp8_gemm_norm_fp8out(&d, static_cast<uint8_t*>(p[0]), static_cast<float*>(p[1]), static_cast<uint8_t*>(p[2]),
                                         static_cast<float*>(p[3]), p[4], p[5], static_cast<uint8_t*>(ptr(oq)),
                                         static_cast<float*>(ptr(so)), y.defined() ? static_cast<float*>(ptr(y)) : nullptr,
                                         ws.defined() ? ptr(ws) : nullptr, ws.defined() ? static_cast<size_t>(ws.numel()) : 0, st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_fp8_gemm_norm_fp8out");
    return pack({oq, so, y});
    END_HANDLE_TH_ERRORS
}

// linear_norm(desc, x, wq, sw, gamma, beta, want_y, want_sx, out) -> (out, y or None, sx or None)
PyObject* linear_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 9)) return nullptr;
    const loka_gemm_desc d = desc_of(a[0]);
    const at::Device dev = tensor(a[1]).device();
    const int64_t rows = d.batch * d.M;
    const int want_y = PyObject_IsTrue(a[6]), want_sx = PyObject_IsTrue(a[7]);
    if (want_y < 0 || want_sx < 0) return nullptr;
    at::Tensor out = given_or(a[8], {rows, d.N}, at::kBFloat16, dev);
    at::Tensor y = want_y ? empty({rows, d.N}, at::kFloat, dev) : at::Tensor();
    at::Tensor sx = want_sx ? empty({rows}, at::kFloat, dev) : at::Tensor();
    void* const p[5] = {ptr_or_null(a[1]), ptr_or_null(a[2]), ptr_or_null(a[3]), ptr_or_null(a[4]), ptr_or_null(a[5])};
    void* st_ = stream();
    const loka_status st = unlocked([&] {
        return loka_fp8_linear_norm(&d, p[0], static_cast<uint8_t*>(p[1]), static_cast<float*>(p[2]), p[3], p[4], ptr(out),
                                    y.defined() ? static_cast<float*>(ptr(y)) : nullptr,
                                    sx.defined() ? static_cast<float*>(ptr(sx)) : nullptr, st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_fp8_linear_norm");
    return pack({out, y, sx});
    END_HANDLE_TH_ERRORS
}

// linear_norm_xq(desc, x, wq, sw, gamma, beta, want_y, out, xq, sx) -> (out, y or None, xq, sx)
PyObject* linear_norm_xq(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 10)) return nullptr;
    const loka_gemm_desc d = desc_of(a[0]);
    const at::Device dev = tensor(a[1]).device();
    const int64_t rows = d.batch * d.M;
    const int want_y = PyObject_IsTrue(a[6]);
    if (want_y < 0) return nullptr;
    at::Tensor out = given_or(a[7], {rows, d.N}, at::kBFloat16, dev);
    at::Tensor xq = given_or(a[8], {rows, d.K}, at::kByte, dev);
    at::Tensor sx = given_or(a[9], {rows}, at::kFloat, dev);
    at::Tensor y = want_y ? empty({rows, d.N}, at::kFloat, dev) : at::Tensor();
    void* const p[5] = {ptr_or_null(a[1]), ptr_or_null(a[2]), ptr_or_null(a[3]), ptr_or_null(a[4]), ptr_or_null(a[5])};
    void* st_ = stream();
    const loka_status st = unlocked([&] {
        return loka_fp8_linear_norm_xq(&d, p[0], static_cast<uint8_t*>(ptr(xq)), static_cast<float*>(ptr(sx)),
                                       static_cast<uint8_t*>(p[1]), static_cast<float*>(p[2]), p[3], p[4], ptr(out),
                                       y.defined() ? static_cast<float*>(ptr(y)) : nullptr, st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_fp8_linear_norm_xq");
    return pack({out, y, xq, sx});
    END_HANDLE_TH_ERRORS
}

// bf16_gemm(desc, x, w, yref, workspace) -> yref
PyObject* bf16_gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 5)) return nullptr;
    loka_gemm_desc d = desc_of(a[0]);
    if (d.strideW) d.strideW = d.K * d.N;           // the weights lie as [batch][K, N] here
    const at::Device dev = tensor(a[1]).device();
    at::Tensor yref = given_or(a[3], {d.batch * d.M, d.N}, at::kFloat, dev);
    at::Tensor ws = a[4] == Py_None ? scratch(loka_bf16_gemm_workspace(&d), dev) : tensor(a[4]);
    void* const p[2] = {ptr_or_null(a[1]), ptr_or_null(a[2])};
    void* st_ = stream();
    const loka_status st = unlocked([&] {
        return loka_bf16_gemm(&d, p[0], p[1], static_cast<float*>(ptr(yref)), ws.defined() ? ptr(ws) : nullptr,
                              ws.defined() ? static_cast<size_t>(ws.numel()) : 0, st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_bf16_gemm");
    return wrap(yref);
    END_HANDLE_TH_ERRORS
}

// probe_error(y, yref, stats, rowmax, workspace) -> (stats, rowmax)
PyObject* probe_error(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 5)) return nullptr;
    const at::Tensor& y = tensor(a[0]);
    const at::Tensor& yref = tensor(a[1]);
    if (y.scalar_type() != at::kFloat || yref.scalar_type() != at::kFloat || y.dim() != 2 || !y.sizes().equals(yref.sizes())) {
        PyErr_SetString(PyExc_AssertionError, "y, yref: fp32 [M, N] of one shape");
        return nullptr;
    }
    const at::Device dev = y.device();
    const int64_t M = y.size(0), N = y.size(1);
    at::Tensor stats = given_or(a[2], {5}, at::kDouble, dev);
    at::Tensor rowmax = given_or(a[3], {M}, at::kFloat, dev);
    at::Tensor ws = a[4] == Py_None ? scratch(loka_probe_error_workspace(M, N), dev) : tensor(a[4]);
    void* st_ = stream();
    const loka_status st = unlocked([&] {
        return loka_probe_error(static_cast<float*>(ptr(y)), static_cast<float*>(ptr(yref)), M, N, y.stride(0),
                                static_cast<loka_probe_stats*>(ptr(stats)), static_cast<float*>(ptr(rowmax)),
                                ws.defined() ? ptr(ws) : nullptr, ws.defined() ? static_cast<size_t>(ws.numel()) : 0, st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_probe_error");
    return pack({stats, rowmax});
    END_HANDLE_TH_ERRORS
}

// tracker_update(x, n_old, mu, sigma, workspace) -> n_old + rows of x
PyObject* tracker_update(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 5)) return nullptr;
    const at::Tensor& x = tensor(a[0]);
    if (x.dim() != 2) {
        PyErr_SetString(PyExc_ValueError, "x: [rows, features]");
        return nullptr;
    }
    const long long n_old = PyLong_AsLongLong(a[1]);
    if (n_old == -1 && PyErr_Occurred()) return nullptr;
    const int64_t rows = x.size(0), K = x.size(1);
    at::Tensor ws = a[4] == Py_None ? scratch(loka_tracker_update_workspace(rows, K), x.device()) : tensor(a[4]);
    void* const p[2] = {ptr_or_null(a[2]), ptr_or_null(a[3])};
    void* st_ = stream();
    const loka_status st = unlocked([&] {
        return loka_tracker_update(ptr(x), rows, K, x.stride(0), n_old, static_cast<float*>(p[0]), static_cast<float*>(p[1]),
                                   ws.defined() ? ptr(ws) : nullptr, ws.defined() ? static_cast<size_t>(ws.numel()) : 0, st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_tracker_update");
    return PyLong_FromLongLong(n_old + rows);
    END_HANDLE_TH_ERRORS
}

// ---- MXFP4 and the residual norm.  Their buffers' sizes follow from the arguments, so every tensor is looked at before its
// address is handed on; the calls run on the tensors' own device, on that device's current stream.
PyObject* refuse(const char* what) {
    PyErr_SetString(PyExc_AssertionError, what);
    return nullptr;
}
// bf16 [rows, cols] with contiguous rows
bool is_rows(const at::Tensor& t) { return t.scalar_type() == at::kBFloat16 && t.dim() == 2 && (t.stride(1) == 1 || t.size(1) == 1); }
bool is_rows_of(const at::Tensor& t, int64_t rows, int64_t cols) { return is_rows(t) && t.size(0) == rows && t.size(1) == cols; }
// a contiguous tensor of at least n elements
bool holds(const at::Tensor& t, at::ScalarType type, int64_t n) { return t.scalar_type() == type && t.is_contiguous() && t.numel() >= n; }
// row stride of a matrix; of a single row it is free
int64_t row_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : (t.size(1) + 7) / 8 * 8; }
bool on_gpu(const at::Device& dev, std::initializer_list<const at::Tensor*> ts) {
    if (!dev.is_cuda()) return false;
    for (const at::Tensor* t : ts)
        if (t && t->defined() && t->device() != dev) return false;
    return true;
}
at::Tensor given(PyObject* o) { return o == Py_None ? at::Tensor() : tensor(o); }
// a workspace that may be written for its nbytes() from its address on
bool is_run(const at::Tensor& ws) { return !ws.defined() || ws.is_contiguous(); }
template <class T>
T* at_or_null(const at::Tensor& t) { return t.defined() ? static_cast<T*>(t.data_ptr()) : nullptr; }
void* stream_of(const at::Device& dev) { return c10::hip::getCurrentHIPStream(dev.index()).stream(); }

// mxfp4_quantize(x, transpose_out) -> (codes, scales)
PyObject* mxfp4_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 2)) return nullptr;
    const at::Tensor& x = tensor(a[0]);
    const int tr = PyObject_IsTrue(a[1]);
    if (tr < 0) return nullptr;
    if (!is_rows(x)) return refuse("x: bf16 [rows, cols] with contiguous rows");
    const int64_t rows = x.size(0), cols = x.size(1);
    if (rows <= 0 || cols <= 0) return fail(LOKA_ERR_SHAPE, "loka_mxfp4_quantize");
    const at::Device dev = x.device();
    if (!on_gpu(dev, {})) return refuse("x: a tensor on the GPU");
    const c10::DeviceGuard guard(dev);
    const int64_t r = tr ? cols : rows, kp = loka_mxfp4_padded(tr ? rows : cols);
    at::Tensor q = empty({r, kp / 2}, at::kByte, dev), s = empty({r, kp / 32}, at::kByte, dev);
    void* st_ = stream_of(dev);
    const loka_status st = unlocked([&] {
        return loka_mxfp4_quantize(ptr(x), rows, cols, row_stride(x), tr, static_cast<uint8_t*>(ptr(q)), static_cast<uint8_t*>(ptr(s)), st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_mxfp4_quantize");
    return pack({q, s});
    END_HANDLE_TH_ERRORS
}

// codes and scales of a stored operand of `rows` rows of `cols` elements
bool is_stored(const at::Tensor& q, const at::Tensor& s, int64_t rows, int64_t cols) {
    const int64_t kp = loka_mxfp4_padded(cols);
    return holds(q, at::kByte, rows * (kp / 2)) && holds(s, at::kByte, rows * (kp / 32));
}

// mxfp4_dequantize(q, scales, cols, out) -> out
PyObject* mxfp4_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 4)) return nullptr;
    const at::Tensor &q = tensor(a[0]), &s = tensor(a[1]);
    const long long cols = PyLong_AsLongLong(a[2]);
    if (cols == -1 && PyErr_Occurred()) return nullptr;
    if (q.dim() != 2 || cols <= 0) return fail(LOKA_ERR_SHAPE, "loka_mxfp4_dequantize");
    const int64_t rows = q.size(0);
    if (q.size(1) != loka_mxfp4_padded(cols) / 2 || !is_stored(q, s, rows, cols)) return refuse("q, scales: uint8 [rows, padded cols / 2] and [rows, padded cols / 32]");
    const at::Device dev = q.device();
    at::Tensor out = given(a[3]);
    if (!on_gpu(dev, {&s, &out})) return refuse("tensors on one GPU");
    const c10::DeviceGuard guard(dev);
    if (!out.defined()) out = empty({rows, cols}, at::kBFloat16, dev);
    else if (!is_rows_of(out, rows, cols)) return refuse("out: bf16 [rows, cols] with contiguous rows");
    void* st_ = stream_of(dev);
    const loka_status st = unlocked([&] {
        return loka_mxfp4_dequantize(static_cast<uint8_t*>(ptr(q)), static_cast<uint8_t*>(ptr(s)), rows, cols, ptr(out), row_stride(out), st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_mxfp4_dequantize");
    return wrap(out);
    END_HANDLE_TH_ERRORS
}

// outputs of a product: out (where wanted or given) and y (likewise); false with an exception set
bool product_outputs(PyObject* want_out, PyObject* want_y, PyObject* out_o, PyObject* y_o, int64_t numel, int64_t rows, int64_t cols, const at::Device& dev,
                     at::Tensor& out, at::Tensor& y) {
    const int wo = PyObject_IsTrue(want_out), wy = PyObject_IsTrue(want_y);
    if (wo < 0 || wy < 0) return false;
    if (wo || out_o != Py_None) out = given_or(out_o, {rows, cols}, at::kBFloat16, dev);
    if (wy || y_o != Py_None) y = given_or(y_o, {rows, cols}, at::kFloat, dev);
    if ((out.defined() && !holds(out, at::kBFloat16, numel)) || (y.defined() && !holds(y, at::kFloat, numel))) {
        refuse("out, y: contiguous bf16 / fp32 [batch * M, N]");
        return false;
    }
    if (!on_gpu(dev, {&out, &y})) {
        refuse("tensors on one GPU");
        return false;
    }
    return true;
}
// elements that `batch` problems `stride` apart span, `each` of them the last (0: shared)
int64_t span(int64_t batch, int64_t stride, int64_t each) { return (batch - 1) * stride + each; }
constexpr int64_t kMost = INT64_C(1) << 31, kMostElements = INT64_C(1) << 46;      // of a size; of a whole operand
bool sizes_ok(const loka_gemm_desc& d) {
    return d.M > 0 && d.N > 0 && d.K > 0 && d.batch > 0 && d.M < kMost && d.N < kMost && d.K < kMost && d.batch < kMost;
}
// (read where there are several problems)
bool strides_ok(const loka_gemm_desc& d) {
    auto ok = [&](int64_t stride) { return stride >= 0 && stride < kMostElements && d.batch * (stride / 1024 + 1) < kMostElements / 1024; };
    return d.batch == 1 || (ok(d.strideX) && ok(d.strideW) && ok(d.strideO));
}

// mxfp4_gemm(desc, xq, sx, wq, sw, want_out, want_y, out, y, workspace) -> (out or None, y or None)
PyObject* mxfp4_gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 10)) return nullptr;
    const loka_gemm_desc d = desc_of(a[0]);
    const at::Tensor &xq = tensor(a[1]), &sx = tensor(a[2]), &wq = tensor(a[3]), &sw = tensor(a[4]);
    if (!sizes_ok(d) || !strides_ok(d)) return fail(LOKA_ERR_SHAPE, "loka_mxfp4_gemm");
    const int64_t kp = loka_mxfp4_padded(d.K);
    const int64_t nx = span(d.batch, d.strideX, d.M * kp), nw = span(d.batch, d.strideW, d.N * kp);
    if (!holds(xq, at::kByte, nx / 2) || !holds(sx, at::kByte, nx / 32) || !holds(wq, at::kByte, nw / 2) || !holds(sw, at::kByte, nw / 32))
        return refuse("xq, sx, wq, sw: stored operands [batch, M, K] and [batch, N, K], contiguous uint8");
    const at::Device dev = xq.device();
    at::Tensor ws = given(a[9]);
    if (!is_run(ws)) return refuse("workspace: contiguous");
    if (!on_gpu(dev, {&sx, &wq, &sw, &ws})) return refuse("tensors on one GPU");
    const c10::DeviceGuard guard(dev);
    at::Tensor out, y;
    if (!product_outputs(a[5], a[6], a[7], a[8], span(d.batch, d.batch > 1 ? d.strideO : 0, d.M * d.N), d.batch * d.M, d.N, dev, out, y)) return nullptr;
    if (!ws.defined()) ws = scratch(loka_mxfp4_gemm_workspace(&d), dev);
    void* st_ = stream_of(dev);
    const loka_status st = unlocked([&] {
        return loka_mxfp4_gemm(&d, static_cast<uint8_t*>(ptr(xq)), static_cast<uint8_t*>(ptr(sx)), static_cast<uint8_t*>(ptr(wq)),
                               static_cast<uint8_t*>(ptr(sw)), at_or_null<void>(out), at_or_null<float>(y), at_or_null<void>(ws),
                               ws.defined() ? ws.nbytes() : 0, st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_mxfp4_gemm");
    return pack({out, y});
    END_HANDLE_TH_ERRORS
}

// mxfp4_linear(desc, x, wq, sw, want_out, want_y, out, y, workspace) -> (out or None, y or None)
PyObject* mxfp4_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 9)) return nullptr;
    const loka_gemm_desc d = desc_of(a[0]);
    const at::Tensor &x = tensor(a[1]), &wq = tensor(a[2]), &sw = tensor(a[3]);
    if (!sizes_ok(d)) return fail(LOKA_ERR_SHAPE, "loka_mxfp4_linear");
    if (!is_rows_of(x, d.M, d.K)) return refuse("x: bf16 [M, K] with contiguous rows");
    if (!is_stored(wq, sw, d.N, d.K)) return refuse("wq, sw: a stored operand [N, K], contiguous uint8");
    const at::Device dev = x.device();
    at::Tensor ws = given(a[8]);
    if (!is_run(ws)) return refuse("workspace: contiguous");
    if (!on_gpu(dev, {&wq, &sw, &ws})) return refuse("tensors on one GPU");
    const c10::DeviceGuard guard(dev);
    at::Tensor out, y;
    if (!product_outputs(a[4], a[5], a[6], a[7], d.M * d.N, d.M, d.N, dev, out, y)) return nullptr;
    if (!ws.defined()) ws = scratch(loka_mxfp4_linear_workspace(&d), dev);
    void* st_ = stream_of(dev);
    const loka_status st = unlocked([&] {
        return loka_mxfp4_linear(&d, ptr(x), row_stride(x), static_cast<uint8_t*>(ptr(wq)), static_cast<uint8_t*>(ptr(sw)), at_or_null<void>(out),
                                 at_or_null<float>(y), at_or_null<void>(ws), ws.defined() ? ws.nbytes() : 0, st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_mxfp4_linear");
    return pack({out, y});
    END_HANDLE_TH_ERRORS
}

// add_rmsnorm(x, residual, gamma, eps, out, out_mode, ckpt_mode, want_h, want_rstd, h_out) -> (h, y, scales, hq, hs, rstd)
PyObject* add_rmsnorm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 10)) return nullptr;
    const at::Tensor& x = tensor(a[0]);
    const at::Tensor res = given(a[1]), gamma = given(a[2]);
    const double eps = PyFloat_AsDouble(a[3]);
    const long out = PyLong_AsLong(a[4]), out_mode = PyLong_AsLong(a[5]);
    const bool ckpt = a[6] != Py_None;
    const long ckpt_mode = ckpt ? PyLong_AsLong(a[6]) : 0;
    const int want_h = PyObject_IsTrue(a[7]), want_rstd = PyObject_IsTrue(a[8]);
    if (PyErr_Occurred()) return nullptr;
    if (!is_rows(x)) return refuse("x: bf16 [rows, cols] with contiguous rows");
    loka_rms_desc d{};
    d.rows = x.size(0);
    d.cols = x.size(1);
    d.ld_x = row_stride(x);
    d.out = static_cast<int32_t>(out);
    d.out_mode = static_cast<int32_t>(out_mode);
    d.ckpt_mode = static_cast<int32_t>(ckpt_mode);
    d.eps = static_cast<float>(eps);
    if (res.defined() && !is_rows_of(res, d.rows, d.cols)) return refuse("residual: bf16 [rows, cols] with contiguous rows");
    d.ld_r = res.defined() ? row_stride(res) : 0;
    if (gamma.defined() && !(holds(gamma, at::kBFloat16, d.cols) && gamma.numel() == d.cols)) return refuse("gamma: contiguous bf16 [cols]");
    if (d.rows <= 0 || d.cols <= 0) return fail(LOKA_ERR_SHAPE, "loka_add_rmsnorm");
    const bool e4m3 = out == LOKA_RMS_OUT_E4M3, mx = out == LOKA_RMS_OUT_MXFP4;
    const int64_t groups = e4m3 ? loka_scale_count(static_cast<loka_scale_mode>(out_mode), d.rows, d.cols) : 0;
    const int64_t hgroups = ckpt ? loka_scale_count(static_cast<loka_scale_mode>(ckpt_mode), d.rows, d.cols) : 0;
    if (groups < 0 || hgroups < 0) return fail(LOKA_ERR_SHAPE, "loka_scale_count");
    const at::Device dev = x.device();
    at::Tensor h = given(a[9]);
    if (!on_gpu(dev, {&res, &gamma, &h})) return refuse("tensors on one GPU");
    const c10::DeviceGuard guard(dev);
    if (h.defined()) {
        if (!(holds(h, at::kBFloat16, d.rows * d.cols) && is_rows_of(h, d.rows, d.cols))) return refuse("h_out: contiguous bf16 [rows, cols]");
    } else if (want_h) {
        h = empty({d.rows, d.cols}, at::kBFloat16, dev);
    }
    const int64_t kp = loka_mxfp4_padded(d.cols);
    at::Tensor y = mx ? empty({d.rows, kp / 2}, at::kByte, dev) : empty({d.rows, d.cols}, e4m3 ? at::kByte : at::kBFloat16, dev), s, hq, hs, rstd;
    if (e4m3) s = out_mode == LOKA_SCALE_ROW ? empty({groups}, at::kFloat, dev) : empty({d.rows, groups / d.rows}, at::kFloat, dev);
    if (mx) s = empty({d.rows, kp / 32}, at::kByte, dev);
    if (ckpt) {
        hq = empty({d.rows, d.cols}, at::kByte, dev);
        hs = ckpt_mode == LOKA_SCALE_ROW ? empty({hgroups}, at::kFloat, dev) : empty({d.rows, hgroups / d.rows}, at::kFloat, dev);
    }
    if (want_rstd) rstd = empty({d.rows}, at::kFloat, dev);
    void* st_ = stream_of(dev);
    const loka_status st = unlocked([&] {
        return loka_add_rmsnorm(&d, ptr(x), at_or_null<void>(res), at_or_null<void>(gamma), at_or_null<void>(h), ptr(y), at_or_null<void>(s),
                                at_or_null<uint8_t>(hq), at_or_null<float>(hs), at_or_null<float>(rstd), st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_add_rmsnorm");
    return pack({h, y, s, hq, hs, rstd});
    END_HANDLE_TH_ERRORS
}

// rmsnorm_backward(dy, hq, hs, rstd, gamma, dh, ckpt_mode, want_dgamma, dx, workspace) -> (dx, dgamma or None)
PyObject* rmsnorm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 10)) return nullptr;
    const at::Tensor &dy = tensor(a[0]), &hq = tensor(a[1]), &hs = tensor(a[2]), &rstd = tensor(a[3]);
    const at::Tensor gamma = given(a[4]), dh = given(a[5]);
    const long mode = PyLong_AsLong(a[6]);
    const int want_dgamma = PyObject_IsTrue(a[7]);
    if (PyErr_Occurred()) return nullptr;
    if (!is_rows(dy)) return refuse("dy: bf16 [rows, cols] with contiguous rows");
    loka_rms_desc d{};
    d.rows = dy.size(0);
    d.cols = dy.size(1);
    d.ld_x = row_stride(dy);
    d.ckpt_mode = static_cast<int32_t>(mode);
    if (dh.defined() && !is_rows_of(dh, d.rows, d.cols)) return refuse("dh: bf16 [rows, cols] with contiguous rows");
    d.ld_r = dh.defined() ? row_stride(dh) : 0;
    if (d.rows <= 0 || d.cols <= 0) return fail(LOKA_ERR_SHAPE, "loka_rmsnorm_backward");
    const int64_t groups = loka_scale_count(static_cast<loka_scale_mode>(mode), d.rows, d.cols);
    if (groups < 0) return fail(LOKA_ERR_SHAPE, "loka_scale_count");
    if (!holds(hq, at::kByte, d.rows * d.cols) || hq.numel() != d.rows * d.cols || !holds(hs, at::kFloat, groups) || hs.numel() != groups ||
        !holds(rstd, at::kFloat, d.rows) || rstd.numel() != d.rows)
        return refuse("hq, hs, rstd: contiguous uint8 [rows, cols], its fp32 scales, fp32 [rows]");
    if (gamma.defined() && !(holds(gamma, at::kBFloat16, d.cols) && gamma.numel() == d.cols)) return refuse("gamma: contiguous bf16 [cols]");
    const at::Device dev = dy.device();
    at::Tensor dx = given(a[8]), ws = given(a[9]);
    if (!is_run(ws)) return refuse("workspace: contiguous");
    if (!on_gpu(dev, {&hq, &hs, &rstd, &gamma, &dh, &dx, &ws})) return refuse("tensors on one GPU");
    const c10::DeviceGuard guard(dev);
    if (!dx.defined()) dx = empty({d.rows, d.cols}, at::kBFloat16, dev);
    else if (!(holds(dx, at::kBFloat16, d.rows * d.cols) && is_rows_of(dx, d.rows, d.cols))) return refuse("dx: contiguous bf16 [rows, cols]");
    at::Tensor dg = want_dgamma ? empty({d.cols}, at::kFloat, dev) : at::Tensor();
    if (!ws.defined() && want_dgamma) ws = scratch(loka_rmsnorm_backward_workspace(&d), dev);
    void* st_ = stream_of(dev);
    const loka_status st = unlocked([&] {
        return loka_rmsnorm_backward(&d, ptr(dy), static_cast<uint8_t*>(ptr(hq)), static_cast<float*>(ptr(hs)), static_cast<float*>(ptr(rstd)),
                                     at_or_null<void>(gamma), at_or_null<void>(dh), ptr(dx), at_or_null<float>(dg), at_or_null<void>(ws),
                                     ws.defined() ? ws.nbytes() : 0, st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_rmsnorm_backward");
    return pack({dx, dg});
    END_HANDLE_TH_ERRORS
}

// ---- a layer of experts
template <class D>
D bytes_of(PyObject* o, const char* what) {      // a ctypes structure: its bytes are the descriptor
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) {
        PyErr_Clear();
        throw std::invalid_argument(what);
    }
    D d;
    const bool ok = b.len == static_cast<Py_ssize_t>(sizeof(d));
    if (ok) memcpy(&d, b.buf, sizeof(d));
    PyBuffer_Release(&b);
    if (!ok) throw std::invalid_argument(what);
    return d;
}
bool is_int32(const at::Tensor& t, int64_t n) { return holds(t, at::kInt, n) && t.numel() == n; }
bool is_matrix(const at::Tensor& t, at::ScalarType type, int64_t rows, int64_t cols) {
    return t.scalar_type() == type && t.is_contiguous() && t.dim() == 2 && t.size(0) == rows && t.size(1) == cols;
}
// the routing problem that the logits and the options describe; false with an exception set
bool route_desc(const at::Tensor& logits, PyObject* const* a, loka_route_desc& d) {      // a: top_k, score, renorm, scale
    const long k = PyLong_AsLong(a[0]), score = PyLong_AsLong(a[1]);
    const int renorm = PyObject_IsTrue(a[2]);
    const double scale = PyFloat_AsDouble(a[3]);
    if (PyErr_Occurred()) return false;
    const bool bf16 = logits.scalar_type() == at::kBFloat16;
    if ((!bf16 && logits.scalar_type() != at::kFloat) || logits.dim() != 2 || (logits.size(1) > 1 && logits.stride(1) != 1)) {
        refuse("logits: bf16 or fp32 [tokens, experts] with contiguous rows");
        return false;
    }
    if (logits.size(0) <= 0 || logits.size(1) <= 0 || logits.size(1) > 1024 || k <= 0 || k > 16) {
        fail(LOKA_ERR_SHAPE, "loka_route");
        return false;
    }
    d = loka_route_desc{logits.size(0), logits.size(0) > 1 ? logits.stride(0) : logits.size(1), static_cast<int32_t>(logits.size(1)), static_cast<int32_t>(k),
                        static_cast<int32_t>(score), renorm, bf16, static_cast<float>(scale)};
    return true;
}

// A contiguous tensor of 4-byte elements that is a part of `whole`'s memory (an allocation of its own costs a small call half a microsecond)
at::Tensor part_of(const at::Tensor& whole, int64_t from, at::IntArrayRef size, at::ScalarType type) {
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(whole.storage()), c10::DispatchKeySet(c10::DispatchKey::CUDA), c10::scalarTypeToTypeMeta(type));
    t.unsafeGetTensorImpl()->set_storage_offset(from);
    t.unsafeGetTensorImpl()->set_sizes_contiguous(size);
    return t;
}

// route(logits, top_k, score, renorm, scale, workspace) -> (expert, weight, slot, row, offsets)
PyObject* route(PyObject*, PyObject* const* a, Py_ssize_t args) {
    HANDLE_TH_ERRORS
    if (!need_args(args, 6)) return nullptr;
    const at::Tensor& logits = tensor(a[0]);
    loka_route_desc d;
    if (!route_desc(logits, a + 1, d)) return nullptr;
    const at::Device dev = logits.device();
    at::Tensor ws = given(a[5]);
    if (!is_run(ws)) return refuse("workspace: contiguous");
    if (!on_gpu(dev, {&ws})) return refuse("tensors on one GPU");
    const c10::DeviceGuard guard(dev);
    const int64_t n = d.tokens * d.top_k;
    const at::Tensor whole = empty({4 * n + d.experts + 1}, at::kInt, dev);
    at::Tensor expert = part_of(whole, 0, {d.tokens, d.top_k}, at::kInt), weight = part_of(whole, n, {d.tokens, d.top_k}, at::kFloat),
               slot = part_of(whole, 2 * n, {d.tokens, d.top_k}, at::kInt), row = part_of(whole, 3 * n, {n}, at::kInt), offsets = part_of(whole, 4 * n, {d.experts + 1}, at::kInt);
    if (!ws.defined()) ws = scratch(loka_route_workspace(&d), dev);
    void* st_ = stream_of(dev);
    const loka_status st = unlocked([&] {
        return loka_route(&d, ptr(logits), static_cast<int32_t*>(ptr(expert)), static_cast<float*>(ptr(weight)), static_cast<int32_t*>(ptr(slot)),
                          static_cast<int32_t*>(ptr(row)), static_cast<int32_t*>(ptr(offsets)), at_or_null<void>(ws), ws.defined() ? ws.nbytes() : 0, st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_route");
    return pack({expert, weight, slot, row, offsets});
    END_HANDLE_TH_ERRORS
}

// route_backward(logits, expert, dweight, score, renorm, scale, dlogits) -> dlogits
PyObject* route_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 7)) return nullptr;
    const at::Tensor &logits = tensor(a[0]), &expert = tensor(a[1]), &dweight = tensor(a[2]);
    if (expert.dim() != 2) return refuse("expert: contiguous int32 [tokens, top_k]");
    PyObject* const k = PyLong_FromLongLong(expert.size(1));
    if (!k) return nullptr;
    PyObject* const options[4] = {k, a[3], a[4], a[5]};
    loka_route_desc d;
    const bool ok = route_desc(logits, options, d);
    Py_DECREF(k);
    if (!ok) return nullptr;
    if (!is_matrix(expert, at::kInt, d.tokens, d.top_k) || !is_matrix(dweight, at::kFloat, d.tokens, d.top_k))
        return refuse("expert, dweight: contiguous int32 and fp32 [tokens, top_k]");
    const at::Device dev = logits.device();
    at::Tensor dl = given(a[6]);
    if (!on_gpu(dev, {&expert, &dweight, &dl})) return refuse("tensors on one GPU");
    const c10::DeviceGuard guard(dev);
    if (!dl.defined()) dl = empty({d.tokens, d.experts}, logits.scalar_type(), dev);
    else if (!is_matrix(dl, logits.scalar_type(), d.tokens, d.experts)) return refuse("dlogits: contiguous [tokens, experts] of the logits' type");
    void* st_ = stream_of(dev);
    const loka_status st = unlocked([&] {
        return loka_route_backward(&d, ptr(logits), static_cast<int32_t*>(ptr(expert)), static_cast<float*>(ptr(dweight)), ptr(dl), st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_route_backward");
    return wrap(dl);
    END_HANDLE_TH_ERRORS
}

// grouped_quantize(x, groups, offsets, index, along, turned, q, scales, qt, st) -> (q, scales, qt, st)
PyObject* grouped_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 10)) return nullptr;
    const at::Tensor& x = tensor(a[0]);
    const long long groups = PyLong_AsLongLong(a[1]);
    const at::Tensor offsets = given(a[2]), index = given(a[3]);
    int along = PyObject_IsTrue(a[4]), turned = PyObject_IsTrue(a[5]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor q = given(a[6]), s = given(a[7]), qt = given(a[8]), st = given(a[9]);
    along |= q.defined() || s.defined();       // (a buffer that is given is written)
    turned |= qt.defined() || st.defined();
    if (!is_rows(x)) return refuse("x: bf16 [rows, cols] with contiguous rows");
    if (offsets.defined() && !(holds(offsets, at::kInt, 2) && offsets.dim() == 1)) return refuse("offsets: contiguous int32 [groups + 1]");
    if (index.defined() && !(holds(index, at::kInt, 0) && index.dim() == 1)) return refuse("index: contiguous int32 [rows]");
    if (!along && !turned) return refuse("one of the two forms at least");
    const int64_t g = offsets.defined() ? offsets.numel() - 1 : groups;
    loka_grouped_quantize_desc d{index.defined() ? index.numel() : x.size(0), x.size(1), row_stride(x), x.size(0), static_cast<int32_t>(g)};
    if (g <= 0 || g > 1024 || d.rows <= 0 || d.rows >= kMost || x.size(0) <= 0 || d.cols <= 0 || d.cols >= kMost || (!offsets.defined() && d.rows % g)) return fail(LOKA_ERR_SHAPE, "loka_grouped_quantize");
    const int64_t kb = (d.cols + 127) / 128, blocks = offsets.defined() ? loka_grouped_blocks(d.rows, g) : (d.rows / g + 127) / 128 * g;
    const at::Device dev = x.device();
    if (!on_gpu(dev, {&offsets, &index, &q, &s, &qt, &st})) return refuse("tensors on one GPU");
    const c10::DeviceGuard guard(dev);
    if (along) {
        if (!q.defined()) q = empty({d.rows, kb * 128}, at::kByte, dev);
        if (!s.defined()) s = empty({d.rows, kb}, at::kFloat, dev);
        if (!holds(q, at::kByte, d.rows * kb * 128) || !holds(s, at::kFloat, d.rows * kb)) return refuse("q, scales: contiguous uint8 [rows, padded cols] and fp32 [rows, padded cols / 128]");
    }
    if (turned) {
        if (!qt.defined()) qt = empty({blocks, d.cols, 128}, at::kByte, dev);
        if (!st.defined()) st = empty({blocks, d.cols}, at::kFloat, dev);
        if (!holds(qt, at::kByte, blocks * d.cols * 128) || !holds(st, at::kFloat, blocks * d.cols)) return refuse("qt, st: contiguous uint8 [blocks, cols, 128] and fp32 [blocks, cols]");
    }
    void* st_ = stream_of(dev);
    const loka_status status = unlocked([&] {
        return loka_grouped_quantize(&d, ptr(x), at_or_null<int32_t>(index), at_or_null<int32_t>(offsets), at_or_null<uint8_t>(q), at_or_null<float>(s),
                                     at_or_null<uint8_t>(qt), at_or_null<float>(st), st_);
    });
    if (status != LOKA_OK) return fail(status, "loka_grouped_quantize");
    return pack({q, s, qt, st});
    END_HANDLE_TH_ERRORS
}

// sizes of a grouped product within what the library takes, so that they can be multiplied
bool grouped_ok(const loka_grouped_desc& d) {
    constexpr int64_t width = INT64_C(1) << 20;
    return d.rows > 0 && d.rows < kMost && d.N > 0 && d.N <= width && d.K > 0 && d.K <= width && d.groups > 0 && d.groups <= 1024;
}
bool is_weights(const at::Tensor& q, const at::Tensor& s, const loka_grouped_desc& d) {
    const int64_t n = d.groups * ((d.K + 127) / 128) * d.N;
    return holds(q, at::kByte, n * 128) && q.numel() == n * 128 && holds(s, at::kFloat, n) && s.numel() == n;
}

// grouped_gemm(desc, xq, sx, wq, sw, offsets, index, want_out, want_y, out, y) -> (out or None, y or None)
PyObject* grouped_gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 11)) return nullptr;
    loka_grouped_desc d = bytes_of<loka_grouped_desc>(a[0], "expected a GroupedDesc");
    const at::Tensor &xq = tensor(a[1]), &sx = tensor(a[2]), &wq = tensor(a[3]), &sw = tensor(a[4]), &offsets = tensor(a[5]);
    const at::Tensor index = given(a[6]);
    if (!grouped_ok(d)) return fail(LOKA_ERR_SHAPE, "loka_grouped_gemm");
    const int64_t kb = (d.K + 127) / 128;
    if (!(holds(xq, at::kByte, 1) && xq.dim() == 2 && xq.size(1) == kb * 128) || !holds(sx, at::kFloat, xq.size(0) * kb) || (!index.defined() && xq.size(0) < d.rows))
        return refuse("xq, sx: contiguous uint8 [rows, padded K] and fp32 [rows, padded K / 128]");
    if (!is_weights(wq, sw, d)) return refuse("wq, sw: stored weights of every group, contiguous uint8 and fp32");
    if (!is_int32(offsets, d.groups + 1) || (index.defined() && !is_int32(index, d.rows))) return refuse("offsets, index: contiguous int32 [groups + 1] and [rows]");
    d.x_rows = xq.size(0);
    const at::Device dev = xq.device();
    if (!on_gpu(dev, {&sx, &wq, &sw, &offsets, &index})) return refuse("tensors on one GPU");
    const c10::DeviceGuard guard(dev);
    at::Tensor out, y;
    if (!product_outputs(a[7], a[8], a[9], a[10], d.rows * d.N, d.rows, d.N, dev, out, y)) return nullptr;
    void* st_ = stream_of(dev);
    const loka_status st = unlocked([&] {
        return loka_grouped_gemm(&d, static_cast<uint8_t*>(ptr(xq)), static_cast<float*>(ptr(sx)), at_or_null<int32_t>(index), static_cast<int32_t*>(ptr(offsets)),
                                 static_cast<uint8_t*>(ptr(wq)), static_cast<float*>(ptr(sw)), at_or_null<void>(out), at_or_null<float>(y), st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_grouped_gemm");
    return pack({out, y});
    END_HANDLE_TH_ERRORS
}

// grouped_linear(desc, x, wq, sw, offsets, index, want_out, want_y, out, y, workspace) -> (out or None, y or None)
PyObject* grouped_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 11)) return nullptr;
    loka_grouped_desc d = bytes_of<loka_grouped_desc>(a[0], "expected a GroupedDesc");
    const at::Tensor &x = tensor(a[1]), &wq = tensor(a[2]), &sw = tensor(a[3]), &offsets = tensor(a[4]);
    const at::Tensor index = given(a[5]);
    if (!grouped_ok(d)) return fail(LOKA_ERR_SHAPE, "loka_grouped_linear");
    if (!is_rows(x) || x.size(1) != d.K || x.size(0) <= 0 || x.size(0) >= kMost || (!index.defined() && x.size(0) < d.rows)) return refuse("x: bf16 [tokens, K] with contiguous rows");
    if (!is_weights(wq, sw, d)) return refuse("wq, sw: stored weights of every group, contiguous uint8 and fp32");
    if (!is_int32(offsets, d.groups + 1) || (index.defined() && !is_int32(index, d.rows))) return refuse("offsets, index: contiguous int32 [groups + 1] and [rows]");
    d.x_rows = x.size(0);
    const at::Device dev = x.device();
    at::Tensor ws = given(a[10]);
    if (!is_run(ws)) return refuse("workspace: contiguous");
    if (!on_gpu(dev, {&wq, &sw, &offsets, &index, &ws})) return refuse("tensors on one GPU");
    const c10::DeviceGuard guard(dev);
    at::Tensor out, y;
    if (!product_outputs(a[6], a[7], a[8], a[9], d.rows * d.N, d.rows, d.N, dev, out, y)) return nullptr;
    if (!ws.defined()) ws = scratch(loka_grouped_linear_workspace(&d, index.defined()), dev);
    void* st_ = stream_of(dev);
    const loka_status st = unlocked([&] {
        return loka_grouped_linear(&d, ptr(x), row_stride(x), at_or_null<int32_t>(index), static_cast<int32_t*>(ptr(offsets)), static_cast<uint8_t*>(ptr(wq)),
                                   static_cast<float*>(ptr(sw)), at_or_null<void>(out), at_or_null<float>(y), at_or_null<void>(ws), ws.defined() ? ws.nbytes() : 0, st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_grouped_linear");
    return pack({out, y});
    END_HANDLE_TH_ERRORS
}

// grouped_wgrad(desc, xt, sxt, dyt, sdyt, offsets, want_out, want_y, out, y, workspace) -> (dw bf16 or None, dw fp32 or None)
PyObject* grouped_wgrad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 11)) return nullptr;
    const loka_grouped_desc d = bytes_of<loka_grouped_desc>(a[0], "expected a GroupedDesc");
    const at::Tensor &xt = tensor(a[1]), &sxt = tensor(a[2]), &dyt = tensor(a[3]), &sdyt = tensor(a[4]), &offsets = tensor(a[5]);
    if (!grouped_ok(d)) return fail(LOKA_ERR_SHAPE, "loka_grouped_wgrad");
    const int64_t blocks = loka_grouped_blocks(d.rows, d.groups);
    if (!holds(xt, at::kByte, blocks * d.K * 128) || !holds(sxt, at::kFloat, blocks * d.K) || !holds(dyt, at::kByte, blocks * d.N * 128) || !holds(sdyt, at::kFloat, blocks * d.N))
        return refuse("xt, sxt, dyt, sdyt: turned forms of [rows, K] and [rows, N], contiguous uint8 and fp32");
    if (!is_int32(offsets, d.groups + 1)) return refuse("offsets: contiguous int32 [groups + 1]");
    const at::Device dev = xt.device();
    at::Tensor ws = given(a[10]);
    if (!is_run(ws)) return refuse("workspace: contiguous");
    if (!on_gpu(dev, {&sxt, &dyt, &sdyt, &offsets, &ws})) return refuse("tensors on one GPU");
    const c10::DeviceGuard guard(dev);
    at::Tensor out, y;
    if (!product_outputs(a[6], a[7], a[8], a[9], d.groups * d.K * d.N, d.groups * d.K, d.N, dev, out, y)) return nullptr;
    if (a[8] == Py_None && out.defined()) out = out.view({d.groups, d.K, d.N});
    if (a[9] == Py_None && y.defined()) y = y.view({d.groups, d.K, d.N});
    if (!ws.defined()) ws = scratch(loka_grouped_wgrad_workspace(&d), dev);
    void* st_ = stream_of(dev);
    const loka_status st = unlocked([&] {
        return loka_grouped_wgrad(&d, static_cast<uint8_t*>(ptr(xt)), static_cast<float*>(ptr(sxt)), static_cast<uint8_t*>(ptr(dyt)), static_cast<float*>(ptr(sdyt)),
                                  static_cast<int32_t*>(ptr(offsets)), at_or_null<void>(out), at_or_null<float>(y), at_or_null<void>(ws), ws.defined() ? ws.nbytes() : 0, st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_grouped_wgrad");
    return pack({out, y});
    END_HANDLE_TH_ERRORS
}

// the slots [tokens, top_k], their weights, and y [rows, cols] or a matrix of the tokens; false with an exception set
bool combine_desc(const at::Tensor& slot, const at::Tensor& weight, int64_t rows, int64_t cols, loka_combine_desc& d) {
    if (!(slot.scalar_type() == at::kInt && slot.is_contiguous() && slot.dim() == 2) || (weight.defined() && !is_matrix(weight, at::kFloat, slot.size(0), slot.size(1)))) {
        refuse("slot, weight: contiguous int32 and fp32 [tokens, top_k]");
        return false;
    }
    if (slot.size(0) <= 0 || slot.size(1) <= 0 || slot.size(1) > 16 || rows <= 0 || cols <= 0) {
        fail(LOKA_ERR_SHAPE, "loka_combine");
        return false;
    }
    d = loka_combine_desc{slot.size(0), cols, rows, static_cast<int32_t>(slot.size(1))};
    return true;
}

// combine(y, slot, weight, residual, out) -> out
PyObject* combine(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 5)) return nullptr;
    const at::Tensor &y = tensor(a[0]), &slot = tensor(a[1]);
    const at::Tensor weight = given(a[2]), res = given(a[3]);
    at::Tensor out = given(a[4]);
    if (!(y.dim() == 2 && y.scalar_type() == at::kBFloat16 && y.is_contiguous())) return refuse("y: contiguous bf16 [rows, cols]");
    loka_combine_desc d;
    if (!combine_desc(slot, weight, y.size(0), y.size(1), d)) return nullptr;
    if ((res.defined() && !is_matrix(res, at::kBFloat16, d.tokens, d.cols)) || (out.defined() && !is_matrix(out, at::kBFloat16, d.tokens, d.cols)))
        return refuse("residual, out: contiguous bf16 [tokens, cols]");
    const at::Device dev = y.device();
    if (!on_gpu(dev, {&slot, &weight, &res, &out})) return refuse("tensors on one GPU");
    const c10::DeviceGuard guard(dev);
    if (!out.defined()) out = empty({d.tokens, d.cols}, at::kBFloat16, dev);
    void* st_ = stream_of(dev);
    const loka_status st = unlocked([&] {
        return loka_combine(&d, ptr(y), static_cast<int32_t*>(ptr(slot)), at_or_null<float>(weight), at_or_null<void>(res), ptr(out), st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_combine");
    return wrap(out);
    END_HANDLE_TH_ERRORS
}

// combine_backward(dout, y, slot, weight, rows, want_dy, want_dweight, dy) -> (dy or None, dweight or None)
PyObject* combine_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!need_args(n, 8)) return nullptr;
    const at::Tensor &dout = tensor(a[0]), &slot = tensor(a[2]);
    const at::Tensor y = given(a[1]), weight = given(a[3]);
    const long long rows_of = PyLong_AsLongLong(a[4]);
    const int want_dy = PyObject_IsTrue(a[5]), want_dweight = PyObject_IsTrue(a[6]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor dy = given(a[7]);
    if (!(dout.dim() == 2 && dout.scalar_type() == at::kBFloat16 && dout.is_contiguous())) return refuse("dout: contiguous bf16 [tokens, cols]");
    if (want_dweight && !y.defined()) return refuse("y: what dweight is taken from");
    if (!want_dweight && !want_dy && !dy.defined()) return refuse("one of the two gradients at least");
    const int64_t rows = y.defined() ? y.size(0) : dy.defined() ? dy.size(0) : rows_of;
    loka_combine_desc d;
    if (!combine_desc(slot, weight, rows, dout.size(1), d)) return nullptr;
    if (dout.size(0) != d.tokens || (y.defined() && !is_matrix(y, at::kBFloat16, rows, d.cols)) || (dy.defined() && !is_matrix(dy, at::kBFloat16, rows, d.cols)))
        return refuse("dout [tokens, cols], y and dy [rows, cols]: contiguous bf16");
    const at::Device dev = dout.device();
    if (!on_gpu(dev, {&y, &slot, &weight, &dy})) return refuse("tensors on one GPU");
    const c10::DeviceGuard guard(dev);
    if (!dy.defined() && want_dy) dy = empty({rows, d.cols}, at::kBFloat16, dev);
    at::Tensor dw = want_dweight ? empty({d.tokens, d.top_k}, at::kFloat, dev) : at::Tensor();
    void* st_ = stream_of(dev);
    const loka_status st = unlocked([&] {
        return loka_combine_backward(&d, ptr(dout), at_or_null<void>(y), static_cast<int32_t*>(ptr(slot)), at_or_null<float>(weight), at_or_null<void>(dy),
                                     at_or_null<float>(dw), st_);
    });
    if (st != LOKA_OK) return fail(st, "loka_combine_backward");
    return pack({dy, dw});
    END_HANDLE_TH_ERRORS
}

PyObject* set_error(PyObject*, PyObject* cls) {
    Py_INCREF(cls);
    Py_XSETREF(g_error, cls);
    Py_RETURN_NONE;
}

#define LOKA_FAST(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&NAME)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {
    LOKA_FAST(quantize), LOKA_FAST(gemm_norm), LOKA_FAST(gemm_norm_fp8out), LOKA_FAST(linear_norm), LOKA_FAST(linear_norm_xq),
    LOKA_FAST(bf16_gemm), LOKA_FAST(probe_error), LOKA_FAST(tracker_update),
    LOKA_FAST(mxfp4_quantize), LOKA_FAST(mxfp4_dequantize), LOKA_FAST(mxfp4_gemm), LOKA_FAST(mxfp4_linear), LOKA_FAST(add_rmsnorm),
    LOKA_FAST(rmsnorm_backward), LOKA_FAST(route), LOKA_FAST(route_backward), LOKA_FAST(grouped_quantize), LOKA_FAST(grouped_gemm),
    LOKA_FAST(grouped_linear), LOKA_FAST(grouped_wgrad), LOKA_FAST(combine), LOKA_FAST(combine_backward),
    {"set_error", &set_error, METH_O, "the exception class raised for a status other than LOKA_OK"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_host", "marshalling of the per-step calls", -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host(void) { return PyModule_Create(&kModule); }
