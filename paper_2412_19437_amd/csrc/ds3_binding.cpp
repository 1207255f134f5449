// The marshalling of the small calls' hot entry points, in native code: argument
// checks, output tensors from torch's allocator, the current stream, one call of
// the C entry point.  The Python functions of the package keep their signatures
// and defaults and end here.
//
// In Python (ctypes, torch.empty, views, a Stream object) a call took 12-17 us
// of host time, now 4.8 us, most of it the launch: a small layer's pass of three
// calls (256x512x1024, FP32 input) goes from 45-46 to 16-18 us, its kernels being 12 us.
#include <Python.h>
#include <algorithm>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/ds3.h"

namespace {

PyObject* g_check = nullptr;                 // _check(status, where): raises
PyObject* g_workspaces = nullptr;            // {(device index, stream): uint8 tensor}
PyObject* g_gemm_workspace = nullptr;        // gemm_workspace(nbytes, device): makes one and keeps it there

[[noreturn]] void fail(PyObject* type, const char* text) {
    PyErr_SetString(type, text);
    throw python_error();
}

const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "expected a torch.Tensor");
    return THPVariable_Unpack(o);
}

int64_t integer(PyObject* o) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}

bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();
    return v != 0;
}

// A 2-D tensor with contiguous rows.
struct Mat { int64_t rows, cols, ld; };
Mat rows2d(const at::Tensor& t, const char* name) {
    if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) {
        PyErr_Format(PyExc_ValueError, "%s must be 2-D with contiguous rows", name);
        throw python_error();
    }
    const int64_t s0 = t.stride(0);
    return {t.size(0), t.size(1), t.size(0) > 1 ? s0 : std::max(t.size(1), s0)};
}

ds3_dtype dtype_of(const at::Tensor& t) {
    if (t.scalar_type() == at::kFloat) return DS3_F32;
    if (t.scalar_type() == at::kBFloat16) return DS3_BF16;
    PyErr_Format(PyExc_TypeError, "unsupported dtype torch.%s", c10::getDtypeNames(t.scalar_type()).first.c_str());
    throw python_error();
}

at::Tensor empty2d(int64_t rows, int64_t cols, int64_t ld, at::ScalarType type, const at::Tensor& like) {
    at::Tensor t = at::empty({rows, ld}, at::TensorOptions().dtype(type).device(like.device()));
    return ld == cols ? t : t.narrow(1, 0, cols);
}
int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int64_t blocks(int64_t v) { return (v + 127) / 128; }

// uint8 [rows][cols], leading dimension padded to a multiple of 16
at::Tensor codes(int64_t rows, int64_t cols, const at::Tensor& like) { return empty2d(rows, cols, up(cols, 16), at::kByte, like); }
// logical [rows][nb] FP32; k_major stores it as [nb][rows]
at::Tensor scales(int64_t rows, int64_t nb, bool k_major, const at::Tensor& like) {
    const auto opt = at::TensorOptions().dtype(at::kFloat).device(like.device());
    return k_major ? at::empty_strided({rows, nb}, {1, std::max<int64_t>(rows, 1)}, opt) : at::empty({rows, nb}, opt);
}
at::Tensor gemm_out(int64_t rows, int64_t cols, at::ScalarType type, const at::Tensor& like) {
    return empty2d(rows, cols, up(cols, 8), type, like);
}

template <typename T = uint8_t> T* ptr(const at::Tensor& t) { return static_cast<T*>(t.data_ptr()); }
void* stream() { return c10::hip::getCurrentHIPStream(-1).stream(); }

// The interpreter lock is released while one of these exists, and taken again however its scope is left.
struct Unlocked {
    PyThreadState* const save = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(save); }
};

// The C call without the interpreter lock; a status other than DS3_OK is raised by the package.  What the call
// is given (a tensor's pointer and strides may throw) is worked out by the caller, under the lock.
template <typename F, typename... A> void call(const char* where, F* fn, A... args) {
    ds3_status st;
    {
        const Unlocked unlocked;
        st = fn(args...);
    }
    if (st == DS3_OK) return;
    PyObject* r = PyObject_CallFunction(g_check, "is", (int)st, where);
    Py_XDECREF(r);
    throw python_error();
}

PyObject* pair(const at::Tensor& q, const at::Tensor& s) {
    PyObject* a = THPVariable_Wrap(q);
    PyObject* b = a ? THPVariable_Wrap(s) : nullptr;
    PyObject* t = b ? PyTuple_Pack(2, a, b) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    return t;
}

void need(Py_ssize_t n, Py_ssize_t want) {
    if (n != want) fail(PyExc_TypeError, "wrong number of arguments");
}

// `workspace` of the GEMM calls: "auto" (the kept one of this device and stream), None or a tensor.
struct Workspace { void* p = nullptr; size_t n = 0; at::Tensor hold; };
Workspace workspace_of(PyObject* o, size_t nbytes, PyObject* a_obj, const at::Tensor& a, void* st) {
    Workspace w;
    if (o == Py_None) return w;
    if (PyUnicode_Check(o)) {
        if (nbytes == 0) return w;
        const int64_t index = a.device().has_index() ? a.device().index() : 0;
        PyObject* key = Py_BuildValue("(LK)", (long long)index, (unsigned long long)reinterpret_cast<uintptr_t>(st));
        if (!key) throw python_error();
        PyObject* kept = PyDict_GetItemWithError(g_workspaces, key);      // borrowed
        Py_DECREF(key);
        if (!kept && PyErr_Occurred()) throw python_error();
        if (kept) w.hold = tensor(kept);
        if (!kept || (size_t)w.hold.numel() < nbytes) {
            PyObject* dev = PyObject_GetAttrString(a_obj, "device");
            PyObject* made = dev ? PyObject_CallFunction(g_gemm_workspace, "KO", (unsigned long long)nbytes, dev) : nullptr;
            Py_XDECREF(dev);
            if (!made) throw python_error();
            w.hold = THPVariable_Check(made) ? THPVariable_Unpack(made) : at::Tensor();
            Py_DECREF(made);
        }
    } else {
        w.hold = tensor(o);
    }
    if (w.hold.defined()) { w.p = w.hold.data_ptr(); w.n = (size_t)w.hold.numel(); }
    return w;
}

// (x, k_major_scales, pow2) -> (codes, scales)
PyObject* quant_act_1x128(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 3);
    const at::Tensor& x = tensor(o[0]);
    const bool km = truth(o[1]), p2 = truth(o[2]);
    const Mat m = rows2d(x, "x");
    const at::Tensor q = codes(m.rows, m.cols, x), s = scales(m.rows, blocks(m.cols), km, x);
    const ds3_dtype t = dtype_of(x);
    void* st = stream();
    call(p2 ? "ds3_quant_act_1x128_pow2" : "ds3_quant_act_1x128", p2 ? ds3_quant_act_1x128_pow2 : ds3_quant_act_1x128,
         ptr(x), t, m.rows, m.cols, m.ld, ptr(q), up(m.cols, 16), ptr<float>(s), s.stride(0), s.stride(1), st);
    return pair(q, s);
    END_HANDLE_TH_ERRORS
}

// (x, k_major_scales, pow2) -> (codes of the transpose, scales)
PyObject* quant_act_128x1(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 3);
    const at::Tensor& x = tensor(o[0]);
    const bool km = truth(o[1]), p2 = truth(o[2]);
    const Mat m = rows2d(x, "x");
    const at::Tensor q = codes(m.cols, m.rows, x), s = scales(m.cols, blocks(m.rows), km, x);
    const ds3_dtype t = dtype_of(x);
    void* st = stream();
    call(p2 ? "ds3_quant_act_128x1_pow2" : "ds3_quant_act_128x1", p2 ? ds3_quant_act_128x1_pow2 : ds3_quant_act_128x1,
         ptr(x), t, m.rows, m.cols, m.ld, ptr(q), up(m.rows, 16), ptr<float>(s), s.stride(0), s.stride(1), st);
    return pair(q, s);
    END_HANDLE_TH_ERRORS
}

// (w, pow2) -> (codes, scales)
PyObject* quant_w_128x128(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 2);
    const at::Tensor& w = tensor(o[0]);
    const bool p2 = truth(o[1]);
    const Mat m = rows2d(w, "w");
    const at::Tensor q = codes(m.rows, m.cols, w), s = scales(blocks(m.rows), blocks(m.cols), false, w);
    const ds3_dtype t = dtype_of(w);
    void* st = stream();
    call(p2 ? "ds3_quant_w_128x128_pow2" : "ds3_quant_w_128x128", p2 ? ds3_quant_w_128x128_pow2 : ds3_quant_w_128x128,
         ptr(w), t, m.rows, m.cols, m.ld, ptr(q), up(m.cols, 16), ptr<float>(s), st);
    return pair(q, s);
    END_HANDLE_TH_ERRORS
}

// (w, pow2) -> (codes, scales, codes of the transpose, its scales)
PyObject* quant_w_128x128_dual(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 2);
    const at::Tensor& w = tensor(o[0]);
    const bool p2 = truth(o[1]);
    const Mat m = rows2d(w, "w");
    const at::Tensor q = codes(m.rows, m.cols, w), qt = codes(m.cols, m.rows, w);
    const at::Tensor s = scales(blocks(m.rows), blocks(m.cols), false, w), s_t = scales(blocks(m.cols), blocks(m.rows), false, w);
    const ds3_dtype t = dtype_of(w);
    void* st = stream();
    call(p2 ? "ds3_quant_w_128x128_dual_pow2" : "ds3_quant_w_128x128_dual",
         p2 ? ds3_quant_w_128x128_dual_pow2 : ds3_quant_w_128x128_dual,
         ptr(w), t, m.rows, m.cols, m.ld, ptr(q), up(m.cols, 16), ptr<float>(s), ptr(qt), up(m.rows, 16), ptr<float>(s_t), st);
    PyObject* a = pair(q, s);
    PyObject* b = a ? pair(qt, s_t) : nullptr;
    PyObject* r = b ? PySequence_Concat(a, b) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    return r;
    END_HANDLE_TH_ERRORS
}

// (h, k_major_scales, pow2) -> (codes, scales)
PyObject* swiglu_quant_1x128(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 3);
    const at::Tensor& h = tensor(o[0]);
    const bool km = truth(o[1]), p2 = truth(o[2]);
    const Mat m = rows2d(h, "h");
    if (h.scalar_type() != at::kBFloat16 || m.cols % 2) fail(PyExc_TypeError, "h must be BF16 with an even number of columns");
    const int64_t inter = m.cols / 2;
    const at::Tensor q = codes(m.rows, inter, h), s = scales(m.rows, blocks(inter), km, h);
    void* st = stream();
    call(p2 ? "ds3_swiglu_quant_1x128_pow2" : "ds3_swiglu_quant_1x128", p2 ? ds3_swiglu_quant_1x128_pow2 : ds3_swiglu_quant_1x128,
         ptr(h), m.rows, inter, m.ld, ptr(q), up(inter, 16), ptr<float>(s), s.stride(0), s.stride(1), st);
    return pair(q, s);
    END_HANDLE_TH_ERRORS
}

// (x, gamma, eps, want_y, k_major_scales, pow2) -> (codes, scales[, y])
PyObject* rmsnorm_quant_1x128(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 6);
    const at::Tensor &x = tensor(o[0]), &gamma = tensor(o[1]);
    const double eps = PyFloat_AsDouble(o[2]);
    if (eps == -1.0 && PyErr_Occurred()) throw python_error();
    const bool want_y = truth(o[3]), km = truth(o[4]), p2 = truth(o[5]);
    const Mat m = rows2d(x, "x");
    if (x.scalar_type() != at::kBFloat16 || gamma.scalar_type() != at::kFloat || gamma.numel() != m.cols || !gamma.is_contiguous())
        fail(PyExc_TypeError, "x must be BF16 and gamma a contiguous FP32 vector of x's width");
    const at::Tensor q = codes(m.rows, m.cols, x), s = scales(m.rows, blocks(m.cols), km, x);
    const at::Tensor y = want_y ? empty2d(m.rows, m.cols, m.cols, at::kBFloat16, x) : at::Tensor();
    void* st = stream();
    call(p2 ? "ds3_rmsnorm_quant_1x128_pow2" : "ds3_rmsnorm_quant_1x128",
         p2 ? ds3_rmsnorm_quant_1x128_pow2 : ds3_rmsnorm_quant_1x128,
         ptr(x), m.rows, m.cols, m.ld, ptr<float>(gamma), (float)eps, want_y ? y.data_ptr() : nullptr, m.cols, ptr(q),
         up(m.cols, 16), ptr<float>(s), s.stride(0), s.stride(1), st);
    PyObject* r = pair(q, s);
    if (!r || !want_y) return r;
    PyObject* yo = THPVariable_Wrap(y);
    PyObject* one = yo ? PyTuple_Pack(1, yo) : nullptr;
    PyObject* all = one ? PySequence_Concat(r, one) : nullptr;
    Py_XDECREF(yo);
    Py_XDECREF(one);
    Py_DECREF(r);
    return all;
    END_HANDLE_TH_ERRORS
}

// (q, s, k_major_scales, pow2) -> (codes of the transpose, scales)
PyObject* retile(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 4);
    const at::Tensor &q = tensor(o[0]), &s = tensor(o[1]);
    const bool km = truth(o[2]), p2 = truth(o[3]);
    const Mat m = rows2d(q, "q");
    if (q.scalar_type() != at::kByte || s.scalar_type() != at::kFloat || s.dim() != 2 || s.size(0) != m.rows || s.size(1) != blocks(m.cols))
        fail(PyExc_ValueError, "q: uint8 [T][C]; s: float32 logical [T][ceil(C/128)]");
    const at::Tensor qt = codes(m.cols, m.rows, q), s_t = scales(m.cols, blocks(m.rows), km, q);
    void* st = stream();
    call(p2 ? "ds3_retile_1x128_to_128x1_pow2" : "ds3_retile_1x128_to_128x1",
         p2 ? ds3_retile_1x128_to_128x1_pow2 : ds3_retile_1x128_to_128x1,
         ptr(q), m.rows, m.cols, m.ld, ptr<float>(s), s.stride(0), s.stride(1), ptr(qt), up(m.rows, 16), ptr<float>(s_t),
         s_t.stride(0), s_t.stride(1), st);
    return pair(qt, s_t);
    END_HANDLE_TH_ERRORS
}

// (x, k_major_scales) -> (packed codes, scales)
PyObject* quant_act_1x128_e5m6(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 2);
    const at::Tensor& x = tensor(o[0]);
    const bool km = truth(o[1]);
    const Mat m = rows2d(x, "x");
    if (x.scalar_type() != at::kBFloat16) fail(PyExc_TypeError, "x must be BF16");
    const int64_t width = m.cols * 3 / 2;
    const at::Tensor q = empty2d(m.rows, width, width, at::kByte, x), s = scales(m.rows, blocks(m.cols), km, x);
    void* st = stream();
    call("ds3_quant_act_1x128_e5m6", ds3_quant_act_1x128_e5m6,
         ptr(x), m.rows, m.cols, m.ld, ptr(q), width, ptr<float>(s), s.stride(0), s.stride(1), st);
    return pair(q, s);
    END_HANDLE_TH_ERRORS
}

// (a, sa, b, sb, sb_mode, f32_out, c or None, accumulate, variant, workspace, pow2) -> c
PyObject* gemm(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 11);
    const at::Tensor &a = tensor(o[0]), &sa = tensor(o[1]), &b = tensor(o[2]), &sb = tensor(o[3]);
    const int64_t sb_mode = integer(o[4]), accumulate = integer(o[7]), variant = integer(o[8]);
    const bool f32 = truth(o[5]), p2 = truth(o[10]);
    const Mat ma = rows2d(a, "a"), mb = rows2d(b, "b");
    if (ma.cols != mb.cols) fail(PyExc_ValueError, "a and b disagree on K");
    at::Tensor c = o[6] == Py_None ? gemm_out(ma.rows, mb.rows, f32 ? at::kFloat : at::kBFloat16, a) : tensor(o[6]);
    const Mat mc = rows2d(c, "c");
    const int64_t sar = sa.stride(0), sak = sa.stride(1), sbr = sb.stride(0), sbk = sb.stride(1);     // (fewer than two: an IndexError)
    void* st = stream();
    const size_t bytes = PyUnicode_Check(o[9])
                             ? ds3_gemm_workspace_bytes_v((int)variant, ma.rows, mb.rows, ma.cols, (ds3_bscale)sb_mode) : 0;
    const Workspace w = workspace_of(o[9], bytes, o[0], a, st);
    const ds3_dtype ct = dtype_of(c);
    call(p2 ? "ds3_gemm_fp8_bs_pow2" : "ds3_gemm_fp8_bs_v", p2 ? ds3_gemm_fp8_bs_pow2 : ds3_gemm_fp8_bs_v,
         (int)variant, ma.rows, mb.rows, ma.cols, ptr(a), ma.ld, ptr<float>(sa), sar, sak, ptr(b), mb.ld,
         ptr<float>(sb), sbr, sbk, (ds3_bscale)sb_mode, c.data_ptr(), ct, mc.ld, (int)accumulate, w.p, w.n, st);
    if (o[6] == Py_None) return THPVariable_Wrap(c);
    Py_INCREF(o[6]);
    return o[6];
    END_HANDLE_TH_ERRORS
}

// ---- MXFP4, and rows in expert order and back ------------------------------------------
// The calls below launch on the current device's current stream: their tensors have to be there.
const at::Tensor& here(PyObject* o, const char* name) {
    const at::Tensor& t = tensor(o);
    if (!t.is_cuda() || t.get_device() != c10::hip::current_device()) {
        PyErr_Format(PyExc_ValueError, "%s must be on the current device", name);
        throw python_error();
    }
    return t;
}
// As rows2d; one without elements has no strides to speak of.
Mat mat2d(const at::Tensor& t, const char* name) {
    if (t.dim() == 2 && t.numel() == 0) return {t.size(0), t.size(1), t.size(1)};
    return rows2d(t, name);
}
void need_type(const at::Tensor& t, at::ScalarType type, const char* text) {
    if (t.scalar_type() != type) fail(PyExc_TypeError, text);
}
at::Tensor scale_words(int64_t rows, int64_t nb, bool k_major, const at::Tensor& like) {
    const auto opt = at::TensorOptions().dtype(at::kInt).device(like.device());
    return k_major ? at::empty_strided({rows, nb}, {1, std::max<int64_t>(rows, 1)}, opt) : at::empty({rows, nb}, opt);
}
// Scales of `rows` rows in blocks of 128 elements, logical [rows][nb] with any strides.
void need_scales(const at::Tensor& s, at::ScalarType type, int64_t rows, int64_t nb, const char* text) {
    if (s.scalar_type() != type || s.dim() != 2 || s.size(0) != rows || s.size(1) != nb) fail(PyExc_ValueError, text);
}
PyObject* again(PyObject* given, const at::Tensor& made) {
    if (given == Py_None) return THPVariable_Wrap(made);
    Py_INCREF(given);
    return given;
}

// (x, k_major_scales, transposed) -> (packed codes, scale words)
PyObject* quant_mxfp4(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 3);
    const at::Tensor& x = here(o[0], "x");
    const bool km = truth(o[1]), tr = truth(o[2]);
    const Mat m = mat2d(x, "x");
    const ds3_dtype t = dtype_of(x);
    const int64_t rows = tr ? m.cols : m.rows, cols = tr ? m.rows : m.cols;
    const at::Tensor q = codes(rows, (cols + 1) / 2, x), s = scale_words(rows, blocks(cols), km, x);
    void* st = stream();
    call(tr ? "ds3_quant_mxfp4_t" : "ds3_quant_mxfp4", tr ? ds3_quant_mxfp4_t : ds3_quant_mxfp4, ptr(x), t, m.rows, m.cols, m.ld,
         ptr(q), up((cols + 1) / 2, 16), ptr<uint32_t>(s), s.stride(0), s.stride(1), st);
    return pair(q, s);
    END_HANDLE_TH_ERRORS
}

// (q, s, cols or -1) -> y BF16
PyObject* dequant_mxfp4(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 3);
    const at::Tensor &q = here(o[0], "q"), &s = here(o[1], "s");
    const Mat m = mat2d(q, "q");
    int64_t cols = integer(o[2]);
    if (cols < 0) cols = 2 * m.cols;
    need_type(q, at::kByte, "q must be uint8");
    if ((cols + 1) / 2 != m.cols) fail(PyExc_ValueError, "q must hold two columns a byte");
    need_scales(s, at::kInt, m.rows, blocks(cols), "s must be int32, logical [rows][ceil(cols / 128)]");
    const at::Tensor y = gemm_out(m.rows, cols, at::kBFloat16, q);
    void* st = stream();
    call("ds3_dequant_mxfp4", ds3_dequant_mxfp4, ptr(q), m.rows, cols, m.ld, ptr<uint32_t>(s), s.stride(0), s.stride(1), y.data_ptr(),
         up(cols, 8), st);
    return THPVariable_Wrap(y);
    END_HANDLE_TH_ERRORS
}

// (a, sa, b, sb, f32_out, c or None, accumulate) -> c
PyObject* gemm_mxfp4(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 7);
    const at::Tensor &a = here(o[0], "a"), &sa = here(o[1], "sa"), &b = here(o[2], "b"), &sb = here(o[3], "sb");
    const bool f32 = truth(o[4]), acc = truth(o[6]);
    const Mat ma = mat2d(a, "a"), mb = mat2d(b, "b");
    need_type(a, at::kByte, "a must be uint8");
    need_type(b, at::kByte, "b must be uint8");
    if (ma.cols != mb.cols) fail(PyExc_ValueError, "a and b disagree on K");
    const int64_t k = 2 * ma.cols;
    need_scales(sa, at::kInt, ma.rows, blocks(k), "sa must be int32, logical [M][K / 128]");
    need_scales(sb, at::kInt, mb.rows, blocks(k), "sb must be int32, logical [N][K / 128]");
    const at::Tensor c = o[5] == Py_None ? gemm_out(ma.rows, mb.rows, f32 ? at::kFloat : at::kBFloat16, a) : here(o[5], "c");
    const Mat mc = mat2d(c, "c");
    if (mc.rows != ma.rows || mc.cols != mb.rows) fail(PyExc_ValueError, "c must be [M][N]");
    if (o[5] == Py_None && acc) fail(PyExc_ValueError, "nothing to accumulate into");
    const ds3_dtype ct = dtype_of(c);
    void* st = stream();
    call("ds3_gemm_mxfp4", ds3_gemm_mxfp4, ma.rows, mb.rows, k, ptr(a), ma.ld, ptr<uint32_t>(sa), sa.stride(0), sa.stride(1), ptr(b),
         mb.ld, ptr<uint32_t>(sb), sb.stride(0), sb.stride(1), c.data_ptr(), ct, mc.ld, (int)acc, st);
    return again(o[5], c);
    END_HANDLE_TH_ERRORS
}

// (a, sa, group_offsets, b, sb, f32_out, c or None) -> c
PyObject* grouped_gemm_mxfp4(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 7);
    const at::Tensor &a = here(o[0], "a"), &sa = here(o[1], "sa"), &off = here(o[2], "group_offsets"), &b = here(o[3], "b"), &sb = here(o[4], "sb");
    const bool f32 = truth(o[5]);
    const Mat ma = mat2d(a, "a");
    need_type(a, at::kByte, "a must be uint8");
    need_type(b, at::kByte, "b must be uint8");
    if (b.dim() != 3 || b.size(2) != ma.cols || !b.is_contiguous()) fail(PyExc_ValueError, "b must be contiguous [G][N][K / 2]");
    const int64_t g = b.size(0), nn = b.size(1), k = 2 * ma.cols;
    if (off.scalar_type() != at::kInt || off.dim() != 1 || off.size(0) != g + 1 || !off.is_contiguous())
        fail(PyExc_ValueError, "group_offsets must be contiguous int32 of length G+1");
    need_scales(sa, at::kInt, ma.rows, blocks(k), "sa must be int32, logical [rows][K / 128]");
    if (sb.scalar_type() != at::kInt || sb.dim() != 3 || sb.size(0) != g || sb.size(1) != nn || sb.size(2) != blocks(k) ||
        (g > 1 && sb.stride(0) != nn * blocks(k)))
        fail(PyExc_ValueError, "sb must be int32, logical [G][N][K / 128], one expert's words behind the other's");
    const at::Tensor c = o[6] == Py_None ? gemm_out(ma.rows, nn, f32 ? at::kFloat : at::kBFloat16, a) : here(o[6], "c");
    const Mat mc = mat2d(c, "c");
    if (mc.rows != ma.rows || mc.cols != nn) fail(PyExc_ValueError, "c must be [rows][N]");
    const ds3_dtype ct = dtype_of(c);
    if (g > INT32_MAX) fail(PyExc_ValueError, "too many experts");
    void* st = stream();
    call("ds3_grouped_gemm_mxfp4", ds3_grouped_gemm_mxfp4, (int32_t)g, ptr<int32_t>(off), ma.rows, nn, k, ptr(a), ma.ld, ptr<uint32_t>(sa),
         sa.stride(0), sa.stride(1), ptr(b), ma.cols, ptr<uint32_t>(sb), sb.stride(1), sb.stride(2), c.data_ptr(), ct, mc.ld, st);
    return again(o[6], c);
    END_HANDLE_TH_ERRORS
}

// (expert_ids, G, first_expert) -> (group_offsets, row_of_slot)
PyObject* moe_sort(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 3);
    const at::Tensor& ids = here(o[0], "expert_ids");
    const int64_t g = integer(o[1]), first = integer(o[2]);
    need_type(ids, at::kInt, "expert_ids must be int32");
    const Mat m = mat2d(ids, "expert_ids");
    if (g < 0 || g > 1023 || first < 0 || first > INT32_MAX || m.cols > INT32_MAX) fail(PyExc_ValueError, "num_experts is 0 .. 1023, first_expert 0 .. 2^31 - 1");
    const auto opt = at::TensorOptions().dtype(at::kInt).device(ids.device());
    const at::Tensor off = at::empty({g + 1}, opt), rows = at::empty({m.rows, m.cols}, opt);
    void* st = stream();
    call("ds3_moe_sort", ds3_moe_sort, ptr<int32_t>(ids), m.rows, (int32_t)m.cols, m.ld, (int32_t)first, (int32_t)g, ptr<int32_t>(off),
         ptr<int32_t>(rows), st);
    return pair(off, rows);
    END_HANDLE_TH_ERRORS
}

// row_of_slot [tokens][top_k], contiguous
const at::Tensor& slots(PyObject* o) {
    const at::Tensor& r = here(o, "row_of_slot");
    if (r.scalar_type() != at::kInt || r.dim() != 2 || !r.is_contiguous() || r.size(1) > INT32_MAX)
        fail(PyExc_ValueError, "row_of_slot must be contiguous int32 [tokens][top_k]");
    return r;
}
int64_t rows_given(PyObject* o, const at::Tensor& r) {
    return o == Py_None ? r.numel() : integer(o);
}

// (x, row_of_slot, rows or None, out or None) -> y
PyObject* moe_dispatch(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 4);
    const at::Tensor &x = here(o[0], "x"), &r = slots(o[1]);
    const Mat m = mat2d(x, "x");
    const ds3_dtype t = dtype_of(x);
    if (r.size(0) != m.rows) fail(PyExc_ValueError, "x and row_of_slot disagree on the tokens");
    const int64_t total = rows_given(o[2], r);
    if (total < 0) fail(PyExc_ValueError, "rows must not be negative");
    const at::Tensor y = o[3] == Py_None ? empty2d(total, m.cols, up(m.cols, 8), x.scalar_type(), x) : here(o[3], "out");
    const Mat my = mat2d(y, "out");
    if (y.scalar_type() != x.scalar_type() || my.cols != m.cols || (o[2] != Py_None && my.rows != total))
        fail(PyExc_ValueError, "out must be [rows][columns of x] of x's type");
    void* st = stream();
    call("ds3_moe_dispatch", ds3_moe_dispatch, ptr(x), t, m.rows, m.cols, m.ld, ptr<int32_t>(r), (int32_t)r.size(1), my.rows, y.data_ptr(),
         my.ld, st);
    return again(o[3], y);
    END_HANDLE_TH_ERRORS
}

// (x, row_of_slot, rows or None, out or None, k_major_scales, form) -> (codes, scales); form 0: 1x128, 1: its power-of-two
// form, 2: MXFP4
PyObject* moe_dispatch_quant(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 6);
    const at::Tensor &x = here(o[0], "x"), &r = slots(o[1]);
    const Mat m = mat2d(x, "x");
    const ds3_dtype t = dtype_of(x);
    const bool km = truth(o[4]);
    const int64_t form = integer(o[5]);
    if (r.size(0) != m.rows) fail(PyExc_ValueError, "x and row_of_slot disagree on the tokens");
    const int64_t width = form == 2 ? (m.cols + 1) / 2 : m.cols, nb = blocks(m.cols);
    const at::ScalarType stype = form == 2 ? at::kInt : at::kFloat;
    int64_t total = rows_given(o[2], r);
    if (total < 0) fail(PyExc_ValueError, "rows must not be negative");
    at::Tensor q, s;
    if (o[3] == Py_None) {
        q = codes(total, width, x);
        s = form == 2 ? scale_words(total, nb, km, x) : scales(total, nb, km, x);
    } else {
        if (!PyTuple_Check(o[3]) || PyTuple_GET_SIZE(o[3]) != 2) fail(PyExc_TypeError, "out must be a pair (codes, scales)");
        q = here(PyTuple_GET_ITEM(o[3], 0), "out");
        s = here(PyTuple_GET_ITEM(o[3], 1), "out");
    }
    const Mat mq = mat2d(q, "out");
    if (q.scalar_type() != at::kByte || mq.cols != width || (o[2] != Py_None && mq.rows != total))
        fail(PyExc_ValueError, "out's codes must be uint8 [rows][bytes of a row]");
    need_scales(s, stype, mq.rows, nb, "out's scales must be logical [rows][ceil(columns / 128)], FP32 (MXFP4: int32)");
    if (mq.rows > 1 && nb > 0 && (s.stride(0) == 0 || (nb > 1 && s.stride(1) == 0))) fail(PyExc_ValueError, "out's scales overlap");
    void* st = stream();
    if (form == 2)
        call("ds3_moe_dispatch_quant_mxfp4", ds3_moe_dispatch_quant_mxfp4, ptr(x), t, m.rows, m.cols, m.ld, ptr<int32_t>(r),
             (int32_t)r.size(1), mq.rows, ptr(q), mq.ld, ptr<uint32_t>(s), s.stride(0), s.stride(1), st);
    else
        call(form ? "ds3_moe_dispatch_quant_1x128_pow2" : "ds3_moe_dispatch_quant_1x128",
             form ? ds3_moe_dispatch_quant_1x128_pow2 : ds3_moe_dispatch_quant_1x128, ptr(x), t, m.rows, m.cols, m.ld, ptr<int32_t>(r),
             (int32_t)r.size(1), mq.rows, ptr(q), mq.ld, ptr<float>(s), s.stride(0), s.stride(1), st);
    if (o[3] == Py_None) return pair(q, s);
    Py_INCREF(o[3]);
    return o[3];
    END_HANDLE_TH_ERRORS
}

// weights [tokens][top_k] FP32 contiguous, or None
const float* weights_of(PyObject* o, const at::Tensor& r) {
    if (o == Py_None) return nullptr;
    const at::Tensor& w = here(o, "weights");
    if (w.scalar_type() != at::kFloat || !w.is_contiguous() || !w.sizes().equals(r.sizes()))
        fail(PyExc_ValueError, "weights must be contiguous FP32 [tokens][top_k]");
    return ptr<float>(w);
}

// (y, row_of_slot, weights or None, out type: 0 as y, 1 FP32, 2 BF16, out or None) -> out
PyObject* moe_combine(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 5);
    const at::Tensor &y = here(o[0], "y"), &r = slots(o[1]);
    const Mat m = mat2d(y, "y");
    const ds3_dtype yt = dtype_of(y);
    const float* w = weights_of(o[2], r);
    const int64_t type = integer(o[3]);
    const at::ScalarType otype = type == 1 ? at::kFloat : type == 2 ? at::kBFloat16 : y.scalar_type();
    const at::Tensor out = o[4] == Py_None ? empty2d(r.size(0), m.cols, up(m.cols, 8), otype, y) : here(o[4], "out");
    const Mat mo = mat2d(out, "out");
    const ds3_dtype ot = dtype_of(out);
    if (mo.rows != r.size(0) || mo.cols != m.cols) fail(PyExc_ValueError, "out must be [tokens][columns of y]");
    void* st = stream();
    call("ds3_moe_combine", ds3_moe_combine, y.data_ptr(), yt, m.rows, m.cols, m.ld, ptr<int32_t>(r), w, r.size(0), (int32_t)r.size(1),
         out.data_ptr(), ot, mo.ld, st);
    return again(o[4], out);
    END_HANDLE_TH_ERRORS
}

// (dout, y, row_of_slot, weights or None, dy or None) -> (dy, dweights)
PyObject* moe_combine_bwd(PyObject*, PyObject* const* o, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 5);
    const at::Tensor &d = here(o[0], "dout"), &y = here(o[1], "y"), &r = slots(o[2]);
    const Mat md = mat2d(d, "dout"), m = mat2d(y, "y");
    const ds3_dtype ot = dtype_of(d), yt = dtype_of(y);
    const float* w = weights_of(o[3], r);
    if (md.rows != r.size(0) || md.cols != m.cols) fail(PyExc_ValueError, "dout must be [tokens][columns of y]");
    const at::Tensor dy = o[4] == Py_None ? empty2d(m.rows, m.cols, up(m.cols, 8), y.scalar_type(), y) : here(o[4], "dy");
    const Mat my = mat2d(dy, "dy");
    if (dy.scalar_type() != y.scalar_type() || my.rows != m.rows || my.cols != m.cols) fail(PyExc_ValueError, "dy must be as y");
    const at::Tensor dw = at::empty({r.size(0), r.size(1)}, at::TensorOptions().dtype(at::kFloat).device(y.device()));
    void* st = stream();
    call("ds3_moe_combine_bwd", ds3_moe_combine_bwd, d.data_ptr(), ot, md.ld, y.data_ptr(), yt, m.rows, m.cols, m.ld, ptr<int32_t>(r), w,
         r.size(0), (int32_t)r.size(1), dy.data_ptr(), my.ld, ptr<float>(dw), st);
    return pair(dy, dw);
    END_HANDLE_TH_ERRORS
}

PyMethodDef kMethods[] = {
#define M(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
    M(quant_act_1x128), M(quant_act_128x1), M(quant_w_128x128), M(quant_w_128x128_dual), M(swiglu_quant_1x128), M(rmsnorm_quant_1x128), M(retile),
    M(quant_act_1x128_e5m6), M(gemm), M(quant_mxfp4), M(dequant_mxfp4), M(gemm_mxfp4), M(grouped_gemm_mxfp4),
    M(moe_sort), M(moe_dispatch), M(moe_dispatch_quant), M(moe_combine), M(moe_combine_bwd),
#undef M
    {"init", [](PyObject*, PyObject* args) -> PyObject* {
         PyObject *check, *kept, *make;
         if (!PyArg_ParseTuple(args, "OO!O", &check, &PyDict_Type, &kept, &make)) return nullptr;
         Py_INCREF(check); Py_INCREF(kept); Py_INCREF(make);
         g_check = check; g_workspaces = kept; g_gemm_workspace = make;
         Py_RETURN_NONE;
     }, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "ds3_native", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_ds3_native() { return PyModule_Create(&kModule); }
