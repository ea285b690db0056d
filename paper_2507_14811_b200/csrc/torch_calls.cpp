// The calls a layer makes at run time and when it is built, as functions that take torch tensors: reading shapes, strides, pointers and the
// current stream here costs a fraction of what it costs in Python (an eager 256 x 256 -> 768 layer call: 17.9 us with
// ctypes objects, 8.5 us from here; the three calls of a 2048 x 4608 -> 1152 W4A8 layer: 50.6 -> 32.8 us).  Argument
// marshalling only: every check is the C ABI's (include/segquant.h), every function returns its status (with the tensors
// it allocated, where it did), and the GIL is released around the call.  Reading a tensor can throw (a wrapper or sparse
// tensor without storage, a stride of a 0-dimensional one), so everything is read into locals while the GIL is held; what
// runs without it is a call of the C ABI, which does not throw.
#include <Python.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include "segquant.h"

namespace {

struct BadArgument {};           // a Python exception is set

// Positional arguments of one call.
struct Args {
    PyObject *const *a;

    const at::Tensor &tensor(int i) const
    {
        if (!THPVariable_Check(a[i])) {
            PyErr_Format(PyExc_TypeError, "argument %d must be a tensor, not %s", i, Py_TYPE(a[i])->tp_name);
            throw BadArgument();
        }
        return THPVariable_Unpack(a[i]);
    }
    const at::Tensor &matrix(int i) const
    {
        const at::Tensor &t = tensor(i);
        if (t.dim() != 2) {
            PyErr_Format(PyExc_ValueError, "argument %d must be a matrix, not %d-dimensional", i, int(t.dim()));
            throw BadArgument();
        }
        return t;
    }
    bool none(int i) const { return a[i] == Py_None; }
    void *ptr(int i) const { return none(i) ? nullptr : tensor(i).data_ptr(); }
    float *f32(int i) const { return static_cast<float *>(ptr(i)); }
    size_t bytes(int i) const { return size_t(tensor(i).numel()); }       // byte buffers: as many elements
    long long integer(int i) const
    {
        const long long v = PyLong_AsLongLong(a[i]);
        if (v == -1 && PyErr_Occurred()) throw BadArgument();
        return v;
    }
    bool truth(int i) const
    {
        const int v = PyObject_IsTrue(a[i]);
        if (v < 0) throw BadArgument();
        return v != 0;
    }
    const sq_segtable *seg(int i) const { return reinterpret_cast<const sq_segtable *>(integer(i)); }
};

sq_dtype dtype_of(const at::Tensor &t)
{
    if (t.scalar_type() == at::kFloat) return SQ_F32;
    if (t.scalar_type() == at::kBFloat16) return SQ_BF16;
    PyErr_Format(PyExc_TypeError, "unsupported dtype %s", c10::toString(t.scalar_type()));
    throw BadArgument();
}

void *current_stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

struct GilRelease {
    PyThreadState *state = PyEval_SaveThread();
    ~GilRelease() { PyEval_RestoreThread(state); }
};

template <typename F>
sq_status without_gil(F f)
{
    const GilRelease released;
    return f();
}

// What the C ABI takes of a tensor with rows: read while the GIL is held.
struct Rows {
    void *p;
    int64_t rows, cols, ld;           // cols: of the last dimension
    bool on_host;
    explicit Rows(const at::Tensor &t) : p(t.data_ptr()), on_host(!t.is_cuda())
    {
        const at::IntArrayRef sizes = t.sizes(), strides = t.strides();
        if (sizes.empty()) (void)t.size(0);                           // throws the error that t.stride(0) gives in Python
        rows = sizes.front(), cols = sizes.back(), ld = strides.front();
    }
};

template <typename F>
PyObject *guarded(const char *name, Py_ssize_t n, Py_ssize_t want, F f)
{
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, not %zd", name, want, n);
        return nullptr;
    }
    try {
        return f();
    } catch (const BadArgument &) {
        return nullptr;
    } catch (...) {                  // torch's own errors, as torch's Python methods raise them
        torch::translate_exception_to_python(std::current_exception());
        return nullptr;
    }
}

// code matrix [rows, K] with a 128-byte padded row pitch, as binding.new_codes makes it
at::Tensor new_codes(int64_t rows, int64_t K, const at::Tensor &like)
{
    return at::empty({rows, (K + 127) / 128 * 128}, like.options().dtype(at::kByte)).narrow(1, 0, K);
}

// X, Wq, seg, code, s_pos, s_neg, s_w, bias, Y, scratch, workspace, x_stage, y_stage, flags
PyObject *layer_forward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded("layer_forward", n, 14, [&] {
        const Args a{args};
        const sq_dtype dx = dtype_of(a.matrix(0)), dy = dtype_of(a.tensor(8));
        const Rows X(a.matrix(0)), W(a.tensor(1)), Y(a.tensor(8));
        const sq_segtable *seg = a.seg(2);
        const sq_code code = sq_code(a.integer(3));
        const float *sp = a.f32(4), *sn = a.f32(5), *sw = a.f32(6), *bias = a.f32(7);
        const uint32_t flags = uint32_t(a.integer(13));
        void *scratch = a.ptr(9), *ws = a.ptr(10), *xs = a.ptr(11), *ys = a.ptr(12), *stream = current_stream();
        const size_t scratch_bytes = a.bytes(9), ws_bytes = a.bytes(10);
        return PyLong_FromLong(without_gil([&] {
            return segquant_layer_forward(X.p, X.on_host, xs, dx, X.rows, X.cols, X.ld, W.p, W.ld, W.rows, seg, code, sp, sn, sw,
                                          bias, flags, Y.p, Y.on_host, ys, dy, Y.ld, scratch, scratch_bytes, ws, ws_bytes, stream);
        }));
    });
}

// X, seg, s_pos, s_neg, code, flags, c_pos, c_neg
PyObject *quantize_act(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded("quantize_act", n, 8, [&] {
        const Args a{args};
        const sq_dtype dx = dtype_of(a.matrix(0));
        const Rows X(a.matrix(0)), C(a.tensor(6));
        const sq_segtable *seg = a.seg(1);
        const float *sp = a.f32(2), *sn = a.f32(3);
        const sq_code code = sq_code(a.integer(4));
        const uint32_t flags = uint32_t(a.integer(5));
        void *cn = a.ptr(7), *stream = current_stream();
        return PyLong_FromLong(without_gil([&] {
            return segquant_quantize_act(X.p, dx, X.rows, X.cols, X.ld, seg, sp, sn, code, flags, C.p, cn, C.ld, stream);
        }));
    });
}

// H, seg, s_pos, s_neg, code, flags, act, mult, c_pos, c_neg
PyObject *quantize_act_fused(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded("quantize_act_fused", n, 10, [&] {
        const Args a{args};
        const sq_dtype dh = dtype_of(a.matrix(0));
        const Rows H(a.matrix(0)), C(a.tensor(8));
        const sq_segtable *seg = a.seg(1);
        const float *sp = a.f32(2), *sn = a.f32(3), *mult = a.f32(7);
        const sq_code code = sq_code(a.integer(4));
        const uint32_t flags = uint32_t(a.integer(5));
        const sq_act act = sq_act(a.integer(6));
        const int64_t K = act == SQ_ACT_GEGLU ? H.cols / 2 : H.cols;
        void *cn = a.ptr(9), *stream = current_stream();
        return PyLong_FromLong(without_gil([&] {
            return segquant_quantize_act_fused(H.p, dh, H.rows, K, H.ld, seg, sp, sn, code, flags, act, mult, C.p, cn, C.ld, stream);
        }));
    });
}

// X, seg, number of scales, code, is_weight, dual, workspace, flags -> (status, s_pos, s_neg | None)
PyObject *calib_scales(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded("calib_scales", n, 8, [&]() -> PyObject * {
        const Args a{args};
        const at::Tensor &x = a.matrix(0);
        const sq_dtype dx = dtype_of(x);
        const Rows X(x);
        const sq_segtable *seg = a.seg(1);
        const int64_t scales = a.integer(2);
        const sq_code code = sq_code(a.integer(3));
        const bool is_weight = a.truth(4), dual = a.truth(5);
        void *ws = a.ptr(6), *stream = current_stream();
        const size_t ws_bytes = a.bytes(6);
        const uint32_t flags = uint32_t(a.integer(7));
        const auto f32 = x.options().dtype(at::kFloat);
        at::Tensor sp = at::empty({scales}, f32), sn;
        if (dual && !is_weight) sn = at::empty({scales}, f32);
        float *s_pos = sp.data_ptr<float>(), *s_neg = sn.defined() ? sn.data_ptr<float>() : nullptr;
        const sq_status st = without_gil([&] {
            return segquant_calib_scales(X.p, dx, X.rows, X.cols, X.ld, seg, code, is_weight, dual, flags, s_pos, s_neg, ws, ws_bytes, stream);
        });
        return Py_BuildValue("(iNN)", int(st), THPVariable_Wrap(sp), THPVariable_Wrap(sn));
    });
}

// W, seg, s_w, code, flags, Wq | None -> (status, Wq)
PyObject *quantize_weight(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded("quantize_weight", n, 6, [&]() -> PyObject * {
        const Args a{args};
        const at::Tensor &w = a.matrix(0);
        const sq_dtype dw = dtype_of(w);
        const Rows W(w);
        const sq_segtable *seg = a.seg(1);
        const float *sw = a.f32(2);
        const sq_code code = sq_code(a.integer(3));
        const uint32_t flags = uint32_t(a.integer(4));
        const at::Tensor q = a.none(5) ? new_codes(W.rows, W.cols, w) : a.tensor(5);
        const Rows C(q);
        void *stream = current_stream();
        const sq_status st = without_gil([&] {
            return segquant_quantize_weight(W.p, dw, W.rows, W.cols, W.ld, seg, sw, code, flags, C.p, C.ld, stream);
        });
        return Py_BuildValue("(iN)", int(st), THPVariable_Wrap(q));
    });
}

// Xq_pos, Xq_neg | None, Wq, seg, code, s_pos, s_neg | None, s_w, bias, Y, acc_dump | None, workspace, kind
enum GemmCall : int { kSeglinear = 0, kDualscale = 1, kW4a8 = 2 };
PyObject *gemm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded("gemm", n, 13, [&] {
        const Args a{args};
        const sq_dtype dy = dtype_of(a.tensor(9));
        const Rows X(a.matrix(0)), W(a.tensor(2)), Y(a.tensor(9));
        const sq_segtable *seg = a.seg(3);
        const sq_code code = sq_code(a.integer(4));
        const float *sp = a.f32(5), *sn = a.f32(6), *sw = a.f32(7), *bias = a.f32(8);
        void *xn = a.ptr(1), *dump = a.ptr(10), *ws = a.ptr(11), *stream = current_stream();
        const size_t ws_bytes = a.bytes(11);
        const int kind = int(a.integer(12));
        const int64_t M = X.rows, K = X.cols, N = W.rows;
        return PyLong_FromLong(without_gil([&] {
            if (kind == kW4a8)
                return segquant_w4a8_gemm(X.p, xn, X.ld, W.p, W.ld, M, N, K, seg, sp, sn, sw, bias, Y.p, dy, Y.ld, dump, ws, ws_bytes,
                                          stream);
            if (kind == kDualscale)
                return segquant_dualscale_gemm(X.p, xn, X.ld, W.p, W.ld, M, N, K, seg, code, sp, sn, sw, bias, Y.p, dy, Y.ld, dump, ws,
                                               ws_bytes, stream);
            return segquant_seglinear_gemm(X.p, X.ld, W.p, W.ld, M, N, K, seg, code, sp, sw, bias, Y.p, dy, Y.ld, dump, ws, ws_bytes,
                                           stream);
        }));
    });
}

// X, seg, P, dual, bits, flags -> (status, s_pos, s_neg | None, c_pos, c_neg | None)
PyObject *quantize_per_row(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded("quantize_per_row", n, 6, [&]() -> PyObject * {
        const Args a{args};
        const at::Tensor &x = a.matrix(0);
        const sq_dtype dx = dtype_of(x);
        const Rows X(x);
        const int64_t P = a.integer(2);
        const sq_segtable *seg = a.seg(1);
        const bool dual = a.truth(3);
        const int bits = int(a.integer(4));
        const uint32_t flags = uint32_t(a.integer(5));
        const auto scales = x.options().dtype(at::kFloat);
        at::Tensor sp = at::empty({X.rows, P}, scales), sn, cp = new_codes(X.rows, X.cols, x), cn;
        if (dual) {
            sn = at::empty({X.rows, P}, scales);
            cn = new_codes(X.rows, X.cols, x);
        }
        float *s_pos = sp.data_ptr<float>(), *s_neg = dual ? sn.data_ptr<float>() : nullptr;
        const Rows C(cp);
        void *c_neg = dual ? cn.data_ptr() : nullptr;
        void *stream = current_stream();
        const sq_status st = without_gil([&] {
            return segquant_quantize_per_row(X.p, dx, X.rows, X.cols, X.ld, seg, bits, flags, s_pos, s_neg, C.p, c_neg, C.ld, stream);
        });
        return Py_BuildValue("(iNNNN)", int(st), THPVariable_Wrap(sp), THPVariable_Wrap(sn), THPVariable_Wrap(cp), THPVariable_Wrap(cn));
    });
}

// Wq4, Wq8
PyObject *unpack_w4(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded("unpack_w4", n, 2, [&] {
        const Args a{args};
        const Rows W4(a.matrix(0)), W8(a.tensor(1));
        void *stream = current_stream();
        return PyLong_FromLong(without_gil([&] {
            return segquant_unpack_w4(W4.p, W4.ld, W4.rows, 2 * W4.cols, W8.p, W8.ld, stream);
        }));
    });
}

// ---- 4-bit weights with group scales and block norms: the tensors are held to what the C ABI takes of them

[[noreturn]] void refuse(PyObject *type, const char *format, const char *what)
{
    PyErr_Format(type, format, what);
    throw BadArgument();
}

// A CUDA tensor of the current device.
const at::Tensor &on_device(const at::Tensor &t, const char *what)
{
    if (!t.is_cuda()) refuse(PyExc_ValueError, "%s must be a CUDA tensor", what);
    if (t.get_device() != c10::cuda::current_device()) refuse(PyExc_ValueError, "%s is on another device than the current one", what);
    return t;
}

// A matrix with consecutive columns (int64 pitch in elements); `rows` / `cols` < 0: any.
struct Matrix {
    void *p = nullptr;
    int64_t rows = 0, cols = 0, ld = 0;
    Matrix() = default;
    Matrix(const at::Tensor &t, const char *what, int64_t want_rows = -1, int64_t want_cols = -1)
    {
        if (t.dim() != 2) refuse(PyExc_ValueError, "%s must be a matrix", what);
        rows = t.size(0), cols = t.size(1);
        if ((want_rows >= 0 && rows != want_rows) || (want_cols >= 0 && cols != want_cols)) refuse(PyExc_ValueError, "%s has another shape than the call's", what);
        if (cols > 1 && t.stride(1) != 1) refuse(PyExc_ValueError, "the columns of %s must lie one behind the other", what);
        on_device(t, what);
        p = t.data_ptr();
        ld = rows == 1 ? (cols + 15) / 16 * 16 : t.stride(0);        // the pitch of a single row is nobody's
    }
};

void want_type(const at::Tensor &t, at::ScalarType type, const char *what)
{
    if (t.scalar_type() != type) refuse(PyExc_TypeError, "%s has the wrong dtype", what);
}

// fp32 vector of at least n elements, or None
float *f32_vector(const Args &a, int i, int64_t n, const char *what)
{
    if (a.none(i)) return nullptr;
    const at::Tensor &t = a.tensor(i);
    want_type(t, at::kFloat, what);
    if (t.numel() < n || !t.is_contiguous()) refuse(PyExc_ValueError, "%s is too short or not contiguous", what);
    return static_cast<float *>(on_device(t, what).data_ptr());
}

// [rows, cols] on the device of a CUDA tensor, with rows on boundaries of `unit` elements.  Past the dispatcher and without a view: half
// the time of at::empty and narrow (a call with one output of an odd width 5.9 -> 4.6 us).  The price: torch's modes that watch
// new tensors or fill them do not see these.
at::Tensor new_rows(int64_t rows, int64_t cols, const at::Tensor &like, at::ScalarType type, int64_t unit = 16)
{
    on_device(like, "a tensor");
    return at::Tensor(at::detail::empty_strided_cuda({rows, cols}, {(cols + unit - 1) / unit * unit, 1}, type, like.device()));
}

struct GroupScales {
    Matrix s, z;
    sq_dtype type;
    GroupScales(const Args &a, int is, int iz, int64_t groups, int64_t N) : s(a.matrix(is), "s_w", groups, N), type(dtype_of(a.tensor(is)))
    {
        if (a.none(iz)) return;
        want_type(a.tensor(iz), at::kChar, "z_w");
        z = Matrix(a.tensor(iz), "z_w", groups, N);
    }
};

int64_t groups_of(int64_t K, int64_t group)
{
    if (group <= 0) refuse(PyExc_ValueError, "%s must be positive", "group");
    return (K + group - 1) / group;
}

at::ScalarType real_type(const Args &a, int i) { return a.integer(i) == SQ_F32 ? at::kFloat : at::kBFloat16; }

// X, W4, s_w, group, z_w | None, bias | None, act, Y | None, type of a new Y -> (status, Y)
PyObject *w4_matvec(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded("w4_matvec", n, 9, [&]() -> PyObject * {
        const Args a{args};
        const at::Tensor &x = a.matrix(0);
        const sq_dtype dx = dtype_of(x);
        want_type(a.tensor(1), at::kByte, "Wq4");
        const Matrix X(x, "X"), W(a.matrix(1), "Wq4", -1, (X.cols + 1) / 2);
        const int64_t group = a.integer(3);
        const GroupScales sc(a, 2, 4, groups_of(X.cols, group), W.rows);
        const float *bias = f32_vector(a, 5, W.rows, "bias");
        const sq_act act = sq_act(a.integer(6));
        const at::Tensor y = a.none(7) ? new_rows(X.rows, W.rows, x, real_type(a, 8), 1) : a.tensor(7);
        const sq_dtype dy = dtype_of(y);
        const Matrix Y(y, "Y", X.rows, W.rows);
        void *stream = current_stream();
        const sq_status st = without_gil([&] {
            return segquant_w4_matvec(X.p, dx, X.rows, X.cols, X.ld, act, W.p, W.ld, W.rows, group, sc.s.p, sc.type, sc.s.ld,
                                      static_cast<const int8_t *>(sc.z.p), sc.z.ld, bias, Y.p, dy, Y.ld, stream);
        });
        return Py_BuildValue("(iN)", int(st), THPVariable_Wrap(y));
    });
}

// W, group, type of the scales, zero_points -> (status, W4, s_w, z_w | None)
PyObject *quantize_w4_group(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded("quantize_w4_group", n, 4, [&]() -> PyObject * {
        const Args a{args};
        const at::Tensor &w = a.matrix(0);
        const sq_dtype dw = dtype_of(w);
        const Matrix W(w, "W");
        const int64_t group = a.integer(1), groups = groups_of(W.cols, group), N = W.rows;
        const at::ScalarType ts = real_type(a, 2);
        const bool zp = a.truth(3);
        const at::Tensor q = new_rows(N, (W.cols + 1) / 2, w, at::kByte), s = new_rows(groups, N, w, ts);
        const at::Tensor z = zp ? new_rows(groups, N, w, at::kChar) : at::Tensor();
        const Rows Q(q), S(s);
        int8_t *zp_p = zp ? static_cast<int8_t *>(z.data_ptr()) : nullptr;
        const int64_t ldz = zp ? z.stride(0) : 0;
        void *stream = current_stream();
        const sq_status st = without_gil([&] {
            return segquant_quantize_w4_group(W.p, dw, N, W.cols, W.ld, group, Q.p, Q.ld, S.p, ts == at::kFloat ? SQ_F32 : SQ_BF16, S.ld, zp_p,
                                              ldz, stream);
        });
        return Py_BuildValue("(iNNN)", int(st), THPVariable_Wrap(q), THPVariable_Wrap(s), THPVariable_Wrap(z));
    });
}

// W4, s_w, group, K, z_w | None, W | None, type of a new W -> (status, W)
PyObject *dequantize_w4_group(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded("dequantize_w4_group", n, 7, [&]() -> PyObject * {
        const Args a{args};
        const at::Tensor &q = a.matrix(0);
        want_type(q, at::kByte, "Wq4");
        const int64_t group = a.integer(2), K = a.integer(3);
        const Matrix Q(q, "Wq4", -1, (K + 1) / 2);
        const GroupScales sc(a, 1, 4, groups_of(K, group), Q.rows);
        const at::Tensor w = a.none(5) ? new_rows(Q.rows, K, q, real_type(a, 6)) : a.tensor(5);
        const sq_dtype dw = dtype_of(w);
        const Matrix W(w, "W", Q.rows, K);
        void *stream = current_stream();
        const sq_status st = without_gil([&] {
            return segquant_dequantize_w4_group(Q.p, Q.ld, Q.rows, K, group, sc.s.p, sc.type, sc.s.ld, static_cast<const int8_t *>(sc.z.p),
                                                sc.z.ld, W.p, dw, W.ld, stream);
        });
        return Py_BuildValue("(iN)", int(st), THPVariable_Wrap(w));
    });
}

// The arguments that the two block norms share, 0 .. 14:
// R | None, Y | None, post, post_w, post_b, alpha, gate, pre, w, b, scale, shift, rows_per_sample | None, eps, H | None
struct BlockNorm {
    sq_block_norm norm{};
    sq_dtype dt;
    int64_t M, C;
    Matrix Y, R, H;
    at::Tensor h;
    bool any_vector = false;

    double number(const Args &a, int i)
    {
        const double v = PyFloat_AsDouble(a.a[i]);
        if (v == -1.0 && PyErr_Occurred()) throw BadArgument();
        return v;
    }
    // a vector over the channels, or one per sample (then [samples, C] or [C])
    const void *vector(const Args &a, int i, const char *what, int64_t samples, int64_t *ld)
    {
        if (a.none(i)) return nullptr;
        const at::Tensor &t = a.tensor(i);
        const sq_dtype type = dtype_of(t);
        if (any_vector && type != norm.p_dtype) refuse(PyExc_TypeError, "%s has another dtype than the vectors before it", what);
        any_vector = true;
        norm.p_dtype = type;
        const int64_t d = t.dim();
        if (d < 1 || d > 2 || (d == 2 && !ld) || t.size(d - 1) != C || (C > 1 && t.stride(d - 1) != 1)) refuse(PyExc_ValueError, "%s must be over the channels", what);
        if (d == 2 && t.size(0) != 1 && t.size(0) < samples) refuse(PyExc_ValueError, "%s has fewer rows than there are samples", what);
        if (ld) *ld = d == 2 && t.size(0) > 1 ? t.stride(0) : 0;
        return on_device(t, what).data_ptr();
    }
    explicit BlockNorm(const Args &a)
    {
        if (a.none(0) && a.none(1)) refuse(PyExc_ValueError, "%s", "R and Y are both missing");
        const at::Tensor &x = a.none(0) ? a.matrix(1) : a.matrix(0);
        dt = dtype_of(x);
        M = x.size(0), C = x.size(1);
        if (!a.none(0)) R = Matrix(x, "R");
        if (!a.none(1)) {
            want_type(a.tensor(1), x.scalar_type(), "Y");
            Y = Matrix(a.tensor(1), "Y", M, C);
        }
        int64_t T = M;
        if (!a.none(12)) T = a.integer(12);
        if (T < 1 && M > 0) refuse(PyExc_ValueError, "%s must be positive", "rows_per_sample");
        const int64_t samples = M > 0 ? (M + T - 1) / T : 0;
        norm.rows_per_sample = T;
        norm.post = sq_norm(a.integer(2));
        norm.post_w = vector(a, 3, "post_w", 1, nullptr);
        norm.post_b = vector(a, 4, "post_b", 1, nullptr);
        norm.alpha = float(number(a, 5));
        norm.gate = vector(a, 6, "gate", samples, &norm.ld_gate);
        norm.pre = sq_norm(a.integer(7));
        norm.w = vector(a, 8, "w", 1, nullptr);
        norm.b = vector(a, 9, "b", 1, nullptr);
        norm.scale = vector(a, 10, "scale", samples, &norm.ld_scale);
        norm.shift = vector(a, 11, "shift", samples, &norm.ld_shift);
        norm.eps = float(number(a, 13));
        if (!a.none(14)) {                               // H given: stored there
            h = a.tensor(14);
            want_type(h, x.scalar_type(), "H");
            H = Matrix(h, "H", M, C);
        } else if (!a.none(1)) {                         // a new one, where there is something to add
            h = new_rows(M, C, x, x.scalar_type());
            H = Matrix(h, "H");
        } else {
            h = x;                                       // h = r
        }
    }
};

// .., O | None, whether O is wanted -> (status, H, O | None)
PyObject *block_norm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded("block_norm", n, 17, [&]() -> PyObject * {
        const Args a{args};
        const BlockNorm b(a);
        const at::Tensor &x = a.none(0) ? a.matrix(1) : a.matrix(0);
        at::Tensor o;
        if (a.truth(16)) o = a.none(15) ? new_rows(b.M, b.C, x, x.scalar_type()) : a.tensor(15);
        Matrix O;
        if (o.defined()) {
            want_type(o, x.scalar_type(), "out");
            O = Matrix(o, "out", b.M, b.C);
        }
        void *stream = current_stream();
        const sq_status st = without_gil([&] {
            return segquant_block_norm(b.Y.p, b.Y.ld, b.R.p, b.R.ld, b.dt, b.M, b.C, &b.norm, b.H.p, b.H.ld, O.p, O.ld, stream);
        });
        return Py_BuildValue("(iNN)", int(st), THPVariable_Wrap(b.h), THPVariable_Wrap(o));
    });
}

// .., seg, P, s_pos, s_neg | None, code, flags, c_pos | None, c_neg | None -> (status, H, c_pos, c_neg | None)
PyObject *block_norm_quantize(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded("block_norm_quantize", n, 23, [&]() -> PyObject * {
        const Args a{args};
        const BlockNorm b(a);
        const at::Tensor &x = a.none(0) ? a.matrix(1) : a.matrix(0);
        const sq_segtable *seg = a.seg(15);
        const int64_t P = a.integer(16);
        const float *sp = f32_vector(a, 17, P, "s_pos"), *sn = f32_vector(a, 18, P, "s_neg");
        const sq_code code = sq_code(a.integer(19));
        const uint32_t flags = uint32_t(a.integer(20));
        const at::Tensor cp = a.none(21) ? new_rows(b.M, b.C, x, at::kByte, 128) : a.tensor(21);
        at::Tensor cn;
        if (sn) cn = a.none(22) ? new_rows(b.M, b.C, x, at::kByte, 128) : a.tensor(22);
        want_type(cp, at::kByte, "c_pos");
        const Matrix P1(cp, "c_pos", b.M, b.C);
        Matrix P2;
        if (cn.defined()) {
            want_type(cn, at::kByte, "c_neg");
            P2 = Matrix(cn, "c_neg", b.M, b.C);
            if (P2.ld != P1.ld) refuse(PyExc_ValueError, "%s must have the pitch of c_pos", "c_neg");
        }
        void *stream = current_stream();
        const sq_status st = without_gil([&] {
            return segquant_block_norm_quantize(b.Y.p, b.Y.ld, b.R.p, b.R.ld, b.dt, b.M, b.C, &b.norm, b.H.p, b.H.ld, seg, sp, sn, code, flags, P1.p,
                                                P2.p, P1.ld, stream);
        });
        return Py_BuildValue("(iNNN)", int(st), THPVariable_Wrap(b.h), THPVariable_Wrap(cp), THPVariable_Wrap(cn));
    });
}

// address of a plan
PyObject *plan_run(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded("plan_run", n, 1, [&] {
        const Args a{args};
        const sq_plan *plan = reinterpret_cast<const sq_plan *>(a.integer(0));
        void *stream = current_stream();
        return PyLong_FromLong(without_gil([&] { return segquant_plan_run(plan, stream); }));
    });
}

#define SQ_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SQ_METHOD(layer_forward), SQ_METHOD(quantize_act), SQ_METHOD(quantize_act_fused), SQ_METHOD(gemm),
                         SQ_METHOD(quantize_per_row), SQ_METHOD(calib_scales), SQ_METHOD(quantize_weight), SQ_METHOD(unpack_w4), SQ_METHOD(plan_run),
                         SQ_METHOD(w4_matvec), SQ_METHOD(quantize_w4_group), SQ_METHOD(dequantize_w4_group), SQ_METHOD(block_norm),
                         SQ_METHOD(block_norm_quantize), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module_def); }
