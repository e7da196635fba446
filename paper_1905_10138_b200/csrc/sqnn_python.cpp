// Argument marshalling of the device entry points for Python: torch tensors in, C ABI calls out.
//
// A small layer's kernels take 3 to 6 us, so what a call costs on the host decides how fast layers follow
// one another.  Marshalling the same arguments in Python through ctypes took 9 us (decode) to 12 us (product)
// per call; here it takes well under one, the rest is the kernel launch itself.
//
// The module holds no arithmetic and no state beyond the addresses of the C functions, which the Python
// side hands over once (so that an alternative build of the library can be loaded in its place).
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <numeric>

#include "sqnn.h"

namespace {

decltype(&sqnn_decode) f_decode = nullptr;
decltype(&sqnn_decode_matmul) f_matmul = nullptr;
decltype(&sqnn_decode_matmul_static) f_matmul_static = nullptr;
decltype(&sqnn_rmsnorm_fp8) f_rmsnorm_fp8 = nullptr;
decltype(&sqnn_fp8_matmul) f_fp8_matmul = nullptr;
decltype(&sqnn_moe_fp8) f_moe_fp8 = nullptr;

// The three functions of encrypted layers, and up to three of 8-bit ones (a function without an address cannot be called).
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    if (nargs < 3 || nargs > 6) { PyErr_SetString(PyExc_TypeError, "bind takes three to six addresses"); return nullptr; }
    void *p[6] = {};
    for (Py_ssize_t i = 0; i < nargs; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    f_decode = reinterpret_cast<decltype(f_decode)>(p[0]);
    f_matmul = reinterpret_cast<decltype(f_matmul)>(p[1]);
    f_matmul_static = reinterpret_cast<decltype(f_matmul_static)>(p[2]);
    f_rmsnorm_fp8 = reinterpret_cast<decltype(f_rmsnorm_fp8)>(p[3]);
    f_fp8_matmul = reinterpret_cast<decltype(f_fp8_matmul)>(p[4]);
    f_moe_fp8 = reinterpret_cast<decltype(f_moe_fp8)>(p[5]);
    Py_RETURN_NONE;
}

// The descriptor lives in a ctypes structure, which exports its memory through the buffer protocol.
struct DescArg {
    Py_buffer view{};
    bool held = false;
    const sqnn_desc *get(PyObject *o)
    {
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) return nullptr;
        held = true;
        if (view.len != (Py_ssize_t)sizeof(sqnn_desc)) {
            PyErr_SetString(PyExc_TypeError, "descriptor of the wrong size");
            return nullptr;
        }
        return static_cast<const sqnn_desc *>(view.buf);
    }
    ~DescArg() { if (held) PyBuffer_Release(&view); }
};

// A tensor argument; None stands for a null pointer.
bool tensor_arg(PyObject *o, const at::Tensor **t)
{
    if (o == Py_None) { *t = nullptr; return true; }
    if (!THPVariable_Check(o)) { PyErr_SetString(PyExc_TypeError, "expected a torch.Tensor or None"); return false; }
    *t = &THPVariable_Unpack(o);
    return true;
}
template <typename T>
T *ptr(const at::Tensor *t) { return t ? static_cast<T *>(t->data_ptr()) : nullptr; }
size_t bytes_of(const at::Tensor *t) { return t ? (size_t)t->numel() * t->element_size() : 0; }

// None = torch's current stream of the current device, else an object with a cuda_stream attribute.
bool stream_arg(PyObject *o, void **st)
{
    if (o == Py_None) { *st = c10::cuda::getCurrentCUDAStream().stream(); return true; }
    PyObject *a = PyObject_GetAttrString(o, "cuda_stream");
    if (!a) return false;
    *st = PyLong_AsVoidPtr(a);
    Py_DECREF(a);
    return !PyErr_Occurred();
}

bool enough(Py_ssize_t nargs, Py_ssize_t want)
{
    if (nargs == want) return true;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, nargs);
    return false;
}

// Other Python threads run while a C function is under way: a launch waits when the stream's queue is full, and in
// checked mode the call waits for its stream.  Everything a call needs has been read out of its Python
// arguments before; the caller's references keep them alive until it returns.
class Unlocked {
  public:
    Unlocked() : state_(PyEval_SaveThread()) {}
    ~Unlocked() { PyEval_RestoreThread(state_); }
    Unlocked(const Unlocked &) = delete;
    Unlocked &operator=(const Unlocked &) = delete;

  private:
    PyThreadState *state_;
};

// C++ exceptions of torch (a tensor without storage, for instance) must not cross into C.
template <typename F>
PyObject *guarded(F &&f)
{
    try {
        return f();
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// decode(desc, blob, mask, alpha, mode, out, status, stream) -> status code
PyObject *decode(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        if (!enough(nargs, 8)) return nullptr;
        DescArg desc;
        const sqnn_desc *d = desc.get(a[0]);
        const at::Tensor *blob, *mask, *alpha, *out, *status;
        void *st;
        if (!d || !tensor_arg(a[1], &blob) || !tensor_arg(a[2], &mask) || !tensor_arg(a[3], &alpha) ||
            !tensor_arg(a[5], &out) || !tensor_arg(a[6], &status) || !stream_arg(a[7], &st))
            return nullptr;
        const long mode = PyLong_AsLong(a[4]);
        if (mode == -1 && PyErr_Occurred()) return nullptr;
        void *const p_blob = ptr<void>(blob), *const p_out = ptr<void>(out);
        const uint64_t *const p_mask = ptr<uint64_t>(mask);
        const float *const p_alpha = ptr<float>(alpha);
        uint32_t *const p_status = ptr<uint32_t>(status);
        const size_t out_bytes = bytes_of(out);
        int rc;
        {
            Unlocked u;
            rc = f_decode(d, p_blob, p_mask, p_alpha, (sqnn_out_mode)mode, p_out, out_bytes, p_status, st);
        }
        return PyLong_FromLong(rc);
    });
}

bool product_shapes(const at::Tensor *x, const at::Tensor *y)
{
    if (x && y && x->dim() == 2 && y->dim() == 2 && x->stride(1) == 1 && y->stride(1) == 1) return true;
    PyErr_SetString(PyExc_ValueError, "X and Y must be 2-D with unit inner stride");
    return false;
}

// What both products take out of their tensors.
struct Operands {
    void *blob, *x;
    uint64_t *mask;
    float *alpha, *y;
    uint32_t *status;
    uint32_t batch;
    int64_t ldx, ldy;
    Operands(const at::Tensor *blob_, const at::Tensor *mask_, const at::Tensor *alpha_, const at::Tensor *x_, const at::Tensor *y_,
             const at::Tensor *status_)
        : blob(ptr<void>(blob_)), x(ptr<void>(x_)), mask(ptr<uint64_t>(mask_)), alpha(ptr<float>(alpha_)), y(ptr<float>(y_)),
          status(ptr<uint32_t>(status_)), batch((uint32_t)x_->size(0)), ldx(x_->stride(0)), ldy(y_->stride(0)) {}
};

// matmul(desc, blob, mask, alpha, x, y, workspace, status, stream) -> status code
PyObject *matmul(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        if (!enough(nargs, 9)) return nullptr;
        DescArg desc;
        const sqnn_desc *d = desc.get(a[0]);
        const at::Tensor *blob, *mask, *alpha, *x, *y, *ws, *status;
        void *st;
        if (!d || !tensor_arg(a[1], &blob) || !tensor_arg(a[2], &mask) || !tensor_arg(a[3], &alpha) ||
            !tensor_arg(a[4], &x) || !tensor_arg(a[5], &y) || !tensor_arg(a[6], &ws) || !tensor_arg(a[7], &status) ||
            !product_shapes(x, y))
            return nullptr;
        int xdt;
        if (x->scalar_type() == at::kFloat) xdt = SQNN_X_F32;
        else if (x->scalar_type() == at::kBFloat16) xdt = SQNN_X_BF16;
        else { PyErr_SetString(PyExc_ValueError, "X must be float32 or bfloat16"); return nullptr; }
        if (y->scalar_type() != at::kFloat) { PyErr_SetString(PyExc_ValueError, "Y must be float32"); return nullptr; }
        if (!stream_arg(a[8], &st)) return nullptr;
        const Operands o(blob, mask, alpha, x, y, status);
        void *const p_ws = ptr<void>(ws);
        const size_t ws_bytes = bytes_of(ws);
        int rc;
        {
            Unlocked u;
            rc = f_matmul(d, o.blob, o.mask, o.alpha, o.x, xdt, o.batch, o.ldx, o.y, o.ldy, p_ws, ws_bytes, o.status, st);
        }
        return PyLong_FromLong(rc);
    });
}

// matmul_static(desc, blob, mask, alpha, x, y, status, stream) -> status code
PyObject *matmul_static(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        if (!enough(nargs, 8)) return nullptr;
        DescArg desc;
        const sqnn_desc *d = desc.get(a[0]);
        const at::Tensor *blob, *mask, *alpha, *x, *y, *status;
        void *st;
        if (!d || !tensor_arg(a[1], &blob) || !tensor_arg(a[2], &mask) || !tensor_arg(a[3], &alpha) ||
            !tensor_arg(a[4], &x) || !tensor_arg(a[5], &y) || !tensor_arg(a[6], &status) || !product_shapes(x, y))
            return nullptr;
        if (x->scalar_type() != at::kBFloat16 || y->scalar_type() != at::kFloat) {
            PyErr_SetString(PyExc_ValueError, "X must be bfloat16 and Y float32");
            return nullptr;
        }
        if (!stream_arg(a[7], &st)) return nullptr;
        const Operands o(blob, mask, alpha, x, y, status);
        int rc;
        {
            Unlocked u;
            rc = f_matmul_static(d, o.blob, o.mask, o.alpha, o.x, SQNN_X_BF16, o.batch, o.ldx, o.y, o.ldy, o.status, st);
        }
        return PyLong_FromLong(rc);
    });
}

// ---- layers in 8-bit floating point.  Their tensors are checked here: where they are, their types and shapes.

bool fail(const char *what)
{
    PyErr_SetString(PyExc_ValueError, what);
    return false;
}
template <typename F>
bool bound(F f)
{
    if (f) return true;
    PyErr_SetString(PyExc_RuntimeError, "this function was not bound");
    return false;
}
bool on_device(const at::Tensor *t, const char *name)
{
    if (!t) return true;
    if (t->is_cuda() && t->get_device() == c10::cuda::current_device()) return true;
    PyErr_Format(PyExc_ValueError, "%s must be on the current CUDA device", name);
    return false;
}
// A matrix whose rows are contiguous; `rows` or `cols` < 0: any.
bool matrix(const at::Tensor *t, int64_t rows, int64_t cols, const char *name)
{
    if (!on_device(t, name)) return false;
    if (t->dim() == 2 && (rows < 0 || t->size(0) == rows) && (cols < 0 || t->size(1) == cols) && (t->size(1) == 1 || t->stride(1) == 1))
        return true;
    PyErr_Format(PyExc_ValueError, "%s must be a matrix of the right size with unit inner stride", name);
    return false;
}
// Row stride; the one row of a matrix has whatever torch says, so it gets one that suits every check.
int64_t row_stride(const at::Tensor *t) { return t->size(0) == 1 ? (t->size(1) + 15) / 16 * 16 : t->stride(0); }
bool real_type(const at::Tensor *t, int *dtype, const char *name)
{
    if (t->scalar_type() == at::kFloat) *dtype = SQNN_X_F32;
    else if (t->scalar_type() == at::kBFloat16) *dtype = SQNN_X_BF16;
    else {
        PyErr_Format(PyExc_ValueError, "%s must be float32 or bfloat16", name);
        return false;
    }
    return true;
}
bool of_type(const at::Tensor *t, at::ScalarType type, const char *name)
{
    if (t->scalar_type() == type) return true;
    PyErr_Format(PyExc_ValueError, "%s must be %s", name, at::toString(type));
    return false;
}
constexpr int64_t blocks_of(int64_t n) { return (n + SQNN_FP8_BLOCK - 1) / SQNN_FP8_BLOCK; }

// rmsnorm_fp8(x, weight, eps, q, scale, residual, h, y, stream) -> status code
PyObject *rmsnorm_fp8(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        if (!bound(f_rmsnorm_fp8) || !enough(nargs, 9)) return nullptr;
        const at::Tensor *x, *w, *q, *scale, *r, *h, *y;
        void *st;
        if (!tensor_arg(a[0], &x) || !tensor_arg(a[1], &w) || !tensor_arg(a[3], &q) || !tensor_arg(a[4], &scale) ||
            !tensor_arg(a[5], &r) || !tensor_arg(a[6], &h) || !tensor_arg(a[7], &y))
            return nullptr;
        const double eps = PyFloat_AsDouble(a[2]);
        if (eps == -1.0 && PyErr_Occurred()) return nullptr;
        if (!x || !w) { fail("x and weight are required"); return nullptr; }
        if (!matrix(x, -1, -1, "x")) return nullptr;
        const int64_t batch = x->size(0), n = x->size(1);
        int xt, wt, rt = SQNN_X_F32, yt = SQNN_X_F32;
        if (!real_type(x, &xt, "x") || !real_type(w, &wt, "weight") || !on_device(w, "weight")) return nullptr;
        if (w->dim() != 1 || w->size(0) != n || (n > 1 && w->stride(0) != 1)) { fail("weight must be a vector as long as a row of x"); return nullptr; }
        if (q && (!matrix(q, batch, n, "q") || !of_type(q, at::kFloat8_e4m3fn, "q"))) return nullptr;
        if (scale && (!matrix(scale, batch, blocks_of(n), "scale") || !of_type(scale, at::kFloat, "scale"))) return nullptr;
        if (r && (!matrix(r, batch, n, "residual") || !real_type(r, &rt, "residual"))) return nullptr;
        if (h && (!matrix(h, batch, n, "h") || !r || !of_type(h, r->scalar_type(), "h"))) {
            if (!PyErr_Occurred()) fail("h goes with a residual");
            return nullptr;
        }
        if (y && (!matrix(y, batch, n, "y") || !real_type(y, &yt, "y"))) return nullptr;
        if (batch > 0x7fffffff) { fail("too many rows"); return nullptr; }
        if (!stream_arg(a[8], &st)) return nullptr;
        const auto ld = [](const at::Tensor *t) { return t ? row_stride(t) : 0; };
        const void *const p_x = ptr<void>(x), *const p_r = ptr<void>(r), *const p_w = ptr<void>(w);
        void *const p_h = ptr<void>(h), *const p_y = ptr<void>(y);
        uint8_t *const p_q = ptr<uint8_t>(q);
        float *const p_s = ptr<float>(scale);
        const int64_t ldx = ld(x), ldr = ld(r), ldh = ld(h), ldq = ld(q), lds = ld(scale), ldy = ld(y);
        int rc;
        {
            Unlocked u;
            rc = f_rmsnorm_fp8((uint32_t)batch, (uint64_t)n, p_x, xt, ldx, p_r, rt, ldr, p_h, ldh, p_w, wt, eps, p_q, ldq, p_s, lds, p_y,
                               yt, ldy, st);
        }
        return PyLong_FromLong(rc);
    });
}

bool status_word(const at::Tensor *t)
{
    if (!t) return true;
    if (!on_device(t, "status")) return false;
    return (t->numel() == 1 && t->element_size() == 4) || fail("status must be one 32-bit word");
}

// fp8_matmul(w, w_scale, x, x_scale, y, status, stream) -> status code
PyObject *fp8_matmul(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        if (!bound(f_fp8_matmul) || !enough(nargs, 7)) return nullptr;
        const at::Tensor *w, *ws, *x, *xs, *y, *status;
        void *st;
        if (!tensor_arg(a[0], &w) || !tensor_arg(a[1], &ws) || !tensor_arg(a[2], &x) || !tensor_arg(a[3], &xs) || !tensor_arg(a[4], &y) ||
            !tensor_arg(a[5], &status))
            return nullptr;
        if (!w || !ws || !x || !xs || !y) { fail("weights, activations, their scales and Y are required"); return nullptr; }
        if (!matrix(w, -1, -1, "w")) return nullptr;
        const int64_t m = w->size(0), n = w->size(1);
        if (!matrix(x, -1, n, "x")) return nullptr;
        const int64_t batch = x->size(0);
        int yt;
        if (!matrix(ws, blocks_of(m), blocks_of(n), "w_scale") || !matrix(xs, batch, blocks_of(n), "x_scale") || !matrix(y, batch, m, "y") ||
            !of_type(w, at::kFloat8_e4m3fn, "w") || !of_type(x, at::kFloat8_e4m3fn, "x") || !of_type(ws, at::kFloat, "w_scale") ||
            !of_type(xs, at::kFloat, "x_scale") || !real_type(y, &yt, "y") || !status_word(status))
            return nullptr;
        if (batch > 0x7fffffff) { fail("too many rows"); return nullptr; }
        if (!stream_arg(a[6], &st)) return nullptr;
        const uint8_t *const p_w = ptr<uint8_t>(w), *const p_x = ptr<uint8_t>(x);
        const float *const p_ws = ptr<float>(ws), *const p_xs = ptr<float>(xs);
        void *const p_y = ptr<void>(y);
        uint32_t *const p_status = ptr<uint32_t>(status);
        const int64_t ldw = row_stride(w), ldws = row_stride(ws), ldx = row_stride(x), ldxs = row_stride(xs), ldy = row_stride(y);
        int rc;
        {
            Unlocked u;
            rc = f_fp8_matmul((uint64_t)m, (uint64_t)n, (uint32_t)batch, p_w, ldw, p_ws, ldws, p_x, ldx, p_xs, ldxs, p_y, yt, ldy, p_status, st);
        }
        return PyLong_FromLong(rc);
    });
}

// moe_fp8(x, router, top_k, renormalize, gate_up, gate_up_scale, down, down_scale, y, workspace, ids, probs, status, stream) -> status code
PyObject *moe_fp8(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        if (!bound(f_moe_fp8) || !enough(nargs, 14)) return nullptr;
        const at::Tensor *x, *router, *gu, *gus, *down, *downs, *y, *ws, *ids, *probs, *status;
        void *st;
        if (!tensor_arg(a[12], &status) || !tensor_arg(a[0], &x) || !tensor_arg(a[1], &router) || !tensor_arg(a[4], &gu) || !tensor_arg(a[5], &gus) || !tensor_arg(a[6], &down) ||
            !tensor_arg(a[7], &downs) || !tensor_arg(a[8], &y) || !tensor_arg(a[9], &ws) || !tensor_arg(a[10], &ids) || !tensor_arg(a[11], &probs))
            return nullptr;
        const long top_k = PyLong_AsLong(a[2]);
        if (top_k == -1 && PyErr_Occurred()) return nullptr;
        const int renormalize = PyObject_IsTrue(a[3]);
        if (renormalize < 0) return nullptr;
        if (!x || !router || !gu || !gus || !down || !downs || !y) { fail("x, router, weights, their scales and y are required"); return nullptr; }
        if (!matrix(x, -1, -1, "x")) return nullptr;
        const int64_t tokens = x->size(0), hidden = x->size(1);
        if (!matrix(router, -1, hidden, "router") || !matrix(y, tokens, hidden, "y")) return nullptr;
        const int64_t experts = router->size(0);
        int xt, rt, yt;
        if (!real_type(x, &xt, "x") || !real_type(router, &rt, "router") || !real_type(y, &yt, "y")) return nullptr;
        if (xt != rt) { fail("router must be of x's type"); return nullptr; }
        if (!on_device(gu, "gate_up") || !on_device(gus, "gate_up_scale") || !on_device(down, "down") || !on_device(downs, "down_scale") ||
            !on_device(ws, "workspace") || !on_device(ids, "ids") || !on_device(probs, "probs") || !of_type(gu, at::kFloat8_e4m3fn, "gate_up") ||
            !of_type(down, at::kFloat8_e4m3fn, "down") || !of_type(gus, at::kFloat, "gate_up_scale") || !of_type(downs, at::kFloat, "down_scale"))
            return nullptr;
        if (gu->dim() != 4 || gu->size(0) != experts || gu->size(1) != 2 || gu->size(3) != hidden || (hidden > 1 && gu->stride(3) != 1)) {
            fail("gate_up must be [experts, 2, inner, hidden] with unit inner stride");
            return nullptr;
        }
        const int64_t inner = gu->size(2);
        if (down->dim() != 3 || down->size(0) != experts || down->size(1) != hidden || down->size(2) != inner || (inner > 1 && down->stride(2) != 1)) {
            fail("down must be [experts, hidden, inner] with unit inner stride");
            return nullptr;
        }
        const int64_t gus_shape[4] = {experts, 2, blocks_of(inner), blocks_of(hidden)}, downs_shape[3] = {experts, blocks_of(hidden), blocks_of(inner)};
        if (gus->sizes() != at::IntArrayRef(gus_shape, 4) || !gus->is_contiguous() || downs->sizes() != at::IntArrayRef(downs_shape, 3) || !downs->is_contiguous()) {
            fail("scales must be contiguous, one per 128 x 128 block");
            return nullptr;
        }
        const int64_t pair_shape[2] = {tokens, top_k};
        if (ids && (ids->scalar_type() != at::kInt || ids->sizes() != at::IntArrayRef(pair_shape, 2) || !ids->is_contiguous())) {
            fail("ids must be contiguous int32 [tokens, top_k]");
            return nullptr;
        }
        if (probs && (probs->scalar_type() != at::kFloat || probs->sizes() != at::IntArrayRef(pair_shape, 2) || !probs->is_contiguous())) {
            fail("probs must be contiguous float32 [tokens, top_k]");
            return nullptr;
        }
        if (!status_word(status)) return nullptr;
        if (ws && !ws->is_contiguous()) { fail("workspace must be contiguous"); return nullptr; }
        const int64_t most = 1ll << 31;
        if (tokens >= most || experts >= most || top_k < 0 || top_k >= most || hidden >= most || inner >= most) { fail("too large"); return nullptr; }
        if (!stream_arg(a[13], &st)) return nullptr;
        // the stride of a dimension of one element is whatever torch says: 0 suits every check, and as a row's what the other strides are multiples of
        const auto stride = [](const at::Tensor *t, int64_t d, int64_t one) { return t->size(d) == 1 ? one : t->stride(d); };
        const auto row_of = [](int64_t half, int64_t expert, int64_t cols) {
            const int64_t common = std::gcd(half, expert);
            return common ? common : (cols + 15) / 16 * 16;
        };
        sqnn_moe L = {};
        L.experts = (uint32_t)experts; L.top_k = (uint32_t)top_k; L.hidden = (uint32_t)hidden; L.inner = (uint32_t)inner;
        L.renormalize = (uint32_t)renormalize;
        L.router = ptr<void>(router);
        L.gate_up = ptr<uint8_t>(gu); L.gate_up_scale = ptr<float>(gus);
        L.down = ptr<uint8_t>(down); L.down_scale = ptr<float>(downs);
        L.router_row = row_stride(router);
        L.gate_up_expert = stride(gu, 0, 0); L.gate_up_half = gu->stride(1); L.gate_up_row = stride(gu, 2, row_of(L.gate_up_half, L.gate_up_expert, hidden));
        L.down_expert = stride(down, 0, 0); L.down_row = stride(down, 1, row_of(0, L.down_expert, inner));
        const void *const p_x = ptr<void>(x);
        void *const p_y = ptr<void>(y), *const p_ws = ptr<void>(ws);
        int32_t *const p_ids = ptr<int32_t>(ids);
        float *const p_probs = ptr<float>(probs);
        uint32_t *const p_status = ptr<uint32_t>(status);
        const int64_t ldx = row_stride(x), ldy = row_stride(y);
        const size_t ws_bytes = bytes_of(ws);
        int rc;
        {
            Unlocked u;
            rc = f_moe_fp8(&L, (uint32_t)tokens, p_x, xt, ldx, p_y, yt, ldy, p_ids, p_probs, p_ws, ws_bytes, p_status, st);
        }
        return PyLong_FromLong(rc);
    });
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, "addresses of the C functions"},
    {"decode", (PyCFunction)(void (*)(void))decode, METH_FASTCALL, "sqnn_decode"},
    {"matmul", (PyCFunction)(void (*)(void))matmul, METH_FASTCALL, "sqnn_decode_matmul"},
    {"matmul_static", (PyCFunction)(void (*)(void))matmul_static, METH_FASTCALL, "sqnn_decode_matmul_static"},
    {"rmsnorm_fp8", (PyCFunction)(void (*)(void))rmsnorm_fp8, METH_FASTCALL, "sqnn_rmsnorm_fp8"},
    {"fp8_matmul", (PyCFunction)(void (*)(void))fp8_matmul, METH_FASTCALL, "sqnn_fp8_matmul"},
    {"moe_fp8", (PyCFunction)(void (*)(void))moe_fp8, METH_FASTCALL, "sqnn_moe_fp8"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_sqnn_python", "torch tensors to the C ABI of libsqnn", -1, methods,
                          nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__sqnn_python(void) { return PyModule_Create(&module_def); }
