// Argument marshalling of the layer operators for torch tensors: checks, outputs and workspace from torch's caching
// allocator, and the call of the C entry point.  No arithmetic.  A layer of a small model runs for a few microseconds, which is what the
// same checks take in Python, so they are made here.
#include "ssd_layers.h"

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <string>

namespace {

PyObject *g_error = nullptr;             // SsdError(status, where, detail)
PyObject *g_memory_error = nullptr;      // torch.OutOfMemoryError

struct Entry {
    ssd_status (*workspace)(const void *, int64_t *);
    ssd_status (*call)(const void *, void *, int64_t, void *);
};
Entry g_linear_forward, g_linear_backward, g_gated_forward, g_gated_backward;
ssd_status (*g_clip)(ssd_grad_list *, float, int32_t, float *, void *);
ssd_status (*g_norm)(ssd_grad_list *, float *, void *);
const char *(*g_cuda_error)(void);

struct Fail {
    int status;
    std::string what;
};

struct Mat {
    void *p;
    int64_t ld, rows, cols;
};

struct Call {
    const char *where;
    at::ScalarType dtype;
    c10::Device device;

    Call(const char *where_, PyObject *first) : where(where_), dtype(at::kFloat), device(c10::kCPU)
    {
        if (!THPVariable_Check(first)) throw Fail{SSD_ERR_ARG, "needs float32 or bfloat16 CUDA tensors"};
        const at::Tensor &t = THPVariable_Unpack(first);
        dtype = t.scalar_type();
        if (!t.is_cuda() || (dtype != at::kFloat && dtype != at::kBFloat16) || t.dim() < 1) throw Fail{SSD_ERR_ARG, "needs float32 or bfloat16 CUDA tensors"};
        device = t.device();
        if (device.index() != c10::cuda::current_device()) throw Fail{SSD_ERR_ARG, "the tensors' device is not the current one"};
    }
    int code() const { return code_of(dtype); }
    static int code_of(at::ScalarType t) { return t == at::kBFloat16 ? SSD_BF16 : SSD_F32; }
    void *stream() const { return c10::cuda::getCurrentCUDAStream(device.index()).stream(); }

    const at::Tensor &tensor(PyObject *o, const char *what) const
    {
        if (!THPVariable_Check(o)) throw Fail{SSD_ERR_ARG, std::string(what) + " is not a tensor"};
        return THPVariable_Unpack(o);
    }

    // A matrix, leading dimensions flattened to rows; cols, rows: what it has to have, or -1.
    Mat flat(const at::Tensor &t, int64_t cols, int64_t rows, const char *what, at::ScalarType type) const
    {
        if (t.scalar_type() != type || t.device() != device) throw Fail{SSD_ERR_ARG, std::string(what) + " has another type or device"};
        const int64_t d = t.dim();
        if (d < 1) throw Fail{SSD_ERR_ARG, std::string(what) + " has no dimension"};
        const auto size = t.sizes(), stride = t.strides();
        Mat m{nullptr, 0, 1, size[d - 1]};
        for (int64_t i = 0; i < d - 1; ++i) m.rows *= size[i];
        if ((cols >= 0 && m.cols != cols) || (rows >= 0 && m.rows != rows))
            throw Fail{SSD_ERR_ARG, std::string(what) + " is " + std::to_string(m.rows) + " x " + std::to_string(m.cols) + ", expected " +
                                        std::to_string(rows < 0 ? m.rows : rows) + " x " + std::to_string(cols < 0 ? m.cols : cols)};
        if (m.cols > 1 && stride[d - 1] != 1 && m.rows > 0) throw Fail{SSD_ERR_ARG, std::string("the last dimension of ") + what + " is not contiguous"};
        // the rows' pitch: that of the innermost leading dimension that has more than one row, which the outer ones must continue
        m.ld = m.cols;
        int64_t next = -1;
        for (int64_t i = d - 2; i >= 0 && m.rows > 1; --i) {
            if (size[i] == 1) continue;
            if (next < 0) m.ld = stride[i];
            else if (stride[i] != next) throw Fail{SSD_ERR_ARG, std::string("the leading dimensions of ") + what + " do not flatten to rows"};
            next = stride[i] * size[i];
        }
        if (m.rows > 1 && m.ld < m.cols) throw Fail{SSD_ERR_ARG, std::string("the rows of ") + what + " overlap"};
        m.p = t.data_ptr();
        return m;
    }
    Mat flat(PyObject *o, int64_t cols, int64_t rows, const char *what) const { return flat(tensor(o, what), cols, rows, what, dtype); }

    void *vector(PyObject *o, int64_t n, const char *what, at::ScalarType type) const
    {
        if (o == Py_None) return nullptr;
        const at::Tensor &t = tensor(o, what);
        if (t.scalar_type() != type || t.device() != device || t.dim() != 1 || t.size(0) != n || (n > 1 && t.stride(0) != 1))
            throw Fail{SSD_ERR_ARG, std::string(what) + " is not a contiguous vector of " + std::to_string(n) + " of the expected type on the tensors' device"};
        return t.data_ptr();
    }

    at::Tensor empty(at::IntArrayRef shape, at::ScalarType type) const { return at::detail::empty_cuda(shape, type, device, std::nullopt); }

    // The given output, or a new one where it is wanted; else none.
    at::Tensor output(PyObject *o, bool wanted, at::IntArrayRef shape, const char *what, at::ScalarType type) const
    {
        if (o != Py_None) return tensor(o, what);
        return wanted ? empty(shape, type) : at::Tensor();
    }

    void run(const Entry &e, const void *args, PyObject *given) const
    {
        void *at = nullptr;
        int64_t size = 0;
        at::Tensor room;
        if (given == Py_None) {
            check(e.workspace(args, &size));
            if (size) {
                room = empty({size}, at::kByte);
                at = room.data_ptr();
            }
        } else {
            const at::Tensor &t = tensor(given, "the workspace");
            if (t.device() != device || !t.is_contiguous()) throw Fail{SSD_ERR_ARG, "the workspace is not a contiguous tensor on the tensors' device"};
            at = t.data_ptr();
            size = int64_t(t.nbytes());
        }
        check(e.call(args, at, size, stream()));
    }
    static void check(ssd_status st)
    {
        if (st != SSD_OK) throw Fail{st, st == SSD_ERR_CUDA ? g_cuda_error() : ""};
    }
};

// x's shape with another last dimension.
c10::SmallVector<int64_t, 5> shape_like(const at::Tensor &x, int64_t cols)
{
    c10::SmallVector<int64_t, 5> s(x.sizes().begin(), x.sizes().end());
    s.back() = cols;
    return s;
}

PyObject *wrap(const at::Tensor &t)
{
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}

template <typename... T> PyObject *pack(const T &...t)
{
    PyObject *r = PyTuple_New(sizeof...(t));
    if (!r) return nullptr;
    Py_ssize_t i = 0;
    bool ok = true;
    auto put = [&](const at::Tensor &v) {
        PyObject *o = wrap(v);
        ok = ok && o;
        PyTuple_SET_ITEM(r, i++, o);
    };
    (put(t), ...);
    if (ok) return r;
    Py_DECREF(r);
    return nullptr;
}

int32_t as_int(PyObject *o)
{
    const long v = PyLong_AsLong(o);
    if ((v == -1 && PyErr_Occurred()) || v != int32_t(v)) {
        PyErr_Clear();
        throw Fail{SSD_ERR_ARG, "an integer of 32 bits is expected"};
    }
    return int32_t(v);
}

template <typename F> PyObject *guarded(const char *where, Py_ssize_t n, Py_ssize_t expected, F f)
{
    try {
        if (n != expected) throw Fail{SSD_ERR_ARG, "wrong number of arguments"};
        return f();
    } catch (const Fail &e) {
        PyObject *x = PyObject_CallFunction(g_error, "iss", e.status, where, e.what.c_str());
        if (x) {
            PyErr_SetObject(g_error, x);
            Py_DECREF(x);
        }
    } catch (const c10::OutOfMemoryError &e) {      // torch's allocator
        PyErr_SetString(g_memory_error, e.what_without_backtrace());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// The weight gradients' type: that of the first tensor given for one, else the code (-1: float32).
at::ScalarType grad_type(const Call &c, std::initializer_list<PyObject *> given, int32_t code)
{
    for (PyObject *o : given)
        if (o != Py_None) {
            const at::ScalarType t = c.tensor(o, "a weight gradient").scalar_type();
            if (t != at::kFloat && t != at::kBFloat16) throw Fail{SSD_ERR_ARG, "weight gradients are float32 or bfloat16"};
            return t;
        }
    return code == SSD_BF16 ? at::kBFloat16 : at::kFloat;
}

// (x, weight, y, bias, residual, z, act, keep, workspace)
PyObject *linear_forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded("ssd_linear_forward", n, 9, [&]() -> PyObject * {
        const Call c("ssd_linear_forward", a[0]);
        const at::Tensor &tx = THPVariable_Unpack(a[0]);
        const Mat x = c.flat(a[0], -1, -1, "x"), w = c.flat(a[1], x.cols, -1, "weight");
        const auto shape = shape_like(tx, w.rows);
        const at::Tensor y = c.output(a[2], true, shape, "y", c.dtype), z = c.output(a[5], a[7] == Py_True, shape, "z", c.dtype);
        ssd_linear_fwd s{x.rows, x.cols, w.rows, c.code(), as_int(a[6]), x.p, x.ld, w.p, w.ld};
        s.bias = static_cast<const float *>(c.vector(a[3], w.rows, "bias", at::kFloat));
        if (a[4] != Py_None) {
            const Mat r = c.flat(a[4], w.rows, x.rows, "residual");
            s.residual = r.p;
            s.ldr = r.ld;
        }
        const Mat my = c.flat(y, w.rows, x.rows, "y", c.dtype);
        s.y = my.p;
        s.ldy = my.ld;
        if (z.defined()) {
            const Mat mz = c.flat(z, w.rows, x.rows, "z", c.dtype);
            s.z = mz.p;
            s.ldz = mz.ld;
        }
        c.run(g_linear_forward, &s, a[8]);
        return pack(y, z);
    });
}

// (dy, x, weight, z, act, dx, dweight, dbias, grad code, want dx, want dweight, want dbias, workspace)
PyObject *linear_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded("ssd_linear_backward", n, 13, [&]() -> PyObject * {
        const Call c("ssd_linear_backward", a[0]);
        const Mat dy = c.flat(a[0], -1, -1, "dy"), w = c.flat(a[2], -1, dy.cols, "weight"), x = c.flat(a[1], w.cols, dy.rows, "x");
        const at::ScalarType g = grad_type(c, {a[6], a[7]}, as_int(a[8]));
        const at::Tensor dx = c.output(a[5], a[9] == Py_True, THPVariable_Unpack(a[1]).sizes(), "dx", c.dtype);
        const at::Tensor dw = c.output(a[6], a[10] == Py_True, {dy.cols, w.cols}, "dweight", g), db = c.output(a[7], a[11] == Py_True, {dy.cols}, "dbias", g);
        ssd_linear_bwd s{dy.rows, w.cols, dy.cols, c.code(), as_int(a[4]), Call::code_of(g), 0, dy.p, dy.ld, x.p, x.ld, w.p, w.ld};
        if (a[3] != Py_None) {
            const Mat z = c.flat(a[3], dy.cols, dy.rows, "z");
            s.z = z.p;
            s.ldz = z.ld;
        }
        if (dx.defined()) {
            const Mat m = c.flat(dx, w.cols, dy.rows, "dx", c.dtype);
            s.dx = m.p;
            s.lddx = m.ld;
        }
        if (dw.defined()) {
            const Mat m = c.flat(dw, w.cols, dy.cols, "dweight", g);
            s.dweight = m.p;
            s.lddw = m.ld;
        }
        if (db.defined()) {
            if (a[7] != Py_None) c.vector(a[7], dy.cols, "dbias", g);
            s.dbias = db.data_ptr();
        }
        c.run(g_linear_backward, &s, a[12]);
        return pack(dx, dw, db);
    });
}

// (x, w_gate, w_up, b_gate, b_up, h, gate, up, act, keep, workspace)
PyObject *gated_forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded("ssd_gated_forward", n, 11, [&]() -> PyObject * {
        const Call c("ssd_gated_forward", a[0]);
        const at::Tensor &tx = THPVariable_Unpack(a[0]);
        const Mat x = c.flat(a[0], -1, -1, "x"), g = c.flat(a[1], x.cols, -1, "w_gate"), u = c.flat(a[2], x.cols, g.rows, "w_up");
        const auto shape = shape_like(tx, g.rows);
        const bool keep = a[9] == Py_True;
        const at::Tensor h = c.output(a[5], true, shape, "h", c.dtype), gate = c.output(a[6], keep, shape, "gate", c.dtype), up = c.output(a[7], keep, shape, "up", c.dtype);
        ssd_gated_fwd s{x.rows, x.cols, g.rows, c.code(), as_int(a[8]), x.p, x.ld, g.p, g.ld, u.p, u.ld};
        s.b_gate = static_cast<const float *>(c.vector(a[3], g.rows, "b_gate", at::kFloat));
        s.b_up = static_cast<const float *>(c.vector(a[4], g.rows, "b_up", at::kFloat));
        const Mat mh = c.flat(h, g.rows, x.rows, "h", c.dtype);
        s.h = mh.p;
        s.ldh = mh.ld;
        if (gate.defined()) {
            const Mat m = c.flat(gate, g.rows, x.rows, "gate", c.dtype);
            s.gate = m.p;
            s.ldgate = m.ld;
        }
        if (up.defined()) {
            const Mat m = c.flat(up, g.rows, x.rows, "up", c.dtype);
            s.up = m.p;
            s.ldup = m.ld;
        }
        c.run(g_gated_forward, &s, a[10]);
        return pack(h, gate, up);
    });
}

// (dh, x, w_gate, w_up, gate, up, act, dx, dw_gate, dw_up, db_gate, db_up, grad code, want dx, want dweight, want dbias, workspace)
PyObject *gated_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded("ssd_gated_backward", n, 17, [&]() -> PyObject * {
        const Call c("ssd_gated_backward", a[0]);
        const Mat dh = c.flat(a[0], -1, -1, "dh"), wg = c.flat(a[2], -1, dh.cols, "w_gate"), wu = c.flat(a[3], wg.cols, dh.cols, "w_up");
        const Mat x = c.flat(a[1], wg.cols, dh.rows, "x"), gate = c.flat(a[4], dh.cols, dh.rows, "gate"), up = c.flat(a[5], dh.cols, dh.rows, "up");
        const at::ScalarType g = grad_type(c, {a[8], a[9], a[10], a[11]}, as_int(a[12]));
        const bool want_dw = a[14] == Py_True, want_db = a[15] == Py_True;
        const at::Tensor dx = c.output(a[7], a[13] == Py_True, THPVariable_Unpack(a[1]).sizes(), "dx", c.dtype);
        const at::Tensor dwg = c.output(a[8], want_dw, {dh.cols, wg.cols}, "dw_gate", g), dwu = c.output(a[9], want_dw, {dh.cols, wg.cols}, "dw_up", g);
        const at::Tensor dbg = c.output(a[10], want_db, {dh.cols}, "db_gate", g), dbu = c.output(a[11], want_db, {dh.cols}, "db_up", g);
        ssd_gated_bwd s{dh.rows, wg.cols, dh.cols, c.code(), as_int(a[6]), Call::code_of(g), 0, dh.p, dh.ld, x.p, x.ld,
                        wg.p, wg.ld, wu.p, wu.ld, gate.p, gate.ld, up.p, up.ld};
        if (dx.defined()) {
            const Mat m = c.flat(dx, wg.cols, dh.rows, "dx", c.dtype);
            s.dx = m.p;
            s.lddx = m.ld;
        }
        if (dwg.defined()) {
            const Mat m = c.flat(dwg, wg.cols, dh.cols, "dw_gate", g);
            s.dw_gate = m.p;
            s.lddwg = m.ld;
        }
        if (dwu.defined()) {
            const Mat m = c.flat(dwu, wg.cols, dh.cols, "dw_up", g);
            s.dw_up = m.p;
            s.lddwu = m.ld;
        }
        if (a[10] != Py_None) c.vector(a[10], dh.cols, "db_gate", g);
        if (a[11] != Py_None) c.vector(a[11], dh.cols, "db_up", g);
        s.db_gate = dbg.defined() ? dbg.data_ptr() : nullptr;
        s.db_up = dbu.defined() ? dbu.data_ptr() : nullptr;
        c.run(g_gated_backward, &s, a[16]);
        return pack(dx, dwg, dwu, dbg, dbu);
    });
}

// (list address, device index, groups, max_norm or None for the norms alone, nonfinite, norms, table, the stream that the table is memory of)
PyObject *clip(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    const bool scale = n == 8 && a[3] != Py_None;
    return guarded(scale ? "ssd_clip_grad_norm" : "ssd_grad_norm", n, 8, [&]() -> PyObject * {
        ssd_grad_list *list = static_cast<ssd_grad_list *>(PyLong_AsVoidPtr(a[0]));
        const c10::Device device(c10::kCUDA, c10::DeviceIndex(as_int(a[1])));
        const int64_t groups = as_int(a[2]);
        if (device.index() != c10::cuda::current_device()) throw Fail{SSD_ERR_ARG, "the gradients' device is not the current one"};
        at::Tensor norms;
        if (a[5] == Py_None) {
            norms = at::detail::empty_cuda({groups}, at::kFloat, device, std::nullopt);
        } else {
            if (!THPVariable_Check(a[5])) throw Fail{SSD_ERR_ARG, "norms is not a tensor"};
            norms = THPVariable_Unpack(a[5]);
            if (norms.scalar_type() != at::kFloat || norms.device() != device || norms.numel() != groups || !norms.is_contiguous())
                throw Fail{SSD_ERR_ARG, "norms is not a contiguous float32 tensor with one value per group on the gradients' device"};
        }
        const c10::cuda::CUDAStream current = c10::cuda::getCurrentCUDAStream(device.index());
        void *stream = current.stream();
        // on another stream than its own, the table's memory stays taken until this call is done there
        if (stream != PyLong_AsVoidPtr(a[7]) && list) {
            if (!THPVariable_Check(a[6])) throw Fail{SSD_ERR_ARG, "the list has no table"};
            c10::cuda::CUDACachingAllocator::recordStream(THPVariable_Unpack(a[6]).storage().data_ptr(), current);
        }
        float *out = static_cast<float *>(norms.data_ptr());
        if (scale) {
            const double limit = PyFloat_AsDouble(a[3]);
            if (PyErr_Occurred()) {
                PyErr_Clear();
                throw Fail{SSD_ERR_ARG, "max_norm is not a number"};
            }
            Call::check(g_clip(list, float(limit), as_int(a[4]), out, stream));
        } else {
            Call::check(g_norm(list, out, stream));
        }
        return wrap(norms);
    });
}

// (SsdError, {entry point: address}, torch.OutOfMemoryError)
PyObject *setup(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 3 || !PyDict_Check(a[1])) {
        PyErr_SetString(PyExc_TypeError, "setup(error class, {name: address}, class of the allocator's error)");
        return nullptr;
    }
    bool ok = true;
    auto at = [&](const std::string &name) -> void * {
        PyObject *o = PyDict_GetItemString(a[1], name.c_str());
        ok = ok && o;
        return o ? PyLong_AsVoidPtr(o) : nullptr;
    };
    auto entry = [&](const std::string &name) {
        return Entry{reinterpret_cast<decltype(Entry::workspace)>(at("ssd_" + name + "_workspace")), reinterpret_cast<decltype(Entry::call)>(at("ssd_" + name))};
    };
    g_linear_forward = entry("linear_forward");
    g_linear_backward = entry("linear_backward");
    g_gated_forward = entry("gated_forward");
    g_gated_backward = entry("gated_backward");
    g_clip = reinterpret_cast<decltype(g_clip)>(at("ssd_clip_grad_norm"));
    g_norm = reinterpret_cast<decltype(g_norm)>(at("ssd_grad_norm"));
    g_cuda_error = reinterpret_cast<decltype(g_cuda_error)>(at("ssd_layer_cuda_error"));
    if (!ok || PyErr_Occurred()) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_KeyError, "an entry point is missing");
        return nullptr;
    }
    Py_INCREF(a[0]);
    Py_XDECREF(g_error);
    g_error = a[0];
    Py_INCREF(a[2]);
    Py_XDECREF(g_memory_error);
    g_memory_error = a[2];
    Py_RETURN_NONE;
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {FAST(setup), FAST(linear_forward), FAST(linear_backward), FAST(gated_forward), FAST(gated_backward), FAST(clip), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_ssd_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ssd_torch(void) { return PyModule_Create(&g_module); }
