// Python module _block: the operators next to the adapters, called with torch tensors.
//
// Marshalling only, like the ctypes binding of the other entry points: shapes, types, devices and pitches are
// looked at, outputs and workspaces that the caller did not bring are made, and the C ABI is called.  It is
// native because these calls stand between kernels of a few microseconds: through ctypes a call took 9 - 32 us
// on the host, three quarters of it Python looking at tensors.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/core/grad_mode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <dlfcn.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <optional>
#include <string>

#include "lordba.h"

namespace {

// The entry points of the library that bind() opened.
struct Library {
    decltype(&lordba_int8_quantize_rows) quantize;
    decltype(&lordba_int8_linear_workspace_bytes) linear_bytes;
    decltype(&lordba_int8_linear) linear;
    decltype(&lordba_gated_workspace_bytes) gated_bytes;
    decltype(&lordba_gated_forward) gated;
    decltype(&lordba_gated_backward_workspace_bytes) grad_bytes;
    decltype(&lordba_gated_backward) grad;
    decltype(&lordba_dropout) dropout;
};
Library lib = {};
PyObject *status_error = nullptr;      // LordbaError

// An error on its way to Python: of a type with a message, or a status of the library.
struct Refusal {
    PyObject *type;
    std::string message;
    int status = 0;
};
[[noreturn]] void type_error(const std::string &m) { throw Refusal{PyExc_TypeError, m}; }
[[noreturn]] void value_error(const std::string &m) { throw Refusal{PyExc_ValueError, m}; }
void check(int status, const char *where)
{
    if (status != LORDBA_OK) throw Refusal{status_error, where, status};
}

using at::Tensor;

// The calls record no graph: as torch's own functions with an output argument, they refuse a tensor that asks for a
// gradient while gradients are recorded, rather than lose it.
const Tensor &tensor(PyObject *o, const char *what)
{
    if (!THPVariable_Check(o)) type_error(std::string(what) + " must be a tensor");
    const Tensor &t = THPVariable_Unpack(o);
    if (t.requires_grad() && at::GradMode::is_enabled())
        throw Refusal{PyExc_RuntimeError, std::string(what) + " requires a gradient, and this call records none: make it under "
                                              "torch.no_grad(), in a torch.autograd.Function, or on detached tensors"};
    return t;
}
std::optional<Tensor> optional_tensor(PyObject *o, const char *what)
{
    if (o == Py_None) return std::nullopt;
    return tensor(o, what);
}

at::ScalarType dtype_of(PyObject *o)
{
    if (!THPDtype_Check(o)) type_error("dtype must be a torch.dtype");
    return reinterpret_cast<THPDtype *>(o)->scalar_type;
}

std::string name_of(at::ScalarType t) { return c10::toString(t); }

int code_of(at::ScalarType t, const char *what)
{
    switch (t) {
        case at::kFloat: return LORDBA_F32;
        case at::kBFloat16: return LORDBA_BF16;
        case at::kHalf: return LORDBA_F16;
        default: type_error(std::string(what) + " must be float32, bfloat16 or float16, got " + name_of(t));
    }
}

// What a call runs on: the current device, and the stream given or its current one.
struct Where {
    c10::DeviceIndex device;
    std::optional<c10::cuda::CUDAStream> given;
    void *stream;

    explicit Where(PyObject *s)
    {
        device = c10::cuda::current_device();
        if (s == Py_None) {
            stream = c10::cuda::getCurrentCUDAStream(device).stream();
            return;
        }
        int64_t v[3];
        const char *names[3] = {"stream_id", "device_index", "device_type"};
        for (int i = 0; i < 3; ++i) {
            PyObject *a = PyObject_GetAttrString(s, names[i]);
            if (!a) throw python_error();
            v[i] = PyLong_AsLongLong(a);
            Py_DECREF(a);
            if (v[i] == -1 && PyErr_Occurred()) throw python_error();
        }
        given = c10::cuda::CUDAStream::unpack3(v[0], (c10::DeviceIndex)v[1], (c10::DeviceType)v[2]);
        if (given->device_index() != device) value_error("the stream must be one of the current CUDA device");
        stream = given->stream();
    }

    // A new matrix whose rows start on 16-byte boundaries (what the copy engine takes).  It belongs to the call's
    // stream: its memory is free for that stream's work.
    Tensor rows(int64_t r, int64_t c, at::ScalarType t) const
    {
        const int64_t step = 16 / (int64_t)c10::elementSize(t);
        return make({r, c}, {(c + step - 1) / step * step, 1}, t);
    }
    Tensor values(int64_t n, at::ScalarType t) const { return make({n}, {1}, t); }

private:
    Tensor make(at::IntArrayRef size, at::IntArrayRef stride, at::ScalarType t) const
    {
        const auto options = at::TensorOptions().dtype(t).device(at::kCUDA, device);
        if (!given) return at::empty_strided(size, stride, options);
        c10::cuda::CUDAStreamGuard guard(*given);
        return at::empty_strided(size, stride, options);
    }
};

void check_device(const Tensor &t, const Where &at, const char *what)
{
    if (!t.is_cuda() || t.get_device() != at.device) value_error(std::string(what) + " must be on the current CUDA device");
}

void check_matrix(const Tensor &t, const char *what)
{
    if (t.dim() != 2) value_error(std::string(what) + " must have two dimensions");
}

// Check a matrix with contiguous rows; its row pitch in elements.
int64_t pitch(const Tensor &t, int64_t rows, int64_t cols, at::ScalarType type, const Where &at, const char *what)
{
    if (t.scalar_type() != type) type_error(std::string(what) + " must be " + name_of(type) + ", got " + name_of(t.scalar_type()));
    check_device(t, at, what);
    if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols)
        value_error(std::string(what) + " must be (" + std::to_string(rows) + ", " + std::to_string(cols) + ")");
    const int64_t ld = t.stride(0);
    if (t.stride(1) != 1 && cols > 1) value_error(std::string("rows of ") + what + " must be contiguous");
    if (rows <= 1) return ld > cols ? ld : cols;          // a single row has no pitch of its own
    if (ld < cols) value_error(std::string("rows of ") + what + " overlap");
    return ld;
}

// The pitch that both matrices of a pair have.
int64_t pitch_of_pair(const std::optional<Tensor> &a, const std::optional<Tensor> &b, int64_t rows, int64_t cols, at::ScalarType type,
                      const Where &at, const char *what)
{
    if (!a || !b) value_error(std::string(what) + " come together");
    const int64_t ld = pitch(*a, rows, cols, type, at, what);
    if (pitch(*b, rows, cols, type, at, what) != ld && rows > 1) value_error(std::string(what) + " must have one row pitch");
    return ld;
}

const float *vector(const Tensor &t, int64_t n, const Where &at, const char *what)
{
    check_device(t, at, what);
    if (t.scalar_type() != at::kFloat || t.numel() != n || !t.is_contiguous())
        type_error(std::string(what) + " must be " + std::to_string(n) + " contiguous float32 values");
    return static_cast<const float *>(t.data_ptr());
}

struct Workspace {
    Tensor made;
    void *p = nullptr;
    size_t bytes = 0;
    Workspace(size_t need, PyObject *given, const Where &at)
    {
        if (given != Py_None) {
            const Tensor &t = tensor(given, "workspace");
            check_device(t, at, "workspace");
            p = t.data_ptr();
            bytes = t.nbytes();
        } else if (need) {
            made = at.values((int64_t)need, at::kByte);
            p = made.data_ptr();
            bytes = need;
        }
    }
};

// Autograd's note that a tensor was written, for the caller's own ones (those made here have not been seen by it).
void written(PyObject *o)
{
    if (o == Py_None) return;
    const Tensor &t = THPVariable_Unpack(o);
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

void *data(const std::optional<Tensor> &t) { return t ? t->data_ptr() : nullptr; }

int64_t integer(PyObject *o)
{
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}
uint64_t low64(PyObject *o)
{
    const uint64_t v = PyLong_AsUnsignedLongLongMask(o);
    if (v == (uint64_t)-1 && PyErr_Occurred()) throw python_error();
    return v;
}

PyObject *wrapped(const std::optional<Tensor> &t)
{
    if (t) return THPVariable_Wrap(*t);
    Py_RETURN_NONE;
}
template <typename... T>
PyObject *tuple_of(const T &...t)
{
    PyObject *items[] = {wrapped(t)...};
    constexpr Py_ssize_t n = sizeof...(T);
    PyObject *r = PyTuple_New(n);
    bool good = r != nullptr;
    for (PyObject *i : items) good = good && i;
    for (Py_ssize_t i = 0; i < n; ++i) {
        if (good) PyTuple_SET_ITEM(r, i, items[i]);
        else Py_XDECREF(items[i]);
    }
    if (!good) Py_CLEAR(r);
    return r;
}

// ---- the calls; arguments by position, as lordba.py passes them -------------------------------------------------

PyObject *int8_quantize_rows(PyObject *const *a)
{
    const Tensor &x = tensor(a[0], "x");
    std::optional<Tensor> q = optional_tensor(a[1], "q"), scale = optional_tensor(a[2], "scale");
    const Where at(a[3]);
    check_matrix(x, "x");
    const int64_t T = x.size(0), d = x.size(1);
    const int dtype = code_of(x.scalar_type(), "x");
    const int64_t ldx = pitch(x, T, d, x.scalar_type(), at, "x");
    if (!q) q = at.rows(T, d, at::kChar);
    if (!scale) scale = at.values(T, at::kFloat);
    const int64_t ldq = pitch(*q, T, d, at::kChar, at, "q");
    vector(*scale, T, at, "scale");
    check(lib.quantize(x.data_ptr(), ldx, static_cast<int8_t *>(q->data_ptr()), ldq, static_cast<float *>(scale->data_ptr()), T, d,
                       dtype, at.stream), "lordba_int8_quantize_rows");
    for (int i : {1, 2}) written(a[i]);
    return tuple_of(q, scale);
}

PyObject *int8_linear(PyObject *const *a)
{
    const Tensor &x = tensor(a[0], "x"), &s_x = tensor(a[1], "s_x"), &w = tensor(a[2], "w"), &s_w = tensor(a[3], "s_w");
    std::optional<Tensor> y = optional_tensor(a[4], "y");
    const at::ScalarType wanted = dtype_of(a[5]);
    const Where at(a[7]);
    check_matrix(x, "x");
    check_matrix(w, "w");
    const int64_t T = x.size(0), d_in = x.size(1), d_out = w.size(0);
    const at::ScalarType type = y ? y->scalar_type() : wanted;
    const int code = code_of(type, "y");
    lordba_int8_proj p = {};
    p.d_in = d_in; p.d_out = d_out;
    p.s_x = vector(s_x, T, at, "s_x");
    p.s_w = vector(s_w, d_out, at, "s_w");
    p.ldx = pitch(x, T, d_in, at::kChar, at, "x");
    p.ldw = pitch(w, d_out, d_in, at::kChar, at, "w");
    if (!y) y = at.rows(T, d_out, type);
    p.ldy = pitch(*y, T, d_out, type, at, "y");
    p.x = static_cast<const int8_t *>(x.data_ptr());
    p.w = static_cast<const int8_t *>(w.data_ptr());
    p.y = y->data_ptr();
    const Workspace ws(lib.linear_bytes(&p, T), a[6], at);
    check(lib.linear(&p, T, code, ws.p, ws.bytes, at.stream), "lordba_int8_linear");
    written(a[4]);
    return wrapped(y);
}

PyObject *gated_forward(PyObject *const *a)
{
    const Tensor &x = tensor(a[0], "x"), &w_gate = tensor(a[1], "w_gate"), &w_up = tensor(a[2], "w_up");
    std::optional<Tensor> h = optional_tensor(a[3], "h"), gate_add = optional_tensor(a[7], "gate_add"), up_add = optional_tensor(a[8], "up_add"),
                          gate = optional_tensor(a[9], "gate"), up = optional_tensor(a[10], "up");
    const int save = PyObject_IsTrue(a[11]);
    if (save < 0) throw python_error();
    const Where at(a[13]);
    check_matrix(x, "x");
    check_matrix(w_gate, "w_gate");
    const int64_t T = x.size(0), d_in = x.size(1), n = w_gate.size(0);
    const at::ScalarType kind = x.scalar_type();
    at::ScalarType type = kind;
    lordba_gated g = {};
    if ((kind == at::kChar) != (a[5] != Py_None)) value_error("int8 operands come with scales = (s_x, s_gate, s_up), others without");
    if (kind == at::kChar) {
        if (!PyTuple_Check(a[5]) || PyTuple_GET_SIZE(a[5]) != 3) type_error("scales must be a tuple (s_x, s_gate, s_up)");
        g.s_x = vector(tensor(PyTuple_GET_ITEM(a[5], 0), "s_x"), T, at, "s_x");
        g.s_gate = vector(tensor(PyTuple_GET_ITEM(a[5], 1), "s_gate"), n, at, "s_gate");
        g.s_up = vector(tensor(PyTuple_GET_ITEM(a[5], 2), "s_up"), n, at, "s_up");
        g.flags = LORDBA_GATED_INT8;
        type = h ? h->scalar_type() : a[6] != Py_None ? dtype_of(a[6]) : at::kBFloat16;
    }
    if (a[6] != Py_None && dtype_of(a[6]) != type)
        type_error("dtype is " + name_of(dtype_of(a[6])) + ", but h is " + name_of(type) + (h ? "" : ", like x"));
    const int code = code_of(type, "h");
    g.d_in = d_in; g.d_hidden = n;
    g.act = (int32_t)integer(a[4]);
    g.ldx = pitch(x, T, d_in, kind, at, "x");
    g.ldw = pitch_of_pair(w_gate, w_up, n, d_in, kind, at, "w_gate and w_up");
    if (!h) h = at.rows(T, n, type);
    g.ldh = pitch(*h, T, n, type, at, "h");
    if (gate_add || up_add) g.ld_add = pitch_of_pair(gate_add, up_add, T, n, type, at, "gate_add and up_add");
    if (save && !gate && !up) {
        gate = at.rows(T, n, type);
        up = at.rows(T, n, type);
    }
    if (gate || up) g.ld_pre = pitch_of_pair(gate, up, T, n, type, at, "gate and up");
    g.x = x.data_ptr(); g.w_gate = w_gate.data_ptr(); g.w_up = w_up.data_ptr();
    g.gate_add = data(gate_add); g.up_add = data(up_add); g.gate = data(gate); g.up = data(up); g.h = h->data_ptr();
    const Workspace ws(lib.gated_bytes(&g, T), a[12], at);
    check(lib.gated(&g, T, code, ws.p, ws.bytes, at.stream), "lordba_gated_forward");
    for (int i : {3, 9, 10}) written(a[i]);
    return tuple_of(h, gate, up);
}

PyObject *gated_backward(PyObject *const *a)
{
    const Tensor &dh = tensor(a[0], "dh");
    const std::optional<Tensor> gate = optional_tensor(a[1], "gate"), up = optional_tensor(a[2], "up"), x = optional_tensor(a[3], "x"),
                                w_gate = optional_tensor(a[4], "w_gate"), w_up = optional_tensor(a[5], "w_up");
    std::optional<Tensor> dgate = optional_tensor(a[6], "dgate"), dup = optional_tensor(a[7], "dup"), dx = optional_tensor(a[8], "dx"),
                          dw_gate = optional_tensor(a[9], "dw_gate"), dw_up = optional_tensor(a[10], "dw_up");
    const Where at(a[13]);
    check_matrix(dh, "dh");
    const int64_t T = dh.size(0), n = dh.size(1);
    const at::ScalarType type = dh.scalar_type();
    const int code = code_of(type, "dh");
    lordba_gated_grad g = {};
    g.act = (int32_t)integer(a[11]);
    g.ld_dh = pitch(dh, T, n, type, at, "dh");
    g.ld_pre = pitch_of_pair(gate, up, T, n, type, at, "gate and up");
    if (!dgate && !dup) {
        dgate = at.rows(T, n, type);
        dup = at.rows(T, n, type);
    }
    g.ld_dpre = pitch_of_pair(dgate, dup, T, n, type, at, "dgate and dup");
    int64_t d_in = 1;
    if (w_gate || w_up) {
        if (!w_gate || !w_up) value_error("w_gate and w_up come together");
        check_matrix(*w_gate, "w_gate");
        d_in = w_gate->size(1);
        g.ldw = pitch_of_pair(w_gate, w_up, n, d_in, type, at, "w_gate and w_up");
        if (!dx) dx = at.rows(T, d_in, type);
        g.ld_dx = pitch(*dx, T, d_in, type, at, "dx");
    } else if (dx) {
        value_error("dx needs w_gate and w_up");
    }
    if (x) {
        check_matrix(*x, "x");
        if (w_gate && x->size(1) != d_in) value_error("x must have the width of w_gate and w_up");
        d_in = x->size(1);
        g.ldx = pitch(*x, T, d_in, type, at, "x");
        if (!dw_gate && !dw_up) {
            dw_gate = at.rows(n, d_in, type);
            dw_up = at.rows(n, d_in, type);
        }
        g.ld_dw = pitch_of_pair(dw_gate, dw_up, n, d_in, type, at, "dw_gate and dw_up");
    } else if (dw_gate || dw_up) {
        value_error("dw_gate and dw_up need x");
    }
    g.d_in = d_in; g.d_hidden = n;
    g.dh = dh.data_ptr(); g.gate = data(gate); g.up = data(up); g.x = data(x); g.w_gate = data(w_gate); g.w_up = data(w_up);
    g.dgate = data(dgate); g.dup = data(dup); g.dx = data(dx); g.dw_gate = data(dw_gate); g.dw_up = data(dw_up);
    const Workspace ws(lib.grad_bytes(&g, T), a[12], at);
    check(lib.grad(&g, T, code, ws.p, ws.bytes, at.stream), "lordba_gated_backward");
    for (int i : {6, 7, 8, 9, 10}) written(a[i]);
    return tuple_of(dgate, dup, dx, dw_gate, dw_up);
}

PyObject *dropout(PyObject *const *a)
{
    const Tensor &x = tensor(a[0], "x");
    const double p = PyFloat_AsDouble(a[1]);
    if (p == -1.0 && PyErr_Occurred()) throw python_error();
    const uint64_t seed = low64(a[2]), offset = low64(a[3]);
    const std::optional<Tensor> residual = optional_tensor(a[4], "residual");
    std::optional<Tensor> out = optional_tensor(a[5], "out");
    const Where at(a[6]);
    check_matrix(x, "x");
    const int64_t T = x.size(0), d = x.size(1);
    const at::ScalarType type = x.scalar_type();
    const int code = code_of(type, "x");
    const int64_t ldx = pitch(x, T, d, type, at, "x"), ldr = residual ? pitch(*residual, T, d, type, at, "residual") : 0;
    if (!out) out = at.rows(T, d, type);
    const int64_t ldo = pitch(*out, T, d, type, at, "out");
    check(lib.dropout(x.data_ptr(), ldx, data(residual), ldr, out->data_ptr(), ldo, T, d, (float)p, seed, offset, code, at.stream),
          "lordba_dropout");
    written(a[5]);
    return wrapped(out);
}

// bind(path, LordbaError): take the entry points from a build of the library.
PyObject *bind(PyObject *const *a)
{
    const char *path = PyUnicode_AsUTF8(a[0]);
    if (!path) throw python_error();
    void *handle = dlopen(path, RTLD_NOW | RTLD_LOCAL);
    if (!handle) throw Refusal{PyExc_RuntimeError, std::string(dlerror())};
    Library found = {};
    auto find = [&](auto &f, const char *name) {
        f = reinterpret_cast<std::decay_t<decltype(f)>>(dlsym(handle, name));
        if (!f) throw Refusal{PyExc_RuntimeError, std::string(path) + " has no " + name};
    };
    find(found.quantize, "lordba_int8_quantize_rows");
    find(found.linear_bytes, "lordba_int8_linear_workspace_bytes");
    find(found.linear, "lordba_int8_linear");
    find(found.gated_bytes, "lordba_gated_workspace_bytes");
    find(found.gated, "lordba_gated_forward");
    find(found.grad_bytes, "lordba_gated_backward_workspace_bytes");
    find(found.grad, "lordba_gated_backward");
    find(found.dropout, "lordba_dropout");
    lib = found;
    Py_INCREF(a[1]);
    Py_XSETREF(status_error, a[1]);
    Py_RETURN_NONE;
}

template <PyObject *(*F)(PyObject *const *), int N>
PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected, got %zd", N, n);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Refusal &r) {
        if (r.status) {
            PyObject *v = Py_BuildValue("(is)", r.status, r.message.c_str());
            if (v) {
                PyErr_SetObject(r.type, v);
                Py_DECREF(v);
            }
        } else {
            PyErr_SetString(r.type, r.message.c_str());
        }
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

template <PyObject *(*F)(PyObject *const *), int N>
PyMethodDef method(const char *name)
{
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(&call<F, N>)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<bind, 2>("bind"),
                         method<int8_quantize_rows, 4>("int8_quantize_rows"),
                         method<int8_linear, 8>("int8_linear"),
                         method<gated_forward, 14>("gated_forward"),
                         method<gated_backward, 14>("gated_backward"),
                         method<dropout, 7>("dropout"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_block", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// made_for: the interpreter and the torch that the module was compiled against
PyMODINIT_FUNC PyInit__block(void)
{
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "made_for", MADE_FOR) != 0) Py_CLEAR(m);
    return m;
}
