// The Python side of the operators around the projection (norm, rotary positions, gradient clipping):
// argument checks, output allocation and the C call, without the interpreter in between.  A call of a few
// rows runs for two microseconds on the GPU; marshalling it in Python took seventeen, and a list of 192
// gradients 380.
//
// Every function takes its arguments by position (pamm.py has the signatures and the documentation), runs on
// the current stream of its tensors' device and raises TypeError, ValueError or PammError.  In a thread that is
// preparing a call (pamm.prepared) the C call is written down instead: its name, its arguments and what has to
// stay alive for it.
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <vector>

#include "../../include/pamm.h"

namespace {

using at::Tensor;

PyObject* g_error = nullptr;       // PammError(code, where)
thread_local PyObject* g_record = nullptr;      // list of (name, arguments, kept) while this thread prepares a call

// ---- Python values ------------------------------------------------------------------------------------
struct Failure {};                 // a Python exception is set

[[noreturn]] void fail(PyObject* type, const char* format, ...) {
    va_list args;
    va_start(args, format);
    PyErr_FormatV(type, format, args);
    va_end(args);
    throw Failure();
}
const char* text(c10::ScalarType t) { return c10::toString(t); }

bool is_none(PyObject* o) { return o == Py_None; }
const Tensor& tensor(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "%s is a tensor, got %s", what, Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}
Tensor optional_tensor(PyObject* o, const char* what) { return is_none(o) ? Tensor() : tensor(o, what); }
int64_t integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Failure();
    return v;
}
double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Failure();
    return v;
}
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Failure();
    return v != 0;
}
PyObject* wrapped(const Tensor& t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
template <typename... T>
PyObject* tuple_of(const T&... t) {
    PyObject* all = PyTuple_New(sizeof...(T));
    if (!all) throw Failure();
    Py_ssize_t i = 0;
    (PyTuple_SET_ITEM(all, i++, wrapped(t)), ...);
    return all;
}

// ---- the C call -----------------------------------------------------------------------------------------
PyObject* value(const void* p) { return p ? PyLong_FromVoidPtr(const_cast<void*>(p)) : (Py_INCREF(Py_None), Py_None); }
PyObject* value(int64_t v) { return PyLong_FromLongLong(v); }
PyObject* value(int v) { return PyLong_FromLong(v); }
PyObject* value(size_t v) { return PyLong_FromSize_t(v); }
PyObject* value(double v) { return PyFloat_FromDouble(v); }
PyObject* value(float v) { return PyFloat_FromDouble(v); }
template <typename E, typename = std::enable_if_t<std::is_enum_v<E>>>
PyObject* value(E v) { return PyLong_FromLong((long)v); }

// What a written-down call needs alive besides its caller's tensors (null where the call is made at once).
template <typename... T>
PyObject* keep(const T&... t) { return g_record ? tuple_of(t...) : nullptr; }

// Lets other Python threads run, as ctypes does: a call waits where the launch queue is full.
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    Unlocked() = default;
    ~Unlocked() { PyEval_RestoreThread(state); }
    Unlocked(const Unlocked&) = delete;
};

// `kept`: a new reference, given up here.
template <typename F, typename... A>
void call(const char* name, F function, PyObject* kept, A... a) {
    if (g_record) {
        PyObject* args = PyTuple_New(sizeof...(A));
        Py_ssize_t i = 0;
        if (args) (PyTuple_SET_ITEM(args, i++, value(a)), ...);
        PyObject* entry = args ? Py_BuildValue("(sOO)", name, args, kept) : nullptr;
        Py_DECREF(kept);
        Py_XDECREF(args);
        const int rc = entry ? PyList_Append(g_record, entry) : -1;
        Py_XDECREF(entry);
        if (rc < 0) throw Failure();
        return;
    }
    pamm_status s;
    {
        const Unlocked unlocked;
        s = function(a...);
    }
    if (s != PAMM_OK) {
        PyObject* e = PyObject_CallFunction(g_error, "is", (int)s, name);
        if (e) {
            PyErr_SetObject(g_error, e);
            Py_DECREF(e);
        }
        throw Failure();
    }
}

// ---- checks ---------------------------------------------------------------------------------------------
// The device of the call: the first tensor's, current while this lives; every other tensor is held to it.
struct Place {
    c10::Device device;
    c10::cuda::CUDAGuard guard;
    Place(const Tensor& t, const char* what) : device(checked(t, what)), guard(device) {}
    static c10::Device checked(const Tensor& t, const char* what) {
        if (!t.is_cuda()) fail(PyExc_ValueError, "%s is a CUDA tensor", what);
        return t.device();
    }
    void holds(const Tensor& t, const char* what) const {
        if (t.device() != device) fail(PyExc_ValueError, "%s is on another device than the call's first tensor", what);
    }
    void* stream() const { return c10::cuda::getCurrentCUDAStream(device.index()).stream(); }
    Tensor empty(at::IntArrayRef sizes, c10::ScalarType type) const {
        return at::detail::empty_cuda(sizes, type, device, std::nullopt);
    }
};

bool known(c10::ScalarType t) { return t == at::kFloat || t == at::kBFloat16; }
pamm_dtype type_of(const Tensor& t, const char* what) {
    if (!known(t.scalar_type())) fail(PyExc_TypeError, "%s is float32 or bfloat16, got %s", what, text(t.scalar_type()));
    return t.scalar_type() == at::kFloat ? PAMM_F32 : PAMM_BF16;
}
// Leading dimension of a b x n matrix of the given type with contiguous rows.
int64_t matrix(const Place& at, const Tensor& t, const char* what, int64_t b, int64_t n, c10::ScalarType type) {
    if (t.dim() != 2 || t.size(0) != b || t.size(1) != n)
        fail(PyExc_ValueError, "%s is a %lld x %lld matrix", what, (long long)b, (long long)n);
    if (t.scalar_type() != type) fail(PyExc_TypeError, "%s is of %s, got %s", what, text(type), text(t.scalar_type()));
    at.holds(t, what);
    if (n > 1 && t.stride(1) != 1) fail(PyExc_ValueError, "%s needs contiguous rows (a row stride is allowed)", what);
    return b < 2 ? n : t.stride(0);
}
// Address of a contiguous vector of n entries of the given type (none: null).
void* vector(const Place& at, const Tensor& t, const char* what, int64_t n, c10::ScalarType type) {
    if (!t.defined()) return nullptr;
    if (t.dim() != 1 || t.size(0) != n || !t.is_contiguous()) fail(PyExc_ValueError, "%s is a contiguous vector of %lld", what, (long long)n);
    if (t.scalar_type() != type) fail(PyExc_TypeError, "%s is of %s, got %s", what, text(type), text(t.scalar_type()));
    at.holds(t, what);
    return t.data_ptr();
}
void* address(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
void workspace_ok(const Place& at, const Tensor& t) {
    if (!t.is_contiguous() || t.scalar_type() != at::kByte) fail(PyExc_ValueError, "the workspace is a contiguous uint8 tensor");
    at.holds(t, "the workspace");
}

// ---- norm -------------------------------------------------------------------------------------------------
PyObject* norm_forward(PyObject* const* o) {
    const Tensor &X = tensor(o[0], "X");
    const Tensor weight = optional_tensor(o[1], "weight"), bias = optional_tensor(o[2], "bias"), R = optional_tensor(o[3], "residual");
    const float eps = (float)number(o[4]);
    const bool rms = truth(o[5]);
    Tensor Y = optional_tensor(o[6], "Y"), H = optional_tensor(o[7], "H"), mean = optional_tensor(o[8], "mean"), rstd = optional_tensor(o[9], "rstd");
    const pamm_dtype dt = type_of(X, "X");
    const Place at(X, "X");
    if (X.dim() != 2) fail(PyExc_ValueError, "X is a matrix, got %lld dimensions", (long long)X.dim());
    const int64_t b = X.size(0), n = X.size(1), ldx = matrix(at, X, "X", b, n, X.scalar_type());
    const Tensor& one = weight.defined() ? weight : bias;
    const pamm_dtype w_dt = one.defined() ? type_of(one, "weight") : dt;
    const c10::ScalarType w_type = one.defined() ? one.scalar_type() : X.scalar_type();
    void *w = vector(at, weight, "weight", n, w_type), *c = vector(at, bias, "bias", n, w_type);
    const int64_t ldr = R.defined() ? matrix(at, R, "residual", b, n, X.scalar_type()) : 0;
    if (!Y.defined()) Y = at.empty({b, n}, X.scalar_type());
    if (!H.defined() && R.defined()) H = at.empty({b, n}, X.scalar_type());
    if (!mean.defined() && !rms) mean = at.empty({b}, at::kFloat);
    if (!rstd.defined()) rstd = at.empty({b}, at::kFloat);
    const int64_t ldy = matrix(at, Y, "Y", b, n, X.scalar_type()), ldh = H.defined() ? matrix(at, H, "H", b, n, X.scalar_type()) : 0;
    call("pamm_norm_forward", pamm_norm_forward, keep(Y, H, mean, rstd), rms ? PAMM_NORM_RMS : PAMM_NORM_LAYER, X.data_ptr(), ldx,
         address(R), ldr, b, n, dt, w, c, w_dt, eps, Y.data_ptr(), ldy, address(H), ldh, (float*)vector(at, mean, "mean", b, at::kFloat),
         (float*)vector(at, rstd, "rstd", b, at::kFloat), at.stream());
    return tuple_of(Y, H.defined() ? H : X, rms ? Tensor() : mean, rstd);
}

PyObject* norm_backward(PyObject* const* o) {
    const Tensor &dY = tensor(o[0], "dY"), &X = tensor(o[1], "X");
    const Tensor mean = optional_tensor(o[2], "mean"), &rstd = tensor(o[3], "rstd"), weight = optional_tensor(o[4], "weight");
    const bool bias = truth(o[5]), need_dw = truth(o[10]);
    const Tensor dH = optional_tensor(o[6], "dH");
    Tensor dX = optional_tensor(o[7], "dX"), dw = optional_tensor(o[8], "dw"), dc = optional_tensor(o[9], "dc");
    Tensor workspace = optional_tensor(o[12], "workspace");
    const pamm_dtype dt = type_of(X, "X");
    const Place at(X, "X");
    if (X.dim() != 2) fail(PyExc_ValueError, "X is a matrix, got %lld dimensions", (long long)X.dim());
    const int64_t b = X.size(0), n = X.size(1), ldx = matrix(at, X, "X", b, n, X.scalar_type());
    const int64_t lddy = matrix(at, dY, "dY", b, n, X.scalar_type());
    const pamm_dtype w_dt = weight.defined() ? type_of(weight, "weight") : dt;
    void* w = vector(at, weight, "weight", n, weight.defined() ? weight.scalar_type() : X.scalar_type());
    c10::ScalarType dw_type = dw.defined() ? dw.scalar_type() : dc.defined() ? dc.scalar_type()
                            : weight.defined() ? weight.scalar_type() : X.scalar_type();
    if (!is_none(o[11])) {
        if (!THPDtype_Check(o[11])) fail(PyExc_TypeError, "dw_dtype is a torch type");
        dw_type = reinterpret_cast<THPDtype*>(o[11])->scalar_type;
    }
    if (!known(dw_type)) fail(PyExc_TypeError, "dw is float32 or bfloat16, got %s", text(dw_type));
    const int64_t lddh = dH.defined() ? matrix(at, dH, "dH", b, n, X.scalar_type()) : 0;
    if (!dX.defined()) dX = at.empty({b, n}, X.scalar_type());
    if (need_dw && !dw.defined()) dw = at.empty({n}, dw_type);
    if (need_dw && bias && !dc.defined()) dc = at.empty({n}, dw_type);
    if (!workspace.defined() && (dw.defined() || dc.defined())) {
        const size_t bytes = pamm_workspace_bytes(PAMM_WS_NORM_BACKWARD, b, n, 1, 1, dt);
        workspace = at.empty({bytes == (size_t)-1 ? 256 : (int64_t)bytes}, at::kByte);
    }
    if (workspace.defined()) workspace_ok(at, workspace);
    const int64_t lddx = matrix(at, dX, "dX", b, n, X.scalar_type());
    call("pamm_norm_backward", pamm_norm_backward, keep(dX, dw, dc, workspace), mean.defined() ? PAMM_NORM_LAYER : PAMM_NORM_RMS,
         dY.data_ptr(), lddy, X.data_ptr(), ldx, (const float*)vector(at, mean, "mean", b, at::kFloat),
         (const float*)vector(at, rstd, "rstd", b, at::kFloat), b, n, dt, w, w_dt, address(dH), lddh, dX.data_ptr(), lddx,
         vector(at, dw, "dw", n, dw_type), vector(at, dc, "dc", n, dw_type), dw_type == at::kFloat ? PAMM_F32 : PAMM_BF16,
         address(workspace), workspace.defined() ? (size_t)workspace.numel() : (size_t)0, at.stream());
    return tuple_of(dX, dw, dc);
}

// ---- rotary positions ---------------------------------------------------------------------------------------
PyObject* rotary(PyObject* const* o) {
    const Tensor &X = tensor(o[0], "X"), &table = tensor(o[1], "table"), positions = optional_tensor(o[2], "positions");
    Tensor out = optional_tensor(o[8], "out");
    const pamm_dtype dt = type_of(X, "X");
    const int64_t dims = X.dim();
    if (dims != 3 && dims != 4)
        fail(PyExc_ValueError, "X is (tokens, heads, head_dim) or (batch, tokens, heads, head_dim), got %lld dimensions", (long long)dims);
    const Place at(X, "X");
    const int64_t batch = dims == 4 ? X.size(0) : 1, seq = X.size(dims - 3), heads = X.size(dims - 2), d = X.size(dims - 1);
    at.holds(table, "the table");
    if (table.dim() != 2 || table.scalar_type() != at::kFloat || !table.is_contiguous())
        fail(PyExc_ValueError, "the table is a contiguous float32 matrix");
    const int64_t rot = table.size(1);
    if (!is_none(o[4]) && integer(o[4]) != rot)
        fail(PyExc_ValueError, "the table holds rotations of %lld elements, not %lld", (long long)rot, (long long)integer(o[4]));
    if (d > 1 && X.stride(dims - 1) != 1) fail(PyExc_ValueError, "X needs contiguous heads");
    if (!out.defined()) {
        out = at.empty(X.sizes(), X.scalar_type());
    } else {
        if (out.sizes() != X.sizes() || out.scalar_type() != X.scalar_type()) fail(PyExc_ValueError, "out is a tensor of X's shape and type");
        at.holds(out, "out");
    }
    for (int64_t i = 0; i < dims; ++i)
        if (out.size(i) > 1 && (out.stride(i) == 0 || (i == dims - 1 && out.stride(i) != 1)))
            fail(PyExc_ValueError, "out needs contiguous heads that do not overlap");
    pamm_position_type pos_type = PAMM_POS_I64;
    int64_t pb = 0, ps = 0;
    if (positions.defined()) {
        at.holds(positions, "positions");
        if (positions.scalar_type() != at::kLong && positions.scalar_type() != at::kInt)
            fail(PyExc_TypeError, "positions are int32 or int64, got %s", text(positions.scalar_type()));
        pos_type = positions.scalar_type() == at::kInt ? PAMM_POS_I32 : PAMM_POS_I64;
        if (positions.dim() == 2 && positions.size(0) == batch && positions.size(1) == seq) {
            pb = positions.stride(0);
            ps = positions.stride(1);
        } else if (positions.dim() == 1 && positions.size(0) == seq) {
            ps = positions.stride(0);
        } else {
            fail(PyExc_ValueError, "positions are of shape (%lld,) or (%lld, %lld)", (long long)seq, (long long)batch, (long long)seq);
        }
    }
    const auto stride = [dims](const Tensor& t, int64_t i) { return i < 0 ? (int64_t)0 : t.stride(i); };
    call("pamm_rotary", pamm_rotary, keep(out), X.data_ptr(), stride(X, dims - 4), X.stride(dims - 3), X.stride(dims - 2), out.data_ptr(),
         stride(out, dims - 4), out.stride(dims - 3), out.stride(dims - 2), batch, seq, heads, is_none(o[3]) ? heads : integer(o[3]), d, rot, dt,
         truth(o[5]) ? PAMM_PAIRS_ADJACENT : PAMM_PAIRS_HALF, truth(o[6]) ? 1 : 0, (const float*)table.data_ptr(), table.size(0),
         address(positions), pos_type, pb, ps, integer(o[7]), at.stream());
    return wrapped(out);
}

// ---- gradients --------------------------------------------------------------------------------------------
struct Held {                      // a reference of our own
    PyObject* o;
    explicit Held(PyObject* o) : o(o) { if (!o) throw Failure(); }
    ~Held() { Py_DECREF(o); }
    Held(const Held&) = delete;
};

// Memory without gaps is one row whatever its shape and order; otherwise a matrix with contiguous rows or columns.
// With an output both lie in the same order.
void describe(const Tensor& g, const Tensor* t, std::vector<pamm_tensor>& in, std::vector<pamm_tensor>& out) {
    const pamm_dtype dt = type_of(g, "a gradient");
    const pamm_dtype odt = t ? type_of(*t, "an output") : dt;
    if (t && t->sizes() != g.sizes()) fail(PyExc_ValueError, "a gradient and its output differ in shape");
    const bool flat = t ? (g.is_contiguous() && t->is_contiguous()) ||
                              (g.strides() == t->strides() && g.is_non_overlapping_and_dense())
                        : g.is_non_overlapping_and_dense();
    if (flat) {
        in.push_back({g.data_ptr(), 1, g.numel(), g.numel(), dt});
        if (t) out.push_back({t->data_ptr(), 1, g.numel(), g.numel(), odt});
        return;
    }
    if (g.dim() == 2) {
        for (int unit = 1; unit >= 0; --unit) {            // contiguous rows, then columns
            const int64_t rows = g.size(1 - unit), cols = g.size(unit);
            const auto fits = [&](const Tensor& x) {
                return (x.stride(unit) == 1 || cols == 1) && (x.stride(1 - unit) >= cols || rows == 1);
            };
            if (!fits(g) || (t && !fits(*t))) continue;
            in.push_back({g.data_ptr(), rows, cols, rows > 1 ? g.stride(1 - unit) : cols, dt});
            if (t) out.push_back({t->data_ptr(), rows, cols, rows > 1 ? t->stride(1 - unit) : cols, odt});
            return;
        }
    }
    fail(PyExc_ValueError, t ? "a gradient and its output need the same order of elements in memory, without overlaps"
                             : "a gradient is contiguous, or a matrix with contiguous rows or columns");
}

PyObject* clip(PyObject* const* o) {
    const bool scale = !is_none(o[2]);
    const double max_norm = scale ? number(o[2]) : 0.0;
    const Held grads(PySequence_Fast(o[0], "gradients are a list of tensors"));
    const Held outs(is_none(o[1]) ? (Py_INCREF(Py_None), Py_None) : PySequence_Fast(o[1], "outputs are a list of tensors"));
    const Py_ssize_t count = PySequence_Fast_GET_SIZE(grads.o);
    const bool apart = outs.o != Py_None;
    if (apart && PySequence_Fast_GET_SIZE(outs.o) != count)
        fail(PyExc_ValueError, "%zd gradients and %zd outputs", count, PySequence_Fast_GET_SIZE(outs.o));
    Tensor norm = optional_tensor(o[3], "norm"), workspace = optional_tensor(o[4], "workspace");
    std::vector<pamm_tensor> in, out;
    in.reserve(count);
    out.reserve(apart ? count : 0);
    c10::Device device(c10::kCUDA, count || norm.defined() ? 0 : c10::cuda::current_device());
    if (count) device = tensor(PySequence_Fast_GET_ITEM(grads.o, 0), "a gradient").device();
    else if (norm.defined()) device = Place::checked(norm, "norm");
    for (Py_ssize_t i = 0; i < count; ++i) {
        const Tensor& g = tensor(PySequence_Fast_GET_ITEM(grads.o, i), "a gradient");
        const Tensor* t = apart ? &tensor(PySequence_Fast_GET_ITEM(outs.o, i), "an output") : nullptr;
        type_of(g, "a gradient");
        if (!g.is_cuda() || (t && !t->is_cuda())) fail(PyExc_TypeError, "gradients and outputs are CUDA tensors");
        if (g.device() != device || (t && t->device() != device)) fail(PyExc_ValueError, "gradients and outputs are on one device");
        describe(g, t, in, out);
    }
    const c10::cuda::CUDAGuard guard(device);
    const auto empty = [&](at::IntArrayRef sizes, c10::ScalarType type) { return at::detail::empty_cuda(sizes, type, device, std::nullopt); };
    if (!norm.defined()) norm = empty({}, at::kFloat);
    if (!workspace.defined()) workspace = empty({(int64_t)pamm_workspace_bytes(PAMM_WS_GRAD_NORM, 1, 1, 1, 1, PAMM_F32)}, at::kByte);
    if (norm.numel() != 1 || norm.scalar_type() != at::kFloat || norm.device() != device) fail(PyExc_ValueError, "norm is one float32 on the gradients' device");
    if (!workspace.is_contiguous() || workspace.scalar_type() != at::kByte || workspace.device() != device)
        fail(PyExc_ValueError, "the workspace is a contiguous uint8 tensor on the gradients' device");
    void* stream = c10::cuda::getCurrentCUDAStream(device.index()).stream();
    const pamm_tensor *pin = in.data(), *pout = apart ? out.data() : nullptr;
    PyObject* kept = keep(norm, workspace);
    if (g_record) {               // the written-down call needs the lists as well
        const Held a(PyBytes_FromStringAndSize((const char*)in.data(), in.size() * sizeof(pamm_tensor)));
        const Held b(PyBytes_FromStringAndSize((const char*)out.data(), out.size() * sizeof(pamm_tensor)));
        pin = (const pamm_tensor*)PyBytes_AS_STRING(a.o);
        if (apart) pout = (const pamm_tensor*)PyBytes_AS_STRING(b.o);
        kept = Py_BuildValue("(NOOOO)", kept, a.o, b.o, grads.o, outs.o);
        if (!kept) throw Failure();
    }
    if (scale)
        call("pamm_clip_grad_norm", pamm_clip_grad_norm, kept, pin, pout, (int64_t)count, max_norm, (float*)norm.data_ptr(), workspace.data_ptr(),
             (size_t)workspace.numel(), stream);
    else
        call("pamm_grad_norm", pamm_grad_norm, kept, pin, (int64_t)count, (float*)norm.data_ptr(), workspace.data_ptr(), (size_t)workspace.numel(),
             stream);
    return wrapped(norm);
}

// ---- the module ---------------------------------------------------------------------------------------------
template <PyObject* (*F)(PyObject* const*), Py_ssize_t N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    if (count != N) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, got %zd", N, count);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Failure&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

PyObject* set_error(PyObject*, PyObject* type) {
    Py_INCREF(type);
    Py_XSETREF(g_error, type);
    Py_RETURN_NONE;
}
PyObject* set_record(PyObject*, PyObject* list) {
    if (list == Py_None) {
        Py_CLEAR(g_record);
    } else if (PyList_Check(list)) {
        Py_INCREF(list);
        Py_XSETREF(g_record, list);
    } else {
        PyErr_SetString(PyExc_TypeError, "a list or None");
        return nullptr;
    }
    Py_RETURN_NONE;
}

#define ENTRY(name, n) {#name, (PyCFunction)(void (*)(void))entry<name, n>, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    ENTRY(norm_forward, 10), ENTRY(norm_backward, 13), ENTRY(rotary, 9), ENTRY(clip, 5),
    {"set_error", set_error, METH_O, nullptr}, {"set_record", set_record, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&g_module); }
