// CPython extension module: the calls of layers.py with their tensors taken apart in native code.
//
// A call of an operator is a check of a handful of tensors and a launch or two.  In Python the checks and the marshalling take
// 12 to 18 us, more than the kernels of small calls; here about 1.  A function returns NotImplemented for whatever it does
// not take as it stands -- tensors that are to be refused (those that autograd follows among them), on another device than the
// current one, subclasses of tensors, the library not loaded yet -- and layers.py goes the plain way, which refuses with the reason.
// The module has no link to the library: layers_binding.py loads that through ctypes and hands over the addresses of its entry points.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <cstring>
#include <initializer_list>

#include "mgwfbp_layers.h"

namespace {

// The entry points, in the order of NAMES; written by set_functions, under the interpreter lock.
enum { EMBED, EMBED_GRAD, EMBED_GRAD_WORKSPACE, ACT_STORE, ACT_BACKWARD, ACT_LINEAR_GRAD, ACT_LINEAR_GRAD_WORKSPACE, N_ENTRIES };
const char* const NAMES[N_ENTRIES] = {"mgwfbp_embed", "mgwfbp_embed_grad", "mgwfbp_embed_grad_workspace", "mgwfbp_act_store",
                                      "mgwfbp_act_backward", "mgwfbp_act_linear_grad", "mgwfbp_act_linear_grad_workspace"};
void* g_entry[N_ENTRIES];
PyObject* g_raise = nullptr;     // layers_binding._check

template <typename F> F* entry(int which, F*) { return reinterpret_cast<F*>(g_entry[which]); }
#define ENTRY(which, fn) entry(which, static_cast<decltype(&fn)>(nullptr))

int dtype_of(const at::Tensor& t) {
    switch (t.scalar_type()) {
        case at::kFloat: return MGWFBP_F32;
        case at::kBFloat16: return MGWFBP_BF16;
        case at::kHalf: return MGWFBP_F16;
        default: return -1;
    }
}
int id_type_of(const at::Tensor& t) { return t.scalar_type() == at::kLong ? MGWFBP_I64 : t.scalar_type() == at::kInt ? MGWFBP_I32 : -1; }

// What the tensors of a call have in common: the current device, found with the first of them.
struct Call {
    bool ok = true;
    int device = -1;

    // A tensor, or null for None where `optional`.
    const at::Tensor* tensor(PyObject* o, bool optional = false) {
        if (optional && o == Py_None) return nullptr;
        if (!THPVariable_CheckExact(o)) return fail();
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.layout() != at::kStrided || !t.is_cuda() || t.is_neg()) return fail();      // a negated view's memory is not its values
        if (t.requires_grad() && c10::GradMode::is_enabled()) return fail();
        if (device < 0) {
            device = t.get_device();
            if (device != c10::hip::current_device()) return fail();
        } else if (t.get_device() != device) {
            return fail();
        }
        return &t;
    }
    const at::Tensor* fail() {
        ok = false;
        return nullptr;
    }
    // Distance of the rows of a matrix of a floating type (rows, cols: -1 for any).
    int64_t matrix(const at::Tensor* t, int64_t rows, int64_t cols) {
        if (t == nullptr) return 0;
        if (t->dim() != 2 || dtype_of(*t) < 0) return ok = false, 0;
        const int64_t r = t->size(0), c = t->size(1), s = t->stride(0);
        if ((rows >= 0 && r != rows) || (cols >= 0 && c != cols) || (c > 1 && t->stride(1) != 1) || (r > 1 && s < c)) ok = false;
        return r > 1 ? s : c;
    }
    // A checkpoint: its tokens.
    int64_t act(const at::Tensor* q, const at::Tensor* scale, int64_t channels) {
        if (!ok || q == nullptr || scale == nullptr || q->dim() != 2 || scale->dim() != 2 || q->scalar_type() != at::kChar ||
            scale->scalar_type() != at::kFloat || !q->is_contiguous() || !scale->is_contiguous())
            return ok = false, 0;
        const int64_t tokens = q->size(0), ld = q->size(1);
        if (scale->size(0) != (tokens + MGWFBP_ACT_GROUP - 1) / MGWFBP_ACT_GROUP || scale->size(1) != ld || channels < 0 || channels > ld || ld % 16 != 0)
            ok = false;
        return tokens;
    }
    // Bytes of device memory: `given`, or torch's, which `keep` holds.
    void* workspace(const at::Tensor* given, uint64_t bytes, at::Tensor& keep, uint64_t& size) {
        if (given != nullptr) {
            size = static_cast<uint64_t>(given->numel()) * given->element_size();
            if (!given->is_contiguous() || size < bytes || reinterpret_cast<uintptr_t>(given->data_ptr()) % 256 != 0) ok = false;
            return given->data_ptr();
        }
        keep = at::empty({static_cast<int64_t>(bytes)}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA, static_cast<c10::DeviceIndex>(device)));
        size = bytes;
        return keep.data_ptr();
    }
    void* stream() const { return c10::hip::getCurrentHIPStream(static_cast<c10::DeviceIndex>(device)).stream(); }
};

void* at_or_null(const at::Tensor* t) { return t == nullptr ? nullptr : t->data_ptr(); }

bool integer(PyObject* o, int64_t& v) {
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return overflow == 0;
}
bool number(PyObject* o, float& v) {
    if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return false;
    v = static_cast<float>(PyFloat_AsDouble(o));
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}
bool truth(PyObject* o, int32_t& v) {
    if (o != Py_True && o != Py_False) return false;
    v = o == Py_True;
    return true;
}

PyObject* not_this_way() { Py_RETURN_NOTIMPLEMENTED; }
// The end of a call: the tensors that it has written count as changed (those made in inference mode have no version).
PyObject* done(int which, int status, std::initializer_list<const at::Tensor*> written) {
    if (status == 0) {
        for (const at::Tensor* t : written)
            if (t != nullptr && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
        Py_RETURN_NONE;
    }
    return PyObject_CallFunction(g_raise, "si", NAMES[which], status);     // raises
}

// Runs f, which throws nothing but what torch does (out of memory): that as torch's own Python exception.
template <typename F> PyObject* guarded(F&& f) {
    HANDLE_TH_ERRORS
    return f();
    END_HANDLE_TH_ERRORS
}

// embed(tables, ids, scales, out): lists or tuples of one to four tensors, ids and numbers; out a tensor
PyObject* embed(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return guarded([&]() -> PyObject* {
        if (nargs != 4 || g_entry[EMBED] == nullptr) return not_this_way();
        PyObject* const* items[3];
        Py_ssize_t n = -1;
        for (int i = 0; i < 3; ++i) {
            if (!PyList_CheckExact(args[i]) && !PyTuple_CheckExact(args[i])) return not_this_way();
            const Py_ssize_t size = PySequence_Fast_GET_SIZE(args[i]);
            if (n >= 0 && size != n) return not_this_way();
            n = size;
            items[i] = PySequence_Fast_ITEMS(args[i]);
        }
        if (n < 1 || n > MGWFBP_MAX_TABLES) return not_this_way();
        Call call;
        mgwfbp_table table[MGWFBP_MAX_TABLES];
        const at::Tensor *first = nullptr, *ids0 = nullptr;
        for (Py_ssize_t k = 0; k < n; ++k) {
            const at::Tensor *t = call.tensor(items[0][k]), *i = call.tensor(items[1][k]);
            float scale;
            if (!call.ok || !number(items[2][k], scale) || t->dim() != 2 || !i->is_contiguous() || id_type_of(*i) < 0) return not_this_way();
            if (k == 0) {
                first = t;
                ids0 = i;
            } else if (t->scalar_type() != first->scalar_type() || i->sizes() != ids0->sizes()) {
                return not_this_way();
            }
            table[k] = {t->data_ptr(), i->data_ptr(), t->size(0), call.matrix(t, -1, first->size(1)), scale, id_type_of(*i)};
        }
        const at::Tensor* out = call.tensor(args[3]);
        if (!call.ok) return not_this_way();
        const int64_t tokens = ids0->numel(), dim = first->size(1);
        int64_t stride;
        if (out->dim() == 2) {
            stride = call.matrix(out, tokens, dim);
        } else {                                             // the ids' shape and the columns
            if (dtype_of(*out) < 0 || !out->is_contiguous() || out->dim() != ids0->dim() + 1 || out->size(-1) != dim) return not_this_way();
            for (int64_t d = 0; d < ids0->dim(); ++d)
                if (out->size(d) != ids0->size(d)) return not_this_way();
            stride = dim;
        }
        if (!call.ok) return not_this_way();
        void *const to = out->data_ptr(), *const stream = call.stream();
        const int table_type = dtype_of(*first), out_type = dtype_of(*out);
        int status;
        Py_BEGIN_ALLOW_THREADS
        status = ENTRY(EMBED, mgwfbp_embed)(table, static_cast<int32_t>(n), table_type, tokens, dim, to, stride, out_type, stream);
        Py_END_ALLOW_THREADS
        return done(EMBED, status, {out});
    });
}

// embed_grad(dy, ids, grad, scale, padding_row, accumulate, workspace)
PyObject* embed_grad(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return guarded([&]() -> PyObject* {
        float scale;
        int64_t padding;
        int32_t accumulate;
        if (nargs != 7 || g_entry[EMBED_GRAD] == nullptr || !number(args[3], scale) || !integer(args[4], padding) || !truth(args[5], accumulate))
            return not_this_way();
        Call call;
        const at::Tensor *dy = call.tensor(args[0]), *ids = call.tensor(args[1]), *grad = call.tensor(args[2]), *given = call.tensor(args[6], true);
        if (!call.ok || dy->dim() != 2 || grad->dim() != 2 || !ids->is_contiguous() || id_type_of(*ids) < 0) return not_this_way();
        const int64_t tokens = ids->numel(), rows = grad->size(0), dim = grad->size(1);
        const int64_t grad_stride = call.matrix(grad, -1, -1), dy_stride = call.matrix(dy, tokens, dim);
        uint64_t bytes = 0, size = 0;
        if (!call.ok || ENTRY(EMBED_GRAD_WORKSPACE, mgwfbp_embed_grad_workspace)(tokens, rows, dim, &bytes) != 0) return not_this_way();
        at::Tensor keep;
        void* const space = call.workspace(given, bytes, keep, size);
        if (!call.ok) return not_this_way();
        void *const d = dy->data_ptr(), *const i = ids->data_ptr(), *const g = grad->data_ptr(), *const stream = call.stream();
        const int dy_type = dtype_of(*dy), grad_type = dtype_of(*grad), id_type = id_type_of(*ids);
        int status;
        Py_BEGIN_ALLOW_THREADS
        status = ENTRY(EMBED_GRAD, mgwfbp_embed_grad)(i, id_type, tokens, d, dy_stride, dy_type, scale, padding, accumulate, g, rows, dim, grad_stride, grad_type,
                                                      space, size, stream);
        Py_END_ALLOW_THREADS
        return done(EMBED_GRAD, status, {grad});
    });
}

// act_store(x, q, scale, channels, kind, y)
PyObject* act_store(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return guarded([&]() -> PyObject* {
        int64_t channels, kind;
        if (nargs != 6 || g_entry[ACT_STORE] == nullptr || !integer(args[3], channels) || !integer(args[4], kind)) return not_this_way();
        Call call;
        const at::Tensor *x = call.tensor(args[0]), *q = call.tensor(args[1]), *scale = call.tensor(args[2]), *y = call.tensor(args[5], true);
        const int64_t tokens = call.act(q, scale, channels);
        if (!call.ok || (y != nullptr && y->scalar_type() != x->scalar_type())) return not_this_way();
        const int64_t x_stride = call.matrix(x, tokens, channels), y_stride = call.matrix(y, tokens, channels);
        if (!call.ok) return not_this_way();
        void *const xp = x->data_ptr(), *const yp = at_or_null(y), *const stream = call.stream();
        int8_t* const qp = static_cast<int8_t*>(q->data_ptr());
        float* const sp = static_cast<float*>(scale->data_ptr());
        const int64_t ld = q->size(1);
        const int type = dtype_of(*x);
        int status;
        Py_BEGIN_ALLOW_THREADS
        status = ENTRY(ACT_STORE, mgwfbp_act_store)(xp, x_stride, type, tokens, channels, static_cast<int32_t>(kind), qp, sp, ld, yp, y_stride, stream);
        Py_END_ALLOW_THREADS
        return done(ACT_STORE, status, {q, scale, y});
    });
}

// act_backward(q, scale, channels, dy, kind, dx, y): dy and dx both or neither, y or None
PyObject* act_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return guarded([&]() -> PyObject* {
        int64_t channels, kind;
        if (nargs != 7 || g_entry[ACT_BACKWARD] == nullptr || !integer(args[2], channels) || !integer(args[4], kind)) return not_this_way();
        Call call;
        const at::Tensor *q = call.tensor(args[0]), *scale = call.tensor(args[1]), *dy = call.tensor(args[3], true), *dx = call.tensor(args[5], true),
                         *y = call.tensor(args[6], true);
        const int64_t tokens = call.act(q, scale, channels);
        const at::Tensor* one = dy != nullptr ? dy : y;
        if (!call.ok || one == nullptr || (dy == nullptr) != (dx == nullptr) || (dx != nullptr && dx->scalar_type() != one->scalar_type()) ||
            (y != nullptr && y->scalar_type() != one->scalar_type()))
            return not_this_way();
        const int64_t dy_stride = call.matrix(dy, tokens, channels), dx_stride = call.matrix(dx, tokens, channels), y_stride = call.matrix(y, tokens, channels);
        if (!call.ok) return not_this_way();
        void *const dyp = at_or_null(dy), *const dxp = at_or_null(dx), *const yp = at_or_null(y), *const stream = call.stream();
        const int8_t* const qp = static_cast<const int8_t*>(q->data_ptr());
        const float* const sp = static_cast<const float*>(scale->data_ptr());
        const int64_t ld = q->size(1);
        const int type = dtype_of(*one);
        int status;
        Py_BEGIN_ALLOW_THREADS
        status = ENTRY(ACT_BACKWARD, mgwfbp_act_backward)(qp, sp, ld, tokens, channels, static_cast<int32_t>(kind), dyp, dy_stride, dxp, dx_stride, yp, y_stride, type,
                                                          stream);
        Py_END_ALLOW_THREADS
        return done(ACT_BACKWARD, status, {dx, y});
    });
}

// act_linear_grad(dy, q, scale, channels, dw, db, accumulate, workspace)
PyObject* act_linear_grad(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return guarded([&]() -> PyObject* {
        int64_t channels;
        int32_t accumulate;
        if (nargs != 8 || g_entry[ACT_LINEAR_GRAD] == nullptr || !integer(args[3], channels) || !truth(args[6], accumulate)) return not_this_way();
        Call call;
        const at::Tensor *dy = call.tensor(args[0]), *q = call.tensor(args[1]), *scale = call.tensor(args[2]), *dw = call.tensor(args[4]),
                         *db = call.tensor(args[5], true), *given = call.tensor(args[7], true);
        const int64_t tokens = call.act(q, scale, channels);
        if (!call.ok || dy->dim() != 2) return not_this_way();
        const int64_t outputs = dy->size(1), dy_stride = call.matrix(dy, tokens, -1), dw_stride = call.matrix(dw, outputs, channels);
        if (db != nullptr && (db->dim() != 1 || db->size(0) != outputs || db->scalar_type() != dw->scalar_type() || (outputs > 1 && db->stride(0) != 1)))
            return not_this_way();
        uint64_t bytes = 0, size = 0;
        if (!call.ok || ENTRY(ACT_LINEAR_GRAD_WORKSPACE, mgwfbp_act_linear_grad_workspace)(tokens, channels, outputs, &bytes) != 0) return not_this_way();
        at::Tensor keep;
        void* const space = call.workspace(given, bytes, keep, size);
        if (!call.ok) return not_this_way();
        void *const d = dy->data_ptr(), *const w = dw->data_ptr(), *const b = at_or_null(db), *const stream = call.stream();
        const int8_t* const qp = static_cast<const int8_t*>(q->data_ptr());
        const float* const sp = static_cast<const float*>(scale->data_ptr());
        const int64_t ld = q->size(1);
        const int dy_type = dtype_of(*dy), grad_type = dtype_of(*dw);
        int status;
        Py_BEGIN_ALLOW_THREADS
        status = ENTRY(ACT_LINEAR_GRAD, mgwfbp_act_linear_grad)(qp, sp, ld, tokens, channels, d, dy_stride, dy_type, outputs, accumulate, w, dw_stride, b, grad_type,
                                                                space, size, stream);
        Py_END_ALLOW_THREADS
        return done(ACT_LINEAR_GRAD, status, {dw, db});
    });
}

// set_functions(check, {name: address}): None for the table takes the entry points away again
PyObject* set_functions(PyObject*, PyObject* args) {
    PyObject *check, *table;
    if (!PyArg_ParseTuple(args, "OO", &check, &table)) return nullptr;
    void* found[N_ENTRIES] = {};
    if (table != Py_None)
        for (int i = 0; i < N_ENTRIES; ++i) {
            PyObject* a = PyDict_Check(table) ? PyDict_GetItemString(table, NAMES[i]) : nullptr;
            if (a == nullptr || !PyLong_Check(a)) {
                PyErr_Format(PyExc_KeyError, "%s", NAMES[i]);
                return nullptr;
            }
            found[i] = reinterpret_cast<void*>(static_cast<uintptr_t>(PyLong_AsUnsignedLongLongMask(a)));
        }
    Py_INCREF(check);
    Py_XSETREF(g_raise, check);
    std::memcpy(g_entry, found, sizeof found);
    Py_RETURN_NONE;
}

template <typename F> PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }
PyMethodDef functions[] = {{"embed", fast(embed), METH_FASTCALL, "embed(tables, ids, scales, out)"},
                           {"embed_grad", fast(embed_grad), METH_FASTCALL, "embed_grad(dy, ids, grad, scale, padding_row, accumulate, workspace)"},
                           {"act_store", fast(act_store), METH_FASTCALL, "act_store(x, q, scale, channels, kind, y)"},
                           {"act_backward", fast(act_backward), METH_FASTCALL, "act_backward(q, scale, channels, dy, kind, dx, y)"},
                           {"act_linear_grad", fast(act_linear_grad), METH_FASTCALL, "act_linear_grad(dy, q, scale, channels, dw, db, accumulate, workspace)"},
                           {"set_functions", set_functions, METH_VARARGS, "set_functions(check, {name: address} or None)"},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_layers_calls", "calls of layers", -1, functions, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layers_calls(void) { return PyModule_Create(&module); }
