// The calls of layers.py in native code, as binding.cpp has those of mxq.py: every function either does what the Python form
// does or returns None BEFORE it has done anything, and then the Python form runs and raises its errors.
#include "binding_common.hpp"

#include "../../include/mxq_layers.h"

namespace {

// libmxq's functions and the tuples of layers.py, handed over by layers.py.
decltype(&mxq_add_rmsnorm) p_norm;
decltype(&mxq_add_rmsnorm_backward) p_norm_back;
decltype(&mxq_add_rmsnorm_backward_workspace_size) p_norm_back_size;
decltype(&mxq_swiglu) p_swiglu;
decltype(&mxq_swiglu_backward) p_swiglu_back;
decltype(&mxq_linear) p_linear;
decltype(&mxq_linear_workspace_size) p_linear_size;
PyObject *q8_class, *norm_class, *swiglu_class;

// A plain 2-D tensor on the GPU whose rows are contiguous, or null.
const at::Tensor* rows_of(PyObject* o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || t.key_set().has_any(kNotPlain) || !t.has_storage() || t.dim() != 2 ||
        (t.size(1) > 1 && t.stride(1) != 1))
        return nullptr;
    return &t;
}

bool like(const at::Tensor* t, const at::Tensor& x)
{
    return t && t->scalar_type() == x.scalar_type() && t->sizes() == x.sizes() && t->device() == x.device();
}

// A plain contiguous tensor of a type and shape on a device.
const at::Tensor* whole(PyObject* o, at::IntArrayRef shape, at::ScalarType type, const at::Device& device)
{
    const at::Tensor* t = plain(o);
    return t && t->scalar_type() == type && t->sizes() == shape && t->device() == device ? t : nullptr;
}

// Codes and scales of a Q8 tuple of that shape.
struct Bits {
    at::Tensor codes, scales;
    bool set(PyObject* o, int64_t rows, int64_t cols, const at::Device& device)
    {
        if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 2) return false;
        const at::Tensor* c = whole(PyTuple_GET_ITEM(o, 0), {rows, cols}, at::kFloat8_e4m3fn, device);
        const at::Tensor* s = whole(PyTuple_GET_ITEM(o, 1), {rows, cols / MXQ_Q8_BLOCK}, at::kFloat8_e8m0fnu, device);
        if (!c || !s) return false;
        codes = *c;
        scales = *s;
        return true;
    }
    void make(NewOutputs& new_empty, const at::Tensor& x)
    {
        codes = new_empty(x.sizes(), at::kFloat8_e4m3fn, x);
        scales = new_empty({x.size(0), x.size(1) / MXQ_Q8_BLOCK}, at::kFloat8_e8m0fnu, x);
    }
    uint8_t* c() const { return codes.defined() ? (uint8_t*)codes.data_ptr() : nullptr; }
    uint8_t* s() const { return scales.defined() ? (uint8_t*)scales.data_ptr() : nullptr; }
};

void* ptr_or_null(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// New references taken over; null if one of them is.
PyObject* tuple_as(PyObject* type, std::initializer_list<PyObject*> items)
{
    PyObject* args[4];
    Py_ssize_t n = 0;
    bool ok = true;
    for (PyObject* o : items) {
        ok &= o != nullptr;
        args[n++] = o;
    }
    PyObject* r = nullptr;
    if (ok && type) {
        r = PyObject_Vectorcall(type, args, (size_t)n, nullptr);
    } else if (ok && (r = PyTuple_New(n))) {
        for (Py_ssize_t i = 0; i < n; ++i) {
            Py_INCREF(args[i]);
            PyTuple_SET_ITEM(r, i, args[i]);
        }
    }
    for (Py_ssize_t i = 0; i < n; ++i) Py_XDECREF(args[i]);
    return r;
}

PyObject* q8(const Bits& b) { return tuple_as(q8_class, {wrapped(b.codes), wrapped(b.scales)}); }

PyObject* new_none() { Py_RETURN_NONE; }

bool real(PyObject* o, float* out)
{
    if (PyFloat_CheckExact(o)) *out = (float)PyFloat_AS_DOUBLE(o);
    else return false;
    return true;
}

// True or False itself.
bool flag(PyObject* o, bool* out)
{
    *out = o == Py_True;
    return o == Py_True || o == Py_False;
}

// add_rmsnorm(x, weight, residual, eps, dense, checkpoint, hidden_out)
PyObject* add_rmsnorm(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor* x = n == 7 && !modes_active() ? rows_of(a[0]) : nullptr;
    float eps;
    bool dense, checkpoint;
    if (!x || dtype_code(*x) < 0 || !real(a[3], &eps) || !flag(a[4], &dense) || !flag(a[5], &checkpoint)) return none();
    const int64_t rows = x->size(0), cols = x->size(1);
    if (cols % MXQ_Q8_BLOCK != 0) return none();
    const at::Tensor *weight = nullptr, *residual = nullptr;
    at::Tensor hidden;
    if (a[1] != Py_None && !(weight = whole(a[1], {cols}, x->scalar_type(), x->device()))) return none();
    if (a[2] != Py_None && (!(residual = rows_of(a[2])) || !like(residual, *x))) return none();
    NewOutputs new_empty;
    if (a[6] != Py_None) {
        const at::Tensor* given = residual ? whole(a[6], x->sizes(), x->scalar_type(), x->device()) : nullptr;
        if (!given) return none();
        hidden = *given;
    } else if (residual) {
        hidden = new_empty(x->sizes(), x->scalar_type(), *x);
    }
    Bits y, norm;
    at::Tensor out, rstd;
    if (dense) out = new_empty(x->sizes(), x->scalar_type(), *x);
    else y.make(new_empty, *x);
    if (checkpoint) {
        norm.make(new_empty, *x);
        rstd = new_empty({rows}, at::kFloat, *x);
    }
    int status;
    {
        void* st = stream();
        Unlocked u;
        status = p_norm(ptr(*x), x->stride(0), residual ? ptr(*residual) : nullptr, residual ? residual->stride(0) : 0,
                        weight ? ptr(*weight) : nullptr, rows, cols, eps, dtype_code(*x), ptr_or_null(hidden), y.c(), y.s(),
                        ptr_or_null(out), norm.c(), norm.s(), (float*)ptr_or_null(rstd), st);
    }
    if (status != MXQ_OK) return PyLong_FromLong(status);
    PyObject* same = a[0];
    Py_INCREF(same);
    return tuple_as(nullptr, {dense ? wrapped(out) : q8(y), residual ? (Py_DECREF(same), wrapped(hidden)) : same,
                              checkpoint ? tuple_as(norm_class, {q8(norm), wrapped(rstd)}) : new_none()});
    END_HANDLE_TH_ERRORS
}

// add_rmsnorm_backward(dy, saved, weight, dhidden, dx_out, want_dweight)
PyObject* add_rmsnorm_backward(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor* dy = n == 6 && !modes_active() ? rows_of(a[0]) : nullptr;
    bool want;
    if (!dy || dtype_code(*dy) < 0 || !PyTuple_Check(a[1]) || PyTuple_GET_SIZE(a[1]) != 2 || !flag(a[5], &want)) return none();
    const int64_t rows = dy->size(0), cols = dy->size(1);
    Bits norm;
    const at::Tensor *rstd = whole(PyTuple_GET_ITEM(a[1], 1), {rows}, at::kFloat, dy->device()), *weight = nullptr, *dhidden = nullptr;
    if (cols % MXQ_Q8_BLOCK != 0 || !rstd || !norm.set(PyTuple_GET_ITEM(a[1], 0), rows, cols, dy->device())) return none();
    if (a[2] != Py_None && !(weight = whole(a[2], {cols}, dy->scalar_type(), dy->device()))) return none();
    if (a[3] != Py_None && (!(dhidden = rows_of(a[3])) || !like(dhidden, *dy))) return none();
    const at::Tensor* given = a[4] != Py_None ? whole(a[4], dy->sizes(), dy->scalar_type(), dy->device()) : nullptr;
    if (a[4] != Py_None && !given) return none();
    NewOutputs new_empty;
    const at::Tensor dx = given ? *given : new_empty(dy->sizes(), dy->scalar_type(), *dy);
    at::Tensor dweight, workspace;
    size_t bytes = 0;
    if (weight && want) {
        dweight = new_empty({cols}, at::kFloat, *dy);
        bytes = p_norm_back_size(rows, cols);
        workspace = new_empty({(int64_t)(bytes < 16 ? 16 : bytes)}, at::kByte, *dy);
    }
    int status;
    {
        void* st = stream();
        Unlocked u;
        status = p_norm_back(ptr(*dy), dy->stride(0), norm.c(), norm.s(), (const float*)ptr(*rstd), weight ? ptr(*weight) : nullptr,
                             dhidden ? ptr(*dhidden) : nullptr, dhidden ? dhidden->stride(0) : 0, rows, cols, dtype_code(*dy), ptr(dx),
                             (float*)ptr_or_null(dweight), ptr_or_null(workspace), bytes, st);
    }
    if (status != MXQ_OK) return PyLong_FromLong(status);
    return tuple_of({dx, dweight});
    END_HANDLE_TH_ERRORS
}

// swiglu(gate, up, dense, checkpoint)
PyObject* swiglu(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor* gate = n == 4 && !modes_active() ? rows_of(a[0]) : nullptr;
    const at::Tensor* up = gate ? rows_of(a[1]) : nullptr;
    bool dense, checkpoint;
    if (!up || dtype_code(*gate) < 0 || !like(up, *gate) || !flag(a[2], &dense) || !flag(a[3], &checkpoint) || gate->size(1) % MXQ_Q8_BLOCK != 0)
        return none();
    NewOutputs new_empty;
    Bits h, g, u8;
    at::Tensor out;
    if (dense) out = new_empty(gate->sizes(), gate->scalar_type(), *gate);
    else h.make(new_empty, *gate);
    if (checkpoint) {
        g.make(new_empty, *gate);
        u8.make(new_empty, *gate);
    }
    int status;
    {
        void* st = stream();
        Unlocked u;
        status = p_swiglu(ptr(*gate), gate->stride(0), ptr(*up), up->stride(0), gate->size(0), gate->size(1), dtype_code(*gate), h.c(), h.s(),
                          ptr_or_null(out), g.c(), g.s(), u8.c(), u8.s(), st);
    }
    if (status != MXQ_OK) return PyLong_FromLong(status);
    return tuple_as(nullptr, {dense ? wrapped(out) : q8(h), checkpoint ? tuple_as(swiglu_class, {q8(g), q8(u8)}) : new_none()});
    END_HANDLE_TH_ERRORS
}

// swiglu_backward(dh, saved, again)
PyObject* swiglu_backward(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor* dh = n == 3 && !modes_active() ? rows_of(a[0]) : nullptr;
    bool again;
    if (!dh || dtype_code(*dh) < 0 || !PyTuple_Check(a[1]) || PyTuple_GET_SIZE(a[1]) != 2 || !flag(a[2], &again)) return none();
    const int64_t rows = dh->size(0), cols = dh->size(1);
    Bits g, u8;
    if (cols % MXQ_Q8_BLOCK != 0 || !g.set(PyTuple_GET_ITEM(a[1], 0), rows, cols, dh->device()) ||
        !u8.set(PyTuple_GET_ITEM(a[1], 1), rows, cols, dh->device()))
        return none();
    NewOutputs new_empty;
    const at::Tensor both = new_empty({rows, 2 * cols}, dh->scalar_type(), *dh), dgate = both.narrow(1, 0, cols), dup = both.narrow(1, cols, cols);
    at::Tensor h;
    if (again) h = new_empty(dh->sizes(), dh->scalar_type(), *dh);
    int status;
    {
        void* st = stream();
        Unlocked u;
        status = p_swiglu_back(ptr(*dh), dh->stride(0), g.c(), g.s(), u8.c(), u8.s(), rows, cols, dtype_code(*dh), dgate.data_ptr(), 2 * cols,
                               dup.data_ptr(), 2 * cols, ptr_or_null(h), st);
    }
    if (status != MXQ_OK) return PyLong_FromLong(status);
    return tuple_of({dgate, dup, h});
    END_HANDLE_TH_ERRORS
}

// linear(x, w, adapters, ids, out_dtype, sums), the output made here
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 6 || modes_active() || !PyTuple_Check(a[1]) || PyTuple_GET_SIZE(a[1]) != 5 || !THPDtype_Check(a[4])) return none();
    mxq_linear_args g = {};
    if (!integer(a[5], 0, 255, &g.sums)) return none();
    const at::Tensor* x = nullptr;
    Bits bits;
    if (PyTuple_Check(a[0])) {
        const at::Tensor* c = PyTuple_GET_SIZE(a[0]) == 2 ? plain(PyTuple_GET_ITEM(a[0], 0)) : nullptr;
        if (!c || c->dim() != 2 || !bits.set(a[0], c->size(0), c->size(1), c->device())) return none();
        x = &bits.codes;
        g.x_codes = bits.c();
        g.x_scales = bits.s();
    } else {
        x = rows_of(a[0]);
        if (!x || x->scalar_type() != at::kBFloat16) return none();
        g.x = ptr(*x);
        g.ld_x = x->stride(0);
    }
    const at::Device device = x->device();
    g.m = x->size(0);
    g.k = x->size(1);
    const at::Tensor* codes = plain(PyTuple_GET_ITEM(a[1], 0));
    if (!codes || codes->dim() != 2 || codes->scalar_type() != at::kByte || codes->device() != device || codes->size(1) != g.k / 2) return none();
    g.n = codes->size(0);
    if (!block_size(PyTuple_GET_ITEM(a[1], 2), &g.block) || !integer(PyTuple_GET_ITEM(a[1], 3), 0, 255, &g.scale_fmt)) return none();
    const at::Tensor* scales = whole(PyTuple_GET_ITEM(a[1], 1), {g.n, g.k / g.block}, at::kByte, device);
    if (!scales) return none();
    g.w_codes = (const uint8_t*)ptr(*codes);
    g.w_scales = (const uint8_t*)ptr(*scales);
    g.tensor_scale = 1.0f;
    if (!number(PyTuple_GET_ITEM(a[1], 4), &g.tensor_scale)) {
        const at::Tensor* t = buffer(PyTuple_GET_ITEM(a[1], 4), 4, at::kFloat);
        if (!t) return none();
        g.tensor_scale_dev = (const float*)ptr(*t);
    }
    if (a[2] != Py_None) {
        if (!PyTuple_Check(a[2]) || PyTuple_GET_SIZE(a[2]) != 3) return none();
        const at::Tensor* A = plain(PyTuple_GET_ITEM(a[2], 0));
        if (!A || A->dim() != 3 || A->scalar_type() != at::kBFloat16 || A->device() != device || A->size(2) != g.k) return none();
        const int64_t count = A->size(0), rank = A->size(1);
        const at::Tensor* B = whole(PyTuple_GET_ITEM(a[2], 1), {count, g.n, rank}, at::kBFloat16, device);
        const at::Tensor* s = whole(PyTuple_GET_ITEM(a[2], 2), {count}, at::kFloat, device);
        if (!B || !s || count < 1 || count > INT32_MAX || rank > 64 || (a[3] == Py_None && count != 1)) return none();
        if (a[3] != Py_None) {
            const at::Tensor* ids = whole(a[3], {g.m}, at::kInt, device);
            if (!ids) return none();
            g.adapter_ids = (const int32_t*)ptr(*ids);
        }
        g.adapter_a = ptr(*A);
        g.adapter_b = ptr(*B);
        g.adapter_scaling = (const float*)ptr(*s);
        g.adapter_count = (int)count;
        g.adapter_rank = (int)rank;
    } else if (a[3] != Py_None) {
        return none();
    }
    const at::ScalarType type = reinterpret_cast<THPDtype*>(a[4])->scalar_type;
    if (type != at::kBFloat16 && type != at::kFloat) return none();
    NewOutputs new_empty;
    const at::Tensor y = new_empty({g.m, g.n}, type, *x);
    g.y = ptr(y);
    g.ld_y = g.n;
    g.y_dtype = dtype_code(y);
    at::Tensor workspace;
    g.workspace_bytes = p_linear_size(&g);
    if (g.workspace_bytes > 0) {
        workspace = new_empty({(int64_t)g.workspace_bytes}, at::kByte, *x);
        g.workspace = ptr(workspace);
    }
    int status;
    {
        void* st = stream();
        Unlocked u;
        status = p_linear(&g, st);
    }
    return status != MXQ_OK ? PyLong_FromLong(status) : wrapped(y);
    END_HANDLE_TH_ERRORS
}

// built_for(): as in binding.cpp
PyObject* built_for(PyObject*, PyObject*) { return Py_BuildValue("(ss)", MXQ_CALLS_ABI, MXQ_HEADER_ID); }

// use(seven addresses in the order of the declarations above, Q8, SavedNorm, SavedSwiglu)
PyObject* use(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    void* p[7];
    if (n != 10) { PyErr_SetString(PyExc_TypeError, "seven addresses and three classes"); return nullptr; }
    for (int i = 0; i < 7; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address"); return nullptr; }
    }
    p_norm = (decltype(p_norm))p[0];
    p_norm_back = (decltype(p_norm_back))p[1];
    p_norm_back_size = (decltype(p_norm_back_size))p[2];
    p_swiglu = (decltype(p_swiglu))p[3];
    p_swiglu_back = (decltype(p_swiglu_back))p[4];
    p_linear = (decltype(p_linear))p[5];
    p_linear_size = (decltype(p_linear_size))p[6];
    q8_class = a[7];
    norm_class = a[8];
    swiglu_class = a[9];
    for (int i = 7; i < 10; ++i) Py_INCREF(a[i]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {MXQ_METHOD(add_rmsnorm), MXQ_METHOD(add_rmsnorm_backward), MXQ_METHOD(swiglu), MXQ_METHOD(swiglu_backward),
                         MXQ_METHOD(linear), MXQ_METHOD(use), {"built_for", built_for, METH_NOARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_mxq_layer_calls", "The calls of layers.py in native code.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__mxq_layer_calls(void) { return PyModule_Create(&module); }
