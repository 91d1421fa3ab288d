// What the native halves of the Python binding share: checks of tensor arguments, outputs, workspaces, streams, results.
#pragma once

#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/ssm_learn.h"

namespace {

constexpr auto F32 = c10::kFloat;
constexpr auto C64 = c10::kComplexFloat;
constexpr auto U8 = c10::kByte;

// One tensor argument.  ok: absent where that is allowed, or a contiguous GPU tensor of the type and shape wanted.
struct Arg {
    const at::Tensor *t = nullptr;
    bool none = false, bad = false;
    explicit Arg(PyObject *o)
    {
        if (o == Py_None) none = true;
        else if (THPVariable_Check(o)) t = &THPVariable_Unpack(o);
        else bad = true;
    }
    bool is(c10::ScalarType dt, std::initializer_list<int64_t> shape, bool optional = false) const
    {
        if (none) return optional;
        return !bad && t->is_cuda() && t->scalar_type() == dt && t->sizes() == c10::IntArrayRef(shape.begin(), shape.size()) &&
               t->is_contiguous();
    }
    int64_t dim() const { return t ? t->dim() : -1; }
    int64_t size(int i) const { return t->size(i); }
    template <class T> T *ptr() const { return t ? static_cast<T *>(t->data_ptr()) : nullptr; }
    const ssm_c64 *c64() const { return ptr<const ssm_c64>(); }
    const float *f32() const { return ptr<const float>(); }
    const uint8_t *u8() const { return ptr<const uint8_t>(); }
};

at::Tensor empty(std::initializer_list<int64_t> shape, c10::ScalarType dt, const at::Tensor &like)
{
    return at::Tensor(at::detail::empty_cuda(c10::IntArrayRef(shape.begin(), shape.size()), dt, like.device(), std::nullopt));
}
template <class T> T *raw(const at::Tensor &t) { return t.defined() ? static_cast<T *>(t.data_ptr()) : nullptr; }
ssm_c64 *c64(const at::Tensor &t) { return raw<ssm_c64>(t); }
float *f32(const at::Tensor &t) { return raw<float>(t); }

// An output: the caller's tensor when there is one, else a new one when it is wanted.
at::Tensor output(PyObject *given, bool wanted, std::initializer_list<int64_t> shape, c10::ScalarType dt, const at::Tensor &like, bool &bad)
{
    if (given && given != Py_None) {
        if (!THPVariable_Check(given)) { bad = true; return at::Tensor(); }
        return THPVariable_Unpack(given);
    }
    return wanted ? empty(shape, dt, like) : at::Tensor();
}

// A caller's workspace has to be memory of the GPU, all of its elements next to each other: its address goes to kernels.
bool workspace_ok(const Arg &given) { return given.t && given.t->is_cuda() && given.t->is_contiguous(); }

// The workspace: the caller's, or one of n bytes that lives until the call returns (its kernels are queued on the
// stream it was allocated on, so the allocator hands the block out again behind them).
struct Workspace {
    at::Tensor own;
    void *p = nullptr;
    size_t n = 0;
    bool bad = false;
    Workspace(const Arg &given, size_t need, const at::Tensor &like)
    {
        if (given.none) {
            if (need == 0) { bad = true; return; }
            own = empty({(int64_t)need}, U8, like);
            p = own.data_ptr(); n = need;
        } else if (workspace_ok(given)) {
            p = given.t->data_ptr(); n = (size_t)given.t->numel();
        } else {
            bad = true;
        }
    }
};

// Raw handle of the stream: the one given (an int), or the current one.  A workspace of this call's own is only
// allocated for the current stream.
bool stream_of(PyObject *o, const Arg *workspace, void *&s)
{
    if (o == Py_None) { s = c10::hip::getCurrentHIPStream().stream(); return true; }
    if (workspace && workspace->none) return false;
    s = PyLong_AsVoidPtr(o);
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}
bool yes(PyObject *o)
{
    if (o == Py_True || o == Py_False) return o == Py_True;
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();                 // (its error is the caller's)
    return v > 0;
}

PyObject *wrap(const at::Tensor &t)
{
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
struct Named { const char *name; const at::Tensor *t; };
PyObject *dict(std::initializer_list<Named> items)
{
    PyObject *d = PyDict_New();
    for (const Named &i : items) {
        PyObject *v = wrap(*i.t);
        PyDict_SetItemString(d, i.name, v);
        Py_DECREF(v);
    }
    return d;
}
PyObject *tuple(std::initializer_list<const at::Tensor *> items)
{
    PyObject *r = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t k = 0;
    for (const at::Tensor *t : items) PyTuple_SET_ITEM(r, k++, wrap(*t));
    return r;
}
PyObject *item(PyObject *d, const char *key) { return d == Py_None ? nullptr : PyDict_GetItemString(d, key); }

// The C call without the interpreter's lock.  Its arguments are values by then: taking a tensor's data pointer can throw (a
// tensor without storage, for instance a batched one), and an exception must find the lock held.
template <class... P, class... A>
ssm_status call_without_gil(ssm_status (*entry)(P...), A... args)
{
    static_assert(sizeof...(P) == sizeof...(A) && (std::is_trivially_copyable_v<A> && ...), "pointers and numbers");
    ssm_status rc;
    Py_BEGIN_ALLOW_THREADS
    rc = entry(args...);
    Py_END_ALLOW_THREADS
    return rc;
}

#define GENERAL_PATH_UNLESS(cond) do { if (!(cond)) Py_RETURN_NONE; } while (0)
#define CALL(...) \
    const ssm_status rc = call_without_gil(__VA_ARGS__); \
    if (rc != SSM_OK) return PyLong_FromLong((long)rc)
#define ENTRY(name) PyObject *name(PyObject *, PyObject *const *a, Py_ssize_t n)
// (torch's own translation: an allocation that fails raises torch.OutOfMemoryError here as on the general path)
#define TRY_BEGIN HANDLE_TH_ERRORS
#define TRY_END END_HANDLE_TH_ERRORS

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(name)), METH_FASTCALL, nullptr}

}  // namespace
