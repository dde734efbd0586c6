// The usual calls of binding.py in native code.  A small call is bound by the host: of the 6.6 us that one
// spinner_apply_signs took through ctypes (27 us for a layer's forward and backward), 3.2 us are the launch; tensor
// checks, the allocation through torch's Python face and the marshalling of a dozen arguments were the rest.
//
// Each function takes the arguments of its namesake in binding.py, all of them, by position, and returns its result, or
// None when anything about the call is out of the ordinary: a tensor that is no plain contiguous CUDA tensor of the
// type and size expected, a number that is no Python number, an explicit stream, a status that the library finds before it
// launches anything.  binding.py then takes the call its long way, which knows every check and error.  SPINNER_ERR_HIP
// alone may come with kernels already on their way: that call is not made again, its SpinnerError is raised from here.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPStream.h>
#include <pybind11/pybind11.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "spinner.h"

namespace {

using at::Tensor;

// a plain tensor on a GPU with memory of its own (subclasses and wrapped tensors go the long way)
const Tensor* gpu_tensor(PyObject* o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const Tensor& t = THPVariable_Unpack(o);
    return t.has_storage() && t.is_cuda() && t.is_contiguous() ? &t : nullptr;
}
const Tensor* typed_tensor(PyObject* o, at::ScalarType type)
{
    const Tensor* t = gpu_tensor(o);
    return t && t->scalar_type() == type ? t : nullptr;
}
const Tensor* floats(PyObject* o) { return typed_tensor(o, at::kFloat); }
const Tensor* floats(PyObject* o, int64_t count)
{
    const Tensor* t = floats(o);
    return t && t->numel() == count ? t : nullptr;
}
// rows [batch][n]; n has to fit the int of the C ABI
const Tensor* rows(PyObject* o, long* batch, int* n)
{
    const Tensor* t = floats(o);
    if (!t || t->dim() != 2 || t->size(1) > INT_MAX) return nullptr;
    *batch = (long)t->size(0);
    *n = (int)t->size(1);
    return t;
}
bool whole(PyObject* o, int* v)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    const long l = PyLong_AsLongAndOverflow(o, &overflow);
    if (overflow || l < INT_MIN || l > INT_MAX) return false;
    *v = (int)l;
    return true;
}
// the number of kept rows: None stands for n
bool kept(PyObject* o, int n, int* m)
{
    if (o == Py_None) *m = n;
    else if (!whole(o, m)) return false;
    return *m >= 1 && *m <= n;
}
bool number(PyObject* o, float* v)
{
    if (PyFloat_CheckExact(o)) { *v = (float)PyFloat_AS_DOUBLE(o); return true; }
    int i;
    if (!whole(o, &i)) return false;
    *v = (float)i;
    return true;
}
bool choice(PyObject* o, const char* const* names, int count, int* v)
{
    if (PyUnicode_CheckExact(o)) {
        for (int i = 0; i < count; ++i)
            if (PyUnicode_CompareWithASCIIString(o, names[i]) == 0) { *v = i; return true; }
        return false;
    }
    return whole(o, v) && *v >= 0 && *v < count;
}
bool epilogue(PyObject* o, int* v)
{
    static const char* const names[] = {"none", "cossin"};
    static_assert(SPINNER_EPI_NONE == 0 && SPINNER_EPI_COSSIN == 1, "the order of the names");
    return choice(o, names, 2, v);
}
bool struct_kind(PyObject* o, int* v)
{
    static const char* const names[] = {"circulant", "skew_circulant", "toeplitz", "hankel"};
    static_assert(SPINNER_STRUCT_CIRCULANT == 0 && SPINNER_STRUCT_SKEW_CIRCULANT == 1 && SPINNER_STRUCT_TOEPLITZ == 2 &&
                      SPINNER_STRUCT_HANKEL == 3, "the order of the names");
    return choice(o, names, 4, v);
}

// Memory that the caller may bring: `given` is null where the argument was None, and is checked by usable() before anything
// is allocated.
struct Buffer {
    const Tensor* given = nullptr;
    bool usable(PyObject* o, at::ScalarType type, int64_t count)
    {
        if (o == Py_None) return true;
        given = typed_tensor(o, type);
        return given && given->numel() == count;
    }
    bool usable_bytes(PyObject* o, size_t need)
    {
        if (o == Py_None) return true;
        given = gpu_tensor(o);
        return given && (size_t)given->nbytes() >= need;
    }
    Tensor get(at::IntArrayRef sizes, at::ScalarType type, const Tensor& like) const
    {
        return given ? *given : at::empty(sizes, at::TensorOptions().dtype(type).device(like.device()));
    }
    // scratch: no tensor at all where none is needed
    Tensor scratch(size_t need, const Tensor& like) const
    {
        return given || need ? get({(int64_t)need}, at::kByte, like) : Tensor();
    }
};
template <typename T = float>
T* ptr(const Tensor& t) { return t.defined() ? static_cast<T*>(t.data_ptr()) : nullptr; }
template <typename T = float>
T* ptr(const Tensor* t) { return t ? static_cast<T*>(t->data_ptr()) : nullptr; }
void* current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// packed sign words of `count` triples from triple `first` on
const void* sign_words(PyObject* o, int n, int first, int count)
{
    const Tensor* t = typed_tensor(o, at::kByte);
    const size_t one = spinner_signs_bytes(n, 1);
    if (!t || one == 0 || first < 0 || count < 1 || (size_t)t->numel() < ((size_t)first + count) * one) return nullptr;
    return static_cast<const char*>(t->data_ptr()) + first * one;
}

// a status other than SPINNER_OK: the long way, or the error itself
PyObject* refused(int rc)
{
    if (rc != SPINNER_ERR_HIP) Py_RETURN_NONE;
    const auto error = pybind11::module_::import("paper_1610_06209_amd.binding").attr("SpinnerError");
    PyErr_SetObject(error.ptr(), error(rc).ptr());
    return nullptr;
}

using Args = PyObject* const*;
#define LONG_WAY Py_RETURN_NONE
#define ENTRY(NAME, COUNT)                                                          \
    PyObject* NAME(PyObject*, Args a, Py_ssize_t given)                             \
    {                                                                               \
        HANDLE_TH_ERRORS                                                            \
        if (given != COUNT) { PyErr_SetString(PyExc_TypeError, #NAME ": " #COUNT " arguments"); return nullptr; }
#define ENTRY_END                                                                   \
        END_HANDLE_TH_ERRORS                                                        \
    }

// Memory of a stream that is not the current one: sizes, dtype, device, handle of the stream, whether it is scratch.  A result is noted as used on the
// current stream too.  (The same from Python, with torch's context of a stream, takes 12 us a tensor.)
ENTRY(_new_on, 5)
    int device;
    if (!PyTuple_Check(a[0]) || !THPDtype_Check(a[1]) || !whole(a[2], &device)) { PyErr_SetString(PyExc_TypeError, "_new_on: sizes, dtype, device, stream, scratch"); return nullptr; }
    std::vector<int64_t> sizes;
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(a[0]); ++i) sizes.push_back(PyLong_AsLongLong(PyTuple_GET_ITEM(a[0], i)));
    void* handle = PyLong_AsVoidPtr(a[3]);
    if (PyErr_Occurred()) return nullptr;
    const at::ScalarType type = reinterpret_cast<THPDtype*>(a[1])->scalar_type;
    const bool scratch = PyObject_IsTrue(a[4]);
    Tensor t;
    {
        pybind11::gil_scoped_release free;
        const auto current = c10::hip::getCurrentHIPStream((c10::DeviceIndex)device);
        struct Back {
            c10::hip::HIPStream to;
            ~Back() { c10::hip::setCurrentHIPStream(to); }
        } back{current};
        c10::hip::setCurrentHIPStream(handle ? c10::hip::getStreamFromExternal(static_cast<hipStream_t>(handle), (c10::DeviceIndex)device)
                                             : c10::hip::getDefaultHIPStream((c10::DeviceIndex)device));
        t = at::empty(sizes, at::TensorOptions().dtype(type).device(at::kCUDA, (c10::DeviceIndex)device));
        if (!scratch) c10::hip::HIPCachingAllocator::recordStream(t.storage().data_ptr(), current);
    }
    return THPVariable_Wrap(std::move(t));
ENTRY_END

// x, signs, m, epilogue, scale, out, workspace, stream, triple
ENTRY(apply_signs, 9)
    long batch;
    int n, m, epi, triple;
    float scale;
    const Tensor* x = rows(a[0], &batch, &n);
    if (!x || a[7] != Py_None || !kept(a[2], n, &m) || !epilogue(a[3], &epi) || !number(a[4], &scale) || !whole(a[8], &triple)) LONG_WAY;
    const void* words = sign_words(a[1], n, triple, 1);
    const int64_t width = epi == SPINNER_EPI_COSSIN ? 2LL * m : m;
    const size_t need = spinner_workspace_bytes(n, batch, m, epi);
    Buffer o, w;
    if (!words || !o.usable(a[5], at::kFloat, batch * width) || !w.usable_bytes(a[6], need)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = o.get({batch, width}, at::kFloat, *x);
        const Tensor ws = w.scratch(need, *x);
        rc = spinner_apply_signs(ptr(x), n, batch, words, m, epi, scale, ptr(out), ptr<void>(ws), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// x, d1, d2, d3, m, epilogue, scale, out, workspace, stream
ENTRY(apply, 10)
    long batch;
    int n, m, epi;
    float scale;
    const Tensor* x = rows(a[0], &batch, &n);
    if (!x || a[9] != Py_None || !kept(a[4], n, &m) || !epilogue(a[5], &epi) || !number(a[6], &scale)) LONG_WAY;
    const Tensor *d1 = floats(a[1], n), *d2 = floats(a[2], n), *d3 = floats(a[3], n);
    const int64_t width = epi == SPINNER_EPI_COSSIN ? 2LL * m : m;
    const size_t need = spinner_workspace_bytes(n, batch, m, epi);
    Buffer o, w;
    if (!d1 || !d2 || !d3 || !o.usable(a[7], at::kFloat, batch * width) || !w.usable_bytes(a[8], need)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = o.get({batch, width}, at::kFloat, *x);
        const Tensor ws = w.scratch(need, *x);
        rc = spinner_apply(ptr(x), n, batch, ptr(d1), ptr(d2), ptr(d3), m, epi, scale, ptr(out), ptr<void>(ws), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// x, diag_sets, m, epilogue, scale, out, workspace, stream
ENTRY(apply_blocks, 8)
    long batch;
    int n, m, epi;
    float scale;
    const Tensor *x = rows(a[0], &batch, &n), *d = floats(a[1]);
    if (!x || !d || a[7] != Py_None || !kept(a[2], n, &m) || !epilogue(a[3], &epi) || !number(a[4], &scale)) LONG_WAY;
    if (d->dim() != 3 || d->size(0) > INT_MAX || d->size(1) != 3 || d->size(2) != n) LONG_WAY;
    const int L = (int)d->size(0);
    const int64_t width = (epi == SPINNER_EPI_COSSIN ? 2LL * m : m) * L;
    const size_t need = spinner_blocks_workspace_bytes(n, batch, m, epi);
    Buffer o, w;
    if (!o.usable(a[5], at::kFloat, batch * width) || !w.usable_bytes(a[6], need)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = o.get({batch, width}, at::kFloat, *x);
        const Tensor ws = w.scratch(need, *x);
        rc = spinner_apply_blocks(ptr(x), n, batch, L, ptr(d), m, epi, scale, ptr(out), ptr<void>(ws), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// x, diag_sets, out_idx, stream
ENTRY(hash, 4)
    long batch;
    int n;
    const Tensor *x = rows(a[0], &batch, &n), *d = floats(a[1]);
    if (!x || !d || a[3] != Py_None || d->dim() != 3 || d->size(0) > INT_MAX || d->size(1) != 3 || d->size(2) != n) LONG_WAY;
    const int L = (int)d->size(0);
    Buffer o;
    if (!o.usable(a[2], at::kInt, (int64_t)batch * L)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = o.get({batch, L}, at::kInt, *x);
        rc = spinner_hash(ptr(x), n, batch, L, ptr(d), ptr<int>(out), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// x, signs, L, out_idx, stream
ENTRY(hash_signs, 5)
    long batch;
    int n, L;
    const Tensor* x = rows(a[0], &batch, &n);
    if (!x || a[4] != Py_None || !whole(a[2], &L)) LONG_WAY;
    const void* words = sign_words(a[1], n, 0, L);
    Buffer o;
    if (!words || !o.usable(a[3], at::kInt, (int64_t)batch * L)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = o.get({batch, L}, at::kInt, *x);
        rc = spinner_hash_signs(ptr(x), n, batch, L, words, ptr<int>(out), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// x, d1, d2, d3, m, codes, workspace, stream
ENTRY(sign_codes, 8)
    long batch;
    int n, m;
    const Tensor* x = rows(a[0], &batch, &n);
    if (!x || a[7] != Py_None || !kept(a[4], n, &m) || spinner_code_bytes(m) == 0) LONG_WAY;
    const Tensor *d1 = floats(a[1], n), *d2 = floats(a[2], n), *d3 = floats(a[3], n);
    const int64_t words = (int64_t)spinner_code_bytes(m) / 8;
    const size_t need = spinner_codes_workspace_bytes(n, batch);
    Buffer o, w;
    if (!d1 || !d2 || !d3 || !o.usable(a[5], at::kLong, batch * words) || !w.usable_bytes(a[6], need)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = o.get({batch, words}, at::kLong, *x);
        const Tensor ws = w.scratch(need, *x);
        rc = spinner_sign_codes(ptr(x), n, batch, ptr(d1), ptr(d2), ptr(d3), m, ptr<void>(out), ptr<void>(ws), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// x, signs, m, codes, workspace, stream, triple
ENTRY(sign_codes_signs, 7)
    long batch;
    int n, m, triple;
    const Tensor* x = rows(a[0], &batch, &n);
    if (!x || a[5] != Py_None || !kept(a[2], n, &m) || spinner_code_bytes(m) == 0 || !whole(a[6], &triple)) LONG_WAY;
    const void* signs = sign_words(a[1], n, triple, 1);
    const int64_t words = (int64_t)spinner_code_bytes(m) / 8;
    const size_t need = spinner_codes_workspace_bytes(n, batch);
    Buffer o, w;
    if (!signs || !o.usable(a[3], at::kLong, batch * words) || !w.usable_bytes(a[4], need)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = o.get({batch, words}, at::kLong, *x);
        const Tensor ws = w.scratch(need, *x);
        rc = spinner_sign_codes_signs(ptr(x), n, batch, signs, m, ptr<void>(out), ptr<void>(ws), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// codes_a, codes_b, m, out, stream
ENTRY(angular_gram, 5)
    int m;
    const Tensor *p = typed_tensor(a[0], at::kLong), *q = typed_tensor(a[1], at::kLong);
    if (!p || !q || a[4] != Py_None || !whole(a[2], &m) || spinner_code_bytes(m) == 0) LONG_WAY;
    const int64_t words = (int64_t)spinner_code_bytes(m) / 8;
    if (p->dim() != 2 || q->dim() != 2 || p->size(1) != words || q->size(1) != words) LONG_WAY;
    const long na = (long)p->size(0), nb = (long)q->size(0);
    Buffer o;
    if (!o.usable(a[3], at::kFloat, (int64_t)na * nb)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = o.get({na, nb}, at::kFloat, *p);
        rc = spinner_angular_gram(ptr<void>(p), na, ptr<void>(q), nb, m, ptr(out), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// x, d1, d2, d3, scale, y, saved, stream
ENTRY(layer_forward, 8)
    long batch;
    int n;
    float scale;
    const Tensor* x = rows(a[0], &batch, &n);
    if (!x || a[7] != Py_None || !number(a[4], &scale)) LONG_WAY;
    const Tensor *d1 = floats(a[1], n), *d2 = floats(a[2], n), *d3 = floats(a[3], n);
    Buffer o, s;
    if (!d1 || !d2 || !d3 || !o.usable(a[5], at::kFloat, (int64_t)batch * n) || !s.usable(a[6], at::kFloat, 2LL * batch * n)) LONG_WAY;
    Tensor y, saved;
    int rc;
    {
        pybind11::gil_scoped_release free;
        y = o.get({batch, n}, at::kFloat, *x);
        saved = s.get({2, batch, n}, at::kFloat, *x);
        rc = spinner_layer_forward(ptr(x), n, batch, ptr(d1), ptr(d2), ptr(d3), scale, ptr(y), ptr<void>(saved), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(y)), THPVariable_Wrap(std::move(saved)));
ENTRY_END

// dy, x, saved, d1, d2, d3, scale, dx, dd, workspace, stream
ENTRY(layer_backward, 11)
    long batch, dy_batch;
    int n, dy_n;
    float scale;
    const Tensor *dy = rows(a[0], &dy_batch, &dy_n), *x = rows(a[1], &batch, &n);
    if (!dy || !x || dy_batch != batch || dy_n != n || a[10] != Py_None || !number(a[6], &scale)) LONG_WAY;
    const Tensor *saved = floats(a[2], 2LL * batch * n), *d1 = floats(a[3], n), *d2 = floats(a[4], n), *d3 = floats(a[5], n);
    size_t need = spinner_layer_workspace_bytes(n, batch);
    Buffer o, g, w;
    if (!saved || !d1 || !d2 || !d3 || !o.usable(a[7], at::kFloat, (int64_t)batch * n) || !g.usable(a[8], at::kFloat, 3LL * n) ||
        !w.usable_bytes(a[9], need))
        LONG_WAY;
    Tensor dx, dd;
    int rc;
    {
        pybind11::gil_scoped_release free;
        dx = o.get({batch, n}, at::kFloat, *x);
        dd = g.get({3, n}, at::kFloat, *x);
        const Tensor ws = w.scratch(need < 16 ? 16 : need, *x);
        rc = spinner_layer_backward(ptr(dy), ptr(x), ptr<void>(saved), n, batch, ptr(d1), ptr(d2), ptr(d3), scale, ptr(dx), ptr(dd),
                                    ptr<void>(ws), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(dx)), THPVariable_Wrap(std::move(dd)));
ENTRY_END

// A, w, d1, d2, d3, m, scale, out, workspace, stream
ENTRY(sketch, 10)
    long n_rows;
    int d, m;
    float scale;
    const Tensor* A = rows(a[0], &n_rows, &d);
    if (!A || n_rows > INT_MAX || a[9] != Py_None || !kept(a[5], (int)n_rows, &m) || !number(a[6], &scale)) LONG_WAY;
    const int n = (int)n_rows;
    const Tensor *weights = a[1] == Py_None ? nullptr : floats(a[1], n), *d1 = floats(a[2], n), *d2 = floats(a[3], n), *d3 = floats(a[4], n);
    const size_t need = spinner_sketch_workspace_bytes(n, d, m);
    Buffer o, w;
    if ((!weights && a[1] != Py_None) || !d1 || !d2 || !d3 || !o.usable(a[7], at::kFloat, (int64_t)m * d) || !w.usable_bytes(a[8], need))
        LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = o.get({m, d}, at::kFloat, *A);
        const Tensor ws = w.scratch(need < 16 ? 16 : need, *A);
        rc = spinner_sketch(ptr(A), n, d, ptr(weights), ptr(d1), ptr(d2), ptr(d3), m, scale, ptr(out), ptr<void>(ws), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// B, out, workspace, stream
ENTRY(sketch_gram, 4)
    long m_rows;
    int d;
    const Tensor* B = rows(a[0], &m_rows, &d);
    if (!B || m_rows > INT_MAX || a[3] != Py_None) LONG_WAY;
    const int m = (int)m_rows;
    const size_t need = spinner_sketch_gram_workspace_bytes(m, d);
    Buffer o, w;
    if (!o.usable(a[1], at::kFloat, (int64_t)d * d) || !w.usable_bytes(a[2], need)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = o.get({d, d}, at::kFloat, *B);
        const Tensor ws = w.scratch(need, *B);
        rc = spinner_sketch_gram(ptr(B), m, d, ptr(out), ptr<void>(ws), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// x, kind, spectrum, d1, d2, m, scale, out, workspace, stream
ENTRY(struct_apply_ws, 10)
    long batch;
    int n, m, kind;
    float scale;
    const Tensor *x = rows(a[0], &batch, &n), *spectrum = gpu_tensor(a[2]);
    if (!x || !spectrum || a[9] != Py_None || !struct_kind(a[1], &kind) || !kept(a[5], n, &m) || !number(a[6], &scale)) LONG_WAY;
    const Tensor *d1 = floats(a[3], n), *d2 = floats(a[4], n);
    const size_t need = spinner_struct_workspace_bytes(kind, n, batch);
    Buffer o, w;
    if ((size_t)spectrum->nbytes() < spinner_struct_spectrum_bytes(kind, n) || !d1 || !d2 || !o.usable(a[7], at::kFloat, (int64_t)batch * m) || !w.usable_bytes(a[8], need)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = o.get({batch, m}, at::kFloat, *x);
        const Tensor ws = w.scratch(need, *x);
        rc = spinner_struct_apply_ws(ptr(x), n, batch, kind, ptr<void>(spectrum), ptr(d1), ptr(d2), m, scale, ptr(out), ptr<void>(ws),
                                     current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// ---- 4-bit numbers and products of rows grouped by expert
bool element_type(at::ScalarType t, int* code)
{
    if (t == at::kFloat) *code = SPINNER_F32;
    else if (t == at::kBFloat16) *code = SPINNER_BF16;
    else if (t == at::kHalf) *code = SPINNER_F16;
    else return false;
    return true;
}
bool dtype_of(PyObject* o, at::ScalarType* type, int* code)
{
    if (!THPDtype_Check(o)) return false;
    *type = reinterpret_cast<THPDtype*>(o)->scalar_type;
    return element_type(*type, code);
}
// a contiguous tensor on the GPU that the call runs on
const Tensor* here(PyObject* o)
{
    const Tensor* t = gpu_tensor(o);
    return t && t->get_device() == c10::hip::current_device() ? t : nullptr;
}
const Tensor* here(PyObject* o, at::ScalarType type)
{
    const Tensor* t = here(o);
    return t && t->scalar_type() == type ? t : nullptr;
}
// rows of plain numbers
const Tensor* number_rows(PyObject* o, long* count, int* width, int* code)
{
    const Tensor* t = here(o);
    if (!t || t->dim() != 2 || t->size(1) > INT_MAX || !element_type(t->scalar_type(), code)) return nullptr;
    *count = (long)t->size(0);
    *width = (int)t->size(1);
    return t;
}
const Tensor* byte_rows(PyObject* o, long count, int64_t width)
{
    const Tensor* t = here(o, at::kByte);
    return t && t->dim() == 2 && t->size(0) == count && t->size(1) == width ? t : nullptr;
}
// [n][k] or [experts][n][k]
bool weights(const Tensor* t, int* experts, int* n, int64_t* k)
{
    if (!t || (t->dim() != 2 && t->dim() != 3) || t->size(-2) > INT_MAX || t->size(0) > INT_MAX) return false;
    *experts = t->dim() == 3 ? (int)t->size(0) : 1;
    *n = (int)t->size(-2);
    *k = t->size(-1);
    return true;
}
bool expert_ends(PyObject* o, int experts, const long long** ends)
{
    *ends = nullptr;
    if (o == Py_None) return experts == 1;
    const Tensor* t = here(o, at::kLong);
    if (!t || t->dim() != 1 || t->numel() != experts) return false;
    *ends = static_cast<const long long*>(t->data_ptr());
    return true;
}
bool result_rows(PyObject* o, const Tensor** given, at::ScalarType type, long count, int width)
{
    *given = nullptr;
    if (o == Py_None) return true;
    const Tensor* t = here(o, type);
    if (!t || t->dim() != 2 || t->size(0) != count || t->size(1) != width) return false;
    *given = t;
    return true;
}
Tensor result(const Tensor* given, at::IntArrayRef sizes, at::ScalarType type, const Tensor& like)
{
    return given ? *given : at::empty(sizes, at::TensorOptions().dtype(type).device(like.device()));
}
bool rotation(PyObject* diag, PyObject* block, int k, const Tensor** d, int* b)
{
    *d = nullptr;
    if (!whole(block, b)) return false;
    if (diag == Py_None) return true;
    *d = here(diag, at::kFloat);
    return *d && (*d)->dim() == 1 && (*d)->numel() == k;
}

// x, diag, block, codes, scales, stream
ENTRY(mx_quantize, 6)
    long count;
    int k, code, block;
    const Tensor *x = number_rows(a[0], &count, &k, &code), *d, *gc = nullptr, *gs = nullptr;
    if (!x || a[5] != Py_None || k % 32 || !rotation(a[1], a[2], k, &d, &block)) LONG_WAY;
    if (a[3] != Py_None && !(gc = byte_rows(a[3], count, k / 2))) LONG_WAY;
    if (a[4] != Py_None && !(gs = byte_rows(a[4], count, k / 32))) LONG_WAY;
    Tensor codes, scales;
    int rc;
    {
        pybind11::gil_scoped_release free;
        codes = result(gc, {count, k / 2}, at::kByte, *x);
        scales = result(gs, {count, k / 32}, at::kByte, *x);
        rc = spinner_mx_quantize(ptr<void>(x), code, count, k, k, ptr(d), block, ptr<void>(codes), ptr<void>(scales), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    PyObject *c = THPVariable_Wrap(std::move(codes)), *s = c ? THPVariable_Wrap(std::move(scales)) : nullptr;
    if (!s) { Py_XDECREF(c); return nullptr; }
    PyObject* both = PyTuple_Pack(2, c, s);
    Py_DECREF(c);
    Py_DECREF(s);
    return both;
ENTRY_END

// codes, scales, dtype, out, stream
ENTRY(mx_dequantize, 5)
    const Tensor *codes = here(a[0], at::kByte), *given;
    at::ScalarType type;
    int code;
    if (!codes || codes->dim() != 2 || codes->size(1) % 16 || codes->size(1) > INT_MAX / 2 || a[4] != Py_None || !dtype_of(a[2], &type, &code)) LONG_WAY;
    const long count = (long)codes->size(0);
    const int k = 2 * (int)codes->size(1);
    const Tensor* scales = byte_rows(a[1], count, k / 32);
    if (!scales || !result_rows(a[3], &given, type, count, k)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = result(given, {count, k}, type, *codes);
        rc = spinner_mx_dequantize(ptr<void>(codes), ptr<void>(scales), count, k, ptr<void>(out), code, k, current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// a_codes, a_scales, w_codes, w_scales, ends, dtype, out, stream
ENTRY(mx_matmul, 8)
    const Tensor *codes = here(a[0], at::kByte), *wc = here(a[2], at::kByte), *ws = here(a[3], at::kByte), *given;
    at::ScalarType type;
    int code, experts, n, experts_s, n_s;
    int64_t half, blocks;
    const long long* ends;
    if (!codes || codes->dim() != 2 || codes->size(1) % 16 || codes->size(1) > INT_MAX / 2 || a[7] != Py_None || !dtype_of(a[5], &type, &code)) LONG_WAY;
    const long count = (long)codes->size(0);
    const int k = 2 * (int)codes->size(1);
    const Tensor* scales = byte_rows(a[1], count, k / 32);
    if (!scales || !weights(wc, &experts, &n, &half) || !weights(ws, &experts_s, &n_s, &blocks) || half != k / 2 || blocks != k / 32) LONG_WAY;
    if (wc->dim() != ws->dim() || experts_s != experts || n_s != n || !expert_ends(a[4], experts, &ends) || !result_rows(a[6], &given, type, count, n)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = result(given, {count, n}, type, *codes);
        rc = spinner_mx_matmul(ptr<void>(codes), ptr<void>(scales), count, k, ptr<void>(wc), ptr<void>(ws), n, experts, ends, ptr<void>(out),
                                code, n, current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// x, w_codes, w_scales, diag, block, ends, out, workspace, stream
ENTRY(mx_linear, 9)
    long count;
    int k, code, block, experts, n, experts_s, n_s;
    int64_t half, blocks;
    const long long* ends;
    const Tensor *x = number_rows(a[0], &count, &k, &code), *wc = here(a[1], at::kByte), *ws = here(a[2], at::kByte), *d, *given;
    if (!x || a[8] != Py_None || k % 32 || !rotation(a[3], a[4], k, &d, &block)) LONG_WAY;
    if (!weights(wc, &experts, &n, &half) || !weights(ws, &experts_s, &n_s, &blocks) || half != k / 2 || blocks != k / 32) LONG_WAY;
    if (wc->dim() != ws->dim() || experts_s != experts || n_s != n || !expert_ends(a[5], experts, &ends)) LONG_WAY;
    if (!result_rows(a[6], &given, x->scalar_type(), count, n)) LONG_WAY;
    const size_t need = spinner_mx_linear_workspace_bytes(count, k);
    Buffer w;
    if ((a[7] != Py_None && !here(a[7])) || !w.usable_bytes(a[7], need)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = result(given, {count, n}, x->scalar_type(), *x);
        const auto call = [&](void* scratch) {
            return spinner_mx_linear(ptr<void>(x), code, count, k, k, ptr(d), block, ptr<void>(wc), ptr<void>(ws), n, experts, ends, ptr<void>(out), n,
                                     scratch, current_stream());
        };
        // a few rows need none, and making it is a tenth of such a call's time
        rc = call(ptr<void>(w.given));
        if (rc == SPINNER_ERR_WORKSPACE) rc = call(ptr<void>(w.scratch(need, *x)));
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

PyObject* grouped(Args a, bool across)
{
    long count;
    int depth, code, experts, n;
    int64_t k;
    const long long* ends;
    const Tensor *x = number_rows(a[0], &count, &depth, &code), *w = here(a[1]), *given;
    if (!x || a[4] != Py_None || !weights(w, &experts, &n, &k) || k > INT_MAX || w->scalar_type() != x->scalar_type()) LONG_WAY;
    if (depth != (across ? k : n) || !expert_ends(a[2], experts, &ends)) LONG_WAY;
    const int width = across ? n : (int)k;
    if (!result_rows(a[3], &given, x->scalar_type(), count, width)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = result(given, {count, width}, x->scalar_type(), *x);
        rc = (across ? spinner_grouped_matmul : spinner_grouped_matmul_dx)(ptr<void>(x), code, count, depth, depth, ptr<void>(w), width, experts, ends,
                                                                           ptr<void>(out), width, current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
}
// x, w, ends, out, stream
ENTRY(grouped_matmul, 5)
    return grouped(a, true);
ENTRY_END
// dy, w, ends, dx, stream
ENTRY(grouped_matmul_dx, 5)
    return grouped(a, false);
ENTRY_END

// dy, x, ends, dtype, dw, workspace, stream
ENTRY(grouped_matmul_dw, 7)
    long count, x_count;
    int n, k, code, x_code, dw_code, experts = 1;
    at::ScalarType type;
    const long long* ends = nullptr;
    const Tensor *dy = number_rows(a[0], &count, &n, &code), *x = number_rows(a[1], &x_count, &k, &x_code), *given = nullptr;
    if (!dy || !x || a[6] != Py_None || x_count != count || x_code != code || !dtype_of(a[3], &type, &dw_code)) LONG_WAY;
    if (a[2] != Py_None) {
        const Tensor* e = here(a[2], at::kLong);
        if (!e || e->dim() != 1 || e->numel() < 1 || e->numel() > INT_MAX) LONG_WAY;
        experts = (int)e->numel();
        ends = static_cast<const long long*>(e->data_ptr());
    }
    const std::vector<int64_t> sizes = ends ? std::vector<int64_t>{experts, n, k} : std::vector<int64_t>{n, k};
    if (a[4] != Py_None) {
        given = here(a[4], type);
        if (!given || given->sizes() != at::IntArrayRef(sizes)) LONG_WAY;
    }
    const size_t need = spinner_grouped_matmul_dw_workspace_bytes(count, n, k, experts);
    Buffer w;
    if ((a[5] != Py_None && !here(a[5])) || !w.usable_bytes(a[5], need)) LONG_WAY;
    Tensor dw;
    int rc;
    {
        pybind11::gil_scoped_release free;
        dw = result(given, sizes, type, *dy);
        const Tensor scratch = w.scratch(need, *dy);
        rc = spinner_grouped_matmul_dw(ptr<void>(dy), ptr<void>(x), code, count, n, k, n, k, experts, ends, ptr<void>(dw), dw_code, ptr<void>(scratch),
                                       current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(dw));
ENTRY_END

// ------------------------------------------------------------------ 8-bit whole numbers
int64_t int_width(int64_t k) { return (k + 15) / 16 * 16; }
PyObject* two(Tensor&& a, Tensor&& b)
{
    PyObject *x = THPVariable_Wrap(std::move(a)), *y = x ? THPVariable_Wrap(std::move(b)) : nullptr;
    if (!y) { Py_XDECREF(x); return nullptr; }
    PyObject* both = PyTuple_Pack(2, x, y);
    Py_DECREF(x);
    Py_DECREF(y);
    return both;
}
const Tensor* shaped(PyObject* o, at::ScalarType type, at::IntArrayRef sizes)
{
    const Tensor* t = here(o, type);
    return t && t->sizes() == sizes ? t : nullptr;
}
// memory that the caller may bring, of this shape
bool given_as(PyObject* o, const Tensor** t, at::ScalarType type, at::IntArrayRef sizes)
{
    *t = nullptr;
    return o == Py_None || (*t = shaped(o, type, sizes));
}
bool places_of(PyObject* o, long rows, const int** p, int* top)
{
    *p = nullptr;
    *top = 1;
    if (o == Py_None) return true;
    const Tensor* t = here(o, at::kInt);
    if (!t || t->dim() != 2 || t->size(0) != rows || t->size(1) < 1 || t->size(1) > 32 || rows > INT_MAX) return false;
    *p = ptr<const int>(t);
    *top = (int)t->size(1);
    return true;
}
bool int_weights(PyObject* codes, PyObject* scales, int64_t width, int* experts, int* n, const Tensor** wc, const Tensor** ws)
{
    int64_t w;
    *wc = here(codes, at::kChar);
    *ws = here(scales, at::kFloat);
    return weights(*wc, experts, n, &w) && w == width && *ws && (*ws)->sizes() == (*wc)->sizes().slice(0, (*wc)->dim() - 1);
}

// x, diag, block, places, codes, scales, stream
ENTRY(int_quantize, 7)
    long count;
    int k, code, block, top;
    const int* places;
    const Tensor *x = number_rows(a[0], &count, &k, &code), *d, *gc, *gs;
    if (!x || a[6] != Py_None || !rotation(a[1], a[2], k, &d, &block) || !places_of(a[3], count, &places, &top)) LONG_WAY;
    const int64_t slots = count * top, width = int_width(k);
    if (!given_as(a[4], &gc, at::kChar, {slots, width}) || !given_as(a[5], &gs, at::kFloat, {slots})) LONG_WAY;
    Tensor codes, scales;
    int rc;
    {
        pybind11::gil_scoped_release free;
        codes = result(gc, {slots, width}, at::kChar, *x);
        scales = result(gs, {slots}, at::kFloat, *x);
        rc = spinner_int_quantize(ptr<void>(x), code, count, k, k, ptr(d), block, places, top, ptr<void>(codes), ptr(scales), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return two(std::move(codes), std::move(scales));
ENTRY_END

// codes, scales, dtype, k, out, stream
ENTRY(int_dequantize, 6)
    const Tensor *codes = here(a[0], at::kChar), *given;
    at::ScalarType type;
    int code, k;
    if (!codes || codes->dim() != 2 || codes->size(1) > INT_MAX || a[5] != Py_None || !dtype_of(a[2], &type, &code)) LONG_WAY;
    const long count = (long)codes->size(0);
    if (a[3] == Py_None) k = (int)codes->size(1);
    else if (!whole(a[3], &k)) LONG_WAY;
    const Tensor* scales = shaped(a[1], at::kFloat, {count});
    if (!scales || int_width(k) != codes->size(1) || !result_rows(a[4], &given, type, count, k)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = result(given, {count, k}, type, *codes);
        rc = spinner_int_dequantize(ptr<void>(codes), ptr(scales), count, k, ptr<void>(out), code, k, current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// a_codes, a_scales, w_codes, w_scales, ends, dtype, out, stream
ENTRY(int_matmul, 8)
    const Tensor *codes = here(a[0], at::kChar), *wc, *ws, *given;
    at::ScalarType type;
    int code, experts, n;
    const long long* ends;
    if (!codes || codes->dim() != 2 || codes->size(1) % 16 || codes->size(1) > INT_MAX || a[7] != Py_None || !dtype_of(a[5], &type, &code)) LONG_WAY;
    const long count = (long)codes->size(0);
    const int k = (int)codes->size(1);
    const Tensor* scales = shaped(a[1], at::kFloat, {count});
    if (!scales || !int_weights(a[2], a[3], k, &experts, &n, &wc, &ws) || !expert_ends(a[4], experts, &ends) || !result_rows(a[6], &given, type, count, n)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = result(given, {count, n}, type, *codes);
        rc = spinner_int_matmul(ptr<void>(codes), ptr(scales), count, k, ptr<void>(wc), ptr(ws), n, experts, ends, ptr<void>(out), code, n, current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// x, w_codes, w_scales, diag, block, ends, places, out, workspace, stream
ENTRY(int_linear, 10)
    long count;
    int k, code, block, experts, n, top;
    const long long* ends;
    const int* places;
    const Tensor *x = number_rows(a[0], &count, &k, &code), *wc, *ws, *d, *given;
    if (!x || a[9] != Py_None || !rotation(a[3], a[4], k, &d, &block) || !int_weights(a[1], a[2], int_width(k), &experts, &n, &wc, &ws)) LONG_WAY;
    if (!expert_ends(a[5], experts, &ends) || !places_of(a[6], count, &places, &top)) LONG_WAY;
    const long slots = count * top;
    if (!result_rows(a[7], &given, x->scalar_type(), slots, n)) LONG_WAY;
    const size_t need = spinner_int_linear_workspace_bytes(slots, k);
    Buffer w;
    if ((a[8] != Py_None && !here(a[8])) || !w.usable_bytes(a[8], need)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = result(given, {slots, n}, x->scalar_type(), *x);
        const auto call = [&](void* scratch) {
            return spinner_int_linear(ptr<void>(x), code, count, k, k, ptr(d), block, places, top, ptr<void>(wc), ptr(ws), n, experts, ends, ptr<void>(out), n,
                                      scratch, current_stream());
        };
        // (a few rows need none)
        rc = call(ptr<void>(w.given));
        if (rc == SPINNER_ERR_WORKSPACE) rc = call(ptr<void>(w.scratch(need, *x)));
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// ------------------------------------------------------------------ routing
bool score_of(PyObject* o, int* v)
{
    static const char* const names[] = {"softmax", "sigmoid"};
    static_assert(SPINNER_SCORE_SOFTMAX == 0 && SPINNER_SCORE_SIGMOID == 1, "the order of the names");
    return choice(o, names, 2, v);
}

// logits, top, bias, mask, score, groups, top_groups, group_top, renormalise, scale, weights, experts, stream
ENTRY(route, 13)
    long count;
    int width, code, top, score, groups, top_groups, group_top;
    float scale;
    const Tensor *x = number_rows(a[0], &count, &width, &code), *bias = nullptr, *mask = nullptr, *gw, *ge;
    if (!x || a[12] != Py_None || !whole(a[1], &top) || top < 1 || !score_of(a[4], &score) || !whole(a[5], &groups) || !whole(a[6], &top_groups)) LONG_WAY;
    if (!whole(a[7], &group_top) || !PyBool_Check(a[8]) || !number(a[9], &scale)) LONG_WAY;
    if (a[2] != Py_None && !(bias = shaped(a[2], at::kFloat, {width}))) LONG_WAY;
    if (a[3] != Py_None && !(mask = shaped(a[3], at::kBool, {count}))) LONG_WAY;
    if (!given_as(a[10], &gw, at::kFloat, {count, top}) || !given_as(a[11], &ge, at::kInt, {count, top})) LONG_WAY;
    Tensor w, e;
    int rc;
    {
        pybind11::gil_scoped_release free;
        w = result(gw, {count, top}, at::kFloat, *x);
        e = result(ge, {count, top}, at::kInt, *x);
        rc = spinner_route(ptr<void>(x), code, count, width, width, ptr(bias), ptr<void>(mask), score, groups, top_groups, group_top, top, a[8] == Py_True, scale,
                           ptr(w), ptr<int>(e), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return two(std::move(w), std::move(e));
ENTRY_END

// dweights, logits, experts, score, renormalise, scale, dlogits, stream
ENTRY(route_grad, 8)
    long count;
    int width, code, score;
    float scale;
    const Tensor *x = number_rows(a[1], &count, &width, &code), *e = here(a[2], at::kInt), *given;
    if (!x || !e || e->dim() != 2 || e->size(0) != count || e->size(1) > INT_MAX || a[7] != Py_None || !score_of(a[3], &score)) LONG_WAY;
    const Tensor* dw = shaped(a[0], at::kFloat, e->sizes());
    if (!dw || !PyBool_Check(a[4]) || !number(a[5], &scale) || !result_rows(a[6], &given, x->scalar_type(), count, width)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = result(given, {count, width}, x->scalar_type(), *x);
        rc = spinner_route_grad(ptr(dw), ptr<void>(x), code, count, width, width, ptr<int>(e), score, (int)e->size(1), a[4] == Py_True, scale, ptr<void>(out), width,
                                current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// experts, count, places, ends, workspace, stream
ENTRY(route_order, 6)
    const Tensor *e = here(a[0], at::kInt), *gp, *ge;
    int experts;
    if (!e || e->dim() != 2 || a[5] != Py_None || !whole(a[1], &experts) || experts < 1) LONG_WAY;
    if (!given_as(a[2], &gp, at::kInt, e->sizes()) || !given_as(a[3], &ge, at::kLong, {experts})) LONG_WAY;
    const size_t need = spinner_route_order_workspace_bytes((long)e->numel(), experts);
    Buffer w;
    if ((a[4] != Py_None && !here(a[4])) || !w.usable_bytes(a[4], need)) LONG_WAY;
    Tensor places, ends;
    int rc;
    {
        pybind11::gil_scoped_release free;
        places = result(gp, e->sizes(), at::kInt, *e);
        ends = result(ge, {experts}, at::kLong, *e);
        const Tensor scratch = w.scratch(need, *e);
        rc = spinner_route_order(ptr<int>(e), (long)e->numel(), experts, ptr<int>(places), ptr<long long>(ends), ptr<void>(scratch), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return two(std::move(places), std::move(ends));
ENTRY_END

// x, places, out, stream
ENTRY(dispatch, 4)
    long count;
    int n, code, top;
    const int* places;
    const Tensor *x = number_rows(a[0], &count, &n, &code), *given;
    if (!x || a[3] != Py_None || a[1] == Py_None || !places_of(a[1], count, &places, &top) || !result_rows(a[2], &given, x->scalar_type(), count * top, n)) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = result(given, {count * top, n}, x->scalar_type(), *x);
        rc = spinner_dispatch(ptr<void>(x), code, count, n, n, places, top, ptr<void>(out), n, current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// y, places, weights, out, stream
ENTRY(combine, 5)
    long slots;
    int n, code, top;
    const int* places;
    const Tensor *y = number_rows(a[0], &slots, &n, &code), *p = here(a[1], at::kInt), *w = nullptr, *given;
    if (!y || !p || p->dim() != 2 || p->numel() != slots || a[4] != Py_None) LONG_WAY;
    const long count = (long)p->size(0);
    if (!places_of(a[1], count, &places, &top) || !result_rows(a[3], &given, y->scalar_type(), count, n)) LONG_WAY;
    if (a[2] != Py_None && !(w = shaped(a[2], at::kFloat, {count, top}))) LONG_WAY;
    Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release free;
        out = result(given, {count, n}, y->scalar_type(), *y);
        rc = spinner_combine(ptr<void>(y), code, count, n, n, places, ptr(w), top, ptr<void>(out), n, current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return THPVariable_Wrap(std::move(out));
ENTRY_END

// dout, y, places, weights, dy, dweights, stream
ENTRY(combine_grad, 7)
    long count, slots;
    int n, code, y_n, y_code, top;
    const int* places;
    const Tensor *d = number_rows(a[0], &count, &n, &code), *y = number_rows(a[1], &slots, &y_n, &y_code), *gy, *gw;
    if (!d || !y || y_n != n || y_code != code || a[6] != Py_None || a[2] == Py_None || !places_of(a[2], count, &places, &top) || slots != count * top) LONG_WAY;
    const Tensor* w = shaped(a[3], at::kFloat, {count, top});
    if (!w || !given_as(a[4], &gy, y->scalar_type(), {slots, n}) || !given_as(a[5], &gw, at::kFloat, {count, top})) LONG_WAY;
    Tensor dy, dw;
    int rc;
    {
        pybind11::gil_scoped_release free;
        dy = result(gy, {slots, n}, y->scalar_type(), *y);
        dw = result(gw, {count, top}, at::kFloat, *y);
        rc = spinner_combine_grad(ptr<void>(d), ptr<void>(y), code, count, n, n, n, places, ptr(w), top, ptr<void>(dy), n, ptr(dw), current_stream());
    }
    if (rc != SPINNER_OK) return refused(rc);
    return two(std::move(dy), std::move(dw));
ENTRY_END

#define METHOD(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(NAME)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(apply_signs), METHOD(apply), METHOD(apply_blocks), METHOD(hash), METHOD(hash_signs), METHOD(sign_codes),
                         METHOD(sign_codes_signs), METHOD(angular_gram), METHOD(layer_forward), METHOD(layer_backward), METHOD(sketch),
                         METHOD(sketch_gram), METHOD(struct_apply_ws), METHOD(_new_on), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};
// the calls of the 4-bit and grouped products, in a module of their own inside the first
PyMethodDef product_methods[] = {METHOD(mx_quantize), METHOD(mx_dequantize), METHOD(mx_matmul), METHOD(mx_linear), METHOD(grouped_matmul),
                                 METHOD(grouped_matmul_dx), METHOD(grouped_matmul_dw), {nullptr, nullptr, 0, nullptr}};
PyModuleDef product_module_def = {PyModuleDef_HEAD_INIT, "_native._products", nullptr, -1, product_methods, nullptr, nullptr, nullptr, nullptr};
// and those of routing and of 8-bit layers
PyMethodDef expert_methods[] = {METHOD(int_quantize), METHOD(int_dequantize), METHOD(int_matmul), METHOD(int_linear), METHOD(route), METHOD(route_grad),
                                METHOD(route_order), METHOD(dispatch), METHOD(combine), METHOD(combine_grad), {nullptr, nullptr, 0, nullptr}};
PyModuleDef expert_module_def = {PyModuleDef_HEAD_INIT, "_native._experts", nullptr, -1, expert_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native()
{
    PyObject* module = PyModule_Create(&module_def);
    const auto add = [&](const char* name, PyModuleDef* def) {
        PyObject* inner = module ? PyModule_Create(def) : nullptr;
        if (inner && PyModule_AddObject(module, name, inner) == 0) return true;
        Py_XDECREF(inner);
        return false;
    };
    if (!add("_products", &product_module_def) || !add("_experts", &expert_module_def)) {
        Py_XDECREF(module);
        return nullptr;
    }
    return module;
}
