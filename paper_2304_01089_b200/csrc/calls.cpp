// Argument marshalling of the paged cache's calls for Python: tensors are looked at through PyTorch's own C++ objects, because a call from
// a decode loop takes less time on the GPU than reading some forty attributes takes in the interpreter (attention 8.0 us a call with
// ctypes, 3.8 of it the call itself, 2.4 here). Nothing is computed here: checks of types, shapes, devices and distances, then the library's function.
//
// Each function returns the library's status; arguments that cannot be handed to it raise ValueError.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "rptq.h"

namespace {

// What a KvCache knows of its handle.
struct Cache {
    const rptq_kv_cache_t* handle;
    int64_t channels, head_dim, k_row_bytes, v_row_bytes, k_page_bytes, v_page_bytes;
    int device;
};

struct Refused {};                             // a Python exception is set

[[noreturn]] void refuse(const char* text)
{
    PyErr_SetString(PyExc_ValueError, text);
    throw Refused();
}

const at::Tensor& tensor(PyObject* o, const char* what, const Cache& c)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_ValueError, "%s: expected a tensor", what);
        throw Refused();
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.layout() != c10::kStrided || (t.is_cuda() ? (int)t.get_device() : -1) != c.device) {
        PyErr_Format(PyExc_ValueError, "%s: expected a tensor on the cache's device", what);
        throw Refused();
    }
    return t;
}

// A 2-D tensor with at least n_rows contiguous rows of n_cols; *ld: elements between rows.
void* rows(const at::Tensor& t, const char* what, int64_t n_rows, int64_t n_cols, int64_t* ld)
{
    if (t.dim() != 2 || t.size(0) < n_rows || t.size(1) < n_cols || (t.stride(1) != 1 && t.size(1) > 1)) {
        PyErr_Format(PyExc_ValueError, "%s: expected at least %lld contiguous rows of %lld", what, (long long)n_rows, (long long)n_cols);
        throw Refused();
    }
    *ld = t.size(0) > 1 ? t.stride(0) : t.size(1);
    return t.data_ptr();
}

int rows_type(const at::Tensor& t, const char* what)
{
    switch (t.scalar_type()) {
        case at::kFloat: return RPTQ_ROWS_F32;
        case at::kHalf: return RPTQ_ROWS_F16;
        case at::kByte: return RPTQ_ROWS_CODES;
        case at::kBFloat16: return RPTQ_ROWS_BF16;
        default: break;
    }
    PyErr_Format(PyExc_ValueError, "%s: fp32, fp16, bf16 or uint8 code rows are expected", what);
    throw Refused();
}

void* pool(const at::Tensor& t, const char* what, int64_t page_bytes, int64_t n_pages)
{
    if (t.scalar_type() != at::kByte || t.dim() != 2 || t.size(1) != page_bytes || t.size(0) != n_pages || !t.is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s: a pool is a contiguous uint8 tensor [n_pages][%lld], the two of a cache with as many pages", what, (long long)page_bytes);
        throw Refused();
    }
    return t.data_ptr();
}

int count(int64_t n, const char* what)
{
    if (n > INT32_MAX) {
        PyErr_Format(PyExc_ValueError, "%s: too many", what);
        throw Refused();
    }
    return (int)n;
}

void* stream_of(PyObject* o, const Cache& c)
{
    if (o == Py_None) return c.device < 0 ? nullptr : (void*)c10::cuda::getCurrentCUDAStream().stream();
    PyObject* at = PyObject_GetAttrString(o, "cuda_stream");       // a torch stream, or the number itself
    if (!at) {
        PyErr_Clear();
        at = Py_NewRef(o);
    }
    void* p = PyLong_AsVoidPtr(at);
    Py_DECREF(at);
    if (PyErr_Occurred()) throw Refused();
    return p;
}

const Cache& cache_of(PyObject* o)
{
    auto* c = static_cast<Cache*>(PyCapsule_GetPointer(o, "rptq_kv_cache"));
    if (!c) throw Refused();
    return *c;
}

template <class F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F f)
{
    if (n != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return PyLong_FromLong(f());
    } catch (const Refused&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// describe(handle, channels, head_dim, k_row_bytes, v_row_bytes, k_page_bytes, v_page_bytes, device)
PyObject* describe(PyObject*, PyObject* args)
{
    unsigned long long handle;
    Cache c{};
    long long n[6];
    if (!PyArg_ParseTuple(args, "KLLLLLLi", &handle, n, n + 1, n + 2, n + 3, n + 4, n + 5, &c.device)) return nullptr;
    c.handle = reinterpret_cast<const rptq_kv_cache_t*>(handle);
    c.channels = n[0]; c.head_dim = n[1]; c.k_row_bytes = n[2]; c.v_row_bytes = n[3]; c.k_page_bytes = n[4]; c.v_page_bytes = n[5];
    return PyCapsule_New(new Cache(c), "rptq_kv_cache", [](PyObject* o) { delete static_cast<Cache*>(PyCapsule_GetPointer(o, "rptq_kv_cache")); });
}

struct RowArgs {
    void *k, *v, *k_pages, *v_pages;
    int64_t ldk, ldv, n_pages;
    const int64_t* slots;
    int n, type;
};
RowArgs row_args(const Cache& c, PyObject* k_o, PyObject* v_o, PyObject* slots_o, PyObject* kp_o, PyObject* vp_o)
{
    const at::Tensor &k = tensor(k_o, "k", c), &v = tensor(v_o, "v", c), &slots = tensor(slots_o, "slots", c), &kp = tensor(kp_o, "k_pages", c), &vp = tensor(vp_o, "v_pages", c);
    RowArgs a;
    if (slots.scalar_type() != at::kLong || slots.dim() != 1 || !slots.is_contiguous()) refuse("slots: expected a contiguous 1-D tensor of int64");
    a.n = count(slots.size(0), "slots");
    a.slots = static_cast<const int64_t*>(slots.data_ptr());
    a.type = rows_type(k, "k");
    if (v.scalar_type() != k.scalar_type()) refuse("k and v have different types");
    a.k = rows(k, "k", a.n, a.type == RPTQ_ROWS_CODES ? c.k_row_bytes : c.channels, &a.ldk);
    a.v = rows(v, "v", a.n, a.type == RPTQ_ROWS_CODES ? c.v_row_bytes : c.channels, &a.ldv);
    a.n_pages = kp.dim() == 2 ? kp.size(0) : -1;
    a.k_pages = pool(kp, "k_pages", c.k_page_bytes, a.n_pages);
    a.v_pages = pool(vp, "v_pages", c.v_page_bytes, a.n_pages);
    return a;
}

// kv_cache_write(cache, k, v, slots, k_pages, v_pages, stream)
PyObject* kv_cache_write(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    return guarded(n, 7, [&] {
        const Cache& c = cache_of(o[0]);
        const RowArgs a = row_args(c, o[1], o[2], o[3], o[4], o[5]);
        return rptq_kv_cache_write(c.handle, a.k, a.ldk, a.v, a.ldv, a.type, a.slots, a.n, a.k_pages, a.v_pages, a.n_pages, stream_of(o[6], c));
    });
}

// kv_cache_read(cache, k_pages, v_pages, slots, k_out, v_out, stream)
PyObject* kv_cache_read(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    return guarded(n, 7, [&] {
        const Cache& c = cache_of(o[0]);
        const RowArgs a = row_args(c, o[4], o[5], o[3], o[1], o[2]);
        return rptq_kv_cache_read(c.handle, a.k_pages, a.v_pages, a.n_pages, a.slots, a.n, a.k, a.ldk, a.v, a.ldv, a.type, stream_of(o[6], c));
    });
}

// attention_paged(cache, q, k_pages, v_pages, page_table, seq_lens, out, qk_scale, n_q_heads, workspace, workspace bytes, stream)
PyObject* attention_paged(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    return guarded(n, 12, [&] {
        const Cache& c = cache_of(o[0]);
        const at::Tensor &q = tensor(o[1], "q", c), &kp = tensor(o[2], "k_pages", c), &vp = tensor(o[3], "v_pages", c), &table = tensor(o[4], "page_table", c),
                         &lens = tensor(o[5], "seq_lens", c), &out = tensor(o[6], "out", c), &ws = tensor(o[9], "workspace", c);
        const double scale = PyFloat_AsDouble(o[7]);
        const long heads = PyLong_AsLong(o[8]);
        const long long need = PyLong_AsLongLong(o[10]);
        if (PyErr_Occurred()) throw Refused();
        if (lens.scalar_type() != at::kInt || lens.dim() != 1 || !lens.is_contiguous()) refuse("seq_lens: expected a contiguous 1-D tensor of int32");
        const int n_seq = count(lens.size(0), "seq_lens");
        int64_t ldq, ldo, ld_table;
        const int type = rows_type(q, "q");
        if (out.scalar_type() != q.scalar_type()) refuse("q and out have different types");
        void* q_at = rows(q, "q", n_seq, heads * c.head_dim, &ldq);
        void* out_at = rows(out, "out", n_seq, heads * c.head_dim, &ldo);
        if (table.scalar_type() != at::kInt) refuse("page_table: expected int32");
        void* table_at = rows(table, "page_table", n_seq, 0, &ld_table);
        const int64_t n_pages = kp.dim() == 2 ? kp.size(0) : -1;
        void *k_at = pool(kp, "k_pages", c.k_page_bytes, n_pages), *v_at = pool(vp, "v_pages", c.v_page_bytes, n_pages);
        if ((long long)ws.nbytes() < need || !ws.is_contiguous()) refuse("workspace: too few contiguous bytes (see attention_paged_workspace_bytes)");
        return rptq_attention_paged(c.handle, q_at, ldq, type, (int)heads, n_seq, k_at, v_at, n_pages, static_cast<const int32_t*>(table_at), ld_table,
                                    count(table.size(1), "page_table"), static_cast<const int32_t*>(lens.data_ptr()), (float)scale, out_at, ldo, ws.data_ptr(),
                                    stream_of(o[11], c));
    });
}

template <class F>
PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {
    {"describe", describe, METH_VARARGS, nullptr},
    {"kv_cache_write", fast(kv_cache_write), METH_FASTCALL, nullptr},
    {"kv_cache_read", fast(kv_cache_read), METH_FASTCALL, nullptr},
    {"attention_paged", fast(attention_paged), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
extern "C" __attribute__((used, visibility("default"))) const char rptq_calls_tag[] = RPTQ_CALLS_TAG;     // (build.py looks for it)
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&module); }
