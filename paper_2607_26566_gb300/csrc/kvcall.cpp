// kvcall.cpp -- CPython entry points for the calls of the key/value cache
// (kv.py): they read the tensors' addresses, types, shapes and strides, fill the
// call's descriptor and pass it to libt2istore.so. A call has up to fifteen
// tensors, and each attribute of one costs about 100 ns in Python (a call of the
// cache 30 us on a Grace host), so tensors are read through torch's C++ headers.
// Marshalling only; the interpreter lock is kept for the call, as in pycall.c.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/TensorBase.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>
#include <initializer_list>
#include <string>

#include "t2istore.h"

namespace {

// The binding's side of a cache (a capsule).
struct Cache {
    t2i_kv* kv;
    int device;
    at::ScalarType dtype;
    int64_t kv_heads, head_dim, max_seqs, max_pages;
    PyObject* table;  // the cache's own page table
};

constexpr const char* kCapsule = "t2i_kv";

struct PyFail {};  // a Python error is set

[[noreturn]] void type_error(const std::string& e) {
    PyErr_SetString(PyExc_TypeError, e.c_str());
    throw PyFail{};
}
[[noreturn]] void value_error(const std::string& e) {
    PyErr_SetString(PyExc_ValueError, e.c_str());
    throw PyFail{};
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) type_error(std::string(name) + " must be a tensor");
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.requires_grad() && c10::GradMode::is_enabled())
        value_error(std::string(name) + " requires a gradient, and the cache's calls have none: detach it, or call under torch.no_grad()");
    return t;
}

int64_t integer(PyObject* o, const char* name, int64_t most) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw PyFail{};
    if (v < 0 || v > most) value_error(std::string(name) + " is out of range");
    return v;
}
uint32_t u32(PyObject* o, const char* name) { return uint32_t(integer(o, name, 0xFFFFFFFFll)); }
float real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PyFail{};
    return float(v);
}

// A token array [n, heads, head_dim], the heads of a token side by side.
struct Rows {
    void* p;
    int64_t n, heads;
    uint64_t stride;
};
Rows rows(const Cache& c, PyObject* o, int64_t heads, const char* name, const at::ScalarType* dtype) {
    const at::Tensor& t = tensor(o, name);
    if (t.dim() != 3 || (heads >= 0 && t.size(1) != heads) || t.size(2) != c.head_dim || !t.is_cuda())
        value_error(std::string(name) + " must be a CUDA tensor [tokens, heads, head_dim] of the right heads and head_dim");
    if (dtype && t.scalar_type() != *dtype) type_error(std::string(name) + " has the wrong dtype");
    if (t.stride(2) != 1 || (t.stride(1) != c.head_dim && t.size(1) > 1))
        value_error(std::string("the heads of a token of ") + name + " must lie next to one another");
    return {t.data_ptr(), t.size(0), t.size(1), uint64_t(t.stride(0))};
}

// Address of a contiguous tensor of this type and shape; null for None.
void* plain(PyObject* o, at::ScalarType dtype, std::initializer_list<int64_t> shape, const char* name) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, name);
    if (t.scalar_type() != dtype) type_error(std::string(name) + " has the wrong dtype");
    if (!t.is_cuda() || !t.is_contiguous() || t.sizes() != at::IntArrayRef(shape.begin(), shape.size()))
        value_error(std::string(name) + " must be a contiguous CUDA tensor of the right shape");
    return t.data_ptr();
}

uint32_t dtype_of(const at::Tensor& t, const char* name) {
    switch (t.scalar_type()) {
        case at::kBFloat16: return T2I_BF16;
        case at::kHalf: return T2I_F16;
        case at::kFloat: return T2I_F32;
        default: type_error(std::string(name) + " must be bfloat16, float16 or float32");
    }
}

Cache& cache(PyObject* o) {
    Cache* c = static_cast<Cache*>(PyCapsule_GetPointer(o, kCapsule));
    if (!c) throw PyFail{};
    if (!c->kv) value_error("the cache is closed");
    return *c;
}

void* stream_of(const Cache& c, PyObject* o) {
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream(c10::DeviceIndex(c.device)).stream();
    if (PyLong_Check(o)) {
        void* s = PyLong_AsVoidPtr(o);
        if (!s && PyErr_Occurred()) throw PyFail{};
        return s;
    }
    PyObject* a = PyObject_GetAttrString(o, "cuda_stream");
    if (!a) throw PyFail{};
    void* s = PyLong_AsVoidPtr(a);
    Py_DECREF(a);
    if (!s && PyErr_Occurred()) throw PyFail{};
    return s;
}

// The page table of a call: the cache's own rows, or the caller's.
void table(const Cache& c, PyObject* o, int64_t n_seqs, const int32_t** p, uint64_t* stride, uint32_t* pages) {
    if (o == Py_None) {
        if (n_seqs > c.max_seqs) value_error("more sequences than the cache has");
        o = c.table;
    }
    const at::Tensor& t = tensor(o, "table");
    if (t.scalar_type() != at::kInt) type_error("table must be int32");
    if (t.dim() != 2 || t.size(0) < n_seqs || t.size(1) < 1 || !t.is_cuda() || (t.stride(1) != 1 && t.size(1) > 1) ||
        (t.stride(0) < t.size(1) && t.size(0) > 1))
        value_error("table must be a CUDA tensor [sequences, pages], the pages of a row side by side");
    *p = static_cast<const int32_t*>(t.data_ptr());
    *stride = uint64_t(std::max(t.stride(0), t.size(1)));
    *pages = uint32_t(t.size(1));
}

t2i_kv_batch batch(const Cache& c, int64_t n, PyObject* lens, PyObject* starts, PyObject* max_new, PyObject* layer,
                   PyObject* tab) {
    const at::Tensor& l = tensor(lens, "lens");
    if (l.dim() != 1) value_error("lens must be a CUDA tensor [sequences]");
    const int64_t s = l.size(0);
    t2i_kv_batch b{};
    table(c, tab, s, &b.table, &b.table_stride, &b.table_pages);
    b.lens = static_cast<const int32_t*>(plain(lens, at::kInt, {s}, "lens"));
    b.starts = static_cast<const int32_t*>(plain(starts, at::kInt, {s + 1}, "starts"));
    if (n > 0x7FFFFFFF || s > 0x7FFFFFFF) value_error("too many tokens or sequences");
    b.n_seqs = uint32_t(s);
    b.n_tokens = uint32_t(n);
    b.max_new = u32(max_new, "max_new");
    b.layer = u32(layer, "layer");
    return b;
}

// A call's workspace, from torch's allocator, for as long as the call takes: memory that is given back comes to
// later calls on its stream alone, behind this call's kernels. While torch captures a graph on the stream it is the
// graph's memory, and stays that. So nothing outlives a call, and threads, streams and graphs share none.
class Workspace {
  public:
    Workspace(int device, uint64_t bytes, void* stream) {
        if (!bytes) return;
        const c10::cuda::CUDAGuard g{c10::DeviceIndex(device)};
        p_ = c10::cuda::CUDACachingAllocator::raw_alloc_with_stream(bytes, static_cast<cudaStream_t>(stream));
    }
    ~Workspace() {
        if (p_) c10::cuda::CUDACachingAllocator::raw_delete(p_);
    }
    Workspace(const Workspace&) = delete;
    Workspace& operator=(const Workspace&) = delete;
    void* get() const { return p_; }

  private:
    void* p_ = nullptr;
};

// append(cache, k, v, lens, q, q_out, starts, max_new, layer, q_norm, k_norm, eps,
//        cos, sin, interleaved, positions, table, stream) -> status
PyObject* append(PyObject* const* a) {
    const Cache& c = cache(a[0]);
    const at::Tensor& kt = tensor(a[1], "k");
    const at::ScalarType in = kt.scalar_type();
    t2i_kv_append_desc d{};
    d.in_dtype = dtype_of(kt, "k");
    const Rows k = rows(c, a[1], c.kv_heads, "k", nullptr), v = rows(c, a[2], c.kv_heads, "v", &in);
    d.k = k.p, d.v = v.p, d.k_stride = k.stride, d.v_stride = v.stride;
    if (v.n != k.n) value_error("k and v must have as many tokens");
    if (a[4] != Py_None) {
        const Rows q = rows(c, a[4], -1, "q", &in), o = rows(c, a[5], q.heads, "q_out", &c.dtype);
        if (q.n != k.n || o.n != k.n) value_error("q, q_out and k must have as many tokens");
        d.q = q.p, d.q_out = o.p, d.q_stride = q.stride, d.q_out_stride = o.stride;
        d.q_heads = uint32_t(q.heads);
    } else if (a[5] != Py_None) {
        value_error("q_out without q");
    }
    d.batch = batch(c, k.n, a[3], a[6], a[7], a[8], a[16]);
    d.q_norm = static_cast<const float*>(plain(a[9], at::kFloat, {c.head_dim}, "q_norm"));
    d.k_norm = static_cast<const float*>(plain(a[10], at::kFloat, {c.head_dim}, "k_norm"));
    d.eps = real(a[11]);
    if ((a[12] == Py_None) != (a[13] == Py_None)) value_error("cos and sin go together");
    if (a[12] != Py_None) {
        const at::Tensor& t = tensor(a[12], "cos");
        if (t.dim() != 2 || t.size(0) > 0x7FFFFFFF || t.size(1) > c.head_dim) value_error("cos must be [positions, rotary_dim / 2]");
        d.cos_table = static_cast<const float*>(plain(a[12], at::kFloat, {t.size(0), t.size(1)}, "cos"));
        d.sin_table = static_cast<const float*>(plain(a[13], at::kFloat, {t.size(0), t.size(1)}, "sin"));
        d.n_positions = uint32_t(t.size(0));
        d.rotary_dim = uint32_t(2 * t.size(1));
    }
    const int turns = PyObject_IsTrue(a[14]);
    if (turns < 0) throw PyFail{};
    d.interleaved = uint32_t(turns);
    d.positions = static_cast<const int32_t*>(plain(a[15], at::kInt, {k.n}, "positions"));
    return PyLong_FromLong(t2i_kv_append(c.kv, &d, stream_of(c, a[17])));
}

// attend(cache, q, lens, out, lse, starts, max_new, layer, scale, softcap, slopes,
//        window, spans, tree, max_len, table, stream) -> status
PyObject* attend(PyObject* const* a) {
    const Cache& c = cache(a[0]);
    const Rows q = rows(c, a[1], -1, "q", &c.dtype), o = rows(c, a[3], q.heads, "out", &c.dtype);
    if (o.n != q.n) value_error("q and out must have as many tokens");
    t2i_kv_attend_desc d{};
    d.batch = batch(c, q.n, a[2], a[5], a[6], a[7], a[15]);
    d.q = q.p, d.out = o.p, d.q_stride = q.stride, d.out_stride = o.stride;
    d.q_heads = uint32_t(q.heads);
    d.lse = static_cast<float*>(plain(a[4], at::kFloat, {q.n, q.heads}, "lse"));
    d.scale = real(a[8]);
    d.softcap = real(a[9]);
    d.slopes = static_cast<const float*>(plain(a[10], at::kFloat, {q.heads}, "slopes"));
    d.window = u32(a[11], "window");
    d.spans = static_cast<const int32_t*>(plain(a[12], at::kInt, {q.n, 2}, "spans"));
    d.tree = static_cast<const uint64_t*>(plain(a[13], at::kLong, {q.n}, "tree"));
    d.max_len = u32(a[14], "max_len");
    void* s = stream_of(c, a[16]);
    const t2i_status st = t2i_kv_workspace_bytes(c.kv, d.batch.n_seqs, d.batch.n_tokens, d.q_heads, &d.workspace_bytes);
    if (st != T2I_OK || d.batch.n_tokens == 0) d.workspace_bytes = 0;
    const Workspace w(c.device, d.workspace_bytes, s);
    d.workspace = w.get();
    return PyLong_FromLong(t2i_kv_attend(c.kv, &d, s));
}

// commit(cache, ctx, path, counts, table, stream) -> status
PyObject* commit(PyObject* const* a) {
    const Cache& c = cache(a[0]);
    const at::Tensor& p = tensor(a[2], "path");
    if (p.dim() != 2 || p.size(0) > 0x7FFFFFFF || p.size(1) > 0x7FFFFFFF) value_error("path must be [sequences, any]");
    const int64_t n = p.size(0);
    t2i_kv_commit_desc d{};
    table(c, a[4], n, &d.table, &d.table_stride, &d.table_pages);
    d.ctx = static_cast<const int32_t*>(plain(a[1], at::kInt, {n}, "ctx"));
    d.path = static_cast<const int32_t*>(plain(a[2], at::kInt, {n, p.size(1)}, "path"));
    d.counts = static_cast<const int32_t*>(plain(a[3], at::kInt, {n}, "counts"));
    d.n_seqs = uint32_t(n);
    d.max_path = uint32_t(p.size(1));
    return PyLong_FromLong(t2i_kv_commit(c.kv, &d, stream_of(c, a[5])));
}

// cache(kv, device, fp16, kv_heads, head_dim, table) -> capsule
PyObject* make(PyObject* const* a) {
    const at::Tensor& t = tensor(a[5], "table");
    Cache* c = new Cache{};
    PyObject* cap = PyCapsule_New(c, kCapsule, [](PyObject* o) {
        Cache* d = static_cast<Cache*>(PyCapsule_GetPointer(o, kCapsule));
        Py_XDECREF(d->table);
        delete d;
    });
    if (!cap) {
        delete c;
        throw PyFail{};
    }
    try {
        c->kv = static_cast<t2i_kv*>(PyLong_AsVoidPtr(a[0]));
        if (!c->kv) value_error("no cache handle");
        c->device = int(integer(a[1], "device", 127));
        c->dtype = integer(a[2], "fp16", 1) ? at::kHalf : at::kBFloat16;
        c->kv_heads = integer(a[3], "kv_heads", 1 << 20);
        c->head_dim = integer(a[4], "head_dim", 1 << 20);
        c->max_seqs = t.size(0);
        c->max_pages = t.size(1);
    } catch (...) {
        Py_DECREF(cap);
        throw;
    }
    Py_INCREF(a[5]);
    c->table = a[5];
    return cap;
}

// close(capsule): later calls are refused
PyObject* shut(PyObject* const* a) {
    Cache* c = static_cast<Cache*>(PyCapsule_GetPointer(a[0], kCapsule));
    if (!c) throw PyFail{};
    c->kv = nullptr;
    Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject* const*), Py_ssize_t N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != N) return PyErr_Format(PyExc_TypeError, "%zd arguments wanted, %zd given", N, n);
    try {
        return F(args);
    } catch (const PyFail&) {
        return nullptr;
    } catch (const c10::OutOfMemoryError& e) {
        PyObject* torch = PyImport_ImportModule("torch");
        PyObject* type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
        if (type) PyErr_SetString(type, e.what_without_backtrace());
        Py_XDECREF(type);
        Py_XDECREF(torch);
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

#define ENTRY(name, f, n, doc) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<f, n>)), METH_FASTCALL, doc}
PyMethodDef methods[] = {ENTRY("cache", make, 6, "a cache's binding"),
                         ENTRY("close", shut, 1, "refuses later calls"),
                         ENTRY("append", append, 18, "t2i_kv_append"),
                         ENTRY("attend", attend, 17, "t2i_kv_attend"),
                         ENTRY("commit", commit, 6, "t2i_kv_commit"),
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kvcall", "CPython entry points for the calls of the key/value cache", -1,
                      methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kvcall(void) { return PyModule_Create(&module); }
