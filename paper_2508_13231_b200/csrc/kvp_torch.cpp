// Native side of the Python binding for calls so short that Python's own work would be most of them (scoring, and the calls of
// a decode step): scoring a schedule is
// 4 us of host time in the library, and took 25 with output tensors, stream and arguments handled in Python (2.4 us for
// each of five torch.empty, 3.2 for the current stream). Argument handling only; the work is libkvp.so's.
// Every function turns what torch throws into the Python exception torch itself raises for it (out of memory, no device, a
// tensor without storage): nothing may be thrown through the interpreter, which would end the process.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cmath>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/kvp.h"

// A library without these still serves the scoring calls (Python loads this module with all references bound, and the tests put a stand-in with the scoring
// calls alone in the library's place); the calls that need them say so.
#pragma weak kvp_cache_append
#pragma weak kvp_cache_read
#pragma weak kvp_attend
#pragma weak kvp_attend_workspace
#pragma weak kvp_trace_weights
#pragma weak kvp_evict

namespace {

PyObject* missing(const char* name)
{
    PyErr_Format(PyExc_ImportError, "libkvp.so has no %s: build it with `python -m paper_2508_13231_b200.build`", name);
    return nullptr;
}

PyObject* value_error(const char* what)
{
    PyErr_SetString(PyExc_ValueError, what);
    return nullptr;
}

// the checks of kvp._ptr; null is allowed for None
bool device_ptr(PyObject* o, at::ScalarType dtype, bool check, void** out)
{
    if (o == Py_None) { *out = nullptr; return true; }
    if (!THPVariable_Check(o)) { PyErr_SetString(PyExc_TypeError, "expected a tensor"); return false; }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) { value_error("expected a contiguous CUDA tensor"); return false; }
    if (check && t.scalar_type() != dtype) { value_error("expected dtype torch.int32"); return false; }
    *out = t.data_ptr();
    return true;
}

bool problem_of(PyObject* const* args, kvp_problem** p, unsigned long long* steps, unsigned long long* w32)
{
    *p = static_cast<kvp_problem*>(PyLong_AsVoidPtr(args[0]));
    *steps = PyLong_AsUnsignedLongLong(args[1]);
    *w32 = PyLong_AsUnsignedLongLong(args[2]);
    return !PyErr_Occurred();
}

// how many schedules a tensor holds
bool batch_of(PyObject* o, unsigned long long per, uint32_t* n)
{
    if (!THPVariable_Check(o)) { PyErr_SetString(PyExc_TypeError, "expected a tensor"); return false; }
    const uint64_t total = (uint64_t)THPVariable_Unpack(o).numel();
    if (total % per) { value_error("schedules must be [n][steps][W32]"); return false; }
    *n = (uint32_t)(total / per);
    return true;
}

bool stream_of(PyObject* o, int device, void** st)
{
    if (o == Py_None) { *st = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); return true; }
    *st = PyLong_AsVoidPtr(o);
    return !PyErr_Occurred();
}

// Other Python threads run meanwhile: a call into the library launches, may allocate, and waits when the stream's launch
// queue is full. (Arguments stay alive: the caller's frame holds them.)
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};

at::Tensor make(at::IntArrayRef size, at::ScalarType dtype, c10::Device dev) { return at::detail::empty_cuda(size, dtype, dev, std::nullopt); }

PyObject* k_step_ticks; PyObject* k_total_ticks; PyObject* k_step_seconds; PyObject* k_total_seconds; PyObject* k_bad_step;

bool put(PyObject* dict, PyObject* key, const at::Tensor& t)
{
    if (!t.defined()) return PyDict_SetItem(dict, key, Py_None) == 0;
    PyObject* v = THPVariable_Wrap(t);
    if (!v) return false;
    const int rc = PyDict_SetItem(dict, key, v);
    Py_DECREF(v);
    return rc == 0;
}

// eval(problem, steps, w32, schedules, want_steps, want_seconds, stream or None) -> dict of tensors, or an error code
PyObject* eval(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (nargs != 7) return value_error("eval takes 7 arguments");
    kvp_problem* p;
    unsigned long long S, w32;
    uint32_t n;
    void *sched, *st;
    if (!problem_of(args, &p, &S, &w32) || !batch_of(args[3], S * w32, &n) || !device_ptr(args[3], at::kInt, true, &sched)) return nullptr;
    const bool steps = PyObject_IsTrue(args[4]), seconds = PyObject_IsTrue(args[5]);
    const c10::Device dev = THPVariable_Unpack(args[3]).device();
    if (!stream_of(args[6], dev.index(), &st)) return nullptr;
    at::Tensor a, b, c, d, e;
    const int64_t rows[2] = {(int64_t)n, (int64_t)S}, one[1] = {(int64_t)n};
    int rc;
    {
        Unlocked unlocked;
        if (steps) a = make(rows, at::kLong, dev);
        b = make(one, at::kLong, dev);
        if (steps && seconds) c = make(rows, at::kDouble, dev);
        if (seconds) d = make(one, at::kDouble, dev);
        e = make(one, at::kInt, dev);
        rc = kvp_eval(p, static_cast<uint32_t*>(sched), n, steps ? static_cast<uint64_t*>(a.data_ptr()) : nullptr,
                      static_cast<uint64_t*>(b.data_ptr()), c.defined() ? static_cast<double*>(c.data_ptr()) : nullptr,
                      seconds ? static_cast<double*>(d.data_ptr()) : nullptr, static_cast<int32_t*>(e.data_ptr()), st);
    }
    if (rc) return PyLong_FromLong(rc);
    PyObject* out = PyDict_New();
    if (!out || !put(out, k_step_ticks, a) || !put(out, k_total_ticks, b) || !put(out, k_step_seconds, c) ||
        !put(out, k_total_seconds, d) || !put(out, k_bad_step, e)) {
        Py_XDECREF(out);
        return nullptr;
    }
    return out;
    END_HANDLE_TH_ERRORS
}

// eval_noalloc(problem, steps, w32, schedules, step_ticks, total_ticks, step_seconds, total_seconds, bad_step, stream or
// None) -> error code
PyObject* eval_noalloc(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (nargs != 10) return value_error("eval_noalloc takes 10 arguments");
    kvp_problem* p;
    unsigned long long S, w32;
    uint32_t n;
    void *sched, *o[5], *st;
    if (!problem_of(args, &p, &S, &w32) || !batch_of(args[3], S * w32, &n) || !device_ptr(args[3], at::kInt, true, &sched)) return nullptr;
    for (int i = 0; i < 5; ++i)
        if (!device_ptr(args[4 + i], at::kInt, false, &o[i])) return nullptr;
    if (!stream_of(args[9], THPVariable_Unpack(args[3]).device().index(), &st)) return nullptr;
    int rc;
    {
        Unlocked unlocked;
        rc = kvp_eval_noalloc(p, static_cast<uint32_t*>(sched), n, static_cast<uint64_t*>(o[0]), static_cast<uint64_t*>(o[1]),
                              static_cast<double*>(o[2]), static_cast<double*>(o[3]), static_cast<int32_t*>(o[4]), st);
    }
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// eval_counts(problem, steps, w32, schedules, stream or None) -> tensor, or an error code
PyObject* eval_counts(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (nargs != 5) return value_error("eval_counts takes 5 arguments");
    kvp_problem* p;
    unsigned long long S, w32;
    uint32_t n;
    void *sched, *st;
    if (!problem_of(args, &p, &S, &w32) || !batch_of(args[3], S * w32, &n) || !device_ptr(args[3], at::kInt, true, &sched)) return nullptr;
    const c10::Device dev = THPVariable_Unpack(args[3]).device();
    if (!stream_of(args[4], dev.index(), &st)) return nullptr;
    const int64_t shape[3] = {(int64_t)n, (int64_t)S, 4};
    at::Tensor t;
    int rc;
    {
        Unlocked unlocked;
        t = make(shape, at::kInt, dev);
        rc = kvp_eval_counts(p, static_cast<uint32_t*>(sched), n, static_cast<uint32_t*>(t.data_ptr()), st);
    }
    return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(t);
    END_HANDLE_TH_ERRORS
}

// ---- the calls between a model's attention and the placement problem ----
// Outputs and workspaces are allocated on the stream the call runs on, so that their memory is not given to another call before
// the kernels are done with it; the device is that of the tensors, whichever is current.

const at::Tensor* tensor_of(PyObject* o, const char* what)
{
    if (!THPVariable_Check(o)) { PyErr_Format(PyExc_TypeError, "%s: expected a tensor", what); return nullptr; }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda()) { PyErr_Format(PyExc_ValueError, "%s: expected a CUDA tensor", what); return nullptr; }
    return &t;
}

// a contiguous tensor of `dtype` on `dev`; *out is null where None is given and allowed
bool dense(PyObject* o, const char* what, at::ScalarType dtype, c10::Device dev, bool none, const at::Tensor** out)
{
    *out = nullptr;
    if (none && o == Py_None) return true;
    const at::Tensor* t = tensor_of(o, what);
    if (!t) return false;
    if (t->device() != dev) { PyErr_Format(PyExc_ValueError, "%s: on another device", what); return false; }
    if (!t->is_contiguous()) { PyErr_Format(PyExc_ValueError, "%s: expected a contiguous CUDA tensor", what); return false; }
    if (t->scalar_type() != dtype) { PyErr_Format(PyExc_ValueError, "%s: expected dtype torch.%s", what, dtype == at::kInt ? "int32" : dtype == at::kLong ? "int64" : dtype == at::kByte ? "uint8" : "float32"); return false; }
    *out = t;
    return true;
}

void* data_of(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

int dtype_code(at::ScalarType t) { return t == at::kBFloat16 ? (int)KVP_BF16 : t == at::kHalf ? (int)KVP_F16 : t == at::kFloat ? (int)KVP_F32 : -1; }

bool u32_of(PyObject* o, const char* what, uint32_t* v)
{
    const long long x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) return false;
    if (x < 0 || x > 0xFFFFFFFFll) { PyErr_Format(PyExc_ValueError, "%s: out of range", what); return false; }
    *v = (uint32_t)x;
    return true;
}

bool size_fits(int64_t n, const char* what, uint32_t* v)
{
    if (n < 0 || n > 0xFFFFFFFFll) { PyErr_Format(PyExc_ValueError, "%s: too large", what); return false; }
    *v = (uint32_t)n;
    return true;
}

// [pages][kv_heads][bytes of a page] uint8
bool cache_of(PyObject* o, int64_t head_dim, kvp_cache_shape* c, const at::Tensor** out)
{
    const at::Tensor* t = tensor_of(o, "cache");
    if (!t || !dense(o, "cache", at::kByte, t->device(), false, out)) return false;
    if (t->dim() != 3) { value_error("cache must be [pages][kv_heads][page bytes]"); return false; }
    if (reinterpret_cast<uintptr_t>(t->data_ptr()) % 16) { value_error("cache must be 16-byte aligned"); return false; }
    const int64_t bytes = t->size(2);
    if (head_dim <= 0 || bytes <= 0 || bytes % (20 * head_dim)) { value_error("cache: the bytes of a page do not belong to this head_dim"); return false; }
    c->reserved = 0;
    return size_fits(t->size(0), "pages", &c->pages) && size_fits(t->size(1), "kv_heads", &c->kv_heads) &&
           size_fits(head_dim, "head_dim", &c->head_dim) && size_fits(bytes / (20 * head_dim) * 16, "page_tokens", &c->page_tokens);
}

bool cuda_stream_of(PyObject* o, c10::Device dev, c10::cuda::CUDAStream* out)
{
    if (o == Py_None) { *out = c10::cuda::getCurrentCUDAStream(dev.index()); return true; }
    void* p = PyLong_AsVoidPtr(o);
    if (PyErr_Occurred()) return false;
    *out = c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(p), dev.index());
    return true;
}

// keys or values [tokens][kv_heads][head_dim], dims contiguous
bool rows_of(PyObject* o, const char* what, const kvp_cache_shape& c, c10::Device dev, const at::Tensor** out)
{
    const at::Tensor* t = tensor_of(o, what);
    if (!t) return false;
    if (t->dim() != 3 || t->size(1) != (int64_t)c.kv_heads) { PyErr_Format(PyExc_ValueError, "%s must be [tokens][kv_heads][head_dim]", what); return false; }
    if (t->device() != dev) { PyErr_Format(PyExc_ValueError, "%s: on another device", what); return false; }
    if (t->stride(2) != 1) { PyErr_Format(PyExc_ValueError, "%s: dims must be contiguous", what); return false; }
    *out = t;
    return true;
}

// cache_append(cache, k, v, slots, stream or None) -> error code
PyObject* cache_append(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (!kvp_cache_append) return missing("kvp_cache_append");
    if (nargs != 5) return value_error("cache_append takes 5 arguments");
    kvp_cache_shape c;
    const at::Tensor *k = tensor_of(args[1], "k"), *v, *slots, *cache;
    if (!k) return nullptr;
    if (k->dim() != 3) return value_error("k must be [tokens][kv_heads][head_dim]");
    if (!cache_of(args[0], k->size(2), &c, &cache)) return nullptr;
    const c10::Device dev = cache->device();
    if (!rows_of(args[1], "k", c, dev, &k) || !rows_of(args[2], "v", c, dev, &v) || !dense(args[3], "slots", at::kLong, dev, false, &slots)) return nullptr;
    uint32_t tokens;
    const int code = dtype_code(k->scalar_type());
    if (code < 0 || v->scalar_type() != k->scalar_type()) return value_error("k and v must both be bfloat16, float16 or float32");
    if (v->sizes() != k->sizes() || slots->numel() != k->size(0)) return value_error("k, v and slots must have the same number of tokens");
    if (!size_fits(k->size(0), "tokens", &tokens)) return nullptr;
    c10::cuda::CUDAStream st = c10::cuda::getDefaultCUDAStream(dev.index());
    if (!cuda_stream_of(args[4], dev, &st)) return nullptr;
    int rc;
    {
        Unlocked unlocked;
        c10::cuda::CUDAStreamGuard guard(st);
        rc = kvp_cache_append(&c, cache->data_ptr(), (uint32_t)code, tokens, k->data_ptr(), k->stride(0), k->stride(1), v->data_ptr(),
                              v->stride(0), v->stride(1), static_cast<const int64_t*>(slots->data_ptr()), st.stream());
    }
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// cache_read(cache, slots, head_dim, a tensor of the dtype or its code, stream or None) -> (k, v), or an error code
PyObject* cache_read(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (!kvp_cache_read) return missing("kvp_cache_read");
    if (nargs != 5) return value_error("cache_read takes 5 arguments");
    kvp_cache_shape c;
    const at::Tensor *cache, *slots;
    uint32_t head_dim, code, tokens;
    if (!u32_of(args[2], "head_dim", &head_dim) || !u32_of(args[3], "dtype", &code) || !cache_of(args[0], head_dim, &c, &cache)) return nullptr;
    const c10::Device dev = cache->device();
    if (!dense(args[1], "slots", at::kLong, dev, false, &slots) || !size_fits(slots->numel(), "tokens", &tokens)) return nullptr;
    if (code > KVP_F32) return value_error("dtype must be bfloat16, float16 or float32");
    c10::cuda::CUDAStream st = c10::cuda::getDefaultCUDAStream(dev.index());
    if (!cuda_stream_of(args[4], dev, &st)) return nullptr;
    at::Tensor k, v;
    int rc;
    {
        Unlocked unlocked;
        c10::cuda::CUDAStreamGuard guard(st);
        const at::ScalarType t = code == KVP_BF16 ? at::kBFloat16 : code == KVP_F16 ? at::kHalf : at::kFloat;
        const int64_t shape[3] = {(int64_t)tokens, (int64_t)c.kv_heads, (int64_t)head_dim};
        k = make(shape, t, dev);
        v = make(shape, t, dev);
        rc = kvp_cache_read(&c, cache->data_ptr(), code, tokens, static_cast<const int64_t*>(slots->data_ptr()), k.data_ptr(), v.data_ptr(), st.stream());
    }
    if (rc) return PyLong_FromLong(rc);
    PyObject *a = THPVariable_Wrap(k), *b = THPVariable_Wrap(v);
    if (!a || !b) { Py_XDECREF(a); Py_XDECREF(b); return nullptr; }
    return Py_BuildValue("(NN)", a, b);
    END_HANDLE_TH_ERRORS
}

PyObject* k_out; PyObject* k_lse; PyObject* k_weights; PyObject* k_kept; PyObject* k_acc;

// attend(q, cache, table, lens, unit_tokens or 0, scale or None, units or None, want_lse, weights: bool or a tensor to write to,
// stream or None) -> dict, or an error code
PyObject* attend(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (!kvp_attend) return missing("kvp_attend");
    if (nargs != 10) return value_error("attend takes 10 arguments");
    const at::Tensor *q = tensor_of(args[0], "q"), *cache, *table, *lens, *units, *weights = nullptr;
    if (!q) return nullptr;
    if (q->dim() != 3 && q->dim() != 4) return value_error("q must be [batch][heads][head_dim] or [batch][queries][heads][head_dim]");
    const int64_t d = q->dim(), head_dim = q->size(d - 1), heads = q->size(d - 2), queries = d == 4 ? q->size(1) : 1;
    kvp_attend_params p;
    if (!cache_of(args[1], head_dim, &p.cache, &cache)) return nullptr;
    const c10::Device dev = cache->device();
    if (q->device() != dev) return value_error("q: on another device");
    if (q->stride(d - 1) != 1) return value_error("q: dims must be contiguous");
    if (q->scalar_type() != at::kBFloat16 && q->scalar_type() != at::kHalf) return value_error("q must be bfloat16 or float16");
    if (!p.cache.kv_heads || heads % p.cache.kv_heads) return value_error("q: heads must be a multiple of the cache's kv_heads");
    if (!dense(args[2], "table", at::kInt, dev, false, &table) || !dense(args[3], "lens", at::kInt, dev, false, &lens) ||
        !dense(args[6], "units", at::kInt, dev, true, &units)) return nullptr;
    if (table->dim() != 2 || table->size(0) != q->size(0) || lens->numel() != q->size(0)) return value_error("table must be [batch][pages] and lens [batch]");
    if (!size_fits(q->size(0), "batch", &p.batch) || !size_fits(queries, "queries", &p.queries) ||
        !size_fits(heads / p.cache.kv_heads, "heads", &p.group) || !size_fits(table->size(1), "table", &p.table_pages) ||
        !u32_of(args[4], "unit_tokens", &p.unit_tokens)) return nullptr;
    if (!p.unit_tokens) p.unit_tokens = p.cache.page_tokens;
    p.dtype = (uint32_t)dtype_code(q->scalar_type());
    const double scale = args[5] == Py_None ? 1.0 / std::sqrt((double)head_dim) : PyFloat_AsDouble(args[5]);
    if (PyErr_Occurred()) return nullptr;
    p.scale = (float)scale;
    p.reserved = 0;
    p.q_batch_stride = q->stride(0);
    p.q_query_stride = d == 4 ? q->stride(1) : 0;
    p.q_head_stride = q->stride(d - 2);
    const bool want_lse = PyObject_IsTrue(args[7]);
    bool want_weights = args[8] == Py_True;
    if (args[8] != Py_True && args[8] != Py_False && args[8] != Py_None) {
        if (!dense(args[8], "weights", at::kFloat, dev, false, &weights)) return nullptr;
        want_weights = true;
    }
    uint64_t bytes = 0;
    int rc = kvp_attend_workspace(&p, want_weights, units != nullptr, &bytes);
    if (rc) return PyLong_FromLong(rc);
    const int64_t n = (int64_t)p.table_pages * p.cache.page_tokens / p.unit_tokens, all = (int64_t)p.batch * p.cache.kv_heads * n;
    if (weights && weights->numel() != all) return value_error("weights must be [batch][kv_heads][units]");
    if (units && units->numel() < (all + 31) / 32) return value_error("units: too few words for batch * kv_heads * units bits");
    c10::cuda::CUDAStream st = c10::cuda::getDefaultCUDAStream(dev.index());
    if (!cuda_stream_of(args[9], dev, &st)) return nullptr;
    at::Tensor out, lse, made;
    {
        Unlocked unlocked;
        c10::cuda::CUDAStreamGuard guard(st);
        out = make(q->sizes(), q->scalar_type(), dev);
        if (want_lse) lse = make(q->sizes().slice(0, d - 1), at::kFloat, dev);
        const int64_t shape[3] = {(int64_t)p.batch, (int64_t)p.cache.kv_heads, n}, room[1] = {(int64_t)bytes};
        if (want_weights) made = weights ? *weights : make(shape, at::kFloat, dev);
        const at::Tensor workspace = make(room, at::kByte, dev);
        rc = kvp_attend(&p, q->data_ptr(), cache->data_ptr(), static_cast<const int32_t*>(table->data_ptr()),
                        static_cast<const int32_t*>(lens->data_ptr()), static_cast<const uint32_t*>(data_of(units)), out.data_ptr(),
                        want_lse ? static_cast<float*>(lse.data_ptr()) : nullptr, want_weights ? static_cast<float*>(made.data_ptr()) : nullptr,
                        workspace.data_ptr(), bytes, st.stream());
    }
    if (rc) return PyLong_FromLong(rc);
    PyObject* r = PyDict_New();
    if (!r || !put(r, k_out, out) || !put(r, k_lse, lse) || !put(r, k_weights, made)) {
        Py_XDECREF(r);
        return nullptr;
    }
    return r;
    END_HANDLE_TH_ERRORS
}

// recorded weights [steps][units], float32; a single step may come without its dimension
bool weights_of(PyObject* o, uint32_t groups, uint32_t* n, uint32_t* steps, const at::Tensor** out)
{
    const at::Tensor* t = tensor_of(o, "weights");
    if (!t || !dense(o, "weights", at::kFloat, t->device(), false, out)) return false;
    if (t->dim() < 1 || t->dim() > 2) { value_error("weights must be [steps][units] or [units]"); return false; }
    const int64_t units = t->size(t->dim() - 1);
    if (!groups || units % groups) { value_error("weights: the units do not divide into the groups"); return false; }
    return size_fits(units / groups, "units", n) && size_fits(t->dim() == 2 ? t->size(0) : 1, "steps", steps);
}

// trace_weights(weights, groups, topk, out or None, stream or None) -> bitmaps, or an error code
PyObject* trace_weights(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (!kvp_trace_weights) return missing("kvp_trace_weights");
    if (nargs != 5) return value_error("trace_weights takes 5 arguments");
    const at::Tensor *w, *given;
    uint32_t groups, n, steps, topk;
    if (!u32_of(args[1], "groups", &groups) || !u32_of(args[2], "topk", &topk) || !weights_of(args[0], groups, &n, &steps, &w)) return nullptr;
    const c10::Device dev = w->device();
    const int64_t shape[2] = {(int64_t)steps, ((int64_t)groups * n + 31) / 32};
    if (!dense(args[3], "out", at::kInt, dev, true, &given)) return nullptr;
    if (given && given->numel() != shape[0] * shape[1]) return value_error("out must be [steps][words]");
    c10::cuda::CUDAStream st = c10::cuda::getDefaultCUDAStream(dev.index());
    if (!cuda_stream_of(args[4], dev, &st)) return nullptr;
    at::Tensor out;
    int rc;
    {
        Unlocked unlocked;
        c10::cuda::CUDAStreamGuard guard(st);
        out = given ? *given : make(shape, at::kInt, dev);
        rc = kvp_trace_weights(groups, n, steps, topk, static_cast<const float*>(w->data_ptr()), static_cast<uint32_t*>(out.data_ptr()), st.stream());
    }
    return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// evict(weights, groups, budget, sink, recent, decay_q, acc or None, kept or None, exist or None, acc_out or None, stream or None, carry)
// -> dict, or an error code
PyObject* evict(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (!kvp_evict) return missing("kvp_evict");
    if (nargs != 12) return value_error("evict takes 12 arguments");
    const at::Tensor *w, *acc, *kept, *exist, *acc_out;
    kvp_evict_params p;
    const int carry = PyObject_IsTrue(args[11]);
    if (carry < 0) return nullptr;
    p.flags = carry ? KVP_EVICT_CARRY : 0;
    if (!u32_of(args[1], "groups", &p.groups) || !u32_of(args[2], "budget", &p.budget) || !u32_of(args[3], "sink", &p.sink) ||
        !u32_of(args[4], "recent", &p.recent) || !u32_of(args[5], "decay_q", &p.decay_q) ||
        !weights_of(args[0], p.groups, &p.units_per_group, &p.steps, &w)) return nullptr;
    const c10::Device dev = w->device();
    if (!dense(args[6], "acc", at::kLong, dev, true, &acc) || !dense(args[7], "kept", at::kInt, dev, true, &kept) ||
        !dense(args[8], "exist", at::kInt, dev, true, &exist) || !dense(args[9], "acc_out", at::kLong, dev, true, &acc_out)) return nullptr;
    const int64_t units = (int64_t)p.groups * p.units_per_group, words = (units + 31) / 32;
    if ((acc && acc->numel() != units) || (acc_out && acc_out->numel() != units)) return value_error("acc must have one entry per unit");
    if (kept && kept->numel() != words) return value_error("kept must be a row of the bitmap");
    if (exist && exist->numel() != (carry ? (int64_t)p.steps : 1) * p.groups)
        return value_error(carry ? "exist must have one entry per step and group" : "exist must have one entry per group");
    c10::cuda::CUDAStream st = c10::cuda::getDefaultCUDAStream(dev.index());
    if (!cuda_stream_of(args[10], dev, &st)) return nullptr;
    at::Tensor rows, sums;
    int rc;
    {
        Unlocked unlocked;
        c10::cuda::CUDAStreamGuard guard(st);
        const int64_t shape[2] = {(int64_t)p.steps, words}, one[1] = {units};
        rows = make(shape, at::kInt, dev);
        sums = acc_out ? *acc_out : make(one, at::kLong, dev);
        rc = kvp_evict(&p, static_cast<const float*>(w->data_ptr()), static_cast<const int64_t*>(data_of(acc)),
                       static_cast<int64_t*>(sums.data_ptr()), static_cast<const uint32_t*>(data_of(kept)),
                       static_cast<const int32_t*>(data_of(exist)), static_cast<uint32_t*>(rows.data_ptr()), st.stream());
    }
    if (rc) return PyLong_FromLong(rc);
    PyObject* r = PyDict_New();
    if (!r || !put(r, k_kept, rows) || !put(r, k_acc, sums)) {
        Py_XDECREF(r);
        return nullptr;
    }
    return r;
    END_HANDLE_TH_ERRORS
}

// current_stream() -> the cudaStream_t of the current device's current stream
PyObject* current_stream(PyObject*, PyObject*)
{
    HANDLE_TH_ERRORS
    return PyLong_FromVoidPtr(c10::cuda::getCurrentCUDAStream().stream());
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"current_stream", current_stream, METH_NOARGS, nullptr},
    {"eval", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(eval)), METH_FASTCALL, nullptr},
    {"eval_noalloc", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(eval_noalloc)), METH_FASTCALL, nullptr},
    {"eval_counts", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(eval_counts)), METH_FASTCALL, nullptr},
    {"cache_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(cache_append)), METH_FASTCALL, nullptr},
    {"cache_read", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(cache_read)), METH_FASTCALL, nullptr},
    {"attend", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attend)), METH_FASTCALL, nullptr},
    {"trace_weights", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(trace_weights)), METH_FASTCALL, nullptr},
    {"evict", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(evict)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kvp_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kvp_torch()
{
    k_step_ticks = PyUnicode_InternFromString("step_ticks");
    k_total_ticks = PyUnicode_InternFromString("total_ticks");
    k_step_seconds = PyUnicode_InternFromString("step_seconds");
    k_total_seconds = PyUnicode_InternFromString("total_seconds");
    k_bad_step = PyUnicode_InternFromString("bad_step");
    k_out = PyUnicode_InternFromString("out");
    k_lse = PyUnicode_InternFromString("lse");
    k_weights = PyUnicode_InternFromString("weights");
    k_kept = PyUnicode_InternFromString("kept");
    k_acc = PyUnicode_InternFromString("acc");
    return PyModule_Create(&module);
}
