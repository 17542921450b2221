// Python entry of the calls that a program makes every iteration: torch tensors -> raw device pointers -> the C
// functions of lq.h on torch's current stream.  The checks are those of binding.py's ctypes route, which still serves the
// calls made once.  What bounds a small iteration is the host: per call the ctypes route took about
// 8 us (eight attribute look-ups and conversions per tensor), this one takes well under 1 us beside the launches.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/core/grad_mode.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "lq.h"

namespace {

PyObject* g_error = nullptr;              // binding.LqError

bool fail(const char* msg)
{
    PyErr_SetString(g_error ? g_error : PyExc_RuntimeError, msg);
    return false;
}

// The tensor's device pointer, or NULL for None; false with an exception set when it is not a contiguous CUDA tensor
// of `type`.
template <typename T>
bool pointer(PyObject* o, at::ScalarType type, T** out)
{
    *out = nullptr;
    if (o == Py_None) return true;
    if (!THPVariable_Check(o)) return fail("expected a contiguous CUDA tensor");
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) return fail("expected a contiguous CUDA tensor");
    if (t.scalar_type() != type) {
        PyErr_Format(g_error ? g_error : PyExc_RuntimeError, "expected dtype %s, got %s", c10::toString(type),
                     c10::toString(t.scalar_type()));
        return false;
    }
    *out = reinterpret_cast<T*>(t.data_ptr());
    return true;
}

bool arity(Py_ssize_t got, Py_ssize_t want)
{
    if (got == want) return true;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, got);
    return false;
}

bool plan_of(PyObject* o, lq_plan** out)
{
    if (o == Py_None) { *out = nullptr; return true; }       // a closed plan: the C function reports it
    *out = static_cast<lq_plan*>(PyLong_AsVoidPtr(o));
    return !(*out == nullptr && PyErr_Occurred());
}

bool int_of(PyObject* o, int32_t* out)
{
    *out = static_cast<int32_t>(PyLong_AsUnsignedLongMask(o));       // (ctypes takes the low 32 bits as well)
    return !PyErr_Occurred();
}

PyObject* done(int code)
{
    if (code == LQ_OK) Py_RETURN_NONE;
    PyErr_Format(g_error ? g_error : PyExc_RuntimeError, "%s (%d): %s", lq_error_string(code), code, lq_last_error());
    return nullptr;
}

// Runs a C function on torch's current stream, without the interpreter lock (a full launch queue blocks the caller).
template <typename F>
PyObject* call(F&& f)
{
    void* s = static_cast<void*>(c10::cuda::getCurrentCUDAStream().stream());
    int code;
    Py_BEGIN_ALLOW_THREADS
    try { code = f(s); } catch (...) { code = LQ_ENOMEM; }    // (nothing but an allocation can throw there)
    Py_END_ALLOW_THREADS
    return done(code);
}

constexpr at::ScalarType kF32 = at::kFloat, kI32 = at::kInt, kI16 = at::kShort, kF64 = at::kDouble;

PyObject* quantize_pack(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    lq_plan* p; float *grads, *norms, *prev_norms; uint32_t *packed, *hist, *prev;
    if (!arity(n, 8) || !plan_of(a[0], &p) || !pointer(a[1], kF32, &grads)) return nullptr;
    const uint32_t step = static_cast<uint32_t>(PyLong_AsUnsignedLongMask(a[2]));
    if (PyErr_Occurred()) return nullptr;
    if (!pointer(a[3], kI32, &packed) || !pointer(a[4], kF32, &norms) || !pointer(a[5], kI32, &hist) ||
        !pointer(a[6], kI32, &prev) || !pointer(a[7], kF32, &prev_norms)) return nullptr;
    return call([&](void* s) { return lq_quantize_pack(p, grads, step, packed, norms, hist, prev, prev_norms, s); });
}

PyObject* step_qoda(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    lq_plan* p; uint32_t* packed; float *norms, *X1, *Y, *Xhalf, *X, *gbar;
    if (!arity(n, 8) || !plan_of(a[0], &p) || !pointer(a[1], kI32, &packed) || !pointer(a[2], kF32, &norms) ||
        !pointer(a[3], kF32, &X1) || !pointer(a[4], kF32, &Y) || !pointer(a[5], kF32, &Xhalf) || !pointer(a[6], kF32, &X) ||
        !pointer(a[7], kF32, &gbar)) return nullptr;
    return call([&](void* s) { return qoda_step(p, packed, norms, X1, Y, Xhalf, X, gbar, s); });
}

PyObject* layer_norms(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    lq_plan* p; float *grads, *norms;
    if (!arity(n, 3) || !plan_of(a[0], &p) || !pointer(a[1], kF32, &grads) || !pointer(a[2], kF32, &norms)) return nullptr;
    return call([&](void* s) { return lq_layer_norms(p, grads, norms, s); });
}

PyObject* decode_aggregate(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    lq_plan* p; uint32_t* packed; float *norms, *gbar;
    if (!arity(n, 4) || !plan_of(a[0], &p) || !pointer(a[1], kI32, &packed) || !pointer(a[2], kF32, &norms) ||
        !pointer(a[3], kF32, &gbar)) return nullptr;
    return call([&](void* s) { return lq_decode_aggregate(p, packed, norms, gbar, s); });
}

PyObject* fit_levels(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    lq_plan* p; uint32_t* hist; float* norms; int32_t z;
    if (!arity(n, 4) || !plan_of(a[0], &p) || !pointer(a[1], kI32, &hist) || !pointer(a[2], kF32, &norms) || !int_of(a[3], &z))
        return nullptr;
    return call([&](void* s) { return lq_fit_levels(p, hist, norms, z, s); });
}

PyObject* level_probabilities(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    lq_plan* p; uint32_t* hist; float* norms; double* probs; int32_t z;
    if (!arity(n, 6) || !plan_of(a[0], &p) || !pointer(a[1], kI32, &hist) || !pointer(a[2], kF32, &norms) || !int_of(a[3], &z) ||
        !pointer(a[5], kF64, &probs)) return nullptr;
    const int staged = PyObject_IsTrue(a[4]);
    if (staged < 0) return nullptr;
    return call([&](void* s) { return lq_level_probabilities(p, hist, norms, z, staged, probs, s); });
}

PyObject* symbol_counts(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    lq_plan* p; uint32_t *packed, *counts;
    if (!arity(n, 3) || !plan_of(a[0], &p) || !pointer(a[1], kI32, &packed) || !pointer(a[2], kI32, &counts)) return nullptr;
    return call([&](void* s) { return lq_symbol_counts(p, packed, counts, s); });
}

// words per row of the [K][capacity] stream buffer
bool capacity_of(PyObject* o, int64_t* out)
{
    if (!THPVariable_Check(o) || THPVariable_Unpack(o).dim() < 2) return fail("stream_words must be a [K][capacity] tensor");
    *out = THPVariable_Unpack(o).size(1);
    return true;
}

PyObject* entropy_encode(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    lq_plan* p; uint32_t *packed, *words, *off; uint16_t* runs; int64_t cap;
    if (!arity(n, 5) || !plan_of(a[0], &p) || !pointer(a[1], kI32, &packed) || !pointer(a[2], kI32, &words) ||
        !capacity_of(a[2], &cap) || !pointer(a[3], kI32, &off) || !pointer(a[4], kI16, &runs)) return nullptr;
    return call([&](void* s) { return lq_entropy_encode(p, packed, words, cap, off, runs, s); });
}

PyObject* entropy_decode(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    lq_plan* p; uint32_t *packed, *words, *off; uint16_t* runs; int64_t cap;
    if (!arity(n, 5) || !plan_of(a[0], &p) || !pointer(a[1], kI32, &words) || !capacity_of(a[1], &cap) ||
        !pointer(a[2], kI32, &off) || !pointer(a[3], kI16, &runs) || !pointer(a[4], kI32, &packed)) return nullptr;
    return call([&](void* s) { return lq_entropy_decode(p, words, cap, off, runs, packed, s); });
}

PyObject* vector_norm_static(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    float *v, *out; uint32_t* st; int32_t q;
    if (!arity(n, 4) || (a[0] == Py_None && !fail("expected a contiguous CUDA tensor")) || !pointer(a[0], kF32, &v) || !int_of(a[1], &q) || !pointer(a[2], kF32, &out) || !pointer(a[3], kI32, &st))
        return nullptr;
    const int64_t len = THPVariable_Unpack(a[0]).numel();
    return call([&](void* s) { return lq_vector_norm_static(v, len, q, out, st, s); });
}

// ---- the key-value cache: its tensors may have strides and have to be on its device, on whose current stream its calls run

struct CacheInfo { lq_cache* cache; int32_t heads, dim, page_size, device; };

bool cache_of(PyObject* o, CacheInfo* c)
{
    c->cache = o == Py_None ? nullptr : static_cast<lq_cache*>(PyLong_AsVoidPtr(o));
    if (PyErr_Occurred()) return false;
    if (lq_cache_info(c->cache, &c->heads, &c->dim, &c->page_size, &c->device) == LQ_OK) return true;
    done(LQ_EINVAL);
    return false;
}

// A tensor on the cache's device of one of the types given; NULL with an exception set otherwise.
const at::Tensor* on_device(PyObject* o, const CacheInfo& c, const char* name)
{
    if (THPVariable_Check(o)) {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.is_cuda() && t.get_device() == c.device) return &t;
    }
    PyErr_Format(g_error ? g_error : PyExc_RuntimeError, "%s: expected a CUDA tensor on the cache's device (cuda:%d)", name, c.device);
    return nullptr;
}

bool wrong(const char* name, const char* what)
{
    PyErr_Format(g_error ? g_error : PyExc_RuntimeError, "%s: expected %s", name, what);
    return false;
}

// Outputs of these calls carry no gradient: a tensor that one would have to pass through is refused, not cut off silently.
bool no_gradient(PyObject* o, const char* name)
{
    if (!THPVariable_Check(o) || !at::GradMode::is_enabled() || !THPVariable_Unpack(o).requires_grad()) return true;
    return wrong(name, "a tensor without a gradient (detach it, or call under torch.no_grad())");
}

// [tokens][heads][head_dim] rows with the coordinates side by side; heads 0: any number.
bool rows_of(PyObject* o, const CacheInfo& c, const char* name, int64_t tokens, int64_t heads, lq_rows* out)
{
    const at::Tensor* t = on_device(o, c, name);
    if (!t) return false;
    const at::ScalarType type = t->scalar_type();
    if (type != at::kFloat && type != at::kHalf && type != at::kBFloat16) return wrong(name, "float32, float16 or bfloat16");
    if (t->dim() != 3 || t->size(0) != tokens || (heads && t->size(1) != heads) || t->size(2) != c.dim) {
        PyErr_Format(g_error ? g_error : PyExc_RuntimeError, "%s: expected the shape [%lld][%lld][%d]", name, (long long)tokens,
                     (long long)(heads ? heads : c.heads), c.dim);
        return false;
    }
    if (t->stride(2) != 1 && t->size(2) != 1) return wrong(name, "coordinates side by side (a last stride of 1)");
    out->data = t->numel() ? t->data_ptr() : nullptr;
    out->token_stride = t->stride(0); out->head_stride = t->stride(1);
    out->type = type == at::kFloat ? LQ_F32 : type == at::kHalf ? LQ_F16 : LQ_BF16;
    return true;
}

// A contiguous tensor of `type` with `dim` dimensions (0: any).
template <typename T>
bool array_of(PyObject* o, const CacheInfo& c, const char* name, at::ScalarType type, int dim, T** out, const at::Tensor** tensor = nullptr)
{
    const at::Tensor* t = on_device(o, c, name);
    if (!t) return false;
    if (t->scalar_type() != type) return wrong(name, c10::toString(type));
    if (!t->is_contiguous() || (dim && t->dim() != dim)) return wrong(name, dim == 1 ? "a contiguous tensor of one dimension" : dim == 2 ? "a contiguous tensor of two dimensions" : "a contiguous tensor");
    *out = t->numel() ? reinterpret_cast<T*>(t->data_ptr()) : nullptr;
    if (tensor) *tensor = t;
    return true;
}

bool pages_of(PyObject* o, const CacheInfo& c, uint32_t** pages, int64_t* num)
{
    const at::Tensor* t;
    if (!array_of(o, c, "pages", at::kInt, 2, pages, &t)) return false;
    if (t->size(1) != lq_cache_page_words(c.cache)) return wrong("pages", "[num_pages][page_words]");
    *num = t->size(0);
    return true;
}

// table and positions (None: none); `interleaved` as a truth value
bool rotary_of(PyObject* table, PyObject* at, PyObject* interleaved, const CacheInfo& c, int64_t tokens, lq_rotary* r, bool* some)
{
    *some = table != Py_None;
    if (!*some) return at == Py_None || fail("positions: expected a rotary table with them");
    float* p;
    const at::Tensor* t;
    if (!array_of(table, c, "rotary", at::kFloat, 2, &p, &t)) return false;
    r->table = p; r->positions = t->size(0); r->at = nullptr;
    if (t->size(1) > c.dim) return wrong("rotary", "[positions][at most head_dim]");
    r->dim = static_cast<int32_t>(t->size(1));
    r->interleaved = PyObject_IsTrue(interleaved);
    if (r->interleaved < 0) return false;
    if (at == Py_None) return true;
    int64_t* q;
    if (!array_of(at, c, "positions", at::kLong, 1, &q, &t)) return false;
    if (t->numel() != tokens) return wrong("positions", "one a token");
    r->at = q;
    return true;
}

template <typename F>
PyObject* call_on(const CacheInfo& c, F&& f)
{
    void* s = static_cast<void*>(c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(c.device)).stream());
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = f(s);
    Py_END_ALLOW_THREADS
    return done(code);
}

// cache, layer, keys, values, slots, pages, step (-1: none), rotary, positions, interleaved
PyObject* cache_write(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    CacheInfo c; lq_rows k, v; int64_t *slots, pages; uint32_t* p; lq_rotary r; bool turned; int32_t layer; const at::Tensor* t;
    if (!arity(n, 10) || !cache_of(a[0], &c) || !int_of(a[1], &layer) || !array_of(a[4], c, "slots", at::kLong, 1, &slots, &t)) return nullptr;
    const int64_t tokens = t->numel(), step = PyLong_AsLongLong(a[6]);
    if (PyErr_Occurred()) return nullptr;
    if (!rows_of(a[2], c, "keys", tokens, c.heads, &k) || !rows_of(a[3], c, "values", tokens, c.heads, &v) || !pages_of(a[5], c, &p, &pages) ||
        !rotary_of(a[7], a[8], a[9], c, tokens, &r, &turned)) return nullptr;
    return call_on(c, [&](void* s) { return lq_cache_write(c.cache, layer, &k, &v, tokens, slots, p, pages, step, turned ? &r : nullptr, s); });
}

// cache, layer, pages, slots, keys, values
PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    CacheInfo c; lq_rows k, v; int64_t *slots, pages; uint32_t* p; int32_t layer; const at::Tensor* t;
    if (!arity(n, 6) || !cache_of(a[0], &c) || !int_of(a[1], &layer) || !pages_of(a[2], c, &p, &pages) ||
        !array_of(a[3], c, "slots", at::kLong, 1, &slots, &t) || !rows_of(a[4], c, "keys", t->numel(), c.heads, &k) ||
        !rows_of(a[5], c, "values", t->numel(), c.heads, &v) || !no_gradient(a[4], "keys") || !no_gradient(a[5], "values")) return nullptr;
    return call_on(c, [&](void* s) { return lq_cache_read(c.cache, layer, p, pages, t->numel(), slots, &k, &v, s); });
}

// cache, layer, queries, pages, table, lengths, out, lse, scale, window, rotary, positions, interleaved
PyObject* cache_attend(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    CacheInfo c; lq_rows q, o; int64_t pages; uint32_t* p; int32_t layer, *table, *lengths; lq_rotary r; bool turned;
    const at::Tensor *t, *l; float* lse = nullptr;
    if (!arity(n, 13) || !cache_of(a[0], &c) || !int_of(a[1], &layer) || !array_of(a[5], c, "lengths", at::kInt, 1, &lengths, &l)) return nullptr;
    const int64_t batch = l->numel();
    if (!rows_of(a[2], c, "queries", batch, 0, &q)) return nullptr;
    const int64_t heads = THPVariable_Unpack(a[2]).size(1);
    if (heads > INT32_MAX) return done(lq_cache_attend(c.cache, layer, &q, batch, -1, nullptr, 0, nullptr, 0, nullptr, 1, 0, nullptr, &q, nullptr, nullptr, 0, nullptr));
    if (!pages_of(a[3], c, &p, &pages) || !array_of(a[4], c, "table", at::kInt, 2, &table, &t)) return nullptr;
    if (t->size(0) != batch) { wrong("table", "a row a sequence"); return nullptr; }
    if (!rows_of(a[6], c, "out", batch, heads, &o)) return nullptr;
    if (!no_gradient(a[2], "queries") || !no_gradient(a[6], "out") || !no_gradient(a[7], "lse")) return nullptr;
    if (a[7] != Py_None) {
        const at::Tensor* e;
        if (!array_of(a[7], c, "lse", at::kFloat, 2, &lse, &e)) return nullptr;
        if (e->size(0) != batch || e->size(1) != heads) { wrong("lse", "[batch][heads]"); return nullptr; }
    }
    const double scale = PyFloat_AsDouble(a[8]);
    const int64_t window = PyErr_Occurred() ? 0 : PyLong_AsLongLong(a[9]);
    if (PyErr_Occurred() || !rotary_of(a[10], a[11], a[12], c, batch, &r, &turned)) return nullptr;
    // from torch's allocator, on the stream that the call runs on: a workspace of its own for every call, also in a graph
    const int64_t bytes = lq_cache_workspace(c.cache, t->size(1), window < 0 ? 0 : window);
    const at::Tensor space = bytes > 0 ? at::empty({bytes}, l->options().dtype(at::kByte)) : at::Tensor();
    return call_on(c, [&](void* s) {
        return lq_cache_attend(c.cache, layer, &q, batch, static_cast<int32_t>(heads), p, pages, table, t->size(1), lengths, static_cast<float>(scale),
                               window, turned ? &r : nullptr, &o, lse, bytes > 0 ? space.data_ptr() : nullptr, bytes, s);
    });
}

PyObject* register_error(PyObject*, PyObject* cls)
{
    Py_INCREF(cls);
    Py_XDECREF(g_error);
    g_error = cls;
    Py_RETURN_NONE;
}

// Every entry runs inside this: torch's accessors throw for tensors without plain memory (sparse ones, subclasses that answer
// for their layout themselves), and no C++ exception may leave through the interpreter's C frames.
template <PyObject* (*kEntry)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    return kEntry(self, a, n);
    END_HANDLE_TH_ERRORS
}

#define LQ_FAST(name, fn) {name, (PyCFunction)(void (*)(void))guarded<fn>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {LQ_FAST("lq_quantize_pack", quantize_pack), LQ_FAST("qoda_step", step_qoda),
                         LQ_FAST("lq_layer_norms", layer_norms), LQ_FAST("lq_decode_aggregate", decode_aggregate),
                         LQ_FAST("lq_fit_levels", fit_levels), LQ_FAST("lq_level_probabilities", level_probabilities),
                         LQ_FAST("lq_symbol_counts", symbol_counts), LQ_FAST("lq_entropy_encode", entropy_encode),
                         LQ_FAST("lq_entropy_decode", entropy_decode),
                         LQ_FAST("lq_vector_norm_static", vector_norm_static), LQ_FAST("lq_cache_write", cache_write),
                         LQ_FAST("lq_cache_read", cache_read), LQ_FAST("lq_cache_attend", cache_attend),
                         {"register_error", register_error, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
#undef LQ_FAST

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
