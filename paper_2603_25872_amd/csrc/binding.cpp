// The argument marshalling of the skip calls and of the attention operators as CPython functions.
//
// One anchor's skip transitions are a 3.4 us kernel behind a call that took 8.1 us: a launch of ~3 us and 5 us of ctypes structures, array
// types and argument conversion.  Here the same conversions and checks are done on the objects themselves: 8.1 -> 6.3 us a call
// (1 x 4096 elements, four targets).  The library's function comes as an address (bind), so this module links to nothing but the interpreter.
// The operators take two to five strided tensors each; a call that rotates one token: 11.2 -> 8.5 us with the allocation of its output, one that norms and
// rotates q and k of 12 x 256 tokens: 17.5 -> 11.9 (6.0 of it on the GPU).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <vector>

#include "../../include/drf.h"

namespace {

typedef drf_status (*SkipFn)(const drf_sched_config*, const float*, const float*, int, const int*, int, int, size_t, const drf_noise*, float*, void*);
SkipFn g_skip = nullptr;

PyObject *k_train_steps, *k_beta_start, *k_beta_end, *k_steps, *k_eta, *k_sampler, *k_shift, *k_get, *k_is_cuda, *k_is_contiguous, *k_dtype, *k_data_ptr, *k_shape, *k_stride, *k_get_device, *k_numel;
PyObject *k_zero, *k_one, *k_ddim;                   // eta, shift and sampler of a schedule that has none

// New reference to d[key], or to d.get(key, fallback) where there is one.
PyObject* item(PyObject* d, PyObject* key, PyObject* fallback)
{
    if (PyDict_CheckExact(d)) {
        PyObject* v = PyDict_GetItemWithError(d, key);
        if (!v && !PyErr_Occurred()) {
            v = fallback;
            if (!v) PyErr_SetObject(PyExc_KeyError, key);
        }
        Py_XINCREF(v);
        return v;
    }
    return fallback ? PyObject_CallMethodObjArgs(d, k_get, key, fallback, nullptr) : PyObject_GetItem(d, key);
}

// A C int as ctypes converts one: integers and what has __index__, the low bits of larger ones.
bool to_int(PyObject* v, int* out)
{
    const unsigned long u = PyLong_AsUnsignedLongMask(v);
    if (u == (unsigned long)-1 && PyErr_Occurred()) return false;
    *out = (int)u;
    return true;
}

// An integer; one with a fallback goes through int() first, a double with one through float() (which also take text).
bool int_item(PyObject* d, PyObject* key, int* out, PyObject* fallback = nullptr)
{
    PyObject* v = item(d, key, fallback);
    if (v && fallback) { PyObject* n = PyNumber_Long(v); Py_DECREF(v); v = n; }
    if (!v) return false;
    const bool ok = to_int(v, out);
    Py_DECREF(v);
    return ok;
}

bool double_item(PyObject* d, PyObject* key, double* out, PyObject* fallback = nullptr)
{
    PyObject* v = item(d, key, fallback);
    if (v && fallback) { PyObject* f = PyNumber_Float(v); Py_DECREF(v); v = f; }
    if (!v) return false;
    *out = PyFloat_AsDouble(v);
    Py_DECREF(v);
    return !(*out == -1.0 && PyErr_Occurred());
}

bool schedule(PyObject* d, drf_sched_config* sc)
{
    int which = 0;
    if (!int_item(d, k_train_steps, &sc->train_steps) || !double_item(d, k_beta_start, &sc->beta_start) ||
        !double_item(d, k_beta_end, &sc->beta_end) || !int_item(d, k_steps, &sc->steps) || !double_item(d, k_eta, &sc->eta, k_zero) ||
        !int_item(d, k_sampler, &which, k_ddim) || !double_item(d, k_shift, &sc->shift, k_one)) return false;
    sc->sampler = (decltype(sc->sampler))which;
    return true;
}

// Device pointer of a contiguous device tensor of the given dtype; None: NULL.
bool device_pointer(PyObject* t, PyObject* dtype, void** out)
{
    *out = nullptr;
    if (t == Py_None) return true;
    PyObject* v = PyObject_GetAttr(t, k_is_cuda);
    if (!v) return false;
    int ok = PyObject_IsTrue(v);
    Py_DECREF(v);
    if (ok > 0) {
        v = PyObject_CallMethodNoArgs(t, k_is_contiguous);
        if (!v) return false;
        ok = PyObject_IsTrue(v);
        Py_DECREF(v);
    }
    if (ok < 0) return false;
    if (!ok) { PyErr_SetString(PyExc_AssertionError, "need a contiguous device tensor"); return false; }
    v = PyObject_GetAttr(t, k_dtype);
    if (!v) return false;
    if (v != dtype) {                               // (dtypes are singletons)
        PyErr_Format(PyExc_AssertionError, "expected %S, got %S", dtype, v);
        Py_DECREF(v);
        return false;
    }
    Py_DECREF(v);
    v = PyObject_CallMethodNoArgs(t, k_data_ptr);
    if (!v) return false;
    *out = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return !(!*out && PyErr_Occurred());
}

// skip(sched, x_from, net_from, s_from, s_to, noise_address, out, float32, stream) -> status.  stream: a handle, or what gives the current one,
// which is asked last (it initialises the device, which a call that is refused has no need of).
PyObject* skip(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 9 || !g_skip) { PyErr_SetString(PyExc_TypeError, "skip() takes 9 arguments, after bind()"); return nullptr; }
    drf_sched_config sc{};
    if (!schedule(a[0], &sc)) return nullptr;
    PyObject* shape = PyObject_GetAttr(a[1], k_shape);
    if (!shape) return nullptr;
    PyObject* dims = PySequence_Tuple(shape);
    Py_DECREF(shape);
    if (!dims) return nullptr;
    size_t batch = 1, elems = 1;                    // a tensor without dimensions: one sample of one element
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(dims); ++i) {
        const size_t v = PyLong_AsSize_t(PyTuple_GET_ITEM(dims, i));
        if (v == (size_t)-1 && PyErr_Occurred()) { Py_DECREF(dims); return nullptr; }
        (i == 0 ? batch : elems) *= v;
    }
    Py_DECREF(dims);
    if (!batch) elems = 0;
    const Py_ssize_t m = PyObject_Length(a[4]);
    if (m < 0) return nullptr;
    // a tuple of our own: an element's __index__ is anybody's code (a device tensor's gives up the interpreter lock) and may change the caller's list
    PyObject* seq = PySequence_Tuple(a[4]);
    if (!seq) return nullptr;
    int few[16];
    std::vector<int> many;
    int* to = few;
    bool ok = PyTuple_GET_SIZE(seq) == m;
    if (!ok) PyErr_SetString(PyExc_IndexError, "invalid index");
    if (ok && m > 16) {
        try { many.resize((size_t)m); to = many.data(); } catch (...) { PyErr_NoMemory(); ok = false; }
    }
    for (Py_ssize_t i = 0; ok && i < m; ++i) ok = to_int(PyTuple_GET_ITEM(seq, i), &to[i]);
    Py_DECREF(seq);
    int s_from = 0;
    void *x = nullptr, *net = nullptr, *out = nullptr, *noise = nullptr, *stream = nullptr;
    ok = ok && device_pointer(a[1], a[7], &x) && device_pointer(a[2], a[7], &net) && to_int(a[3], &s_from) && device_pointer(a[6], a[7], &out);
    if (!ok) return nullptr;
    if (a[5] != Py_None && !(noise = PyLong_AsVoidPtr(a[5])) && PyErr_Occurred()) return nullptr;
    PyObject* handle = PyLong_Check(a[8]) ? Py_NewRef(a[8]) : PyObject_CallNoArgs(a[8]);
    if (!handle) return nullptr;
    stream = PyLong_AsVoidPtr(handle);
    Py_DECREF(handle);
    if (!stream && PyErr_Occurred()) return nullptr;
    drf_status rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_skip(&sc, (const float*)x, (const float*)net, s_from, to, (int)m, (int)batch, elems, (const drf_noise*)noise, (float*)out, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)rc);
}

// bind(address of drf_skip_transition_noise)
PyObject* bind(PyObject*, PyObject* address)
{
    void* p = PyLong_AsVoidPtr(address);
    if (!p) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "NULL address");
        return nullptr;
    }
    g_skip = reinterpret_cast<SkipFn>(p);
    Py_RETURN_NONE;
}

// ---- attention operators ------------------------------------------------------------------------------

struct Operators {
    decltype(&drf_rope) rope; decltype(&drf_qk_norm_rope) qk; decltype(&drf_block_words) words; decltype(&drf_block_select_scratch_bytes) scratch;
    decltype(&drf_block_select) select; decltype(&drf_block_attention_scratch_bytes) parts; decltype(&drf_block_attention_split) attend;
} g_ops = {};
PyObject *g_f32, *g_bf16, *g_i32, *g_device, *g_stream;     // dtypes; what gives the current device, and the current stream of a device

bool refuse(const char* text) { PyErr_SetString(PyExc_AssertionError, text); return false; }

bool attr_is(PyObject* t, PyObject* name, PyObject* want, bool* is)
{
    PyObject* v = PyObject_GetAttr(t, name);
    if (!v) return false;
    *is = v == want;                                        // (dtypes are singletons)
    Py_DECREF(v);
    return true;
}

// The four numbers of a tensor's shape or strides.
bool four(PyObject* v, long long (&out)[4])
{
    if (!v) return false;
    bool ok = PyTuple_Check(v) && PyTuple_GET_SIZE(v) == 4;
    if (!ok) refuse("need a device tensor [slots, tokens, heads, head_dim]");
    for (int i = 0; ok && i < 4; ++i) {
        out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(v, i));
        ok = !(out[i] == -1 && PyErr_Occurred());
    }
    Py_DECREF(v);
    return ok;
}

bool device_of(PyObject* t, long* device)
{
    PyObject* v = PyObject_GetAttr(t, k_is_cuda);
    if (!v) return false;
    const int cuda = PyObject_IsTrue(v);
    Py_DECREF(v);
    if (cuda < 0) return false;
    if (!cuda) return refuse("need a device tensor [slots, tokens, heads, head_dim]");
    v = PyObject_CallMethodNoArgs(t, k_get_device);
    if (!v) return false;
    *device = PyLong_AsLong(v);
    Py_DECREF(v);
    return !(*device == -1 && PyErr_Occurred());
}

struct Tensor { drf_heads h; long long size[4]; long device; drf_dtype dtype; };
// A tensor of heads, of the device and type of `like` if there is one, of its shape if `same`.
bool heads(PyObject* t, const Tensor* like, bool same, Tensor* out)
{
    bool is = false;
    long long stride[4];
    if (!device_of(t, &out->device) || !four(PyObject_GetAttr(t, k_shape), out->size) || !four(PyObject_CallMethodNoArgs(t, k_stride), stride)) return false;
    if (stride[3] != 1 && out->size[3] > 1) return refuse("a head's columns must be contiguous");
    if (!attr_is(t, k_dtype, g_bf16, &is)) return false;
    out->dtype = DRF_BF16;
    if (!is) {
        if (!attr_is(t, k_dtype, g_f32, &is)) return false;
        if (!is) return refuse("expected bfloat16 or float32");
        out->dtype = DRF_F32;
    }
    if (like && out->dtype != like->dtype) return refuse("tensors of two types");
    if (like && out->device != like->device) return refuse("tensors on two devices");
    for (int i = 0; i < 4; ++i) {
        if (out->size[i] > 0x7fffffff) return refuse("a size that does not fit 32 bits");
        if (same && out->size[i] != like->size[i]) return refuse("an output must have the shape of its input");
    }
    PyObject* p = PyObject_CallMethodNoArgs(t, k_data_ptr);
    if (!p) return false;
    out->h = { PyLong_AsVoidPtr(p), stride[0], stride[1], stride[2] };
    Py_DECREF(p);
    return !(!out->h.data && PyErr_Occurred());
}

// Device pointer of a contiguous tensor of `dtype` with n elements on `device`; None: NULL.
bool vector(PyObject* t, PyObject* dtype, long long n, long device, const char* what, void** out)
{
    *out = nullptr;
    if (t == Py_None) return true;
    if (!device_pointer(t, dtype, out)) return false;
    long d = -1;
    if (!device_of(t, &d)) return false;
    if (d != device) return refuse("tensors on two devices");
    PyObject* v = PyObject_CallMethodNoArgs(t, k_numel);
    if (!v) return false;
    const long long have = PyLong_AsLongLong(v);
    Py_DECREF(v);
    if (have == -1 && PyErr_Occurred()) return false;
    if (have != n) { PyErr_Format(PyExc_AssertionError, "%s must have %lld elements", what, n); return false; }
    return true;
}

// Positions [tokens, axes] or [slots, tokens, axes].
bool positions(PyObject* t, const drf_rope_config* rope, const Tensor& x, void** out, size_t* stride)
{
    *out = nullptr;
    *stride = 0;
    if (t == Py_None) return true;
    if (!rope) { PyErr_SetString(PyExc_ValueError, "positions without a rotation"); return false; }
    PyObject* shape = PyObject_GetAttr(t, k_shape);
    if (!shape) return false;
    const Py_ssize_t dims = PyTuple_Check(shape) ? PyTuple_GET_SIZE(shape) : -1;
    const long long want[3] = { x.size[0], x.size[1], rope->n_axes };
    bool ok = dims == 2 || dims == 3;
    for (Py_ssize_t i = 0; ok && i < dims; ++i) ok = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i)) == want[i + 3 - dims];
    Py_DECREF(shape);
    if (!ok) return !PyErr_Occurred() && refuse("positions must be [tokens, axes] or [slots, tokens, axes]");
    if (dims == 3) *stride = (size_t)(x.size[1] * rope->n_axes);
    return vector(t, g_f32, (dims == 3 ? x.size[0] : 1) * x.size[1] * rope->n_axes, x.device, "positions", out);
}

// The current stream, if x is on the current device.
bool current(const Tensor& x, void** stream)
{
    PyObject* v = PyObject_CallNoArgs(g_device);
    if (!v) return false;
    const long device = PyLong_AsLong(v);
    bool ok = !(device == -1 && PyErr_Occurred());
    if (ok && device != x.device) ok = refuse("the tensors are not on the current device");
    PyObject* s = ok ? PyObject_CallOneArg(g_stream, v) : nullptr;
    Py_DECREF(v);
    if (!s) return false;
    *stream = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    return !(!*stream && PyErr_Occurred());
}

bool address(PyObject* v, void** out)
{
    *out = nullptr;
    return v == Py_None || (*out = PyLong_AsVoidPtr(v)) || !PyErr_Occurred();
}

bool ready(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want && g_ops.rope) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments are taken, after bind_operators()", want);
    return false;
}

#define DRF_RUN(expr) drf_status rc; Py_BEGIN_ALLOW_THREADS rc = expr; Py_END_ALLOW_THREADS return PyLong_FromLong((long)rc)

// rope(x, out, address of the configuration, positions, lens) -> status
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Tensor x, y;
    void *rc_ = nullptr, *pos = nullptr, *lens = nullptr, *stream = nullptr;
    size_t pos_stride = 0;
    if (!ready(n, 5) || !heads(a[0], nullptr, false, &x) || !heads(a[1], &x, true, &y) || !address(a[2], &rc_)) return nullptr;
    const drf_rope_config* cfg = (const drf_rope_config*)rc_;
    if (!positions(a[3], cfg, x, &pos, &pos_stride) || !vector(a[4], g_i32, x.size[0], x.device, "lens", &lens) || !current(x, &stream)) return nullptr;
    DRF_RUN(g_ops.rope(cfg, x.dtype, (int)x.size[0], (int)x.size[1], (int)x.size[2], (int)x.size[3], (const int32_t*)lens, (const float*)pos, pos_stride, &x.h, &y.h, stream));
}

// qk_norm_rope(q, k, q_out, k_out, norm, eps, q_scale, q_gain, q_bias, k_gain, k_bias, address of the configuration or None, positions, lens) -> status
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Tensor q, k, qo, ko;
    void *rc_ = nullptr, *pos = nullptr, *lens = nullptr, *stream = nullptr, *par[4];
    size_t pos_stride = 0;
    int norm = 0;
    if (!ready(n, 14) || !heads(a[0], nullptr, false, &q) || !heads(a[1], &q, false, &k) || !heads(a[2], &q, true, &qo) || !heads(a[3], &k, true, &ko)) return nullptr;
    if (q.size[0] != k.size[0] || q.size[1] != k.size[1] || q.size[3] != k.size[3]) { refuse("k must have the slots, tokens and head width of q"); return nullptr; }
    drf_qk_config cfg{};
    if (!to_int(a[4], &norm)) return nullptr;
    cfg.norm = (drf_qk_norm)norm;
    cfg.eps = PyFloat_AsDouble(a[5]);
    if (cfg.eps == -1.0 && PyErr_Occurred()) return nullptr;
    const double scale = PyFloat_AsDouble(a[6]);
    if (scale == -1.0 && PyErr_Occurred()) return nullptr;
    cfg.q_scale = (float)scale;
    for (int i = 0; i < 4; ++i)
        if (!vector(a[7 + i], g_f32, q.size[3], q.device, "a norm's parameters", &par[i])) return nullptr;
    cfg.q_gain = (const float*)par[0]; cfg.q_bias = (const float*)par[1]; cfg.k_gain = (const float*)par[2]; cfg.k_bias = (const float*)par[3];
    if (!address(a[11], &rc_)) return nullptr;
    const drf_rope_config* rcfg = (const drf_rope_config*)rc_;
    if (!positions(a[12], rcfg, q, &pos, &pos_stride) || !vector(a[13], g_i32, q.size[0], q.device, "lens", &lens) || !current(q, &stream)) return nullptr;
    const drf_attn_shape s = { q.dtype, (int)q.size[0], (int)q.size[1], (int)k.size[1], (int)q.size[2], (int)k.size[2], (int)q.size[3], (const int32_t*)lens, nullptr };
    DRF_RUN(g_ops.qk(&cfg, rcfg, &s, (const float*)pos, pos_stride, &q.h, &k.h, &qo.h, &ko.h, stream));
}

bool attn_shape(PyObject* q_, PyObject* k_, PyObject* q_lens, PyObject* kv_lens, Tensor* q, Tensor* k, drf_attn_shape* s)
{
    void *ql = nullptr, *kl = nullptr;
    if (!heads(q_, nullptr, false, q) || !heads(k_, q, false, k)) return false;
    if (q->size[0] != k->size[0] || q->size[3] != k->size[3]) return refuse("k must have the slots and head width of q");
    if (!vector(q_lens, g_i32, q->size[0], q->device, "q_lens", &ql) || !vector(kv_lens, g_i32, q->size[0], q->device, "kv_lens", &kl)) return false;
    *s = { q->dtype, (int)q->size[0], (int)q->size[1], (int)k->size[1], (int)q->size[2], (int)k->size[2], (int)q->size[3], (const int32_t*)ql, (const int32_t*)kl };
    return true;
}

// Words of the bit masks of a shape.
long long mask_words(const drf_attn_shape& s, int q_block, int kv_block)
{
    const long long nq = q_block > 0 ? ((long long)s.q_tokens + q_block - 1) / q_block : 0;
    return nq * s.slots * s.q_heads * (long long)g_ops.words(s.kv_tokens, kv_block);
}

// block_select(q, k, out, q_block, kv_block, topk, q_lens, kv_lens, scratch) -> status
PyObject* block_select(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Tensor q, k;
    drf_attn_shape s;
    int qb = 0, kb = 0, topk = 0;
    void *out = nullptr, *scratch = nullptr, *stream = nullptr;
    if (!ready(n, 9) || !attn_shape(a[0], a[1], a[6], a[7], &q, &k, &s) || !to_int(a[3], &qb) || !to_int(a[4], &kb) || !to_int(a[5], &topk)) return nullptr;
    const size_t bytes = g_ops.scratch(&s, qb, kb);
    if (!vector(a[2], g_i32, mask_words(s, qb, kb), q.device, "the blocks' words", &out) || !vector(a[8], g_f32, (long long)(bytes / 4), q.device, "scratch", &scratch) ||
        !current(q, &stream)) return nullptr;
    DRF_RUN(g_ops.select(&s, qb, kb, topk, &q.h, &k.h, scratch, bytes, (uint32_t*)out, stream));
}

// block_attention(q, k, v, blocks, out, q_block, kv_block, scale, q_lens, kv_lens, scratch) -> status
PyObject* block_attention(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Tensor q, k, v, out;
    drf_attn_shape s;
    int qb = 0, kb = 0;
    void *blocks = nullptr, *scratch = nullptr, *stream = nullptr;
    if (!ready(n, 11) || !attn_shape(a[0], a[1], a[8], a[9], &q, &k, &s) || !heads(a[2], &k, true, &v) || !heads(a[4], &q, true, &out)) return nullptr;
    if (!to_int(a[5], &qb) || !to_int(a[6], &kb)) return nullptr;
    const double scale = PyFloat_AsDouble(a[7]);
    if (scale == -1.0 && PyErr_Occurred()) return nullptr;
    const size_t bytes = a[10] == Py_None ? 0 : g_ops.parts(&s);
    if (!vector(a[3], g_i32, mask_words(s, qb, kb), q.device, "the blocks' words", &blocks) || !vector(a[10], g_f32, (long long)(bytes / 4), q.device, "scratch", &scratch) ||
        !current(q, &stream)) return nullptr;
    DRF_RUN(g_ops.attend(&s, qb, kb, (float)scale, (const uint32_t*)blocks, &q.h, &k.h, &v.h, &out.h, scratch, bytes, stream));
}

// bind_operators((addresses), float32, bfloat16, int32, current device, current stream of a device)
PyObject* bind_operators(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 6 || !PyTuple_Check(a[0]) || PyTuple_GET_SIZE(a[0]) != 7) { PyErr_SetString(PyExc_TypeError, "bind_operators() takes seven addresses and five objects"); return nullptr; }
    void* p[7];
    for (int i = 0; i < 7; ++i)
        if (!(p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(a[0], i)))) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "NULL address");
            return nullptr;
        }
    PyObject** keep[5] = { &g_f32, &g_bf16, &g_i32, &g_device, &g_stream };
    for (int i = 0; i < 5; ++i) { Py_INCREF(a[1 + i]); Py_XSETREF(*keep[i], a[1 + i]); }
    g_ops = { (decltype(g_ops.rope))p[0], (decltype(g_ops.qk))p[1], (decltype(g_ops.words))p[2], (decltype(g_ops.scratch))p[3], (decltype(g_ops.select))p[4],
              (decltype(g_ops.parts))p[5], (decltype(g_ops.attend))p[6] };
    Py_RETURN_NONE;
}

#define DRF_FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL
PyMethodDef kMethods[] = {
    { "rope", DRF_FAST(rope), "status of drf_rope on these arguments" },
    { "qk_norm_rope", DRF_FAST(qk_norm_rope), "status of drf_qk_norm_rope on these arguments" },
    { "block_select", DRF_FAST(block_select), "status of drf_block_select on these arguments" },
    { "block_attention", DRF_FAST(block_attention), "status of drf_block_attention on these arguments" },
    { "bind_operators", DRF_FAST(bind_operators), "addresses of the operators' calls, dtypes, and what gives the current device and stream" },
    { "skip", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(skip)), METH_FASTCALL, "status of drf_skip_transition_noise on these arguments" },
    { "bind", bind, METH_O, "address of drf_skip_transition_noise" },
    { nullptr, nullptr, 0, nullptr },
};
PyModuleDef kModule = { PyModuleDef_HEAD_INIT, "_native", "Argument marshalling of the skip calls and the attention operators", -1, kMethods, nullptr, nullptr, nullptr, nullptr };

}  // namespace

PyMODINIT_FUNC PyInit__native()
{
    struct { PyObject** at; const char* text; } names[] = {
        { &k_train_steps, "train_steps" }, { &k_beta_start, "beta_start" }, { &k_beta_end, "beta_end" }, { &k_steps, "steps" }, { &k_eta, "eta" },
        { &k_sampler, "sampler" }, { &k_shift, "shift" }, { &k_get, "get" }, { &k_is_cuda, "is_cuda" }, { &k_is_contiguous, "is_contiguous" },
        { &k_dtype, "dtype" }, { &k_data_ptr, "data_ptr" }, { &k_shape, "shape" }, { &k_stride, "stride" }, { &k_get_device, "get_device" }, { &k_numel, "numel" } };
    for (auto& n : names)
        if (!(*n.at = PyUnicode_InternFromString(n.text))) return nullptr;
    if (!(k_zero = PyFloat_FromDouble(0.0)) || !(k_one = PyFloat_FromDouble(1.0)) || !(k_ddim = PyLong_FromLong(DRF_DDIM))) return nullptr;
    return PyModule_Create(&kModule);
}
