// ops_binding.cpp -- the Python calls of include/dsim_ops.h: every tensor's
// dtype, shape, layout and device checked, then one call of libdsim.
//
// The operators' smallest calls take the GPU 3 to 9 us.  Marshalled in Python
// through ctypes a call took 14 to 20 us of the host's time, ten tensors'
// attributes at 0.1 to 0.3 us each; here it takes about what the launches do.
#include "call.h"

namespace binding {
PyObject *g_dsim_error;
}

using namespace binding;

namespace {

// cache, block_table, k, v, seq, pos, rope, interleaved, q, q_out, status, stream
void kv_append(PyObject *const *a)
{
    Call c("dsim_kv_append", a[11]);
    const dsim_kv_cache cache = cache_of(c, a[0], a[1], true);
    const at::Tensor &k = *c.get("k", a[2]), &v = *c.get("v", a[3]);
    element_type("k", k, false);
    c.check("k", k, {kAny, cache.n_heads, cache.head_dim});
    const int64_t n = k.size(0);
    c.type_is("v", v, k.scalar_type());
    c.check("v", v, {n, cache.n_heads, cache.head_dim});
    const int32_t *seq = c.vector<int32_t>("seq", a[4], at::kInt, n, false);
    const int32_t *pos = c.vector<int32_t>("pos", a[5], at::kInt, n, false);
    const at::Tensor *rope = c.get("rope", a[6], true), *q = c.get("q", a[8], true), *q_out = c.get("q_out", a[9], true);
    const int interleaved = PyObject_IsTrue(a[7]);
    if (interleaved < 0) throw PythonError();
    if (rope) {
        c.type_is("rope", *rope, at::kFloat);
        c.check("rope", *rope, {kAny, kAny}, true);
        if (rope->size(1) > cache.head_dim || rope->size(1) == 0) refuse("rope", "must have 1 to head_dim columns");
    }
    int64_t heads = 0;
    dsim_rows kr = c.rows(k), vr = c.rows(v), qr{}, qo{};
    if (!q != !q_out) refuse("q and q_out", "come together");
    if (q) {
        c.type_is("q", *q, k.scalar_type());
        c.check("q", *q, {n, kAny, cache.head_dim});
        heads = q->size(1);
        if (heads > INT32_MAX) refuse("q", "is too large");
        c.type_is("q_out", *q_out, k.scalar_type());
        c.check("q_out", *q_out, {n, heads, cache.head_dim});
        qr = c.rows(*q);
        qo = c.rows(*q_out);
        c.writes(*q_out);
    }
    int32_t *status = c.vector<int32_t>("status", a[10], at::kInt, n, true, true);
    c.run([&](void *stream) {
        return dsim_kv_append(&cache, n, dtype_of(k), &kr, &vr, q ? &qr : nullptr, q ? &qo : nullptr, (int32_t)heads, seq,
                              pos, rope ? static_cast<const float *>(c.data(*rope)) : nullptr, rope ? rope->size(0) : 0,
                              rope ? (int32_t)rope->size(1) : 0, interleaved, status, stream);
    });
}

// q, cache, block_table, seq_len, out, scale, window, workspace, lse, status, stream
void paged_attention(PyObject *const *a)
{
    Call c("dsim_paged_attention", a[10]);
    const dsim_kv_cache cache = cache_of(c, a[1], a[2], false);
    const int64_t n = cache.n_seq;
    const at::Tensor &q = *c.get("q", a[0]), &out = *c.get("out", a[4]);
    element_type("q", q, false);
    c.check("q", q, {n, kAny, cache.head_dim});
    const int64_t heads = q.size(1);
    if (heads > INT32_MAX) refuse("q", "is too large");
    c.type_is("out", out, q.scalar_type());
    c.check("out", out, {n, heads, cache.head_dim});
    const int32_t *len = c.vector<int32_t>("seq_len", a[3], at::kInt, n, false);
    const double scale = a[5] == Py_None ? 1.0 / std::sqrt((double)cache.head_dim) : PyFloat_AsDouble(a[5]);
    const long window = PyLong_AsLong(a[6]);
    if (PyErr_Occurred()) throw PythonError();
    if (window < 0 || window > INT32_MAX) refuse("window", "must be in [0, 2^31)");
    const at::Tensor &ws = *c.get("workspace", a[7]), *lse = c.get("lse", a[8], true);
    c.type_is("workspace", ws, at::kByte);
    c.check("workspace", ws, {kAny}, true);
    if (lse) {
        c.type_is("lse", *lse, at::kFloat);
        c.check("lse", *lse, {n, heads}, true);
    }
    int32_t *status = c.vector<int32_t>("status", a[9], at::kInt, n, true, true);
    const dsim_rows qr = c.rows(q), o = c.rows(out);
    c.writes(out);
    c.writes(ws);
    if (lse) c.writes(*lse);
    c.run([&](void *stream) {
        return dsim_paged_attention(&cache, dtype_of(q), &qr, &o, (int32_t)heads, len, (float)scale, (int32_t)window,
                                    lse ? static_cast<float *>(c.data(*lse)) : nullptr, status, c.data(ws),
                                    (size_t)ws.numel(), stream);
    });
}

// logits, out, history, prompt_len, history_len, repetition, frequency,
// presence, bias_id, bias, mask, stream
void logit_adjust(PyObject *const *a)
{
    Call c("dsim_logit_adjust", a[11]);
    const at::Tensor &x = *c.get("logits", a[0]), &y = *c.get("out", a[1]);
    element_type("logits", x, false);
    c.check("logits", x, {kAny, kAny});
    const int64_t n = x.size(0), vocab = x.size(1);
    if (vocab > INT32_MAX) refuse("logits", "is too large");
    c.type_is("out", y, x.scalar_type());
    c.check("out", y, {n, vocab});
    dsim_logits s{};
    s.logits = c.data(x);
    s.out = c.data(y);
    c.writes(y);
    s.logits_stride = x.stride(0);
    s.out_stride = y.stride(0);
    s.n_rows = n;
    s.vocab = (int32_t)vocab;
    s.dtype = dtype_of(x);
    s.prompt_len = c.vector<int32_t>("prompt_len", a[3], at::kInt, n);
    s.history_len = c.vector<int32_t>("history_len", a[4], at::kInt, n);
    if (const at::Tensor *h = c.get("history", a[2], true)) {
        c.type_is("history", *h, at::kInt);
        c.check("history", *h, {n, kAny});
        if (h->size(1) > INT32_MAX) refuse("history", "is too large");
        s.history_width = (int32_t)h->size(1);
        s.history_stride = h->stride(0);
        // (no token of a history of width 0 is read: any address will do)
        s.history = s.history_width ? static_cast<const int32_t *>(c.data(*h)) : s.history_len;
    }
    s.repetition = c.vector<float>("repetition", a[5], at::kFloat, n);
    s.frequency = c.vector<float>("frequency", a[6], at::kFloat, n);
    s.presence = c.vector<float>("presence", a[7], at::kFloat, n);
    const at::Tensor *id = c.get("bias_id", a[8], true), *bias = c.get("bias", a[9], true), *mask = c.get("mask", a[10], true);
    if (!id != !bias) refuse("bias_id and bias", "come together");
    if (id) {
        c.type_is("bias_id", *id, at::kInt);
        c.check("bias_id", *id, {n, kAny}, true);
        c.type_is("bias", *bias, at::kFloat);
        c.check("bias", *bias, {n, id->size(1)}, true);
        if (id->size(1) > INT32_MAX) refuse("bias_id", "is too large");
        s.n_bias = (int32_t)id->size(1);
        s.bias_id = static_cast<const int32_t *>(c.data(*id));
        s.bias = static_cast<const float *>(c.data(*bias));
    }
    if (mask) {
        c.type_is("mask", *mask, at::kInt);
        c.check("mask", *mask, {n, (vocab + 31) / 32});
        s.mask = static_cast<const uint32_t *>(c.data(*mask));
        s.mask_stride = mask->stride(0);
    }
    c.run([&](void *stream) { return dsim_logit_adjust(&s, stream); });
}

// n_q_heads, n_heads, head_dim
PyObject *workspace(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    long v[3] = {0, 0, 0};
    for (Py_ssize_t i = 0; i < 3 && n == 3; ++i) {
        v[i] = PyLong_AsLong(args[i]);
        if (PyErr_Occurred()) return nullptr;
        if (v[i] < 0 || v[i] > INT32_MAX) v[i] = 0;   // (no such heads: 0 bytes)
    }
    return PyLong_FromSize_t(dsim_paged_attention_workspace((int32_t)v[0], (int32_t)v[1], (int32_t)v[2]));
}

PyMethodDef g_methods[] = {ENTRY(kv_append, 12), ENTRY(paged_attention, 11), ENTRY(logit_adjust, 12),
                           {"paged_attention_workspace", (PyCFunction)(void (*)(void))workspace, METH_FASTCALL, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_ops", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops(void)
{
    PyObject *m = PyImport_ImportModule("paper_2111_05426_amd.dsim");
    if (!m) return nullptr;
    g_dsim_error = PyObject_GetAttrString(m, "DsimError");
    Py_DECREF(m);
    PyObject *module = g_dsim_error ? PyModule_Create(&g_module) : nullptr;
    if (module && PyModule_AddFunctions(module, g_multi_methods) < 0) Py_CLEAR(module);
    return module;
}
