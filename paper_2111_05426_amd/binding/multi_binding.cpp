// multi_binding.cpp -- the Python calls of include/dsim_multi_ops.h.
#include <vector>

#include "call.h"

namespace binding {
namespace {

float number(PyObject *o, const char *name)
{
    const double x = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) throw PythonError();
    if (!(x == x)) refuse(name, "must not be NaN");
    return (float)x;
}

// cache, block_table, k, v, seq, slot, pos, rope, sections, interleaved, q,
// q_out, status, stream
void kv_append_axes(PyObject *const *a)
{
    Call c("dsim_kv_append_axes", a[13]);
    const dsim_kv_cache cache = cache_of(c, a[0], a[1], true);
    const at::Tensor &k = *c.get("k", a[2]), &v = *c.get("v", a[3]);
    element_type("k", k, false);
    c.check("k", k, {kAny, cache.n_heads, cache.head_dim});
    const int64_t n = k.size(0);
    c.type_is("v", v, k.scalar_type());
    c.check("v", v, {n, cache.n_heads, cache.head_dim});
    const int32_t *seq = c.vector<int32_t>("seq", a[4], at::kInt, n, false);
    const int32_t *slot = c.vector<int32_t>("slot", a[5], at::kInt, n, false);
    const at::Tensor *rope = c.get("rope", a[7], true), *pos = c.get("pos", a[6], !rope), *q = c.get("q", a[10], true),
                     *q_out = c.get("q_out", a[11], true);
    const int interleaved = PyObject_IsTrue(a[9]);
    if (interleaved < 0) throw PythonError();
    int32_t n_axes = 0, sections[DSIM_MAX_AXES] = {0, 0, 0, 0};
    if (rope) {
        c.type_is("rope", *rope, at::kFloat);
        c.check("rope", *rope, {kAny, kAny}, true);
        if (rope->size(1) > cache.head_dim || rope->size(1) == 0) refuse("rope", "must have 1 to head_dim columns");
        c.type_is("pos", *pos, at::kInt);
        c.check("pos", *pos, {n, kAny}, true);
        if (pos->size(1) < 1 || pos->size(1) > DSIM_MAX_AXES) refuse("pos", "must have 1 to 4 columns");
        n_axes = (int32_t)pos->size(1);
        if (a[8] == Py_None) {
            if (n_axes > 1) refuse("sections", "is required with several axes");
            sections[0] = (int32_t)(rope->size(1) / 2);
        } else {
            PyObject *list = PySequence_Fast(a[8], "sections must be a sequence of whole numbers");
            if (!list) throw PythonError();
            const Py_ssize_t m = PySequence_Fast_GET_SIZE(list);
            for (Py_ssize_t i = 0; i < m && i < n_axes; ++i) {
                const long x = PyLong_AsLong(PySequence_Fast_GET_ITEM(list, i));
                sections[i] = x < 0 || x > INT32_MAX ? -1 : (int32_t)x;
            }
            Py_DECREF(list);
            if (PyErr_Occurred()) throw PythonError();
            if (m != n_axes) refuse("sections", "must have an entry for each column of pos");
        }
    } else if (pos || a[8] != Py_None) {
        refuse("pos and sections", "need rope");
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
    int32_t *status = c.vector<int32_t>("status", a[12], at::kInt, n, true, true);
    c.run([&](void *stream) {
        return dsim_kv_append_axes(&cache, n, dtype_of(k), &kr, &vr, q ? &qr : nullptr, q ? &qo : nullptr, (int32_t)heads,
                                   seq, slot, rope ? static_cast<const int32_t *>(c.data(*pos)) : nullptr, n_axes, sections,
                                   rope ? static_cast<const float *>(c.data(*rope)) : nullptr, rope ? rope->size(0) : 0,
                                   rope ? (int32_t)rope->size(1) : 0, interleaved, status, stream);
    });
}

// The arguments that prompts and trees share.
struct Queries {
    dsim_kv_cache cache;
    dsim_queries q;
};

Queries queries(Call &c, PyObject *q_, PyObject *cache, PyObject *table, PyObject *start, PyObject *len, const char *len_name,
                PyObject *out_, PyObject *scale, PyObject *window, PyObject *cap, PyObject *slopes, PyObject *workspace,
                PyObject *lse_, PyObject *status)
{
    Queries r{cache_of(c, cache, table, false), {}};
    const int64_t n_seq = r.cache.n_seq;
    const at::Tensor &q = *c.get("q", q_), &out = *c.get("out", out_);
    element_type("q", q, false);
    c.check("q", q, {kAny, kAny, r.cache.head_dim});
    const int64_t n = q.size(0), heads = q.size(1);
    if (heads > INT32_MAX) refuse("q", "is too large");
    c.type_is("out", out, q.scalar_type());
    c.check("out", out, {n, heads, r.cache.head_dim});
    r.q.start = c.vector<int32_t>("start", start, at::kInt, n_seq + 1, false);
    r.q.len = c.vector<int32_t>(len_name, len, at::kInt, n_seq, false);
    r.q.scale = scale == Py_None ? (float)(1.0 / std::sqrt((double)r.cache.head_dim)) : number(scale, "scale");
    r.q.cap = number(cap, "cap");
    const long w = PyLong_AsLong(window);
    if (PyErr_Occurred()) throw PythonError();
    if (w < 0 || w > INT32_MAX) refuse("window", "must be in [0, 2^31)");
    r.q.window = (int32_t)w;
    r.q.slopes = c.vector<float>("slopes", slopes, at::kFloat, heads);
    const at::Tensor &ws = *c.get("workspace", workspace), *lse = c.get("lse", lse_, true);
    c.type_is("workspace", ws, at::kByte);
    c.check("workspace", ws, {kAny}, true);
    if (lse) {
        c.type_is("lse", *lse, at::kFloat);
        c.check("lse", *lse, {n, heads}, true);
        c.writes(*lse);
        r.q.lse = static_cast<float *>(c.data(*lse));
    }
    r.q.status = c.vector<int32_t>("status", status, at::kInt, n_seq, true, true);
    r.q.q = c.rows(q);
    r.q.out = c.rows(out);
    r.q.n_tok = n;
    r.q.n_q_heads = (int32_t)heads;
    r.q.dtype = dtype_of(q);
    r.q.workspace = c.data(ws);
    r.q.ws_bytes = (size_t)ws.numel();
    c.writes(out);
    c.writes(ws);
    return r;
}

// q, cache, block_table, start, seq_len, out, scale, window, cap, slopes,
// prefix_len, first_key, workspace, lse, status, stream
void prompt_attention(PyObject *const *a)
{
    Call c("dsim_prompt_attention", a[15]);
    const Queries x = queries(c, a[0], a[1], a[2], a[3], a[4], "seq_len", a[5], a[6], a[7], a[8], a[9], a[12], a[13], a[14]);
    const int32_t *prefix = c.vector<int32_t>("prefix_len", a[10], at::kInt, x.cache.n_seq);
    const int32_t *first = c.vector<int32_t>("first_key", a[11], at::kInt, x.q.n_tok);
    c.run([&](void *stream) { return dsim_prompt_attention(&x.cache, &x.q, prefix, first, stream); });
}

// q, cache, block_table, start, context_len, tree_mask, out, depth, scale,
// window, cap, slopes, workspace, lse, status, stream
void tree_attention(PyObject *const *a)
{
    Call c("dsim_tree_attention", a[15]);
    const Queries x = queries(c, a[0], a[1], a[2], a[3], a[4], "context_len", a[6], a[8], a[9], a[10], a[11], a[12], a[13], a[14]);
    const at::Tensor &mask = *c.get("tree_mask", a[5]);
    c.type_is("tree_mask", mask, at::kInt);
    c.check("tree_mask", mask, {x.q.n_tok, kAny});
    if (mask.size(1) > INT32_MAX) refuse("tree_mask", "is too large");
    const int32_t *depth = c.vector<int32_t>("depth", a[7], at::kInt, x.q.n_tok);
    c.run([&](void *stream) {
        return dsim_tree_attention(&x.cache, &x.q, static_cast<const uint32_t *>(c.data(mask)), mask.stride(0),
                                   (int32_t)mask.size(1), depth, stream);
    });
}

// A pool with its block table, all of it written.
dsim_page_pool pool_of(Call &c, PyObject *pool, PyObject *table, int64_t page_size)
{
    if (!PyDict_Check(pool)) refuse("pool", "must be a dict");
    const Table t = table_of(c, table, true);
    const at::Tensor &refs = *c.get("pool['refs']", item(pool, "refs"));
    c.type_is("pool['refs']", refs, at::kInt);
    c.check("pool['refs']", refs, {kAny}, true);
    c.writes(refs);
    const int64_t n = refs.size(0);
    dsim_page_pool p{};
    p.refs = static_cast<int32_t *>(c.data(refs));
    p.free = reinterpret_cast<uint32_t *>(c.vector<int32_t>("pool['free']", item(pool, "free"), at::kInt, (n + 31) / 32, false, true));
    p.held = c.vector<int32_t>("pool['held']", item(pool, "held"), at::kInt, t.n_seq, false, true);
    p.block_table = t.data;
    p.table_stride = t.stride;
    p.n_seq = t.n_seq;
    p.table_width = t.width;
    p.n_pages = n;
    p.page_size = (int32_t)page_size;
    return p;
}

int64_t page_size_of(PyObject *o)
{
    const long x = PyLong_AsLong(o);
    if (PyErr_Occurred()) throw PythonError();
    if (x < 1 || x > INT32_MAX) refuse("page_size", "must be in 1..2^20");
    return x;
}

// One cache or a sequence of them.
std::vector<dsim_kv_cache> layers_of(Call &c, PyObject *layers)
{
    std::vector<dsim_kv_cache> r;
    if (PyDict_Check(layers)) {
        r.push_back(layer_of(c, layers, true));
        return r;
    }
    if (!PyList_Check(layers) && !PyTuple_Check(layers)) refuse("layers", "must be a cache or a list of caches");
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(layers);
    if (n == 0) refuse("layers", "must not be empty");
    r.reserve((size_t)n);
    for (Py_ssize_t i = 0; i < n; ++i) r.push_back(layer_of(c, PySequence_Fast_GET_ITEM(layers, i), true));
    return r;
}

int32_t count(const std::vector<dsim_kv_cache> &layers)
{
    return layers.size() > 1 << 20 ? 1 << 20 : (int32_t)layers.size();
}

// pool, block_table, page_size, seq_len, new_len, status, stream
void kv_reserve(PyObject *const *a)
{
    Call c("dsim_kv_reserve", a[6]);
    const dsim_page_pool p = pool_of(c, a[0], a[1], page_size_of(a[2]));
    const int32_t *len = c.vector<int32_t>("seq_len", a[3], at::kInt, p.n_seq, false);
    const int32_t *want = c.vector<int32_t>("new_len", a[4], at::kInt, p.n_seq, false);
    int32_t *status = c.vector<int32_t>("status", a[5], at::kInt, p.n_seq, false, true);
    c.run([&](void *stream) { return dsim_kv_reserve(&p, len, want, status, stream); });
}

// pool, block_table, page_size, row, keep_len, status, stream
void kv_release(PyObject *const *a)
{
    Call c("dsim_kv_release", a[6]);
    const dsim_page_pool p = pool_of(c, a[0], a[1], page_size_of(a[2]));
    const at::Tensor &row = *c.get("row", a[3]);
    c.type_is("row", row, at::kInt);
    c.check("row", row, {kAny}, true);
    const int64_t n = row.size(0);
    const int32_t *keep = c.vector<int32_t>("keep_len", a[4], at::kInt, n, false);
    int32_t *status = c.vector<int32_t>("status", a[5], at::kInt, n, true, true);
    c.run([&](void *stream) { return dsim_kv_release(&p, n, static_cast<const int32_t *>(c.data(row)), keep, status, stream); });
}

// layers, pool, block_table, seq_len, src, dst, status, stream
void kv_fork(PyObject *const *a)
{
    Call c("dsim_kv_fork", a[7]);
    const std::vector<dsim_kv_cache> layers = layers_of(c, a[0]);
    const dsim_page_pool p = pool_of(c, a[1], a[2], layers[0].page_size);
    int32_t *len = c.vector<int32_t>("seq_len", a[3], at::kInt, p.n_seq, false, true);
    const at::Tensor &src = *c.get("src", a[4]);
    c.type_is("src", src, at::kInt);
    c.check("src", src, {kAny}, true);
    const int64_t n = src.size(0);
    const int32_t *dst = c.vector<int32_t>("dst", a[5], at::kInt, n, false);
    int32_t *status = c.vector<int32_t>("status", a[6], at::kInt, n, false, true);
    c.run([&](void *stream) {
        return dsim_kv_fork(layers.data(), count(layers), &p, len, n, static_cast<const int32_t *>(c.data(src)), dst, status,
                            stream);
    });
}

// layers, src, dst, stream
void kv_copy_pages(PyObject *const *a)
{
    Call c("dsim_kv_copy_pages", a[3]);
    const std::vector<dsim_kv_cache> layers = layers_of(c, a[0]);
    const at::Tensor &src = *c.get("src", a[1]);
    c.type_is("src", src, at::kInt);
    c.check("src", src, {kAny}, true);
    const int64_t n = src.size(0);
    const int32_t *dst = c.vector<int32_t>("dst", a[2], at::kInt, n, false);
    c.run([&](void *stream) {
        return dsim_kv_copy_pages(layers.data(), count(layers), n, static_cast<const int32_t *>(c.data(src)), dst, stream);
    });
}

// layers, block_table, start, keep, n_keep, status, stream
void kv_compact(PyObject *const *a)
{
    Call c("dsim_kv_compact", a[6]);
    std::vector<dsim_kv_cache> layers = layers_of(c, a[0]);
    const Table t = table_of(c, a[1], false);
    layers[0].block_table = t.data;
    layers[0].table_stride = t.stride;
    layers[0].n_seq = t.n_seq;
    layers[0].table_width = t.width;
    const int32_t *start = c.vector<int32_t>("start", a[2], at::kInt, t.n_seq, false);
    const at::Tensor &keep = *c.get("keep", a[3]);
    c.type_is("keep", keep, at::kInt);
    c.check("keep", keep, {t.n_seq, kAny});
    if (keep.size(1) > INT32_MAX) refuse("keep", "is too large");
    const int32_t *n_keep = c.vector<int32_t>("n_keep", a[4], at::kInt, t.n_seq, false);
    int32_t *status = c.vector<int32_t>("status", a[5], at::kInt, t.n_seq, true, true);
    c.run([&](void *stream) {
        return dsim_kv_compact(layers.data(), count(layers), start, static_cast<const int32_t *>(c.data(keep)),
                               keep.stride(0), (int32_t)keep.size(1), n_keep, status, stream);
    });
}

// n_tok, n_seq, n_q_heads, n_heads, head_dim
PyObject *prompt_attention_workspace(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    long v[5] = {0, 0, 0, 0, 0};
    for (Py_ssize_t i = 0; i < 5 && n == 5; ++i) {
        v[i] = PyLong_AsLong(args[i]);
        if (PyErr_Occurred()) return nullptr;
        if (v[i] < 0 || v[i] > INT32_MAX) v[i] = -1;   // (refused: 0 bytes)
    }
    return PyLong_FromSize_t(dsim_prompt_attention_workspace(v[0], (int32_t)v[1], (int32_t)v[2], (int32_t)v[3], (int32_t)v[4]));
}

}  // namespace

PyMethodDef g_multi_methods[] = {
    ENTRY(kv_append_axes, 14), ENTRY(prompt_attention, 16), ENTRY(tree_attention, 16), ENTRY(kv_reserve, 7),
    ENTRY(kv_release, 7), ENTRY(kv_fork, 8), ENTRY(kv_copy_pages, 4), ENTRY(kv_compact, 7),
    {"prompt_attention_workspace", (PyCFunction)(void (*)(void))prompt_attention_workspace, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

}  // namespace binding
