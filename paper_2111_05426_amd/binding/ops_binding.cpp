// ops_binding.cpp -- the Python calls of include/dsim_ops.h: every tensor's
// dtype, shape, layout and device checked, then one call of libdsim.
//
// The operators' smallest calls take the GPU 3 to 9 us.  Marshalled in Python
// through ctypes a call took 14 to 20 us of the host's time, ten tensors'
// attributes at 0.1 to 0.3 us each; here it takes about what the launches do.
#include <Python.h>

#include <ATen/core/grad_mode.h>
#include <c10/core/AutogradState.h>
#include <c10/hip/HIPStream.h>
#include <hip/hip_runtime.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <string>

#include "dsim_ops.h"

namespace {

PyObject *g_dsim_error;   // the binding's DsimError(function, code, message)

// A refused argument: becomes ValueError.
struct Refused {
    std::string what;
};

[[noreturn]] void refuse(const char *name, const std::string &what) { throw Refused{std::string(name) + " " + what}; }

struct PythonError {};   // the Python error is set

const char *const kTypeNames[] = {"torch.float32", "torch.float16", "torch.bfloat16", "torch.float8_e4m3fn"};

int dtype_of(const at::Tensor &t)
{
    switch (t.scalar_type()) {
    case at::kFloat: return DSIM_F32;
    case at::kHalf: return DSIM_F16;
    case at::kBFloat16: return DSIM_BF16;
    case at::kFloat8_e4m3fn: return DSIM_E4M3;
    default: return -1;
    }
}

std::string shape_text(c10::IntArrayRef s)
{
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + (s[i] < 0 ? "any" : std::to_string(s[i]));
    return r + (s.size() == 1 ? ",)" : ")");
}

constexpr int64_t kAny = -1;

// The tensors of one call: the device they all lie on.
class Call {
  public:
    Call(const char *fn, PyObject *stream) : fn_(fn), stream_(stream) {}

    // A tensor argument; nullptr for None where that is allowed.
    const at::Tensor *get(const char *name, PyObject *o, bool optional = false)
    {
        if (o == Py_None) {
            if (!optional) refuse(name, "is required");
            return nullptr;
        }
        if (!THPVariable_Check(o)) refuse(name, "must be a torch tensor");
        const at::Tensor &t = THPVariable_Unpack(o);
        if (t.layout() != at::kStrided || t.is_neg()) refuse(name, "must be a plain strided tensor");
        // (what autograd recorded of it would end here without a word)
        if (t.requires_grad() && at::GradMode::is_enabled())
            refuse(name, "requires a gradient, which the operator has not: detach it or call under torch.no_grad()");
        if (t._fw_grad(0).defined() && c10::AutogradState::get_tls_state().get_fw_grad_mode())
            refuse(name, "carries a tangent, which the operator has not: take its primal");
        return &t;
    }

    // A tensor that the call writes: one that an earlier operation saved for
    // its backward pass is then known to have changed.
    void writes(const at::Tensor &t) { written_[n_written_++] = &t; }

    // The tensor's shape (kAny entries free), the last dimension contiguous
    // (all of it if `whole`), on a GPU and on the others' device.
    void check(const char *name, const at::Tensor &t, std::initializer_list<int64_t> shape, bool whole = false)
    {
        const auto got = t.sizes();
        bool same = got.size() == shape.size();
        for (size_t i = 0; same && i < got.size(); ++i) same = shape.begin()[i] == kAny || shape.begin()[i] == got[i];
        if (!same)
            refuse(name, "must have shape " + shape_text(c10::IntArrayRef(shape.begin(), shape.size())) + ", not " +
                             shape_text(got));
        if (whole ? !t.is_contiguous() : got.back() > 1 && t.strides().back() != 1)
            refuse(name, whole ? "must be contiguous" : "must be contiguous in its last dimension");
        if (!first_) {
            first_ = name;
            device_ = t.device();
        }
        if (t.device() != device_)
            refuse(name, "must be on " + device_.str() + " with " + first_ + ", not on " + t.device().str());
    }

    template <class T>
    T *vector(const char *name, PyObject *o, at::ScalarType type, int64_t n, bool optional = true, bool written = false)
    {
        const at::Tensor *t = get(name, o, optional);
        if (!t) return nullptr;
        type_is(name, *t, type);
        check(name, *t, {n}, true);
        if (written) writes(*t);
        return static_cast<T *>(data(*t));
    }

    void type_is(const char *name, const at::Tensor &t, at::ScalarType type)
    {
        if (t.scalar_type() != type)
            refuse(name, std::string("must be of dtype ") + at::toString(type) + ", not " + at::toString(t.scalar_type()));
    }

    // The address, once every check of this tensor has passed.  (A tensor on
    // no GPU has its address taken by nobody: run() refuses it first.)
    void *data(const at::Tensor &t) { return device_.is_cuda() ? t.mutable_data_ptr() : nullptr; }

    dsim_rows rows(const at::Tensor &t) { return {data(t), t.strides()[0], t.strides()[1]}; }

    // f(stream) on the tensors' device; its status becomes an exception.
    template <class F> void run(F f)
    {
        if (!device_.is_cuda()) refuse(first_, "must be a GPU tensor, not on " + device_.str());
        const int device = device_.index();
        void *stream;
        if (stream_ == Py_None) {
            stream = c10::hip::getCurrentHIPStream((c10::DeviceIndex)device).stream();
        } else {
            if (!PyLong_Check(stream_)) {
                PyObject *of = PyObject_GetAttrString(stream_, "device_index");
                const long index = of ? PyLong_AsLong(of) : device;
                Py_XDECREF(of);
                PyErr_Clear();   // (another library's stream need not say)
                if (index != device) refuse("stream", "must be on " + device_.str() + " with " + first_);
            }
            PyObject *h = PyLong_Check(stream_) ? Py_NewRef_(stream_) : PyObject_GetAttrString(stream_, "cuda_stream");
            if (!h) throw PythonError();
            stream = PyLong_AsVoidPtr(h);
            Py_DECREF(h);
            if (PyErr_Occurred()) throw PythonError();
        }
        int current = device;
        const hipError_t e = hipGetDevice(&current);
        if (e == hipSuccess && current != device && hipSetDevice(device) != hipSuccess) refuse(first_, "is on a device that cannot be selected");
        const dsim_status st = f(stream);
        if (e == hipSuccess && current != device) (void)hipSetDevice(current);
        if (st != DSIM_OK) {
            PyObject *args = Py_BuildValue("(sis)", fn_, (int)st, dsim_last_error());
            if (args) {
                PyObject *error = PyObject_Call(g_dsim_error, args, nullptr);
                Py_DECREF(args);
                if (error) {
                    PyErr_SetObject(g_dsim_error, error);
                    Py_DECREF(error);
                }
            }
            throw PythonError();
        }
        for (int i = 0; i < n_written_; ++i)   // (tensors of inference mode keep no versions)
            if (!written_[i]->is_inference()) written_[i]->unsafeGetTensorImpl()->bump_version();
    }

  private:
    static PyObject *Py_NewRef_(PyObject *o)
    {
        Py_INCREF(o);
        return o;
    }

    const char *fn_, *first_ = nullptr;
    PyObject *stream_;
    c10::Device device_{c10::kCPU};
    const at::Tensor *written_[4];   // (the most that a call writes)
    int n_written_ = 0;
};

PyObject *item(PyObject *dict, const char *key)
{
    PyObject *o = PyDict_GetItemString(dict, key);   // (borrowed)
    return o ? o : Py_None;
}

void element_type(const char *name, const at::Tensor &t, bool cache)
{
    const int d = dtype_of(t);
    if (d < 0 || (d == DSIM_E4M3 && !cache)) {
        std::string types;
        for (int i = 0; i < (cache ? 4 : 3); ++i) types += (i ? " or " : "") + std::string(kTypeNames[i]);
        refuse(name, "must be of dtype " + types + ", not " + at::toString(t.scalar_type()));
    }
}

dsim_kv_cache cache_of(Call &c, PyObject *cache, PyObject *table, bool written)
{
    if (!PyDict_Check(cache)) refuse("cache", "must be a dict");
    const at::Tensor &k = *c.get("cache['k']", item(cache, "k")), &v = *c.get("cache['v']", item(cache, "v"));
    element_type("cache['k']", k, true);
    c.check("cache['k']", k, {kAny, kAny, kAny, kAny});
    c.type_is("cache['v']", v, k.scalar_type());
    const auto n = k.sizes(), s = k.strides();
    c.check("cache['v']", v, {n[0], n[1], n[2], n[3]});
    for (int i = 0; i < 4; ++i)
        if (n[i] > 1 && v.strides()[i] != s[i]) refuse("cache['v']", "must have the strides of cache['k']");
    if (written) {
        c.writes(k);
        c.writes(v);
    }
    const at::Tensor &t = *c.get("block_table", table);
    c.type_is("block_table", t, at::kInt);
    c.check("block_table", t, {kAny, kAny});
    for (const int64_t x : {n[1], n[2], n[3], t.size(0), t.size(1)})
        if (x > INT32_MAX) refuse("cache", "is too large");
    dsim_kv_cache r{};
    r.k = c.data(k);
    r.v = c.data(v);
    r.k_scale = c.vector<float>("cache['k_scale']", item(cache, "k_scale"), at::kFloat, n[2]);
    r.v_scale = c.vector<float>("cache['v_scale']", item(cache, "v_scale"), at::kFloat, n[2]);
    r.block_table = static_cast<const int32_t *>(c.data(t));
    r.n_pages = n[0];
    r.page_stride = s[0];
    r.slot_stride = s[1];
    r.head_stride = s[2];
    r.table_stride = t.stride(0);
    r.dtype = dtype_of(k);
    r.n_heads = (int32_t)n[2];
    r.head_dim = (int32_t)n[3];
    r.page_size = (int32_t)n[1];
    r.n_seq = (int32_t)t.size(0);
    r.table_width = (int32_t)t.size(1);
    return r;
}

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

template <void (*F)(PyObject *const *), int N> PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected, %d given", N, (int)n);
        return nullptr;
    }
    try {
        F(args);
        Py_RETURN_NONE;
    } catch (const Refused &e) {
        PyErr_SetString(PyExc_ValueError, e.what.c_str());
    } catch (const PythonError &) {
    } catch (const std::exception &e) {   // torch's own refusals
        PyErr_SetString(PyExc_ValueError, e.what());
    }
    return nullptr;
}

#define ENTRY(f, n) {#f, (PyCFunction)(void (*)(void))entry<f, n>, METH_FASTCALL, nullptr}
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
    return g_dsim_error ? PyModule_Create(&g_module) : nullptr;
}
