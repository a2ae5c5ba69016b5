// call.h -- the tensors of a Python call: checked, and handed to libdsim.
#pragma once

#include <Python.h>

#include <ATen/core/grad_mode.h>
#include <c10/core/AutogradState.h>
#include <c10/hip/HIPStream.h>
#include <c10/util/SmallVector.h>
#include <hip/hip_runtime.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <string>

#include "dsim_multi_ops.h"

namespace binding {

extern PyObject *g_dsim_error;   // the binding's DsimError(function, code, message)

// A refused argument: becomes ValueError.
struct Refused {
    std::string what;
};

[[noreturn]] inline void refuse(const char *name, const std::string &what) { throw Refused{std::string(name) + " " + what}; }

struct PythonError {};   // the Python error is set

inline const char *const kTypeNames[] = {"torch.float32", "torch.float16", "torch.bfloat16", "torch.float8_e4m3fn"};

inline int dtype_of(const at::Tensor &t)
{
    switch (t.scalar_type()) {
    case at::kFloat: return DSIM_F32;
    case at::kHalf: return DSIM_F16;
    case at::kBFloat16: return DSIM_BF16;
    case at::kFloat8_e4m3fn: return DSIM_E4M3;
    default: return -1;
    }
}

inline std::string shape_text(c10::IntArrayRef s)
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
    void writes(const at::Tensor &t) { written_.push_back(&t); }

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
        for (const at::Tensor *t : written_)   // (tensors of inference mode keep no versions)
            if (!t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
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
    c10::SmallVector<const at::Tensor *, 8> written_;
};

inline PyObject *item(PyObject *dict, const char *key)
{
    PyObject *o = PyDict_GetItemString(dict, key);   // (borrowed)
    return o ? o : Py_None;
}

inline void element_type(const char *name, const at::Tensor &t, bool cache)
{
    const int d = dtype_of(t);
    if (d < 0 || (d == DSIM_E4M3 && !cache)) {
        std::string types;
        for (int i = 0; i < (cache ? 4 : 3); ++i) types += (i ? " or " : "") + std::string(kTypeNames[i]);
        refuse(name, "must be of dtype " + types + ", not " + at::toString(t.scalar_type()));
    }
}

// A cache without its block table.
inline dsim_kv_cache layer_of(Call &c, PyObject *cache, bool written)
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
    for (const int64_t x : {n[1], n[2], n[3]})
        if (x > INT32_MAX) refuse("cache", "is too large");
    dsim_kv_cache r{};
    r.k = c.data(k);
    r.v = c.data(v);
    r.n_pages = n[0];
    r.page_stride = s[0];
    r.slot_stride = s[1];
    r.head_stride = s[2];
    r.dtype = dtype_of(k);
    r.n_heads = (int32_t)n[2];
    r.head_dim = (int32_t)n[3];
    r.page_size = (int32_t)n[1];
    return r;
}

struct Table {
    int32_t *data;
    int64_t stride;
    int32_t n_seq, width;
};

inline Table table_of(Call &c, PyObject *table, bool written)
{
    const at::Tensor &t = *c.get("block_table", table);
    c.type_is("block_table", t, at::kInt);
    c.check("block_table", t, {kAny, kAny});
    for (const int64_t x : {t.size(0), t.size(1)})
        if (x > INT32_MAX) refuse("block_table", "is too large");
    if (written) c.writes(t);
    return {static_cast<int32_t *>(c.data(t)), t.stride(0), (int32_t)t.size(0), (int32_t)t.size(1)};
}

inline dsim_kv_cache cache_of(Call &c, PyObject *cache, PyObject *table, bool written)
{
    dsim_kv_cache r = layer_of(c, cache, written);
    const Table t = table_of(c, table, false);
    r.k_scale = c.vector<float>("cache['k_scale']", item(cache, "k_scale"), at::kFloat, r.n_heads);
    r.v_scale = c.vector<float>("cache['v_scale']", item(cache, "v_scale"), at::kFloat, r.n_heads);
    r.block_table = t.data;
    r.table_stride = t.stride;
    r.n_seq = t.n_seq;
    r.table_width = t.width;
    return r;
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

extern PyMethodDef g_multi_methods[];   // those of multi_binding.cpp

}  // namespace binding
