// The KV cache's entry points on torch tensors: checks of types, shapes and strides,
// outputs and workspaces from torch's allocator, torch's current stream, then the C ABI.
// A call costs about what its launches cost: from Python, one launch takes 2.5 us,
// reading the tensors and filling in the C arguments another 4 us through ctypes and
// below 1 us here.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/core/LegacyTypeDispatch.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPGuard.h>
#include <c10/hip/HIPStream.h>
#include <hip/hip_runtime_api.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "kvr.h"

namespace {

// A bad argument: a ValueError (or TypeError) with this text.
struct Refused {
    PyObject *type;
    std::string text;
};
[[noreturn]] void refuse(const std::string &text) { throw Refused{PyExc_ValueError, text}; }

const at::Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) throw Refused{PyExc_TypeError, std::string(name) + " must be a tensor"};
    return THPVariable_Unpack(o);
}
bool given(PyObject *o) { return o != Py_None; }

// The device of a call: that of its first tensor; the others must be on it too.
struct Device {
    c10::Device at{c10::DeviceType::CPU};
    void check(const at::Tensor &t, const char *name)
    {
        if (at.is_cpu()) at = t.device();
        else if (t.device() != at)
            refuse(std::string(name) + " must be on " + at.str() + " as the call's other tensors are, not on " +
                   t.device().str());
    }
    void check(int64_t index, const char *name) const
    {
        if (index != at.index())
            refuse(std::string(name) + " must be of " + at.str() + ", not of device " + std::to_string(index));
    }
};

// Calls record no gradients, so tensors that need one are refused rather than cut off.
void no_gradient(const at::Tensor &t, const char *name)
{
    if (t.requires_grad() && c10::GradMode::is_enabled())
        refuse(std::string(name) + " requires gradients, which this call does not record: detach it or "
                                   "call under torch.no_grad()");
}

int64_t integer(PyObject *o, const char *name)
{
    const long long x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Refused{PyExc_TypeError, std::string(name) + " must be an integer"};
    }
    return x;
}
int32_t integer32(PyObject *o, const char *name)
{
    const int64_t x = integer(o, name);
    if (x < INT32_MIN || x > INT32_MAX) refuse(std::string(name) + " is beyond 32 bits");
    return (int32_t)x;
}

int32_t dtype_of(const at::Tensor &t, const char *name)
{
    switch (t.scalar_type()) {
    case at::kBFloat16: return KVR_DT_BF16;
    case at::kHalf: return KVR_DT_FP16;
    case at::kFloat: return KVR_DT_FP32;
    default:
        refuse(std::string(name) + " must be bfloat16, float16 or float32, not " +
               std::string(c10::toString(t.scalar_type())));
    }
}

// A [tokens, heads, dim] tensor with adjacent rows; sizes below 0 are free.
const at::Tensor &rows(PyObject *o, const char *name, Device &on, int64_t tokens, int64_t heads,
                       int64_t dim)
{
    const at::Tensor &t = tensor(o, name);
    if (!t.is_cuda() || t.dim() != 3 || (t.stride(2) != 1 && t.size(2) != 1))
        refuse(std::string(name) + " must be a [tokens, heads, dim] CUDA tensor with adjacent rows");
    on.check(t, name);
    no_gradient(t, name);
    const int64_t want[3] = {tokens, heads, dim};
    for (int i = 0; i < 3; ++i)
        if (want[i] >= 0 && t.size(i) != want[i]) {
            auto one = [](int64_t n) { return n < 0 ? std::string("any") : std::to_string(n); };
            refuse(std::string(name) + " must have shape (" + one(tokens) + ", " + one(heads) + ", " +
                   one(dim) + "), not (" + std::to_string(t.size(0)) + ", " +
                   std::to_string(t.size(1)) + ", " + std::to_string(t.size(2)) + ")");
        }
    return t;
}

// A contiguous [count] tensor.
const at::Tensor &vector(PyObject *o, const char *name, Device &on, at::ScalarType type, int64_t count)
{
    const at::Tensor &t = tensor(o, name);
    if (!t.is_cuda() || t.scalar_type() != type || t.dim() != 1 || t.size(0) != count ||
        !t.is_contiguous())
        refuse(std::string(name) + " must be a contiguous [" + std::to_string(count) + "] " +
               c10::toString(type) + " CUDA tensor");
    on.check(t, name);
    return t;
}
const at::Tensor *status_of(PyObject *o, Device &on)
{
    return given(o) ? &vector(o, "status", on, at::kInt, 1) : nullptr;
}
template <class T>
T *address(const at::Tensor &t)
{
    return static_cast<T *>(t.data_ptr());
}
template <class T>
T *address(const at::Tensor *t)   // nullptr: none
{
    return t ? address<T>(*t) : nullptr;
}

const at::Tensor &table_of(PyObject *o, Device &on)
{
    const at::Tensor &t = tensor(o, "table");
    if (!t.is_cuda() || t.scalar_type() != at::kFloat || t.dim() != 3 || t.size(1) != 2 ||
        !t.is_contiguous() || t.size(2) > (1 << 20))
        refuse("table must be a contiguous [n_pos, 2, rot_dim / 2] float32 CUDA tensor");
    on.check(t, "table");
    no_gradient(t, "table");
    return t;
}
int32_t rot_of(const at::Tensor &table) { return (int32_t)(2 * table.size(2)); }

// A KvCache's handle: the address of the C view, the tensors it was made of (one device), and
// the view's own object, which holds it.
const kvr_kv_cache *cache_of(PyObject *o, Device &on)
{
    void *p = nullptr;
    if (PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 6) p = PyLong_AsVoidPtr(PyTuple_GET_ITEM(o, 0));
    if (!p) {
        PyErr_Clear();
        throw Refused{PyExc_TypeError, "cache must be a KvCache"};
    }
    const at::Tensor &k = tensor(PyTuple_GET_ITEM(o, 1), "cache");
    on.check(k, "cache");
    no_gradient(k, "cache");
    no_gradient(tensor(PyTuple_GET_ITEM(o, 2), "cache"), "cache");
    return static_cast<const kvr_kv_cache *>(p);
}

// A stream of the caller's: its handle and device index.
struct GivenStream {
    bool any;
    hipStream_t handle = nullptr;
    GivenStream(PyObject *o, const Device &on) : any(given(o))
    {
        if (!any) return;
        if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 2)
            throw Refused{PyExc_TypeError, "stream must be a torch.cuda.Stream"};
        on.check(integer(PyTuple_GET_ITEM(o, 1), "stream"), "stream");
        handle = static_cast<hipStream_t>(PyLong_AsVoidPtr(PyTuple_GET_ITEM(o, 0)));
        if (PyErr_Occurred()) {
            PyErr_Clear();
            throw Refused{PyExc_TypeError, "stream must be a torch.cuda.Stream"};
        }
    }
};

// The stream of a call: the caller's, or torch's current one on the call's device.  That is the
// current device as long as this lives: a launch goes to the current device, whatever
// device its tensors are on.  Made when every argument has been checked.
struct Stream {
    c10::hip::OptionalHIPGuard device;
    hipStream_t current, used;
    Stream(const GivenStream &s, const Device &on)
        : current(c10::hip::getCurrentHIPStream(on.at.index()).stream()),
          used(s.any ? s.handle : current)
    {
        if (c10::hip::current_device() != on.at.index()) device.set_index(on.at.index());
    }
    // After an allocation: memory comes from the current stream's pool, where work on what it
    // held before may still be queued, and another stream waits for that.
    void allocated() const
    {
        if (used == current) return;
        hipEvent_t e;
        hipError_t rc = hipEventCreateWithFlags(&e, hipEventDisableTiming);
        if (rc == hipSuccess) {
            rc = hipEventRecord(e, current);
            if (rc == hipSuccess) rc = hipStreamWaitEvent(used, e, 0);
            const hipError_t last = hipEventDestroy(e);   // (once it is no longer needed)
            if (rc == hipSuccess) rc = last;
        }
        if (rc != hipSuccess)
            throw Refused{PyExc_RuntimeError, std::string("streams: ") + hipGetErrorString(rc)};
    }
};

// Notes for autograd that a tensor has been written: it may have been saved for a gradient.
// (Tensors made in inference mode have no version.)
void written(const at::Tensor &t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// A Python tuple of a status code and tensors (undefined ones: None).
template <class... Ts>
PyObject *answer(int rc, const Ts &...ts)
{
    PyObject *r = PyTuple_New(1 + sizeof...(ts));
    if (!r) return nullptr;
    PyTuple_SET_ITEM(r, 0, PyLong_FromLong(rc));
    int i = 1;
    auto put = [&](const at::Tensor &t) {
        PyObject *o = Py_None;
        if (t.defined()) o = THPVariable_Wrap(t);
        else Py_INCREF(o);
        PyTuple_SET_ITEM(r, i++, o);
    };
    (put(ts), ...);
    return r;
}

// No C++ exception leaves an entry point.
template <class F>
PyObject *entry(Py_ssize_t got, Py_ssize_t want, F f)
{
    if (got != want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments expected, not %zd", want, got);
        return nullptr;
    }
    HANDLE_TH_ERRORS
    try {
        const at::AutoDispatchBelowADInplaceOrView plain;   // nothing here records gradients
        return f();
    } catch (const Refused &e) {
        PyErr_SetString(e.type, e.text.c_str());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// The output that is given, like x, or an undefined tensor.
at::Tensor given_like(PyObject *o, const at::Tensor &x, Device &on, const char *message)
{
    if (!given(o)) return at::Tensor();
    at::Tensor out = rows(o, "out", on, x.size(0), x.size(1), x.size(2));
    if (out.scalar_type() != x.scalar_type()) refuse(message);
    return out;
}
at::Tensor new_like(const at::Tensor &x)
{
    return at::empty(x.sizes(), x.options().memory_format(at::MemoryFormat::Contiguous));
}

int32_t fits32(int64_t n, const char *name)
{
    if (n > INT32_MAX) refuse(std::string(name) + " is beyond 32 bits");
    return (int32_t)n;
}

// (x, positions, table, flags, out, status, stream) -> (code, out)
PyObject *rotary(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return entry(n, 7, [&] {
        Device on;
        const at::Tensor &x = rows(a[0], "x", on, -1, -1, -1);
        const int32_t dt = dtype_of(x, "x");
        const int64_t tokens = x.size(0);
        const at::Tensor &pos = vector(a[1], "positions", on, at::kInt, tokens);
        const at::Tensor &t = table_of(a[2], on);
        const int32_t flags = integer32(a[3], "flags");
        at::Tensor out = given_like(a[4], x, on, "out must have the type of x");
        const at::Tensor *status = status_of(a[5], on);
        const int32_t heads = fits32(x.size(1), "heads"), dim = fits32(x.size(2), "head_dim");
        const GivenStream own(a[6], on);
        const Stream stream(own, on);
        if (!out.defined()) {
            out = new_like(x);
            stream.allocated();
        } else {
            written(out);
        }
        const int rc = kvr_rotary(x.data_ptr(), out.data_ptr(), dt, tokens, heads, dim, x.stride(0),
                                  x.stride(1), out.stride(0), out.stride(1), address<int32_t>(pos),
                                  address<float>(t), t.size(0), rot_of(t), flags,
                                  address<int32_t>(status), stream.used);
        return answer(rc, out);
    });
}

// (cache, k, v, slots, positions, table, flags, status, stream) -> (code,)
PyObject *cache_write(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return entry(n, 9, [&] {
        Device on;
        const kvr_kv_cache *c = cache_of(a[0], on);
        const at::Tensor &slots = tensor(a[3], "slots");
        const int64_t tokens = slots.dim() ? slots.size(0) : 0;
        const at::Tensor &k = rows(a[1], "k", on, tokens, c->n_kv_heads, c->head_dim);
        const at::Tensor &v = rows(a[2], "v", on, tokens, c->n_kv_heads, c->head_dim);
        const int32_t dt = dtype_of(k, "k");
        if (v.scalar_type() != k.scalar_type()) refuse("k and v must have one type");
        vector(a[3], "slots", on, at::kLong, tokens);
        const at::Tensor *t = nullptr, *pos = nullptr;
        if (given(a[5])) {
            t = &table_of(a[5], on);
            if (!given(a[4])) refuse("a table needs positions");
            pos = &vector(a[4], "positions", on, at::kInt, tokens);
        } else if (given(a[4])) {
            refuse("positions need a table");
        }
        const int32_t flags = integer32(a[6], "flags");
        const at::Tensor *status = status_of(a[7], on);
        const GivenStream own(a[8], on);
        const Stream stream(own, on);
        for (int i = 1; i <= 4; ++i)   // the cache's tensors, scales among them if it has any
            if (given(PyTuple_GET_ITEM(a[0], i))) written(tensor(PyTuple_GET_ITEM(a[0], i), "cache"));
        return answer(kvr_cache_write(c, k.data_ptr(), v.data_ptr(), dt, tokens, k.stride(0),
                                      k.stride(1), v.stride(0), v.stride(1), address<int64_t>(slots),
                                      address<int32_t>(pos), address<float>(t), t ? t->size(0) : 0,
                                      t ? rot_of(*t) : 0, flags, address<int32_t>(status),
                                      stream.used));
    });
}

// (cache, slots, KVR_DT_* or None, out k, out v, status, stream) -> (code, k, v)
PyObject *cache_read(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return entry(n, 7, [&] {
        Device on;
        const kvr_kv_cache *c = cache_of(a[0], on);
        const at::Tensor &slots = tensor(a[1], "slots");
        const int64_t tokens = slots.dim() ? slots.size(0) : 0;
        vector(a[1], "slots", on, at::kLong, tokens);
        const int64_t heads = c->n_kv_heads, dim = c->head_dim;
        at::Tensor k, v;
        int32_t dt;
        if (!given(a[3])) {
            dt = given(a[2]) ? integer32(a[2], "dtype") : KVR_DT_BF16;
        } else {
            k = rows(a[3], "out k", on, tokens, heads, dim);
            v = rows(a[4], "out v", on, tokens, heads, dim);
            dt = dtype_of(k, "out");
            if (v.scalar_type() != k.scalar_type() || (given(a[2]) && integer32(a[2], "dtype") != dt))
                refuse("out must be two tensors of the type that is asked for");
        }
        const at::Tensor *status = status_of(a[5], on);
        const GivenStream own(a[6], on);
        const Stream stream(own, on);
        if (!k.defined()) {
            const at::ScalarType type = dt == KVR_DT_BF16   ? at::kBFloat16
                                        : dt == KVR_DT_FP16 ? at::kHalf
                                                            : at::kFloat;
            const auto options = slots.options().dtype(type);
            k = at::empty({tokens, heads, dim}, options);
            v = at::empty({tokens, heads, dim}, options);
            stream.allocated();
        } else {
            written(k);
            written(v);
        }
        const int rc = kvr_cache_read(c, address<int64_t>(slots), tokens, k.data_ptr(), v.data_ptr(),
                                      dt, k.stride(0), k.stride(1), v.stride(0), v.stride(1),
                                      address<int32_t>(status), stream.used);
        return answer(rc, k, v);
    });
}

// (cache, q, cu_q, kv_len, page_table, max_q, max_kv, tree_mask, scale, want_lse, out,
// workspace, status, stream) -> (code, out, lse, workspace)
PyObject *tree_attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return entry(n, 14, [&] {
        Device on;
        const kvr_kv_cache *c = cache_of(a[0], on);
        const at::Tensor &q = rows(a[1], "q", on, -1, -1, c->head_dim);
        const int32_t dt = dtype_of(q, "q");
        const at::Tensor &len = tensor(a[3], "kv_len");
        const int64_t seqs = len.dim() ? len.size(0) : 0;
        vector(a[3], "kv_len", on, at::kInt, seqs);
        const at::Tensor &cu_q = vector(a[2], "cu_q", on, at::kInt, seqs + 1);
        const at::Tensor &pages = tensor(a[4], "page_table");
        if (!pages.is_cuda() || pages.scalar_type() != at::kInt || pages.dim() != 2 ||
            pages.size(0) != seqs || (pages.size(1) > 1 && pages.stride(1) != 1))
            refuse("page_table must be a [n_seqs, pages] int32 CUDA tensor");
        on.check(pages, "page_table");
        kvr_sequences s{};
        s.pages_stride = pages.stride(0);
        s.max_pages = pages.size(1);
        s.n_queries = q.size(0);
        s.n_seqs = fits32(seqs, "n_seqs");
        s.max_q = integer32(a[5], "max_q");
        s.max_kv = integer32(a[6], "max_kv");
        const at::Tensor *mask = nullptr;
        int32_t words = 0;
        if (given(a[7])) {
            mask = &tensor(a[7], "tree_mask");
            if (!mask->is_cuda() || mask->scalar_type() != at::kLong || mask->dim() != 2 ||
                mask->size(0) != s.n_queries || !mask->is_contiguous())
                refuse("tree_mask must be a contiguous [n_queries, words] int64 CUDA tensor");
            on.check(*mask, "tree_mask");
            words = fits32(mask->size(1), "tree_mask");
        }
        double scale = 1.0 / std::sqrt((double)c->head_dim);
        if (given(a[8])) {
            scale = PyFloat_AsDouble(a[8]);
            if (scale == -1.0 && PyErr_Occurred()) {
                PyErr_Clear();
                throw Refused{PyExc_TypeError, "scale must be a number"};
            }
        }
        const int want_lse = PyObject_IsTrue(a[9]);
        if (want_lse < 0) {
            PyErr_Clear();
            throw Refused{PyExc_TypeError, "want_lse must be true or false"};
        }
        at::Tensor out = given_like(a[10], q, on, "out must have the type of q");
        at::Tensor lse, ws;
        if (given(a[11])) {
            ws = tensor(a[11], "workspace");
            if (!ws.is_cuda() || ws.scalar_type() != at::kByte || !ws.is_contiguous())
                refuse("workspace must be a contiguous torch.uint8 CUDA tensor");
            on.check(ws, "workspace");
        }
        const at::Tensor *status = status_of(a[12], on);
        const int32_t heads = fits32(q.size(1), "q");
        const GivenStream own(a[13], on);
        const Stream stream(own, on);
        bool allocated = false;
        if (!out.defined()) {
            out = new_like(q);
            allocated = true;
        } else {
            written(out);
        }
        if (want_lse) {
            lse = at::empty({q.size(0), q.size(1)}, q.options().dtype(at::kFloat));
            allocated = true;
        }
        s.d_cu_q = address<int32_t>(cu_q);
        s.d_kv_len = address<int32_t>(len);
        s.d_pages = address<int32_t>(pages);
        size_t bytes = 0;
        auto call = [&](void *space) {
            return kvr_tree_attention(c, &s, q.data_ptr(), dt, heads, q.stride(0), q.stride(1),
                                      address<uint64_t>(mask), words, (float)scale, out.data_ptr(),
                                      out.stride(0), out.stride(1),
                                      lse.defined() ? address<float>(lse) : nullptr,
                                      address<int32_t>(status), space, &bytes, stream.used);
        };
        int rc = call(nullptr);   // the workspace's size
        if (rc != KVR_OK) return answer(rc, out, lse, ws);
        const bool cut = bytes != 0;
        if (cut && (!ws.defined() || (size_t)ws.numel() < bytes)) {
            ws = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
            allocated = true;
        }
        if (allocated) stream.allocated();
        if (!cut) {   // an address that is never used
            alignas(256) static char none[256];
            return answer(call(none), out, lse, at::Tensor());
        }
        bytes = (size_t)ws.numel();
        rc = call(ws.data_ptr());
        return answer(rc, out, lse, ws);
    });
}

#define KVR_FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {KVR_FAST(rotary), KVR_FAST(cache_write), KVR_FAST(cache_read),
                          KVR_FAST(tree_attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "kvr_torch", nullptr, -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject *PyInit_kvr_torch() { return PyModule_Create(&kModule); }
