// The entry points of the caches and their pages on torch tensors: checks of types, shapes and strides,
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

// A LatentCache's handle: the address of the C view, its rows, its scales (or None) and the
// view's own object.
const kvr_latent_cache *latents_of(PyObject *o, Device &on)
{
    void *p = nullptr;
    if (PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 4) p = PyLong_AsVoidPtr(PyTuple_GET_ITEM(o, 0));
    if (!p || !THPVariable_Check(PyTuple_GET_ITEM(o, 1))) {
        PyErr_Clear();
        throw Refused{PyExc_TypeError, "cache must be a LatentCache"};
    }
    const at::Tensor &rows = tensor(PyTuple_GET_ITEM(o, 1), "cache");
    on.check(rows, "cache");
    no_gradient(rows, "cache");
    return static_cast<const kvr_latent_cache *>(p);
}

// A [count, dim] tensor with adjacent rows.
const at::Tensor &matrix(PyObject *o, const char *name, Device &on, int64_t count, int64_t dim)
{
    const at::Tensor &t = tensor(o, name);
    if (!t.is_cuda() || t.dim() != 2 || t.size(0) != count || t.size(1) != dim ||
        (t.stride(1) != 1 && t.size(1) != 1))
        refuse(std::string(name) + " must be a [" + std::to_string(count) + ", " + std::to_string(dim) +
               "] CUDA tensor with adjacent rows");
    on.check(t, name);
    no_gradient(t, name);
    return t;
}

double number(PyObject *o, const char *name)
{
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Refused{PyExc_TypeError, std::string(name) + " must be a number"};
    }
    return x;
}
bool truth(PyObject *o, const char *name)
{
    const int x = PyObject_IsTrue(o);
    if (x < 0) {
        PyErr_Clear();
        throw Refused{PyExc_TypeError, std::string(name) + " must be true or false"};
    }
    return x != 0;
}

// The workspace that is given, or an undefined tensor.
at::Tensor workspace_of(PyObject *o, Device &on)
{
    if (!given(o)) return at::Tensor();
    const at::Tensor &ws = tensor(o, "workspace");
    if (!ws.is_cuda() || ws.scalar_type() != at::kByte || !ws.is_contiguous())
        refuse("workspace must be a contiguous torch.uint8 CUDA tensor");
    on.check(ws, "workspace");
    return ws;
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

// Runs call(workspace, bytes) twice: for the workspace's size, and in earnest.  `allocated`: the
// call has allocated already.  Returns the code; ws: what was used, undefined for none.
template <class Call>
int with_workspace(const Stream &stream, at::Tensor &ws, const at::TensorOptions &options, bool allocated,
                   Call call)
{
    size_t bytes = 0;
    const int rc = call(nullptr, &bytes);
    if (rc != KVR_OK) return rc;
    if (bytes == 0) {   // an address that is never used
        if (allocated) stream.allocated();
        alignas(256) static char none[256];
        ws = at::Tensor();
        return call(none, &bytes);
    }
    if (!ws.defined() || (size_t)ws.numel() < bytes) {
        ws = at::empty({(int64_t)bytes}, options.dtype(at::kByte));
        allocated = true;
    }
    if (allocated) stream.allocated();
    bytes = (size_t)ws.numel();
    return call(ws.data_ptr(), &bytes);
}

// (cache, latent, key, slots, positions, table, norm_weight, eps, flags, status, stream) -> (code,)
PyObject *latent_write(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return entry(n, 11, [&] {
        Device on;
        const kvr_latent_cache *c = latents_of(a[0], on);
        const at::Tensor &slots = tensor(a[3], "slots");
        const int64_t tokens = slots.dim() ? slots.size(0) : 0;
        const at::Tensor &latent = matrix(a[1], "latent", on, tokens, c->rank);
        const at::Tensor &key = matrix(a[2], "key", on, tokens, c->rot);
        const int32_t dt = dtype_of(latent, "latent");
        if (key.scalar_type() != latent.scalar_type()) refuse("latent and key must have one type");
        vector(a[3], "slots", on, at::kLong, tokens);
        const at::Tensor *t = nullptr, *pos = nullptr, *norm = nullptr;
        if (given(a[5])) {
            t = &table_of(a[5], on);
            if (!given(a[4])) refuse("a table needs positions");
            pos = &vector(a[4], "positions", on, at::kInt, tokens);
        } else if (given(a[4])) {
            refuse("positions need a table");
        }
        if (given(a[6])) {
            norm = &vector(a[6], "norm_weight", on, latent.scalar_type(), c->rank);
            no_gradient(*norm, "norm_weight");
        }
        const double eps = number(a[7], "eps");
        const int32_t flags = integer32(a[8], "flags");
        const at::Tensor *status = status_of(a[9], on);
        const GivenStream own(a[10], on);
        const Stream stream(own, on);
        for (int i = 1; i <= 2; ++i)
            if (given(PyTuple_GET_ITEM(a[0], i))) written(tensor(PyTuple_GET_ITEM(a[0], i), "cache"));
        return answer(kvr_latent_write(c, latent.data_ptr(), key.data_ptr(), dt, tokens, latent.stride(0),
                                       key.stride(0), norm ? norm->data_ptr() : nullptr, (float)eps,
                                       address<int64_t>(slots), address<int32_t>(pos), address<float>(t),
                                       t ? t->size(0) : 0, t ? rot_of(*t) : 0, flags,
                                       address<int32_t>(status), stream.used));
    });
}

// (cache, slots, KVR_DT_* or None, out, status, stream) -> (code, out)
PyObject *latent_read(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return entry(n, 6, [&] {
        Device on;
        const kvr_latent_cache *c = latents_of(a[0], on);
        const at::Tensor &slots = tensor(a[1], "slots");
        const int64_t tokens = slots.dim() ? slots.size(0) : 0;
        vector(a[1], "slots", on, at::kLong, tokens);
        const int64_t dim = (int64_t)c->rank + c->rot;
        at::Tensor out;
        int32_t dt;
        if (!given(a[3])) {
            dt = given(a[2]) ? integer32(a[2], "dtype") : KVR_DT_BF16;
        } else {
            out = matrix(a[3], "out", on, tokens, dim);
            dt = dtype_of(out, "out");
            if (given(a[2]) && integer32(a[2], "dtype") != dt) refuse("out must have the type that is asked for");
        }
        const at::Tensor *status = status_of(a[4], on);
        const GivenStream own(a[5], on);
        const Stream stream(own, on);
        if (!out.defined()) {
            const at::ScalarType type = dt == KVR_DT_BF16   ? at::kBFloat16
                                        : dt == KVR_DT_FP16 ? at::kHalf
                                                            : at::kFloat;
            out = at::empty({tokens, dim}, slots.options().dtype(type));
            stream.allocated();
        } else {
            written(out);
        }
        const int rc = kvr_latent_read(c, address<int64_t>(slots), tokens, out.data_ptr(), dt, out.stride(0),
                                       address<int32_t>(status), stream.used);
        return answer(rc, out);
    });
}

// An output [tokens, heads, dim] of x's type: the one that is given, or an undefined tensor.
at::Tensor output_of(PyObject *o, const at::Tensor &x, int64_t dim, Device &on)
{
    if (!given(o)) return at::Tensor();
    at::Tensor out = rows(o, "out", on, x.size(0), x.size(1), dim);
    if (out.scalar_type() != x.scalar_type()) refuse("out must have the type of q");
    return out;
}
// The output, new if none was given, and with want_lse the logarithms; whether memory was allocated.
bool outputs(at::Tensor &out, at::Tensor &lse, bool want_lse, const at::Tensor &q, int64_t dim)
{
    const bool fresh = !out.defined();
    if (fresh) out = at::empty({q.size(0), q.size(1), dim}, q.options());
    else written(out);
    if (want_lse) lse = at::empty({q.size(0), q.size(1)}, q.options().dtype(at::kFloat));
    return fresh || want_lse;
}

// (cache, q, cu_q, kv_len, page_table, max_q, max_kv, scale, tree_mask, want_lse, out,
// workspace, status, stream) -> (code, out, lse, workspace)
PyObject *latent_attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return entry(n, 14, [&] {
        Device on;
        const kvr_latent_cache *c = latents_of(a[0], on);
        const at::Tensor &q = rows(a[1], "q", on, -1, -1, (int64_t)c->rank + c->rot);
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
        const double scale = number(a[7], "scale");
        const at::Tensor *mask = nullptr;
        int32_t words = 0;
        if (given(a[8])) {
            mask = &tensor(a[8], "tree_mask");
            if (!mask->is_cuda() || mask->scalar_type() != at::kLong || mask->dim() != 2 ||
                mask->size(0) != s.n_queries || !mask->is_contiguous())
                refuse("tree_mask must be a contiguous [n_queries, words] int64 CUDA tensor");
            on.check(*mask, "tree_mask");
            words = fits32(mask->size(1), "tree_mask");
        }
        const bool want_lse = truth(a[9], "want_lse");
        at::Tensor out = output_of(a[10], q, c->rank, on), lse, ws = workspace_of(a[11], on);
        const at::Tensor *status = status_of(a[12], on);
        const int32_t heads = fits32(q.size(1), "q");
        const GivenStream own(a[13], on);
        const Stream stream(own, on);
        const bool allocated = outputs(out, lse, want_lse, q, c->rank);
        s.d_cu_q = address<int32_t>(cu_q);
        s.d_kv_len = address<int32_t>(len);
        s.d_pages = address<int32_t>(pages);
        const int rc = with_workspace(stream, ws, q.options(), allocated, [&](void *space, size_t *bytes) {
            return kvr_latent_attention(c, &s, q.data_ptr(), dt, heads, q.stride(0), q.stride(1),
                                        address<uint64_t>(mask), words, (float)scale, out.data_ptr(),
                                        out.stride(0), out.stride(1),
                                        lse.defined() ? address<float>(lse) : nullptr,
                                        address<int32_t>(status), space, bytes, stream.used);
        });
        return answer(rc, out, lse, ws);
    });
}

// (q, k, k_rot, v, cu_q, cu_k, max_q, max_k, causal, scale, want_lse, out, workspace, status,
// stream) -> (code, out, lse, workspace)
PyObject *latent_prompt(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return entry(n, 15, [&] {
        Device on;
        const at::Tensor &q = rows(a[0], "q", on, -1, -1, -1);
        const at::Tensor &k = rows(a[1], "k", on, -1, -1, -1);
        const int64_t nope = k.size(2), rot = q.size(2) - nope;
        if (rot < 1) refuse("q must have the elements of k and those of k_rot");
        const at::Tensor &shared = matrix(a[2], "k_rot", on, k.size(0), rot);
        const at::Tensor &v = rows(a[3], "v", on, k.size(0), k.size(1), nope);
        const int32_t dt = dtype_of(q, "q");
        if (k.scalar_type() != q.scalar_type() || v.scalar_type() != q.scalar_type() ||
            shared.scalar_type() != q.scalar_type())
            refuse("q, k, k_rot and v must have one type");
        const at::Tensor &first = tensor(a[4], "cu_q");
        const int64_t seqs = first.dim() ? first.size(0) - 1 : -1;
        if (seqs < 0) refuse("cu_q must have one element more than there are sequences");
        const at::Tensor &cu_q = vector(a[4], "cu_q", on, at::kInt, seqs + 1);
        const at::Tensor &cu_k = vector(a[5], "cu_k", on, at::kInt, seqs + 1);
        kvr_prompt p{};
        p.d_cu_q = address<int32_t>(cu_q);
        p.d_cu_k = address<int32_t>(cu_k);
        p.n_queries = q.size(0);
        p.n_keys = k.size(0);
        p.n_seqs = fits32(seqs, "n_seqs");
        p.max_q = integer32(a[6], "max_q");
        p.max_k = integer32(a[7], "max_k");
        p.n_q_heads = fits32(q.size(1), "q");
        p.n_kv_heads = fits32(k.size(1), "k");
        p.nope = fits32(nope, "k");
        p.rot = fits32(rot, "k_rot");
        p.causal = truth(a[8], "causal");
        const double scale = given(a[9]) ? number(a[9], "scale") : 1.0 / std::sqrt((double)q.size(2));
        const bool want_lse = truth(a[10], "want_lse");
        at::Tensor out = output_of(a[11], q, nope, on), lse, ws = workspace_of(a[12], on);
        const at::Tensor *status = status_of(a[13], on);
        const GivenStream own(a[14], on);
        const Stream stream(own, on);
        const bool allocated = outputs(out, lse, want_lse, q, nope);
        const int rc = with_workspace(stream, ws, q.options(), allocated, [&](void *space, size_t *bytes) {
            return kvr_latent_prompt(&p, q.data_ptr(), dt, q.stride(0), q.stride(1), k.data_ptr(), k.stride(0),
                                     k.stride(1), shared.data_ptr(), shared.stride(0), v.data_ptr(),
                                     v.stride(0), v.stride(1), (float)scale, out.data_ptr(), out.stride(0),
                                     out.stride(1), lse.defined() ? address<float>(lse) : nullptr,
                                     address<int32_t>(status), space, bytes, stream.used);
        });
        return answer(rc, out, lse, ws);
    });
}

// refs, page_table, kv_len and page_size as the C ABI takes them.
kvr_page_pool pool_of(PyObject *const *a, PyObject *size, Device &on)
{
    const at::Tensor &refs = tensor(a[0], "refs");
    vector(a[0], "refs", on, at::kInt, refs.dim() ? refs.size(0) : 0);
    const at::Tensor &len = tensor(a[2], "kv_len");
    const int64_t seqs = len.dim() ? len.size(0) : 0;
    vector(a[2], "kv_len", on, at::kInt, seqs);
    const at::Tensor &pages = tensor(a[1], "page_table");
    if (!pages.is_cuda() || pages.scalar_type() != at::kInt || pages.dim() != 2 || pages.size(0) != seqs ||
        (pages.size(1) > 1 && pages.stride(1) != 1))
        refuse("page_table must be a [n_seqs, pages] int32 CUDA tensor");
    on.check(pages, "page_table");
    kvr_page_pool p{};
    p.d_refs = address<int32_t>(refs);
    p.d_pages = address<int32_t>(pages);
    p.d_kv_len = address<int32_t>(len);
    p.n_pages = refs.size(0);
    p.pages_stride = pages.stride(0);
    p.max_pages = fits32(pages.size(1), "page_table");
    p.n_seqs = fits32(seqs, "n_seqs");
    p.page_size = integer32(size, "page_size");
    return p;
}
void pool_written(PyObject *const *a)
{
    for (int i = 0; i < 3; ++i) written(THPVariable_Unpack(a[i]));
}

// A contiguous [count, 2] int32 tensor.
const at::Tensor &pairs_of(PyObject *o, const char *name, Device &on, int64_t count)
{
    const at::Tensor &t = tensor(o, name);
    if (!t.is_cuda() || t.scalar_type() != at::kInt || t.dim() != 2 || t.size(1) != 2 ||
        (count >= 0 && t.size(0) != count) || !t.is_contiguous())
        refuse(std::string(name) + " must be a contiguous [" + (count < 0 ? "n" : std::to_string(count)) +
               ", 2] int32 CUDA tensor");
    on.check(t, name);
    return t;
}

// (refs, page_table, kv_len, parent, page_size, status, stream) -> (code,)
PyObject *pages_fork(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return entry(n, 7, [&] {
        Device on;
        const kvr_page_pool p = pool_of(a, a[4], on);
        const at::Tensor &parent = vector(a[3], "parent", on, at::kInt, p.n_seqs);
        const at::Tensor *status = status_of(a[5], on);
        const GivenStream own(a[6], on);
        const Stream stream(own, on);
        pool_written(a);
        return answer(kvr_pages_fork(&p, address<int32_t>(parent), address<int32_t>(status), stream.used));
    });
}

// (refs, page_table, kv_len, new_len, page_size, copies, workspace, status, stream) ->
// (code, copies, workspace)
PyObject *pages_resize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return entry(n, 9, [&] {
        Device on;
        const kvr_page_pool p = pool_of(a, a[4], on);
        const at::Tensor &len = vector(a[3], "new_len", on, at::kInt, p.n_seqs);
        at::Tensor copies, ws = workspace_of(a[6], on);
        if (given(a[5])) copies = pairs_of(a[5], "copies", on, p.n_seqs);
        const at::Tensor *status = status_of(a[7], on);
        const GivenStream own(a[8], on);
        const Stream stream(own, on);
        const bool fresh = !copies.defined();
        if (fresh) copies = at::empty({p.n_seqs, 2}, len.options());
        else written(copies);
        pool_written(a);
        const int rc = with_workspace(stream, ws, len.options(), fresh, [&](void *space, size_t *bytes) {
            return kvr_pages_resize(&p, address<int32_t>(len), address<int32_t>(copies),
                                    address<int32_t>(status), space, bytes, stream.used);
        });
        return answer(rc, copies, ws);
    });
}

// (refs, page_table, kv_len, page_size, max_moves or None, moves, used, workspace, status,
// stream) -> (code, moves, used, workspace)
PyObject *pages_compact(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return entry(n, 10, [&] {
        Device on;
        const kvr_page_pool p = pool_of(a, a[3], on);
        at::Tensor moves, used, ws = workspace_of(a[7], on);
        int64_t most = given(a[4]) ? integer(a[4], "max_moves") : p.n_pages;
        if (most < 0 || most > p.n_pages) refuse("max_moves must be from 0 to the pages of the pool");
        if (given(a[5])) moves = pairs_of(a[5], "moves", on, most);
        if (given(a[6])) used = vector(a[6], "used", on, at::kInt, 1);
        const at::Tensor *status = status_of(a[8], on);
        const GivenStream own(a[9], on);
        const Stream stream(own, on);
        const at::TensorOptions options = THPVariable_Unpack(a[0]).options();
        const bool fresh = !moves.defined() || !used.defined();
        if (!moves.defined()) moves = at::empty({most, 2}, options);
        else written(moves);
        if (!used.defined()) used = at::empty({1}, options);
        else written(used);
        pool_written(a);
        const int rc = with_workspace(stream, ws, options, fresh, [&](void *space, size_t *bytes) {
            return kvr_pages_compact(&p, address<int32_t>(moves), most, address<int32_t>(used),
                                     address<int32_t>(status), space, bytes, stream.used);
        });
        return answer(rc, moves, used, ws);
    });
}

// (PageBuffers' handle: address, count, pages, tensors, array; pairs, status, stream) -> (code,)
PyObject *pages_copy(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return entry(n, 4, [&] {
        Device on;
        if (!PyTuple_Check(a[0]) || PyTuple_GET_SIZE(a[0]) != 5 || !PyTuple_Check(PyTuple_GET_ITEM(a[0], 3)))
            throw Refused{PyExc_TypeError, "buffers must be PageBuffers"};
        const auto *buffers = static_cast<const kvr_page_buffer *>(PyLong_AsVoidPtr(PyTuple_GET_ITEM(a[0], 0)));
        const int32_t count = integer32(PyTuple_GET_ITEM(a[0], 1), "buffers");
        const int64_t n_pages = integer(PyTuple_GET_ITEM(a[0], 2), "buffers");
        PyObject *tensors = PyTuple_GET_ITEM(a[0], 3);
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(tensors); ++i) {
            const at::Tensor &t = tensor(PyTuple_GET_ITEM(tensors, i), "buffers");
            on.check(t, "buffers");
            no_gradient(t, "buffers");
        }
        const at::Tensor &pairs = pairs_of(a[1], "pairs", on, -1);
        const at::Tensor *status = status_of(a[2], on);
        const GivenStream own(a[3], on);
        const Stream stream(own, on);
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(tensors); ++i)
            written(THPVariable_Unpack(PyTuple_GET_ITEM(tensors, i)));
        return answer(kvr_pages_copy(buffers, count, n_pages, address<int32_t>(pairs), pairs.size(0),
                                     address<int32_t>(status), stream.used));
    });
}

#define KVR_FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {KVR_FAST(rotary), KVR_FAST(cache_write), KVR_FAST(cache_read),
                          KVR_FAST(tree_attention), KVR_FAST(latent_write), KVR_FAST(latent_read),
                          KVR_FAST(latent_attention), KVR_FAST(latent_prompt), KVR_FAST(pages_fork),
                          KVR_FAST(pages_resize), KVR_FAST(pages_compact), KVR_FAST(pages_copy),
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "kvr_torch", nullptr, -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject *PyInit_kvr_torch() { return PyModule_Create(&kModule); }
