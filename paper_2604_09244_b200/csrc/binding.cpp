// Native side of the Python binding (module `_native`): turns the arguments of the C-ABI calls -- tensors, sample
// descriptors, output records -- into plain pointers and calls libmvla_prune.so.  No arithmetic of the method here.
//
// A step of the smallest sizes is 12 us of GPU work, so what a call costs on the host is part of its time: the same
// marshalling through ctypes (two structures, some fourteen tensors checked one by one, the current stream) took 8.7 us
// of interpreter work per call, here about 1 us.
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <cstring>

#include "mvla_prune.h"

namespace {

constexpr int kMaxBatch = 64;       // samples per call (the library refuses more)

// Attribute names of StepOutputs, in the order of mvla_outputs, and of the sample descriptors.
enum { OUT_HIDDEN, OUT_K, OUT_V, KEPT, OFFSETS, BUDGETS, ATTN, AHAT, Z, DIAG, PATCH_X, PATCH_XHAT, PATCH_INFO, PATCH_DIAG, N_OUT };
const char* const kOutNames[N_OUT] = {"out_hidden", "out_k", "out_v", "kept_idx", "out_offsets", "budgets", "attn",
                                      "ahat", "z", "diag", "patch_x", "patch_xhat", "patch_info", "patch_diag"};
const char* const kSampleInts[8] = {"seq_off", "off_txt", "n_txt", "off_2d", "n_2d", "off_3d", "n_3d", "state_slot"};
const char* const kSampleFloats[3] = {"keep_2d", "keep_3d", "keep_total"};
PyObject* g_out_names[N_OUT];
PyObject* g_int_names[8];
PyObject* g_float_names[3];
PyObject* g_cuda_stream;            // "cuda_stream"

// Device pointer of a tensor, null for None.  False: a Python exception is set.
bool tensor_ptr(PyObject* o, void** p, const at::Tensor** tensor = nullptr)
{
    *p = nullptr;
    if (o == Py_None) return true;
    if (!THPVariable_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "expected a torch.Tensor or None");
        return false;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) {
        PyErr_SetString(PyExc_AssertionError, "device-resident contiguous tensors only");
        return false;
    }
    *p = t.data_ptr();
    if (tensor) *tensor = &t;
    return true;
}

// Rows of the packed tensor q (its first dimension).
bool rows_of(PyObject* q, int64_t* rows)
{
    if (!THPVariable_Check(q) || THPVariable_Unpack(q).dim() < 1) {
        PyErr_SetString(PyExc_TypeError, "q must be a tensor of [rows, heads, head_dim]");
        return false;
    }
    *rows = THPVariable_Unpack(q).size(0);
    return true;
}

bool int_of(PyObject* o, int64_t* v)
{
    *v = PyLong_AsLongLong(o);
    if (*v == -1 && PyErr_Occurred()) {                       // not an int (a NumPy integer, say): what int() makes of it
        PyErr_Clear();
        PyObject* i = PyNumber_Long(o);
        if (!i) return false;
        *v = PyLong_AsLongLong(i);
        Py_DECREF(i);
        if (*v == -1 && PyErr_Occurred()) return false;
    }
    return true;
}

// One descriptor from an object with the descriptor's field names.
bool sample_from(PyObject* o, mvla_sample* s)
{
    int32_t* const ints[8] = {&s->seq_off, &s->off_txt, &s->n_txt, &s->off_2d, &s->n_2d, &s->off_3d, &s->n_3d, &s->state_slot};
    double* const floats[3] = {&s->keep_2d, &s->keep_3d, &s->keep_total};
    for (int i = 0; i < 8; ++i) {
        PyObject* a = PyObject_GetAttr(o, g_int_names[i]);
        if (!a) {
            if (i < 7 || !PyErr_ExceptionMatches(PyExc_AttributeError)) return false;
            PyErr_Clear();                                    // state_slot may be missing: slot 0
            s->state_slot = 0;
            continue;
        }
        int64_t v = 0;
        const bool ok = int_of(a, &v);
        Py_DECREF(a);
        if (!ok) return false;
        *ints[i] = static_cast<int32_t>(v);
    }
    for (int i = 0; i < 3; ++i) {
        PyObject* a = PyObject_GetAttr(o, g_float_names[i]);
        if (!a) return false;
        *floats[i] = PyFloat_AsDouble(a);
        Py_DECREF(a);
        if (*floats[i] == -1.0 && PyErr_Occurred()) return false;
    }
    return true;
}

// The call's descriptors: the caller's ctypes array as it lies in memory, or a list / tuple of objects converted here.
struct Samples {
    mvla_sample own[kMaxBatch];
    const mvla_sample* ptr = nullptr;
    int n = 0;
    Py_buffer view;
    bool viewed = false;
    ~Samples() { if (viewed) PyBuffer_Release(&view); }
    bool take(PyObject* o)
    {
        if (PyList_Check(o) || PyTuple_Check(o)) {
            const Py_ssize_t len = PySequence_Fast_GET_SIZE(o);
            n = static_cast<int>(len);
            ptr = own;
            // more than the library takes: only the count matters, it answers MVLA_ERR_CAPACITY
            for (Py_ssize_t i = 0; i < len && i < kMaxBatch; ++i)
                if (!sample_from(PySequence_Fast_GET_ITEM(o, i), own + i)) return false;
            return true;
        }
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) == 0) {
            viewed = true;
            if (view.len % static_cast<Py_ssize_t>(sizeof(mvla_sample)) != 0) {
                PyErr_SetString(PyExc_TypeError, "samples: not an array of sample descriptors");
                return false;
            }
            ptr = static_cast<const mvla_sample*>(view.buf);
            n = static_cast<int>(view.len / static_cast<Py_ssize_t>(sizeof(mvla_sample)));
            return true;
        }
        PyErr_Clear();
        PyObject* seq = PySequence_List(o);                   // any other sequence of objects
        if (!seq) return false;
        const bool ok = take(seq);
        Py_DECREF(seq);
        return ok;
    }
    int64_t visual() const
    {
        int64_t v = 0;
        for (int i = 0; i < n && i < kMaxBatch; ++i) v += ptr[i].n_2d + ptr[i].n_3d;
        return v;
    }
};

bool stream_of(PyObject* o, void** st)
{
    if (o == Py_None) {
        *st = c10::cuda::getCurrentCUDAStream().stream();
        return true;
    }
    PyObject* h = PyObject_GetAttr(o, g_cuda_stream);
    if (!h) return false;
    *st = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    return !PyErr_Occurred();
}

bool arg_count(Py_ssize_t got, Py_ssize_t want)
{
    if (got == want) return true;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, got);
    return false;
}

// Pointers of a StepOutputs record; the tensors stay alive through the record.
bool outputs_of(PyObject* out, mvla_outputs* o, unsigned wanted)
{
    std::memset(o, 0, sizeof *o);
    void** const dst[N_OUT] = {&o->out_hidden, &o->out_k, &o->out_v, reinterpret_cast<void**>(&o->kept_idx),
                               reinterpret_cast<void**>(&o->out_offsets), reinterpret_cast<void**>(&o->budgets),
                               reinterpret_cast<void**>(&o->attn), reinterpret_cast<void**>(&o->ahat),
                               reinterpret_cast<void**>(&o->z), reinterpret_cast<void**>(&o->diag),
                               reinterpret_cast<void**>(&o->patch_x), reinterpret_cast<void**>(&o->patch_xhat),
                               reinterpret_cast<void**>(&o->patch_info), reinterpret_cast<void**>(&o->patch_diag)};
    for (int i = 0; i < N_OUT; ++i) {
        if (!((wanted >> i) & 1u)) continue;
        PyObject* a = PyObject_GetAttr(out, g_out_names[i]);
        if (!a) return false;
        const bool ok = tensor_ptr(a, dst[i]);
        Py_DECREF(a);
        if (!ok) return false;
    }
    return true;
}

// The library call itself runs without the interpreter lock: a launch may block when the device's queue is full.
template <class F>
int32_t unlocked(F call)
{
    PyThreadState* save = PyEval_SaveThread();
    const int32_t rc = call();
    PyEval_RestoreThread(save);
    return rc;
}
mvla_ctx* ctx_of(PyObject* h) { return static_cast<mvla_ctx*>(PyLong_AsVoidPtr(h)); }

#define MVLA_TRY try {
#define MVLA_CATCH                                                                    \
    } catch (const std::exception& e) {                                               \
        PyErr_SetString(PyExc_RuntimeError, e.what());                                \
        return nullptr;                                                               \
    }

// prune_step(ctx, point, samples, mode, flags, q, k, v, hidden, rand_u, changed_rows, out, stream) -> rows kept, or < 0
PyObject* py_prune_step(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    MVLA_TRY
    if (!arg_count(n, 13)) return nullptr;
    int64_t point, mode, flags;
    if (!int_of(a[1], &point) || !int_of(a[3], &mode) || !int_of(a[4], &flags)) return nullptr;
    Samples s;
    if (!s.take(a[2])) return nullptr;
    mvla_tensors in;
    std::memset(&in, 0, sizeof in);
    void *q, *k, *v, *hidden, *u, *st;
    if (!tensor_ptr(a[5], &q) || !tensor_ptr(a[6], &k) || !tensor_ptr(a[7], &v) || !tensor_ptr(a[8], &hidden) ||
        !tensor_ptr(a[9], &u) || !rows_of(a[5], &in.rows))
        return nullptr;
    in.q = q; in.k = k; in.v = v; in.hidden = hidden; in.rand_u = static_cast<const float*>(u);
    Py_buffer mask;
    const bool masked = a[10] != Py_None;
    if (masked) {                                             // a host byte per row, read during the call
        if (PyObject_GetBuffer(a[10], &mask, PyBUF_SIMPLE) != 0) return nullptr;
        if (mask.len != in.rows) {
            PyBuffer_Release(&mask);
            PyErr_SetString(PyExc_AssertionError, "one byte per row of the packed tensors");
            return nullptr;
        }
        in.changed_rows = static_cast<const uint8_t*>(mask.buf);
    }
    mvla_outputs out;
    int32_t rc = 0, total = 0;
    const bool ok = outputs_of(a[11], &out, ~0u) && stream_of(a[12], &st);
    mvla_ctx* ctx = ctx_of(a[0]);
    if (ok)
        rc = unlocked([&] {
            return mvla_prune_step(ctx, static_cast<int32_t>(point), s.n, s.ptr, static_cast<int32_t>(mode),
                                   static_cast<uint32_t>(flags), &in, &out, &total, st);
        });
    if (masked) PyBuffer_Release(&mask);
    if (!ok) return nullptr;
    return PyLong_FromLong(rc != MVLA_OK ? rc : total);
    MVLA_CATCH
}

// salience(ctx, samples, q, k, hidden, attn_out, l1_out, stream) -> (status, attn_out, l1_out); a missing attn_out, and a
// missing l1_out beside `hidden`, is allocated on q's device
PyObject* py_salience(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    MVLA_TRY
    if (!arg_count(n, 8)) return nullptr;
    Samples s;
    if (!s.take(a[1])) return nullptr;
    int64_t rows;
    void *q, *k, *hidden, *attn, *l1, *st;
    const at::Tensor* qt = nullptr;
    if (!tensor_ptr(a[2], &q, &qt) || !tensor_ptr(a[3], &k) || !tensor_ptr(a[4], &hidden) || !rows_of(a[2], &rows) ||
        !stream_of(a[7], &st))
        return nullptr;
    PyObject *attn_o = a[5], *l1_o = a[6];
    Py_INCREF(attn_o);
    Py_INCREF(l1_o);
    auto fresh = [&](PyObject** o) {
        Py_DECREF(*o);
        *o = THPVariable_Wrap(at::empty({s.visual()}, qt->options().dtype(at::kFloat)));
    };
    if (attn_o == Py_None) fresh(&attn_o);
    if (l1_o == Py_None && hidden) fresh(&l1_o);
    PyObject* ret = nullptr;
    if (attn_o && l1_o && tensor_ptr(attn_o, &attn) && tensor_ptr(l1_o, &l1)) {
        mvla_ctx* ctx = ctx_of(a[0]);
        const int32_t rc = unlocked([&] {
            return mvla_salience(ctx, s.n, s.ptr, q, k, hidden, rows, static_cast<float*>(attn), static_cast<float*>(l1), st);
        });
        ret = Py_BuildValue("(iOO)", rc, attn_o, l1_o);
    }
    Py_XDECREF(attn_o);
    Py_XDECREF(l1_o);
    return ret;
    MVLA_CATCH
}

// select(ctx, point, samples, mode, flags, attn, l1, out, stream) -> status
PyObject* py_select(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    MVLA_TRY
    if (!arg_count(n, 9)) return nullptr;
    int64_t point, mode, flags;
    if (!int_of(a[1], &point) || !int_of(a[3], &mode) || !int_of(a[4], &flags)) return nullptr;
    Samples s;
    void *attn, *l1, *st;
    mvla_outputs o;
    constexpr unsigned kWanted = 1u << KEPT | 1u << OFFSETS | 1u << BUDGETS | 1u << AHAT | 1u << Z | 1u << DIAG;
    if (!s.take(a[2]) || !tensor_ptr(a[5], &attn) || !tensor_ptr(a[6], &l1) || !outputs_of(a[7], &o, kWanted) ||
        !stream_of(a[8], &st))
        return nullptr;
    mvla_ctx* ctx = ctx_of(a[0]);
    return PyLong_FromLong(unlocked([&] {
        return mvla_select(ctx, static_cast<int32_t>(point), s.n, s.ptr, static_cast<int32_t>(mode),
                           static_cast<uint32_t>(flags), static_cast<const float*>(attn), static_cast<const float*>(l1),
                           o.kept_idx, o.out_offsets, o.budgets, o.ahat, o.z, o.diag, st);
    }));
    MVLA_CATCH
}

// compact(ctx, samples, kept_idx, out_offsets, total, hidden, k, v, out_hidden, out_k, out_v, stream) -> status
PyObject* py_compact(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    MVLA_TRY
    if (!arg_count(n, 12)) return nullptr;
    Samples s;
    int64_t total;
    void *kept, *offs, *src[3], *dst[3], *st;
    if (!s.take(a[1]) || !tensor_ptr(a[2], &kept) || !tensor_ptr(a[3], &offs) || !int_of(a[4], &total)) return nullptr;
    for (int i = 0; i < 3; ++i)
        if (!tensor_ptr(a[5 + i], &src[i]) || !tensor_ptr(a[8 + i], &dst[i])) return nullptr;
    if (!stream_of(a[11], &st)) return nullptr;
    mvla_ctx* ctx = ctx_of(a[0]);
    return PyLong_FromLong(unlocked([&] {
        return mvla_compact(ctx, s.n, s.ptr, static_cast<const int32_t*>(kept), static_cast<const int32_t*>(offs),
                            static_cast<int32_t>(total), src[0], src[1], src[2], dst[0], dst[1], dst[2], st);
    }));
    MVLA_CATCH
}

// patch_indicators(ctx, samples, q, k, hidden, attn_out, x_out, stream) -> status
PyObject* py_patch_indicators(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    MVLA_TRY
    if (!arg_count(n, 8)) return nullptr;
    Samples s;
    int64_t rows;
    void *q, *k, *hidden, *attn, *x, *st;
    if (!s.take(a[1]) || !tensor_ptr(a[2], &q) || !tensor_ptr(a[3], &k) || !tensor_ptr(a[4], &hidden) ||
        !tensor_ptr(a[5], &attn) || !tensor_ptr(a[6], &x) || !rows_of(a[2], &rows) || !stream_of(a[7], &st))
        return nullptr;
    mvla_ctx* ctx = ctx_of(a[0]);
    return PyLong_FromLong(unlocked([&] {
        return mvla_patch_indicators(ctx, s.n, s.ptr, q, k, hidden, rows, static_cast<float*>(attn), static_cast<float*>(x), st);
    }));
    MVLA_CATCH
}

// patch_select(ctx, point, samples, flags, attn, x, rand_u, out, stream) -> status
PyObject* py_patch_select(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    MVLA_TRY
    if (!arg_count(n, 9)) return nullptr;
    int64_t point, flags;
    if (!int_of(a[1], &point) || !int_of(a[3], &flags)) return nullptr;
    Samples s;
    void *attn, *x, *u, *st;
    mvla_outputs o;
    constexpr unsigned kWanted = 1u << KEPT | 1u << OFFSETS | 1u << BUDGETS | 1u << PATCH_XHAT | 1u << PATCH_INFO | 1u << PATCH_DIAG;
    if (!s.take(a[2]) || !tensor_ptr(a[4], &attn) || !tensor_ptr(a[5], &x) || !tensor_ptr(a[6], &u) ||
        !outputs_of(a[7], &o, kWanted) || !stream_of(a[8], &st))
        return nullptr;
    mvla_ctx* ctx = ctx_of(a[0]);
    return PyLong_FromLong(unlocked([&] {
        return mvla_patch_select(ctx, static_cast<int32_t>(point), s.n, s.ptr, static_cast<uint32_t>(flags),
                                 static_cast<const float*>(attn), static_cast<const float*>(x), static_cast<const float*>(u),
                                 o.kept_idx, o.out_offsets, o.budgets, o.patch_xhat, o.patch_info, o.patch_diag, st);
    }));
    MVLA_CATCH
}

// ---- calls around the prune point.  Tensors are looked at here for what the library cannot see: their type, device and rows.

bool expect(bool ok, const char* what)
{
    if (!ok) PyErr_SetString(PyExc_AssertionError, what);
    return ok;
}
// The device of a call: every tensor of it lies there.
bool on_device(const at::Tensor& t, const char* name, int64_t device)
{
    if (t.device().index() == device) return true;
    PyErr_Format(PyExc_AssertionError, "%s: not on the context's device", name);
    return false;
}
// Pointer and tensor of an optional argument of a given type; `dims`: how many it must have.
bool typed(PyObject* o, const char* name, at::ScalarType type, int dims, int64_t device, void** p, const at::Tensor** t)
{
    *t = nullptr;
    if (!tensor_ptr(o, p, t)) return false;
    if (!*t) return true;
    if ((*t)->scalar_type() != type || (*t)->dim() != dims) {
        PyErr_Format(PyExc_AssertionError, "%s: wrong type or number of dimensions", name);
        return false;
    }
    return on_device(**t, name, device);
}
// Sequence descriptors: an array of them as it lies in memory.
struct Seqs {
    const mvla_seq* ptr = nullptr;
    int n = 0;
    Py_buffer view;
    bool viewed = false;
    ~Seqs() { if (viewed) PyBuffer_Release(&view); }
    bool take(PyObject* o)
    {
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) return false;
        viewed = true;
        if (!expect(view.len % static_cast<Py_ssize_t>(sizeof(mvla_seq)) == 0, "seqs: not an array of sequence descriptors")) return false;
        ptr = static_cast<const mvla_seq*>(view.buf);
        n = static_cast<int>(view.len / static_cast<Py_ssize_t>(sizeof(mvla_seq)));
        return true;
    }
};
// The stream of a call on `device`: the given one, or the device's current one.
bool stream_on(PyObject* o, int64_t device, void** st)
{
    if (o != Py_None) return stream_of(o, st);
    *st = c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream();
    return true;
}
// Memory for the time that the stream takes to run the call (torch's allocator keeps it apart from what other streams use, and inside
// a graph capture in the graph's pool).
at::Tensor fresh_on(at::IntArrayRef sizes, at::ScalarType type, int64_t device, PyObject* stream, void* st)
{
    const auto index = static_cast<c10::DeviceIndex>(device);
    const auto options = at::TensorOptions().dtype(type).device(at::kCUDA, index);
    if (stream == Py_None) return at::empty(sizes, options);              // (the device's current stream)
    const c10::cuda::CUDAStreamGuard guard(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(st), index));
    return at::empty(sizes, options);
}
at::ScalarType scalar_of(int64_t dtype)
{
    return dtype == MVLA_DTYPE_FP32 ? at::kFloat : dtype == MVLA_DTYPE_BF16 ? at::kBFloat16 : at::kFloat8_e4m3fn;
}
// What a context is, as PruneContext hands it over with every call: (dtype, heads, kv_heads, head_dim, device) from a[1] on.
struct Shape {
    int64_t dtype, heads, kv_heads, dim, device;
    at::ScalarType kept, wide;
    bool take(PyObject* const* a)
    {
        if (!int_of(a[1], &dtype) || !int_of(a[2], &heads) || !int_of(a[3], &kv_heads) || !int_of(a[4], &dim) || !int_of(a[5], &device)) return false;
        kept = scalar_of(dtype);
        wide = dtype == MVLA_DTYPE_FP32 ? at::kFloat : at::kBFloat16;
        return true;
    }
    bool rows_of_keys(const at::Tensor* t) const { return !t || (t->size(1) == kv_heads && t->size(2) == dim); }
};
bool entries(const at::Tensor* t, int64_t n) { return !t || t->size(0) == n; }

// Rows of [heads, head_dim] with a stride of their own: pointer, stride, rows.
bool strided_rows(PyObject* o, const char* name, const Shape& c, int64_t heads, const void** p, int64_t* stride, int64_t* rows)
{
    *p = nullptr;
    *stride = 0;
    if (o == Py_None) return true;
    if (!expect(THPVariable_Check(o), "expected a torch.Tensor or None")) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != c.wide || t.dim() != 3 || t.size(1) != heads || t.size(2) != c.dim ||
        (t.numel() && (t.stride(2) != 1 || (heads > 1 && t.stride(1) != c.dim)))) {
        PyErr_Format(PyExc_AssertionError, "%s: device tensor [rows, heads, head_dim] of the context's row type with contiguous rows", name);
        return false;
    }
    if (!expect(*rows < 0 || *rows == t.size(0), "q, k and v: as many rows of one as of another")) return false;
    *rows = t.size(0);
    *p = t.data_ptr();
    *stride = t.size(0) > 1 ? t.stride(0) : heads * c.dim;
    return on_device(t, name, c.device);
}

// An object that is held until the scope ends, by an exception too (memory for an output may run out).
struct Held {
    PyObject* o;
    explicit Held(PyObject* held) : o(held) { Py_XINCREF(o); }
    ~Held() { Py_XDECREF(o); }
    Held(const Held&) = delete;
    Held& operator=(const Held&) = delete;
    void take(PyObject* fresh)                               // instead of what it holds; a reference of the caller's
    {
        Py_XDECREF(o);
        o = fresh;
    }
};

// qk_norm_rope(ctx, dtype, heads, kv_heads, dim, device, q, k, v, pos, inv_freq, q_weight, k_weight, flags, eps, q_out, k_out, v_out,
//   out_rows, stream) -> (status, q_out, k_out, v_out); an output that is missing beside its input is allocated
PyObject* py_qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    MVLA_TRY
    if (!arg_count(n, 20)) return nullptr;
    Shape c;
    int64_t flags;
    if (!c.take(a) || !int_of(a[13], &flags)) return nullptr;
    mvla_qk_rope r;
    std::memset(&r, 0, sizeof r);
    r.eps = PyFloat_AsDouble(a[14]);
    if (r.eps == -1.0 && PyErr_Occurred()) return nullptr;
    int64_t rows = -1;
    if (!strided_rows(a[6], "q", c, c.heads, &r.q, &r.q_stride, &rows) || !strided_rows(a[7], "k", c, c.kv_heads, &r.k, &r.k_stride, &rows) ||
        !strided_rows(a[8], "v", c, c.kv_heads, &r.v, &r.v_stride, &rows))
        return nullptr;
    if (!expect(rows >= 0, "qk_norm_rope: none of q, k, v is given")) return nullptr;
    void *pos, *freq, *wq, *wk, *qo, *ko, *vo, *to, *st;
    const at::Tensor *tp, *tf, *twq, *twk, *tqo, *tko, *tvo, *tto;
    if (!typed(a[9], "pos", at::kInt, 1, c.device, &pos, &tp) || !typed(a[10], "inv_freq", at::kDouble, 1, c.device, &freq, &tf) ||
        !typed(a[11], "q_weight", c.wide, 1, c.device, &wq, &twq) || !typed(a[12], "k_weight", c.wide, 1, c.device, &wk, &twk) ||
        !typed(a[15], "q_out", c.kept, 3, c.device, &qo, &tqo) || !typed(a[16], "k_out", c.kept, 3, c.device, &ko, &tko) ||
        !typed(a[17], "v_out", c.kept, 3, c.device, &vo, &tvo) || !typed(a[18], "out_rows", at::kInt, 1, c.device, &to, &tto) ||
        !stream_on(a[19], c.device, &st))
        return nullptr;
    if (!expect(entries(tp, rows) && entries(tto, rows), "pos, out_rows: one entry per row") ||
        !expect(entries(twq, c.dim) && entries(twk, c.dim), "weights: one entry per element of a head") ||
        !expect(!tqo || (tqo->size(0) == rows && tqo->size(1) == c.heads && tqo->size(2) == c.dim), "q_out: [rows, heads, head_dim]") ||
        !expect(c.rows_of_keys(tko) && c.rows_of_keys(tvo), "k_out, v_out: [rows, heads, head_dim]") ||
        !expect(!tko || !tvo || tko->size(0) == tvo->size(0), "k_out, v_out: as many rows of one as of the other") ||
        !expect(!tf || tf->size(0) <= c.dim, "inv_freq: one entry per pair of a head"))
        return nullptr;
    if (!expect(!tto || ((a[7] == Py_None || tko) && (a[8] == Py_None || tvo)), "out_rows: rows of a k_out / v_out that is given")) return nullptr;
    r.n_rows = rows;
    r.q_weight = wq; r.k_weight = wk;
    r.pos = static_cast<const int32_t*>(pos);
    r.inv_freq = static_cast<const double*>(freq);
    r.rot_dim = tf ? static_cast<int32_t>(2 * tf->size(0)) : 0;
    r.flags = static_cast<uint32_t>(flags);
    r.out_rows = static_cast<const int32_t*>(to);
    Held outs[3] = {Held(a[15]), Held(a[16]), Held(a[17])};
    const at::Tensor* const given[3] = {tqo, tko, tvo};
    void* ptr[3] = {qo, ko, vo};
    int64_t kv_rows = tko ? tko->size(0) : tvo ? tvo->size(0) : rows;
    for (int i = 0; i < 3; ++i) {
        if (given[i] || a[6 + i] == Py_None) continue;
        const at::Tensor t = fresh_on({i ? kv_rows : rows, i ? c.kv_heads : c.heads, c.dim}, c.kept, c.device, a[19], st);
        ptr[i] = t.data_ptr();
        outs[i].take(THPVariable_Wrap(t));
        if (!outs[i].o) return nullptr;
    }
    r.q_out = ptr[0]; r.k_out = ptr[1]; r.v_out = ptr[2];
    r.kv_rows = kv_rows;
    mvla_ctx* ctx = ctx_of(a[0]);
    const int32_t rc = unlocked([&] { return mvla_qk_norm_rope(ctx, &r, st); });
    return Py_BuildValue("(iOOO)", rc, outs[0].o, outs[1].o, outs[2].o);
    MVLA_CATCH
}

// window_attention(ctx, dtype, heads, kv_heads, dim, device, seqs, q, k, v, window, sinks, scale, q_pos, kv_pos, kv_len, out, lse, mass,
//   stream) -> (status, out); a missing `out` is allocated
PyObject* py_window_attention(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    MVLA_TRY
    if (!arg_count(n, 20)) return nullptr;
    Shape c;
    int64_t window, sinks;
    if (!c.take(a) || !int_of(a[10], &window) || !int_of(a[11], &sinks)) return nullptr;
    mvla_attention r;
    std::memset(&r, 0, sizeof r);
    r.scale = PyFloat_AsDouble(a[12]);
    if (r.scale == -1.0 && PyErr_Occurred()) return nullptr;
    Seqs s;
    void *q, *k, *v, *qp, *kp, *kl, *out, *lse, *mass, *st;
    const at::Tensor *tq, *tk, *tv, *tqp, *tkp, *tkl, *to, *tl, *tm;
    if (!s.take(a[6]) || !typed(a[7], "q", c.kept, 3, c.device, &q, &tq) || !typed(a[8], "k", c.kept, 3, c.device, &k, &tk) ||
        !typed(a[9], "v", c.kept, 3, c.device, &v, &tv) || !typed(a[13], "q_pos", at::kInt, 1, c.device, &qp, &tqp) ||
        !typed(a[14], "kv_pos", at::kInt, 1, c.device, &kp, &tkp) || !typed(a[15], "kv_len", at::kInt, 1, c.device, &kl, &tkl) ||
        !typed(a[16], "out", c.wide, 3, c.device, &out, &to) || !typed(a[17], "lse", at::kFloat, 2, c.device, &lse, &tl) ||
        !typed(a[18], "mass", at::kFloat, 1, c.device, &mass, &tm) || !stream_on(a[19], c.device, &st))
        return nullptr;
    if (!expect(tq && tk && tv, "q, k and v are needed")) return nullptr;
    const int64_t rows = tq->size(0), kv_rows = tk->size(0);
    if (!expect(tq->size(1) == c.heads && tq->size(2) == c.dim, "q: [rows, heads, head_dim]") ||
        !expect(c.rows_of_keys(tk) && tv->sizes() == tk->sizes(), "k, v: [rows, heads, head_dim], alike") ||
        !expect(entries(tqp, rows) && entries(tkp, kv_rows), "q_pos, kv_pos: one entry per row") ||
        !expect(entries(tkl, s.n), "kv_len: one entry per sequence") || !expect(!to || to->sizes() == tq->sizes(), "out: as q") ||
        !expect(!tl || (tl->size(0) == rows && tl->size(1) == c.heads), "lse: [rows, heads]") || !expect(entries(tm, kv_rows), "mass: one entry per cached row") ||
        !expect(window >= 1 && window <= MVLA_WINDOW_ALL && sinks >= 0 && sinks <= MVLA_WINDOW_ALL, "window, n_sink: out of range"))
        return nullptr;
    r.q = q; r.k = k; r.v = v; r.q_rows = rows; r.kv_rows = kv_rows;
    r.q_pos = static_cast<const int32_t*>(qp);
    r.kv_pos = static_cast<const int32_t*>(kp);
    r.kv_len = static_cast<const int32_t*>(kl);
    r.window = static_cast<int32_t>(window);
    r.n_sink = static_cast<int32_t>(sinks);
    r.lse = static_cast<float*>(lse);
    r.mass = static_cast<float*>(mass);
    mvla_ctx* ctx = ctx_of(a[0]);
    int64_t bytes = 0;
    int32_t rc = mvla_window_attention_workspace(ctx, s.n, s.ptr, &r, &bytes);
    if (rc != MVLA_OK) return Py_BuildValue("(iO)", rc, Py_None);
    at::Tensor ws, fresh;
    if (bytes > 0) ws = fresh_on({bytes}, at::kByte, c.device, a[19], st);
    if (!to) {
        fresh = fresh_on(tq->sizes(), c.wide, c.device, a[19], st);
        out = fresh.data_ptr();
    }
    r.out = out;
    r.workspace = bytes > 0 ? ws.data_ptr() : nullptr;
    r.workspace_bytes = bytes;
    rc = unlocked([&] { return mvla_window_attention(ctx, s.n, s.ptr, &r, st); });
    if (to) return Py_BuildValue("(iO)", rc, a[16]);
    PyObject* o = THPVariable_Wrap(fresh);
    PyObject* ret = o ? Py_BuildValue("(iO)", rc, o) : nullptr;
    Py_XDECREF(o);
    return ret;
    MVLA_CATCH
}

// cache_evict(ctx, dtype, heads, kv_heads, dim, device, seqs, k, v, pos, mass, pos_out, mass_out, kept_idx, kv_len, kv_len_out, sinks,
//   recent, stream) -> status
PyObject* py_cache_evict(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    MVLA_TRY
    if (!arg_count(n, 19)) return nullptr;
    Shape c;
    int64_t sinks, recent;
    if (!c.take(a) || !int_of(a[16], &sinks) || !int_of(a[17], &recent)) return nullptr;
    Seqs s;
    void *k, *v, *pos, *mass, *po, *mo, *idx, *kl, *klo, *st;
    const at::Tensor *tk, *tv, *tp, *tm, *tpo, *tmo, *ti, *tkl, *tklo;
    if (!s.take(a[6]) || !typed(a[7], "k", c.kept, 3, c.device, &k, &tk) || !typed(a[8], "v", c.kept, 3, c.device, &v, &tv) ||
        !typed(a[9], "pos", at::kInt, 1, c.device, &pos, &tp) || !typed(a[10], "mass", at::kFloat, 1, c.device, &mass, &tm) ||
        !typed(a[11], "pos_out", at::kInt, 1, c.device, &po, &tpo) || !typed(a[12], "mass_out", at::kFloat, 1, c.device, &mo, &tmo) ||
        !typed(a[13], "kept_idx", at::kInt, 1, c.device, &idx, &ti) || !typed(a[14], "kv_len", at::kInt, 1, c.device, &kl, &tkl) ||
        !typed(a[15], "kv_len_out", at::kInt, 1, c.device, &klo, &tklo) || !stream_on(a[18], c.device, &st))
        return nullptr;
    if (!expect(tk && tv && tp && tm && tpo && tmo, "k, v, pos and mass are needed")) return nullptr;
    const int64_t rows = tk->size(0);
    if (!expect(c.rows_of_keys(tk) && tv->sizes() == tk->sizes(), "k, v: [rows, heads, head_dim], alike") ||
        !expect(entries(tp, rows) && entries(tm, rows) && entries(tpo, rows) && entries(tmo, rows) && entries(ti, rows),
                "pos, mass, kept_idx: one entry per cached row") ||
        !expect(entries(tkl, s.n) && entries(tklo, s.n), "kv_len: one entry per sequence") ||
        !expect(sinks >= 0 && sinks <= MVLA_WINDOW_ALL && recent >= 0 && recent <= MVLA_WINDOW_ALL, "n_sink, n_recent: out of range"))
        return nullptr;
    mvla_eviction r;
    std::memset(&r, 0, sizeof r);
    r.k = k; r.v = v; r.kv_rows = rows;
    r.pos = static_cast<const int32_t*>(pos);
    r.mass = static_cast<const float*>(mass);
    r.pos_out = static_cast<int32_t*>(po);
    r.mass_out = static_cast<float*>(mo);
    r.kept_idx = static_cast<int32_t*>(idx);
    r.kv_len = static_cast<const int32_t*>(kl);
    r.kv_len_out = static_cast<int32_t*>(klo);
    r.n_sink = static_cast<int32_t>(sinks);
    r.n_recent = static_cast<int32_t>(recent);
    mvla_ctx* ctx = ctx_of(a[0]);
    int64_t bytes = 0;
    const int32_t rc = mvla_cache_evict_workspace(ctx, s.n, s.ptr, &r, &bytes);
    if (rc != MVLA_OK) return PyLong_FromLong(rc);
    const at::Tensor ws = fresh_on({bytes}, at::kByte, c.device, a[18], st);
    r.workspace = ws.data_ptr();
    r.workspace_bytes = bytes;
    return PyLong_FromLong(unlocked([&] { return mvla_cache_evict(ctx, s.n, s.ptr, &r, st); }));
    MVLA_CATCH
}

// A pool of pages as its four tensors (PagePool): keys, values, their scales.  The type of the elements says which kind it is.
struct Pool {
    mvla_pages p;
    bool take(PyObject* const* a, const Shape& c)
    {
        std::memset(&p, 0, sizeof p);
        const at::Tensor* t[4] = {};
        void* ptr[4] = {};
        for (int i = 0; i < 4; ++i)
            if (!tensor_ptr(a[i], &ptr[i], &t[i]) || (t[i] && !on_device(*t[i], "pool", c.device))) return false;
        if (!expect(t[0] && t[1], "pool: k and v are needed")) return false;
        const at::ScalarType type = t[0]->scalar_type();
        p.kind = type == at::kByte ? MVLA_PAGE_E2M1 : type == at::kFloat8_e4m3fn ? MVLA_PAGE_E4M3 : MVLA_PAGE_ROWS;
        if (!expect(p.kind != MVLA_PAGE_ROWS || type == c.wide, "pool: elements of the context's row type, e4m3, or bytes of two e2m1") ||
            !expect(t[0]->dim() == 4 && t[0]->size(1) == c.kv_heads && t[0]->size(3) == (p.kind == MVLA_PAGE_E2M1 ? c.dim / 2 : c.dim) &&
                        t[1]->scalar_type() == type && t[1]->sizes() == t[0]->sizes(),
                    "pool: k, v: [pages, heads, page rows, head_dim] (e2m1: head_dim / 2 bytes), alike") ||
            !expect((p.kind == MVLA_PAGE_ROWS) == !t[2] && !t[2] == !t[3], "pool: scales beside quantised pages, and only there"))
            return false;
        for (int i = 2; i < 4; ++i)
            if (t[i] && !expect(t[i]->scalar_type() == at::kByte && t[i]->dim() == (p.kind == MVLA_PAGE_E4M3 ? 3 : 4) && t[i]->size(0) == t[0]->size(0) &&
                                    t[i]->size(1) == c.kv_heads && t[i]->size(2) == t[0]->size(2) && (p.kind == MVLA_PAGE_E4M3 || t[i]->size(3) == c.dim / 32),
                                "pool: scales: bytes [pages, heads, page rows] (e2m1: and head_dim / 32)"))
                return false;
        if (!expect(t[0]->size(2) <= 0x7FFFFFFF, "pool: page rows out of range")) return false;
        p.k = ptr[0];
        p.v = ptr[1];
        p.k_scale = static_cast<uint8_t*>(ptr[2]);
        p.v_scale = static_cast<uint8_t*>(ptr[3]);
        p.n_pages = t[0]->size(0);
        p.page_rows = static_cast<int32_t>(t[0]->size(2));
        return true;
    }
};
// The table of a call: [sequences, pages].
bool table_of(PyObject* o, const Shape& c, int n, const int32_t** p, int64_t* stride)
{
    void* ptr;
    const at::Tensor* t;
    if (!typed(o, "table", at::kInt, 2, c.device, &ptr, &t) || !expect(t && t->size(0) == n, "table: [sequences, pages]")) return false;
    *p = static_cast<const int32_t*>(ptr);
    *stride = t->size(1);
    return true;
}

// page_rows(ctx, dtype, heads, kv_heads, dim, device, write, seqs, pool k, v, k_scale, v_scale, table, k, v, kv_len, stream) ->
//   (status, k, v); a read that is given neither allocates both
PyObject* py_page_rows(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    MVLA_TRY
    if (!arg_count(n, 17)) return nullptr;
    Shape c;
    int64_t write;
    if (!c.take(a) || !int_of(a[6], &write)) return nullptr;
    Seqs s;
    Pool pool;
    mvla_page_rows r;
    std::memset(&r, 0, sizeof r);
    void *kl, *st;
    const at::Tensor* tkl;
    if (!s.take(a[7]) || !pool.take(a + 8, c) || !table_of(a[12], c, s.n, &r.table, &r.table_stride) || !typed(a[15], "kv_len", at::kInt, 1, c.device, &kl, &tkl) ||
        !stream_on(a[16], c.device, &st) || !expect(entries(tkl, s.n), "kv_len: one entry per sequence"))
        return nullptr;
    r.pages = pool.p;
    r.kv_len = static_cast<const int32_t*>(kl);
    Held rows[2] = {Held(a[13]), Held(a[14])};
    if (a[13] == Py_None && a[14] == Py_None) {
        if (!expect(!write, "k or v is needed")) return nullptr;
        int64_t end = 0;
        for (int i = 0; i < s.n; ++i)
            if (s.ptr[i].n_q >= 0 && s.ptr[i].q_row >= 0 && s.ptr[i].q_row <= 0x7FFFFFFF) end = std::max<int64_t>(end, s.ptr[i].q_row + s.ptr[i].n_q);
        for (Held& h : rows) {
            h.take(THPVariable_Wrap(fresh_on({end, c.kv_heads, c.dim}, c.wide, c.device, a[16], st)));
            if (!h.o) return nullptr;
        }
    }
    const void *k, *v;
    int64_t count = -1;
    if (!strided_rows(rows[0].o, "k", c, c.kv_heads, &k, &r.k_stride, &count) || !strided_rows(rows[1].o, "v", c, c.kv_heads, &v, &r.v_stride, &count)) return nullptr;
    r.k = const_cast<void*>(k);
    r.v = const_cast<void*>(v);
    r.rows = count;
    mvla_ctx* ctx = ctx_of(a[0]);
    const int32_t rc = unlocked([&] { return write ? mvla_page_write(ctx, s.n, s.ptr, &r, st) : mvla_page_read(ctx, s.n, s.ptr, &r, st); });
    return Py_BuildValue("(iOO)", rc, rows[0].o, rows[1].o);
    MVLA_CATCH
}

// page_attention(ctx, dtype, heads, kv_heads, dim, device, seqs, pool k, v, k_scale, v_scale, table, q, window, sinks, scale, kv_len, out, lse,
//   stream) -> (status, out); a missing `out` is allocated
PyObject* py_page_attention(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    MVLA_TRY
    if (!arg_count(n, 20)) return nullptr;
    Shape c;
    int64_t window, sinks;
    if (!c.take(a) || !int_of(a[13], &window) || !int_of(a[14], &sinks)) return nullptr;
    mvla_paged_attention r;
    std::memset(&r, 0, sizeof r);
    r.scale = PyFloat_AsDouble(a[15]);
    if (r.scale == -1.0 && PyErr_Occurred()) return nullptr;
    Seqs s;
    Pool pool;
    void *q, *kl, *out, *lse, *st;
    const at::Tensor *tq, *tkl, *to, *tl;
    if (!s.take(a[6]) || !pool.take(a + 7, c) || !table_of(a[11], c, s.n, &r.table, &r.table_stride) || !typed(a[12], "q", c.wide, 3, c.device, &q, &tq) ||
        !typed(a[16], "kv_len", at::kInt, 1, c.device, &kl, &tkl) || !typed(a[17], "out", c.wide, 3, c.device, &out, &to) ||
        !typed(a[18], "lse", at::kFloat, 2, c.device, &lse, &tl) || !stream_on(a[19], c.device, &st))
        return nullptr;
    if (!expect(tq && tq->size(1) == c.heads && tq->size(2) == c.dim, "q: [rows, heads, head_dim]") || !expect(entries(tkl, s.n), "kv_len: one entry per sequence") ||
        !expect(!to || to->sizes() == tq->sizes(), "out: as q") || !expect(!tl || (tl->size(0) == tq->size(0) && tl->size(1) == c.heads), "lse: [rows, heads]") ||
        !expect(window >= 1 && window <= MVLA_WINDOW_ALL && sinks >= 0 && sinks <= MVLA_WINDOW_ALL, "window, n_sink: out of range"))
        return nullptr;
    r.pages = pool.p;
    r.kv_len = static_cast<const int32_t*>(kl);
    r.q = q;
    r.q_rows = tq->size(0);
    r.window = static_cast<int32_t>(window);
    r.n_sink = static_cast<int32_t>(sinks);
    r.lse = static_cast<float*>(lse);
    mvla_ctx* ctx = ctx_of(a[0]);
    int64_t bytes = 0;
    int32_t rc = mvla_page_attention_workspace(ctx, s.n, s.ptr, &r, &bytes);
    if (rc != MVLA_OK) return Py_BuildValue("(iO)", rc, Py_None);
    at::Tensor ws, fresh;
    if (bytes > 0) ws = fresh_on({bytes}, at::kByte, c.device, a[19], st);
    if (!to) {
        fresh = fresh_on(tq->sizes(), c.wide, c.device, a[19], st);
        out = fresh.data_ptr();
    }
    r.out = out;
    r.workspace = bytes > 0 ? ws.data_ptr() : nullptr;
    r.workspace_bytes = bytes;
    rc = unlocked([&] { return mvla_page_attention(ctx, s.n, s.ptr, &r, st); });
    if (to) return Py_BuildValue("(iO)", rc, a[17]);
    PyObject* o = THPVariable_Wrap(fresh);
    PyObject* ret = o ? Py_BuildValue("(iO)", rc, o) : nullptr;
    Py_XDECREF(o);
    return ret;
    MVLA_CATCH
}

// fill_samples(array, sequence): descriptors from objects with the descriptor's field names, into a ctypes array
PyObject* py_fill_samples(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    MVLA_TRY
    if (!arg_count(n, 2)) return nullptr;
    PyObject* seq = PySequence_Fast(a[1], "samples: expected a sequence");
    if (!seq) return nullptr;
    Py_buffer view;
    bool ok = PyObject_GetBuffer(a[0], &view, PyBUF_WRITABLE) == 0;
    if (ok) {
        const Py_ssize_t len = PySequence_Fast_GET_SIZE(seq);
        if (view.len < len * static_cast<Py_ssize_t>(sizeof(mvla_sample))) {
            PyErr_SetString(PyExc_ValueError, "array too small");
            ok = false;
        }
        for (Py_ssize_t i = 0; ok && i < len; ++i)
            ok = sample_from(PySequence_Fast_GET_ITEM(seq, i), static_cast<mvla_sample*>(view.buf) + i);
        PyBuffer_Release(&view);
    }
    Py_DECREF(seq);
    if (!ok) return nullptr;
    Py_RETURN_NONE;
    MVLA_CATCH
}

#define MVLA_FAST(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fn)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {MVLA_FAST("prune_step", py_prune_step), MVLA_FAST("salience", py_salience),
                          MVLA_FAST("select", py_select), MVLA_FAST("compact", py_compact),
                          MVLA_FAST("patch_indicators", py_patch_indicators), MVLA_FAST("patch_select", py_patch_select),
                          MVLA_FAST("qk_norm_rope", py_qk_norm_rope), MVLA_FAST("window_attention", py_window_attention),
                          MVLA_FAST("cache_evict", py_cache_evict), MVLA_FAST("page_rows", py_page_rows),
                          MVLA_FAST("page_attention", py_page_attention),
                          MVLA_FAST("fill_samples", py_fill_samples), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_native", "Argument marshalling of libmvla_prune.so", -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native()
{
    for (int i = 0; i < N_OUT; ++i) if (!(g_out_names[i] = PyUnicode_InternFromString(kOutNames[i]))) return nullptr;
    for (int i = 0; i < 8; ++i) if (!(g_int_names[i] = PyUnicode_InternFromString(kSampleInts[i]))) return nullptr;
    for (int i = 0; i < 3; ++i) if (!(g_float_names[i] = PyUnicode_InternFromString(kSampleFloats[i]))) return nullptr;
    if (!(g_cuda_stream = PyUnicode_InternFromString("cuda_stream"))) return nullptr;
    return PyModule_Create(&kModule);
}
