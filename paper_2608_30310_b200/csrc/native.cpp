// Fast argument path of the Python binding.  A call's tensors are checked and marshalled here instead of in Python, where the
// checks, the ctypes descriptor and the stream lookup cost some 10 us a call: more than the kernels of a one-request decoding step.
// Whatever this code does not recognise as a correct call (a wrong type or shape, a workspace that has to grow, a tensor whose sizes or
// storage torch does not hand out, which it says with a C++ exception: none may pass a C entry) is answered with None: the caller
// then takes the general path in Python, which raises the errors or makes the allocation.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>
#include <c10/cuda/CUDAStream.h>
#include <string.h>
#include <initializer_list>
#include "gdn_tail_replay.h"

namespace {

using Forward = int32_t (*)(const gdn_desc*, const void*, const void*, const void*, const float*, const float*, const int32_t*,
                            int32_t, void*, float*);
using Decode = int32_t (*)(const gdn_desc*, const void*, const void*, const void*, const float*, const float*, const float*,
                           void*, float*);
Forward g_forward[3] = {};               // gdn_tail_replay, gdn_full_prefill, gdn_tail_replay_static_scratch
Decode g_decode = nullptr;
size_t (*g_workspace_size)(const gdn_desc*) = nullptr;
PyObject *s_by_stream = nullptr, *s_cuda_stream = nullptr, *s_kept = nullptr, *g_workspace_type = nullptr;
int64_t g_device_bytes = 0;              // Workspace.DEVICE

inline const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }
// contiguous, of type dt, on the side given by `cuda`, of shape {s...}
template <typename... S>
inline bool fits(const at::Tensor* t, at::ScalarType dt, bool cuda, S... s)
{
    if (!t || t->scalar_type() != dt || t->is_cuda() != cuda || t->dim() != (int64_t)sizeof...(s) || !t->is_contiguous()) return false;
    const int64_t want[] = {(int64_t)s...};
    for (size_t i = 0; i < sizeof...(s); ++i)
        if (t->size((int64_t)i) != want[i]) return false;
    return true;
}
template <typename... S>
inline bool fits_or_none(PyObject* o, const at::Tensor*& t, at::ScalarType dt, bool cuda, S... s)
{
    t = nullptr;
    if (o == Py_None) return true;
    t = tensor(o);
    return fits(t, dt, cuda, s...);
}
inline void* ptr(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
// the stream argument's handle, or the current stream's
inline bool stream_of(PyObject* o, void*& st)
{
    if (o == Py_None) {
        st = (void*)c10::cuda::getCurrentCUDAStream().stream();
        return true;
    }
    PyObject* h = PyObject_GetAttr(o, s_cuda_stream);
    if (h) st = PyLong_AsVoidPtr(h);
    Py_XDECREF(h);
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}

using Entry = PyObject* (*)(PyObject*, PyObject* const*, Py_ssize_t);
template <Entry F> PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    try {
        return F(self, a, n);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}
// The library's call, with the other Python threads running: it may copy pageable memory, or wait for room in a launch queue that
// only empties when a host callback of another thread's has run.  (The caller's frame holds the arguments.)
template <typename F> PyObject* without_gil(F call)
{
    int32_t rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}
struct Ref {                                 // an owned reference, given back on every way out
    PyObject* o;
    ~Ref() { Py_XDECREF(o); }
};

// Whether a device call, which may be captured, may take the Workspace's buffer: a larger one than such calls need is perhaps the staging of
// calls on host memory, which goes when it is outgrown, until the general path has put it down as kept.
bool kept_when_outgrown(PyObject* workspace, PyObject* key, PyObject* buffer, int64_t bytes)
{
    if (bytes <= g_device_bytes + 256) return true;
    const Ref map{PyObject_GetAttr(workspace, s_kept)};
    return map.o && PyDict_Check(map.o) && PyDict_GetItemWithError(map.o, key) == buffer;
}

// forward(which, q, k, v, g, beta, cu_tail_lens, chunk, out_o, out_state, init_state, workspace, status_word, kernel, stream, raw)
PyObject* forward(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 16) Py_RETURN_NONE;
    const long which = PyLong_AsLong(a[0]), chunk = PyLong_AsLong(a[7]), kernel = PyLong_AsLong(a[13]);
    const int raw = PyObject_IsTrue(a[15]);
    if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    if (which < 0 || which > 2 || chunk != (int32_t)chunk || kernel != (int32_t)kernel) Py_RETURN_NONE;
    const at::Tensor *q = tensor(a[1]), *k = tensor(a[2]), *v = tensor(a[3]), *g = tensor(a[4]), *beta = tensor(a[5]), *cu = tensor(a[6]);
    if (!q || !v || !cu || q->dim() != 3 || v->dim() != 3 || cu->dim() != 1 || cu->size(0) < 1) Py_RETURN_NONE;
    const at::ScalarType dt = q->scalar_type();
    const bool cuda = q->is_cuda();
    const int64_t T = q->size(0), Hq = q->size(1), dk = q->size(2), Hv = v->size(1), dv = v->size(2), N = cu->size(0) - 1;
    if ((dt != at::kBFloat16 && dt != at::kFloat) || N > 0x7fffffff || Hq > 0x7fffffff || Hv > 0x7fffffff || dk > 0x7fffffff || dv > 0x7fffffff)
        Py_RETURN_NONE;
    const at::Tensor *o, *st, *init, *status;
    if (!fits(q, dt, cuda, T, Hq, dk) || !fits(k, dt, cuda, T, Hq, dk) || !fits(v, dt, cuda, T, Hv, dv) ||
        !fits(g, at::kFloat, cuda, T, Hv) || !fits(beta, at::kFloat, cuda, T, Hv) || !fits(cu, at::kInt, cuda, N + 1) ||
        !fits_or_none(a[8], o, dt, cuda, T, Hv, dv) || !fits_or_none(a[9], st, at::kFloat, cuda, N, Hv, dk, dv))
        Py_RETURN_NONE;
    init = status = nullptr;
    if (a[10] != Py_None && (!(init = tensor(a[10])) || init->is_cuda() != cuda || !init->is_contiguous() || init->scalar_type() != at::kFloat ||
                             init->numel() < N * Hv * dk * dv))
        Py_RETURN_NONE;
    if (a[12] != Py_None && (!(status = tensor(a[12])) || !status->is_cuda() || status->nbytes() < 4)) Py_RETURN_NONE;

    gdn_desc d = {};
    d.num_qk_heads = (int32_t)Hq; d.num_v_heads = (int32_t)Hv; d.head_k_dim = (int32_t)dk; d.head_v_dim = (int32_t)dv;
    d.io_dtype = dt == at::kBFloat16 ? GDN_BF16 : GDN_F32;
    d.num_seqs = (int32_t)N; d.total_tokens = T;
    d.memory = cuda ? GDN_MEM_DEVICE : GDN_MEM_HOST;
    d.kernel = (int32_t)kernel;
    d.input_stage = raw ? GDN_INPUT_RAW : GDN_INPUT_READY;
    d.init_state = (const float*)ptr(init);
    if (!stream_of(a[14], d.stream)) Py_RETURN_NONE;
    Ref b{nullptr};
    if (which != 2) {
        // the Workspace's buffer for this stream as it is; making or growing it is the general path's
        if ((PyObject*)Py_TYPE(a[11]) != g_workspace_type) Py_RETURN_NONE;
        const Ref map{PyObject_GetAttr(a[11], s_by_stream)}, key{PyLong_FromVoidPtr(d.stream)};
        if (map.o && key.o && PyDict_Check(map.o)) b.o = PyDict_GetItemWithError(map.o, key.o);
        Py_XINCREF(b.o);                                  // (held over the call: another thread may let the Workspace grow)
        const at::Tensor* buf = b.o ? tensor(b.o) : nullptr;
        const int64_t need = (int64_t)g_workspace_size(&d);
        const bool ok = buf && buf->is_cuda() && buf->element_size() == 1 && buf->numel() >= need && (!cuda || kept_when_outgrown(a[11], key.o, b.o, buf->numel()));
        if (ok) {
            const uintptr_t base = (uintptr_t)buf->data_ptr(), off = (256 - base % 256) % 256;
            d.workspace = (void*)(base + off);
            d.workspace_bytes = (size_t)buf->numel() - off;
        }
        PyErr_Clear();
        if (!ok) Py_RETURN_NONE;
    }
    d.status_word = (int32_t*)ptr(status);
    const void *pq = q->data_ptr(), *pk = k->data_ptr(), *pv = v->data_ptr(), *pg = g->data_ptr(), *pb = beta->data_ptr(), *pc = cu->data_ptr();
    void *po = ptr(o), *ps = ptr(st);
    return without_gil([&]() { return g_forward[which](&d, pq, pk, pv, (const float*)pg, (const float*)pb, (const int32_t*)pc, (int32_t)chunk, po, (float*)ps); });
}

// decode(q, k, v, g, beta, state_in, out_o, state_out, stream)
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 9) Py_RETURN_NONE;
    const at::Tensor *q = tensor(a[0]), *v = tensor(a[2]), *o;
    if (!q || !v || q->dim() != 3 || v->dim() != 3) Py_RETURN_NONE;
    const at::ScalarType dt = q->scalar_type();
    const int64_t N = q->size(0), Hq = q->size(1), dk = q->size(2), Hv = v->size(1), dv = v->size(2);
    if ((dt != at::kBFloat16 && dt != at::kFloat) || N > 0x7fffffff || Hq > 0x7fffffff || Hv > 0x7fffffff || dk > 0x7fffffff || dv > 0x7fffffff)
        Py_RETURN_NONE;
    const at::Tensor *k = tensor(a[1]), *g = tensor(a[3]), *beta = tensor(a[4]), *in = tensor(a[5]), *out = tensor(a[7]);
    if (!fits(q, dt, true, N, Hq, dk) || !fits(k, dt, true, N, Hq, dk) || !fits(v, dt, true, N, Hv, dv) || !fits(g, at::kFloat, true, N, Hv) ||
        !fits(beta, at::kFloat, true, N, Hv) || !fits(in, at::kFloat, true, N, Hv, dk, dv) || !fits(out, at::kFloat, true, N, Hv, dk, dv) ||
        !fits_or_none(a[6], o, dt, true, N, Hv, dv))
        Py_RETURN_NONE;
    gdn_desc d = {};
    d.num_qk_heads = (int32_t)Hq; d.num_v_heads = (int32_t)Hv; d.head_k_dim = (int32_t)dk; d.head_v_dim = (int32_t)dv;
    d.io_dtype = dt == at::kBFloat16 ? GDN_BF16 : GDN_F32;
    d.num_seqs = (int32_t)N; d.total_tokens = N;
    d.memory = GDN_MEM_DEVICE; d.kernel = GDN_KERNEL_AUTO;
    if (!stream_of(a[8], d.stream)) Py_RETURN_NONE;
    const void *pq = q->data_ptr(), *pk = k->data_ptr(), *pv = v->data_ptr(), *pg = g->data_ptr(), *pb = beta->data_ptr(), *pi = in->data_ptr();
    void *po = ptr(o), *ps = out->data_ptr();
    return without_gil([&]() { return g_decode(&d, pq, pk, pv, (const float*)pg, (const float*)pb, (const float*)pi, po, (float*)ps); });
}

// bind(gdn_tail_replay, gdn_full_prefill, gdn_tail_replay_static_scratch, gdn_decode_step, gdn_workspace_size, Workspace): the addresses of
// the library's functions, and the class whose buffers are looked up here
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 6) { PyErr_SetString(PyExc_TypeError, "five addresses and a class"); return nullptr; }
    void* p[5];
    for (int i = 0; i < 5; ++i) p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    for (int i = 0; i < 3; ++i) g_forward[i] = (Forward)p[i];
    g_decode = (Decode)p[3];
    g_workspace_size = (size_t (*)(const gdn_desc*))p[4];
    const Ref bytes{PyObject_GetAttrString(a[5], "DEVICE")};
    g_device_bytes = bytes.o ? PyLong_AsLongLong(bytes.o) : 0;
    if (PyErr_Occurred()) return nullptr;
    Py_INCREF(a[5]);
    Py_XSETREF(g_workspace_type, a[5]);
    Py_RETURN_NONE;
}

// ---- recurrent layers and cache pages: all device tensors, on the current device

struct Library {
    int32_t (*conv)(const gdn_conv_desc*, const void*, const void*, const void*, const int32_t*, const void*, void*, void*);
    int32_t (*conv_step)(const gdn_conv_desc*, const void*, const void*, const void*, const void*, void*, void*);
    int32_t (*scan)(const gdn_scan_desc*, const void*, const void*, const float*, const void*, const void*, const float*, const void*, const float*,
                    const int32_t*, const float*, void*, float*);
    int32_t (*scan_step)(const gdn_scan_desc*, const void*, const void*, const float*, const void*, const void*, const float*, const void*, const float*,
                         const float*, void*, float*);
    int32_t (*copy)(const gdn_cache_desc*, const int32_t*, const int32_t*, int32_t);
    int32_t (*fork)(const gdn_cache_desc*, int32_t*, int32_t*, const int32_t*, const int32_t*, const int32_t*, int32_t);
    int32_t (*free)(const gdn_cache_desc*, int32_t*, int32_t*, const int32_t*, int32_t);
    int32_t (*compact)(const gdn_cache_desc*, const int32_t*, const int32_t*, int32_t*, int32_t*, int32_t*, int32_t*);
    size_t (*workspace_size)(const gdn_cache_desc*, int32_t);
};
Library g_lib = {};

constexpr int64_t kMost = 0x7fffffff;

// A tensor of this call: on the device, of the type and shape.  `any` sizes are taken as they are.
constexpr int64_t kAny = -1;
struct Args {
    c10::DeviceIndex device = c10::cuda::current_device();
    bool ok = true;

    const at::Tensor* take(PyObject* o, at::ScalarType dt, bool optional, std::initializer_list<int64_t> shape)
    {
        if (optional && o == Py_None) return nullptr;
        const at::Tensor* t = tensor(o);
        ok = ok && t && t->is_cuda() && t->device().index() == device && t->scalar_type() == dt && t->dim() == (int64_t)shape.size();
        for (size_t i = 0; ok && i < shape.size(); ++i) {
            const int64_t want = shape.begin()[i], got = t->size((int64_t)i);
            ok = got <= kMost && (want == kAny || want == got);
        }
        return ok ? t : nullptr;
    }
    const at::Tensor* packed(PyObject* o, at::ScalarType dt, std::initializer_list<int64_t> shape, bool optional = false)
    {
        const at::Tensor* t = take(o, dt, optional, shape);
        ok = ok && (!t || t->is_contiguous());
        return ok ? t : nullptr;
    }
    // rows of packed values, `stride` apart
    const at::Tensor* rows(PyObject* o, at::ScalarType dt, std::initializer_list<int64_t> shape, int64_t& stride, bool optional = false)
    {
        const at::Tensor* t = take(o, dt, optional, shape);
        stride = 0;
        if (!ok || !t) return nullptr;
        int64_t values = 1;
        for (int64_t i = t->dim() - 1; i > 0; --i) {
            ok = ok && (t->size(i) == 1 || t->stride(i) == values);
            values *= t->size(i);
        }
        stride = t->size(0) > 1 ? t->stride(0) : values;
        ok = ok && stride >= values;
        return ok ? t : nullptr;
    }
    int32_t* status(PyObject* o)
    {
        if (o == Py_None) return nullptr;
        const at::Tensor* t = tensor(o);
        ok = ok && t && t->is_cuda() && t->device().index() == device && t->nbytes() >= 4;
        return ok ? (int32_t*)t->data_ptr() : nullptr;
    }
    // the Workspace's buffer for the stream, if it is large enough (held by `b` over the call)
    bool workspace(PyObject* o, void* stream, size_t need, Ref& b, void*& base, size_t& bytes)
    {
        if ((PyObject*)Py_TYPE(o) != g_workspace_type) return false;
        const Ref map{PyObject_GetAttr(o, s_by_stream)}, key{PyLong_FromVoidPtr(stream)};
        if (map.o && key.o && PyDict_Check(map.o)) b.o = PyDict_GetItemWithError(map.o, key.o);
        Py_XINCREF(b.o);
        PyErr_Clear();
        const at::Tensor* buf = b.o ? tensor(b.o) : nullptr;
        if (!buf || !buf->is_cuda() || buf->device().index() != device || buf->element_size() != 1) return false;
        const uintptr_t at = (uintptr_t)buf->data_ptr(), off = (256 - at % 256) % 256;
        const bool kept = kept_when_outgrown(o, key.o, b.o, buf->numel());
        PyErr_Clear();
        if (!kept || (size_t)buf->numel() < need + off) return false;
        base = (void*)(at + off);
        bytes = (size_t)buf->numel() - off;
        return true;
    }
};

bool io_type(const at::Tensor* x, at::ScalarType& dt, int32_t& io)
{
    if (!x) return false;
    dt = x->scalar_type();
    io = dt == at::kBFloat16 ? GDN_BF16 : GDN_F32;
    return dt == at::kBFloat16 || dt == at::kFloat;
}

// conv(step, x, weight, bias, cu_tail_lens, init_state, out, out_state, silu, init_slots, out_slots, status_word, stream)
PyObject* conv(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 13 || !g_lib.conv) Py_RETURN_NONE;
    const bool step = a[0] == Py_True;
    const at::Tensor *x = tensor(a[1]), *w = tensor(a[2]);
    at::ScalarType dt;
    gdn_conv_desc d = {};
    if (!io_type(x, dt, d.io_dtype) || !w || x->dim() != 2 || w->dim() != 2 || (a[8] != Py_True && a[8] != Py_False)) Py_RETURN_NONE;
    const int64_t T = x->size(0), C = x->size(1), K = w->size(1);
    Args g;
    g.rows(a[1], dt, {kAny, kAny}, d.x_stride);
    g.packed(a[2], dt, {C, kAny});
    const at::Tensor* bias = g.packed(a[3], dt, {C}, true);
    const at::Tensor* cu = step ? nullptr : g.packed(a[4], at::kInt, {kAny});
    const at::Tensor* in = g.packed(a[5], dt, {kAny, K - 1, C}, !step);
    const at::Tensor* out = g.rows(a[6], dt, {T, C}, d.out_stride);
    const at::Tensor* keep = g.packed(a[7], dt, {kAny, K - 1, C}, !step);
    if (!g.ok || C < 1 || K < 2 || (cu && cu->size(0) < 1)) Py_RETURN_NONE;
    const int64_t N = step ? T : cu->size(0) - 1;
    const at::Tensor *is = g.packed(a[9], at::kInt, {N}, true), *os = g.packed(a[10], at::kInt, {N}, true);
    d.status_word = g.status(a[11]);
    if (!g.ok || !stream_of(a[12], d.stream)) Py_RETURN_NONE;
    d.channels = (int32_t)C; d.width = (int32_t)K; d.num_seqs = (int32_t)N; d.total_tokens = T; d.silu = a[8] == Py_True;
    d.num_init_states = in ? (int32_t)in->size(0) : 0; d.num_out_states = keep ? (int32_t)keep->size(0) : 0;
    d.init_slots = (const int32_t*)ptr(is); d.out_slots = (const int32_t*)ptr(os);
    const void *px = ptr(x), *pw = ptr(w), *pb = ptr(bias), *pi = ptr(in);
    const int32_t* pc = (const int32_t*)ptr(cu);
    void *po = ptr(out), *pk = ptr(keep);
    return without_gil([&]() { return step ? g_lib.conv_step(&d, px, pw, pb, pi, po, pk) : g_lib.conv(&d, px, pw, pb, pc, pi, po, pk); });
}

// scan(step, x, dt, a, b, c, d, z, dt_bias, cu_tail_lens, init_state, out, out_state, softplus, init_slots, out_slots, status_word, stream)
PyObject* scan(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 18 || !g_lib.scan) Py_RETURN_NONE;
    const bool step = a[0] == Py_True;
    const at::Tensor *x = tensor(a[1]), *ta = tensor(a[3]), *b = tensor(a[4]);
    at::ScalarType dt;
    gdn_scan_desc d = {};
    if (!io_type(x, dt, d.io_dtype) || !ta || !b || x->dim() != 2 || ta->dim() != 2 || b->dim() != 3 || (a[13] != Py_True && a[13] != Py_False))
        Py_RETURN_NONE;
    const int64_t T = x->size(0), C = x->size(1), S = ta->size(1), G = b->size(1);
    Args g;
    g.rows(a[1], dt, {kAny, kAny}, d.x_stride);
    const at::Tensor* tdt = g.rows(a[2], dt, {T, C}, d.dt_stride);
    g.packed(a[3], at::kFloat, {C, kAny});
    g.rows(a[4], dt, {T, kAny, S}, d.b_stride);
    const at::Tensor* c = g.rows(a[5], dt, {T, G, S}, d.c_stride);
    const at::Tensor *skip = g.packed(a[6], at::kFloat, {C}, true), *z = g.rows(a[7], dt, {T, C}, d.z_stride, true), *bias = g.packed(a[8], at::kFloat, {C}, true);
    const at::Tensor* cu = step ? nullptr : g.packed(a[9], at::kInt, {kAny});
    const at::Tensor* in = g.packed(a[10], at::kFloat, {kAny, C, S}, !step);
    const at::Tensor* out = g.rows(a[11], dt, {T, C}, d.out_stride);
    const at::Tensor* keep = g.packed(a[12], at::kFloat, {kAny, C, S}, !step);
    if (!g.ok || C < 1 || (cu && cu->size(0) < 1)) Py_RETURN_NONE;
    const int64_t N = step ? T : cu->size(0) - 1;
    const at::Tensor *is = g.packed(a[14], at::kInt, {N}, true), *os = g.packed(a[15], at::kInt, {N}, true);
    d.status_word = g.status(a[16]);
    if (!g.ok || !stream_of(a[17], d.stream)) Py_RETURN_NONE;
    d.channels = (int32_t)C; d.states = (int32_t)S; d.groups = (int32_t)G; d.num_seqs = (int32_t)N; d.total_tokens = T; d.softplus = a[13] == Py_True;
    d.num_init_states = in ? (int32_t)in->size(0) : 0; d.num_out_states = keep ? (int32_t)keep->size(0) : 0;
    d.init_slots = (const int32_t*)ptr(is); d.out_slots = (const int32_t*)ptr(os);
    const void *px = ptr(x), *pd = ptr(tdt), *pb = ptr(b), *pc = ptr(c), *pz = ptr(z);
    const float *pa = (const float*)ptr(ta), *ps = (const float*)ptr(skip), *pt = (const float*)ptr(bias), *pi = (const float*)ptr(in);
    const int32_t* pcu = (const int32_t*)ptr(cu);
    void* po = ptr(out);
    float* pk = (float*)ptr(keep);
    return without_gil([&]() {
        return step ? g_lib.scan_step(&d, px, pd, pa, pb, pc, ps, pz, pt, pi, po, pk) : g_lib.scan(&d, px, pd, pa, pb, pc, ps, pz, pt, pcu, pi, po, pk);
    });
}

constexpr Py_ssize_t kPools = 256;           // more go through the general path
// A list or tuple of pools [pages, ...], packed and with the same number of pages.
bool pools_of(PyObject* o, Args& g, gdn_pool* pools, gdn_cache_desc& d)
{
    const bool list = PyList_Check(o);
    if (!list && !PyTuple_Check(o)) return false;
    const Py_ssize_t n = list ? PyList_GET_SIZE(o) : PyTuple_GET_SIZE(o);
    if (n < 1 || n > kPools) return false;
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::Tensor* t = tensor(list ? PyList_GET_ITEM(o, i) : PyTuple_GET_ITEM(o, i));
        if (!t || !t->is_cuda() || t->device().index() != g.device || t->dim() < 2 || !t->is_contiguous() || t->size(0) < 1 || t->size(0) > kMost) return false;
        if (i == 0) d.num_pages = (int32_t)t->size(0);
        if (t->size(0) != d.num_pages) return false;
        pools[i].base = t->data_ptr();
        pools[i].page_bytes = (int64_t)(t->nbytes() / (size_t)t->size(0));
    }
    d.pools = pools;
    d.num_pools = (int32_t)n;
    return true;
}

// cache_copy(pools, src, dst, status_word, stream)
PyObject* cache_copy(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 5 || !g_lib.copy) Py_RETURN_NONE;
    Args g;
    gdn_pool pools[kPools];
    gdn_cache_desc d = {};
    if (!pools_of(a[0], g, pools, d)) Py_RETURN_NONE;
    const at::Tensor* src = g.packed(a[1], at::kInt, {kAny});
    if (!g.ok) Py_RETURN_NONE;
    const at::Tensor* dst = g.packed(a[2], at::kInt, {src->size(0)});
    d.status_word = g.status(a[3]);
    if (!g.ok || !stream_of(a[4], d.stream)) Py_RETURN_NONE;
    const int32_t *ps = (const int32_t*)ptr(src), *pd = (const int32_t*)ptr(dst), count = (int32_t)src->size(0);
    return without_gil([&]() { return g_lib.copy(&d, ps, pd, count); });
}

// cache_fork(pools, page_tokens, refcounts, tables, parents, children, tokens, workspace, status_word, stream)
PyObject* cache_fork(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 10 || !g_lib.fork) Py_RETURN_NONE;
    Args g;
    gdn_pool pools[kPools];
    gdn_cache_desc d = {};
    const long tokens = PyLong_AsLong(a[1]);
    if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    if (tokens < 1 || tokens > kMost || !pools_of(a[0], g, pools, d)) Py_RETURN_NONE;
    const at::Tensor* counts = g.packed(a[2], at::kInt, {(int64_t)d.num_pages});
    const at::Tensor* tables = g.packed(a[3], at::kInt, {kAny, kAny});
    const at::Tensor* parents = g.packed(a[4], at::kInt, {kAny});
    if (!g.ok) Py_RETURN_NONE;
    const int64_t count = parents->size(0);
    const at::Tensor *children = g.packed(a[5], at::kInt, {count}), *upto = g.packed(a[6], at::kInt, {count});
    d.status_word = g.status(a[8]);
    if (!g.ok || !stream_of(a[9], d.stream)) Py_RETURN_NONE;
    d.page_tokens = (int32_t)tokens; d.num_rows = (int32_t)tables->size(0); d.row_pages = (int32_t)tables->size(1);
    Ref held{nullptr};
    if (!g.workspace(a[7], d.stream, g_lib.workspace_size(&d, (int32_t)count), held, d.workspace, d.workspace_bytes)) Py_RETURN_NONE;
    int32_t *pc = (int32_t*)ptr(counts), *pt = (int32_t*)ptr(tables);
    const int32_t *pp = (const int32_t*)ptr(parents), *pk = (const int32_t*)ptr(children), *pn = (const int32_t*)ptr(upto);
    return without_gil([&]() { return g_lib.fork(&d, pc, pt, pp, pk, pn, (int32_t)count); });
}

// cache_free(refcounts, tables, rows, status_word, stream)
PyObject* cache_free(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 5 || !g_lib.free) Py_RETURN_NONE;
    Args g;
    gdn_cache_desc d = {};
    const at::Tensor *counts = g.packed(a[0], at::kInt, {kAny}), *tables = g.packed(a[1], at::kInt, {kAny, kAny}), *rows = g.packed(a[2], at::kInt, {kAny});
    d.status_word = g.status(a[3]);
    if (!g.ok || !stream_of(a[4], d.stream)) Py_RETURN_NONE;
    d.num_pages = (int32_t)counts->size(0); d.num_rows = (int32_t)tables->size(0); d.row_pages = (int32_t)tables->size(1);
    int32_t *pc = (int32_t*)ptr(counts), *pt = (int32_t*)ptr(tables);
    const int32_t *pr = (const int32_t*)ptr(rows), count = (int32_t)rows->size(0);
    return without_gil([&]() { return g_lib.free(&d, pc, pt, pr, count); });
}

// cache_compact(pools, refcounts, tables, out_refcounts, out_tables, page_map, live, workspace, status_word, stream)
PyObject* cache_compact(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 10 || !g_lib.compact) Py_RETURN_NONE;
    Args g;
    gdn_pool pools[kPools];
    gdn_cache_desc d = {};
    if (!pools_of(a[0], g, pools, d)) Py_RETURN_NONE;
    const int64_t P = d.num_pages;
    const at::Tensor *counts = g.packed(a[1], at::kInt, {P}), *tables = g.packed(a[2], at::kInt, {kAny, kAny});
    if (!g.ok) Py_RETURN_NONE;
    const at::Tensor *oc = g.packed(a[3], at::kInt, {P}), *ot = g.packed(a[4], at::kInt, {tables->size(0), tables->size(1)}),
                     *map = g.packed(a[5], at::kInt, {P}), *live = g.packed(a[6], at::kInt, {1});
    d.status_word = g.status(a[8]);
    if (!g.ok || !stream_of(a[9], d.stream)) Py_RETURN_NONE;
    d.num_rows = (int32_t)tables->size(0); d.row_pages = (int32_t)tables->size(1);
    Ref held{nullptr};
    if (!g.workspace(a[7], d.stream, g_lib.workspace_size(&d, 0), held, d.workspace, d.workspace_bytes)) Py_RETURN_NONE;
    const int32_t *pc = (const int32_t*)ptr(counts), *pt = (const int32_t*)ptr(tables);
    int32_t *qc = (int32_t*)ptr(oc), *qt = (int32_t*)ptr(ot), *qm = (int32_t*)ptr(map), *ql = (int32_t*)ptr(live);
    return without_gil([&]() { return g_lib.compact(&d, pc, pt, qc, qt, qm, ql); });
}

// bind_layers(the addresses of the functions, in the order of Library's)
PyObject* bind_layers(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    void* p[9];
    if (n != 9) { PyErr_SetString(PyExc_TypeError, "nine addresses"); return nullptr; }
    for (int i = 0; i < 9; ++i) p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    static_assert(sizeof p == sizeof g_lib, "one address each");
    memcpy(&g_lib, p, sizeof p);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"conv", (PyCFunction)(void (*)(void))guarded<conv>, METH_FASTCALL, nullptr},
    {"scan", (PyCFunction)(void (*)(void))guarded<scan>, METH_FASTCALL, nullptr},
    {"cache_copy", (PyCFunction)(void (*)(void))guarded<cache_copy>, METH_FASTCALL, nullptr},
    {"cache_fork", (PyCFunction)(void (*)(void))guarded<cache_fork>, METH_FASTCALL, nullptr},
    {"cache_free", (PyCFunction)(void (*)(void))guarded<cache_free>, METH_FASTCALL, nullptr},
    {"cache_compact", (PyCFunction)(void (*)(void))guarded<cache_compact>, METH_FASTCALL, nullptr},
    {"bind_layers", (PyCFunction)(void (*)(void))bind_layers, METH_FASTCALL, nullptr},
    {"forward", (PyCFunction)(void (*)(void))guarded<forward>, METH_FASTCALL, nullptr},
    {"decode", (PyCFunction)(void (*)(void))guarded<decode>, METH_FASTCALL, nullptr},
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__native()
{
    s_by_stream = PyUnicode_InternFromString("by_stream");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    s_kept = PyUnicode_InternFromString("kept");
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for_torch", BUILT_FOR_TORCH) < 0) { Py_DECREF(m); return nullptr; }
    return m;
}
