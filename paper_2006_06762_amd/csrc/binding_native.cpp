// The operators of binding.py for the calls that programs make over and over: plain GPU tensors, a descriptor within
// its fields' ranges.  Anything else (and every error) goes to the Python function of the same
// name, so what is accepted, refused and raised is decided there.
//
// Marshalling in Python took 1.6 to 2.2 us of a call, more than the launch: back to back on the GPU 128 x 128 x 128 ran every 4.6
// us where the launches alone allow 2.8, a depthwise 97 x 8 x 8 every 4.8 of 2.5.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <cstring>
#include <string>
#include <unordered_map>

#include "anr.h"

namespace {

// ---- what binding.py hands over (setup): its functions, the library's entry points
enum Op { GEMM, CONV2D, CONV_BN_RELU, CONV2D_PACKED, CONV_BN_RELU_PACKED, DWCONV, TBG, TBS, NRM, GROUP_NORM, GROUP_NORM_BACKWARD, ROTARY, GATED_FF, GATED_FF_BACKWARD, RMS_NORM, RMS_NORM_BACKWARD, RMS_NORM_Q8,
          QUANTIZE_ROWS, DEQUANTIZE_ROWS, GEMM_I8, OPS };
PyObject* g_python[OPS];
using Call3 = anr_status (*)(const void*, const void*, const void*, void*, void*, size_t, void*);
using CallBn = anr_status (*)(const void*, const void*, const void*, const void*, const void*, const void*, const void*, float, void*, void*, size_t, void*);
using CallNrm = anr_status (*)(const void*, const void*, void*, void*, size_t, void*);
using CallNorm = anr_status (*)(const void*, const void*, const void*, const void*, float, void*, void*, void*, void*, size_t, void*);
using CallNormBackward = anr_status (*)(const void*, const void*, const void*, const void*, const void*, const void*, const void*, void*, void*, void*, void*, size_t, void*);
using CallRotary = anr_status (*)(const void*, const void*, const void*, const void*, const void*, void*, void*, void*, size_t, void*);
using CallFf = anr_status (*)(const void*, const void*, const void*, const void*, const void*, void*, void*, void*, void*, size_t, void*);
using CallFfBackward = anr_status (*)(const void*, const void*, const void*, const void*, const void*, const void*, const void*, const void*, void*, void*, void*, void*, void*,
                                      size_t, void*);
using CallRmsNorm = anr_status (*)(const void*, const void*, const void*, const void*, float, void*, void*, void*, void*, size_t, void*);
using CallRmsNormBackward = anr_status (*)(const void*, const void*, const void*, const void*, const void*, const void*, void*, void*, void*, size_t, void*);
using CallQuantize = anr_status (*)(const void*, const void*, const void*, void*, void*, void*, size_t, void*);
using CallGemmI8 = anr_status (*)(const void*, const void*, const void*, const void*, const void*, const void*, void*, void*, size_t, void*);
using CallFastSize = anr_status (*)(const void*, size_t*);
using CallSize = anr_status (*)(int, const void*, size_t*);
void* g_entry[OPS];
CallFastSize g_fast_size;
CallSize g_size;

// A tensor that is memory on a GPU and nothing else: no subclass, no wrapper of a transform.
const at::Tensor* plain_memory(PyObject* o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined()) return nullptr;
    const c10::TensorImpl* impl = t.unsafeGetTensorImpl();
    constexpr c10::DispatchKeySet usual({c10::DispatchKey::CUDA, c10::DispatchKey::AutogradCUDA, c10::DispatchKey::AutocastCUDA, c10::DispatchKey::ADInplaceOrView});
    if ((impl->key_set().raw_repr() & ~usual.raw_repr()) != 0 || impl->has_symbolic_sizes_strides() || !impl->has_storage()) return nullptr;
    return t.is_cuda() ? &t : nullptr;
}
const at::Tensor* plain(PyObject* o, at::ScalarType type = at::kFloat)
{
    const at::Tensor* const t = plain_memory(o);
    return t && t->scalar_type() == type ? t : nullptr;
}

void* data(const at::Tensor* t) { return t->mutable_data_ptr(); }

// Arguments by position and name, as a Python function with these parameters takes them; absent ones stay null.  False
// where that function would complain.
template <int N>
bool arguments(const char* const (&names)[N], int required, PyObject* const* args, Py_ssize_t n, PyObject* kwnames, PyObject* (&out)[N])
{
    if (n > N) return false;
    for (int i = 0; i < N; ++i) out[i] = i < n ? args[i] : nullptr;
    const Py_ssize_t named = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
    for (Py_ssize_t k = 0; k < named; ++k) {
        PyObject* const name = PyTuple_GET_ITEM(kwnames, k);
        int i = 0;
        while (i < N && PyUnicode_CompareWithASCIIString(name, names[i]) != 0) ++i;
        if (i == N || out[i]) return false;
        out[i] = args[n + k];
    }
    for (int i = 0; i < required; ++i)
        if (!out[i]) return false;
    return true;
}

bool int32(PyObject* o, int32_t* out)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    const long v = PyLong_AsLongAndOverflow(o, &overflow);
    *out = (int32_t)v;
    return !overflow && v == *out;
}

bool pair(PyObject* o, int32_t absent, int32_t* a, int32_t* b)
{
    if (!o) {
        *a = *b = absent;
        return true;
    }
    return PyTuple_CheckExact(o) && PyTuple_GET_SIZE(o) == 2 && int32(PyTuple_GET_ITEM(o, 0), a) && int32(PyTuple_GET_ITEM(o, 1), b);
}

bool fits(int64_t v, int32_t* out)
{
    *out = (int32_t)v;
    return v == *out;
}

// Element strides of a four-dimensional tensor, zeros for a packed one.
void strides4(const at::Tensor* t, int64_t* out)
{
    const bool packed = t->is_contiguous();
    for (int i = 0; i < 4; ++i) out[i] = packed ? 0 : t->stride(i);
}

struct Stream {
    c10::DeviceIndex device = c10::hip::current_device();
    hipStream_t stream = c10::hip::getCurrentHIPStream(device).stream();

    bool capturing() const
    {
        hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
        return hipStreamIsCapturing(stream, &status) != hipSuccess || status != hipStreamCaptureStatusNone;
    }
};

// Smaller workspaces of a thread, one for each of the eight streams it used last: asking the allocator takes 0.9 us of a call, which
// shows where the GPU is done before the host (norms 5.9 against 6.9 us; 1 x 32 x 28 x 28 -> 32, 1.7 MB, 7.9 against 8.3; from
// 8 MB on calls take 15 us and more).  Not of all threads together: another one's launches may come between those of a call.
// Given back when the thread ends.
class Kept {
public:
    static constexpr size_t kMost = (size_t)8 << 20;

    void* get(size_t need, const Stream& s)
    {
        Entry* e = entries_;
        while (e != entries_ + kStreams && !(e->ptr && e->device == s.device && e->stream == s.stream)) ++e;
        if (e == entries_ + kStreams) e = &entries_[next_++ % kStreams];
        else if (e->bytes >= need) return e->ptr;
        size_t bytes = (size_t)1 << 16;
        while (bytes < need) bytes *= 2;
        void* const ptr = c10::hip::HIPCachingAllocator::raw_alloc_with_stream(bytes, s.stream);
        if (e->ptr) c10::hip::HIPCachingAllocator::raw_delete(e->ptr);
        *e = {s.device, s.stream, ptr, bytes};
        return ptr;
    }
    ~Kept()
    {
        for (const Entry& e : entries_) try {
                if (e.ptr) c10::hip::HIPCachingAllocator::raw_delete(e.ptr);
            } catch (...) {                       // (at the end of the process)
            }
    }

private:
    static constexpr int kStreams = 8;
    struct Entry {
        c10::DeviceIndex device;
        hipStream_t stream;
        void* ptr;
        size_t bytes;
    };
    Entry entries_[kStreams] = {};
    unsigned next_ = 0;
};
thread_local Kept t_kept;

// Memory for the launches of one call (see _with_workspace in binding.py); none of zero bytes, and not in a capture, where
// Python looks after it.
struct Workspace {
    const bool here;
    const size_t bytes;
    void* const ptr;

    Workspace(size_t need, const Stream& s) : here(need == 0 || !s.capturing()), bytes(need), ptr(need && here ? take(need, s) : nullptr) {}
    ~Workspace()
    {
        if (ptr && bytes > Kept::kMost) c10::hip::HIPCachingAllocator::raw_delete(ptr);
    }
    Workspace(const Workspace&) = delete;
    Workspace& operator=(const Workspace&) = delete;

private:
    static void* take(size_t need, const Stream& s)
    {
        return need > Kept::kMost ? c10::hip::HIPCachingAllocator::raw_alloc_with_stream(need, s.stream) : t_kept.get(need, s);
    }
};

// Other threads run while the library is called, as they do around a ctypes call: a launch may wait for room in its queue.
struct WithoutGil {
    PyThreadState* const state = PyEval_SaveThread();
    ~WithoutGil() { PyEval_RestoreThread(state); }
};

template <typename Call, typename... Args>
bool accepted(Op op, Args... args)
{
    WithoutGil released;
    return reinterpret_cast<Call>(g_entry[op])(args...) == ANR_OK;
}

// anr_conv2d_fast_workspace_size of a descriptor, asked once for each of up to 4096.
size_t fast_size(const anr_conv_desc& d)
{
    static std::unordered_map<std::string, size_t> known;
    std::string key(reinterpret_cast<const char*>(&d), sizeof d);
    const auto at = known.find(key);
    if (at != known.end()) return at->second;
    size_t bytes = 0;
    if (g_fast_size(&d, &bytes) != ANR_OK) bytes = 0;       // (what is refused here is refused by the call itself)
    if (known.size() >= 4096) known.clear();
    known.emplace(std::move(key), bytes);
    return bytes;
}

bool conv_desc(const at::Tensor* x, const at::Tensor* w, const at::Tensor* y, PyObject* stride, PyObject* pad, PyObject* dil, PyObject* groups, PyObject* route,
               anr_conv_desc* d)
{
    if (x->dim() != 4 || w->dim() != 4 || y->dim() != 4 || !w->is_contiguous()) return false;
    std::memset(d, 0, sizeof *d);
    d->groups = 1;
    d->route = ANR_CONV_ROUTE_AUTO;
    d->layout = ANR_LAYOUT_NCHW;
    strides4(x, d->x_stride);
    strides4(y, d->y_stride);
    return fits(x->size(0), &d->N) && fits(x->size(1), &d->C) && fits(x->size(2), &d->H) && fits(x->size(3), &d->W) && fits(w->size(0), &d->K) &&
           fits(w->size(2), &d->R) && fits(w->size(3), &d->S) && pair(stride, 1, &d->stride_h, &d->stride_w) && pair(pad, 0, &d->pad_h, &d->pad_w) &&
           pair(dil, 1, &d->dil_h, &d->dil_w) && (!groups || int32(groups, &d->groups)) && (!route || int32(route, &d->route));
}

// The operators: true with the call made and accepted; false leaves it to Python, with nothing done.
bool run_gemm(PyObject* const* a)
{
    const at::Tensor *A = plain(a[0]), *B = plain(a[1]), *C = plain(a[2]);
    if (!A || !B || !C) return false;
    const int64_t n = A->dim();
    if ((n != 2 && n != 3) || B->dim() != n || C->dim() != n || A->stride(n - 1) != 1 || B->stride(n - 1) != 1 || C->stride(n - 1) != 1) return false;
    anr_gemm_desc d{};
    d.M = A->size(n - 2);
    d.K = A->size(n - 1);
    d.N = B->size(n - 1);
    d.lda = A->stride(n - 2);
    d.ldb = B->stride(n - 2);
    d.ldc = C->stride(n - 2);
    d.batch = n == 3 ? A->size(0) : 1;
    if (n == 3) {
        d.strideA = A->stride(0);
        d.strideB = B->stride(0);
        d.strideC = C->stride(0);
    }
    return accepted<Call3>(GEMM, &d, data(A), data(B), data(C), nullptr, 0, Stream().stream);
}

bool run_conv2d(PyObject* const* a)
{
    const at::Tensor *x = plain(a[0]), *w = plain(a[1]), *y = plain(a[2]);
    anr_conv_desc d;
    if (!x || !w || !y || (a[5] && a[5] != Py_None) || !conv_desc(x, w, y, a[3], a[4], a[6], a[7], a[8], &d)) return false;
    const Stream s;
    const Workspace ws(fast_size(d), s);
    return ws.here && accepted<Call3>(CONV2D, &d, data(x), data(w), data(y), ws.ptr, ws.bytes, s.stream);
}

bool run_conv_bn_relu(PyObject* const* a)
{
    const at::Tensor *x = plain(a[0]), *w = plain(a[1]), *y = plain(a[7]);
    anr_conv_desc d;
    if (!x || !w || !y || !PyFloat_CheckExact(a[6]) || (a[10] && a[10] != Py_None) || !conv_desc(x, w, y, a[8], a[9], a[11], a[12], a[13], &d)) return false;
    void* bn[4];
    for (int i = 0; i < 4; ++i) {
        const at::Tensor* const v = plain(a[2 + i]);
        if (!v || v->dim() != 1 || v->size(0) != d.K || !v->is_contiguous()) return false;
        bn[i] = data(v);
    }
    const Stream s;
    const Workspace ws(fast_size(d), s);
    return ws.here && accepted<CallBn>(CONV_BN_RELU, &d, data(x), data(w), bn[0], bn[1], bn[2], bn[3], (float)PyFloat_AS_DOUBLE(a[6]), data(y), ws.ptr,
                                       ws.bytes, s.stream);
}

bool run_packed(Op op, PyObject* const* a)
{
    const at::Tensor *x = plain(a[1]), *pack = plain(a[2], at::kByte), *y = plain(a[3]);
    if (!x || !pack || !y || (a[4] && a[4] != Py_None) || x->dim() != 4 || y->dim() != 4 || !x->is_contiguous() || !PyObject_CheckBuffer(a[0])) return false;
    Py_buffer view;
    if (PyObject_GetBuffer(a[0], &view, PyBUF_SIMPLE) != 0) {
        PyErr_Clear();
        return false;
    }
    anr_conv_desc d;
    const bool whole = view.len == (Py_ssize_t)sizeof d;
    if (whole) std::memcpy(&d, view.buf, sizeof d);
    PyBuffer_Release(&view);
    if (!whole) return false;
    for (int i = 0; i < 4; ++i) d.x_stride[i] = 0;
    strides4(y, d.y_stride);
    const Stream s;
    const Workspace ws(fast_size(d), s);
    return ws.here && accepted<Call3>(op, &d, data(x), data(pack), data(y), ws.ptr, ws.bytes, s.stream);
}

bool run_dwconv(PyObject* const* a)
{
    const at::Tensor *x = plain(a[0]), *w = plain(a[1]), *y = plain(a[2]);
    anr_conv_desc d;
    if (!x || !w || !y || !conv_desc(x, w, y, a[3], a[4], a[5], nullptr, nullptr, &d)) return false;
    return accepted<Call3>(DWCONV, &d, data(x), data(w), data(y), nullptr, 0, Stream().stream);
}

bool run_scores(Op op, PyObject* const* a)
{
    const at::Tensor *q = plain(a[0]), *k = plain(a[1]), *out = plain(a[2]);
    if (!q || !k || !out || q->dim() != 4 || k->dim() != 4 || out->dim() != 4) return false;
    anr_tbg_desc d{};
    if (!fits(q->size(0), &d.B) || !fits(q->size(1), &d.S) || !fits(q->size(2), &d.H) || !fits(q->size(3), &d.D)) return false;
    strides4(q, d.q_stride);
    strides4(k, d.k_stride);
    strides4(out, d.o_stride);
    return accepted<Call3>(op, &d, data(q), data(k), data(out), nullptr, 0, Stream().stream);
}

bool run_nrm(PyObject* const* a)
{
    const at::Tensor *x = plain(a[0]), *out = plain(a[1]);
    if (!x || !out || (a[2] && a[2] != Py_None)) return false;
    const int64_t n = x->dim();
    if ((n != 2 && n != 3) || x->stride(n - 1) != 1 || !out->is_contiguous()) return false;
    anr_nrm_desc d{};
    d.N = x->size(n - 2);
    d.M = x->size(n - 1);
    d.ld = x->stride(n - 2);
    d.batch = n == 3 ? x->size(0) : 1;
    d.stride = d.batch > 1 ? x->stride(0) : 0;
    if (out->numel() != d.batch) return false;
    size_t need = 0;
    if (g_size(ANR_OP_NRM, &d, &need) != ANR_OK) return false;
    const Stream s;
    const Workspace ws(need, s);
    return ws.here && accepted<CallNrm>(NRM, &d, data(x), data(out), ws.ptr, ws.bytes, s.stream);
}

// ---- operators with an element type

int type_code(at::ScalarType t) { return t == at::kFloat ? ANR_F32 : t == at::kHalf ? ANR_F16 : t == at::kBFloat16 ? ANR_BF16 : -1; }
bool absent(PyObject* o) { return !o || o == Py_None; }

// Tensors of a call, all of them plain ones on the current device; `fine` tells whether each was as it has to be.
struct Tensors {
    const Stream s;
    bool fine = true;

    // a tensor with these sizes
    const at::Tensor* get(PyObject* o, at::ScalarType type, c10::IntArrayRef sizes)
    {
        const at::Tensor* const t = fine ? plain(o, type) : nullptr;
        fine = t && t->device().index() == s.device && t->sizes() == sizes;
        return fine ? t : nullptr;
    }
    const at::Tensor* optional(PyObject* o, at::ScalarType type, c10::IntArrayRef sizes) { return absent(o) ? nullptr : get(o, type, sizes); }
    const at::Tensor* packed(PyObject* o, at::ScalarType type, c10::IntArrayRef sizes)
    {
        const at::Tensor* const t = optional(o, type, sizes);
        if (t && !t->is_contiguous()) fine = false;
        return t;
    }
    // a matrix, and its leading dimension (0: one row at most)
    const at::Tensor* matrix(PyObject* o, at::ScalarType type, int64_t rows, int64_t cols, int64_t* ld)
    {
        const at::Tensor* const t = optional(o, type, {rows, cols});
        if (!t) return nullptr;
        if ((t->stride(1) != 1 && cols != 1) || (t->stride(0) < cols && rows > 1)) fine = false;
        const int64_t step = rows > 1 ? t->stride(0) : 0;
        if (ld) *ld = step;
        return t;
    }
    // one of two matrices that share a leading dimension
    const at::Tensor* matrix_like(PyObject* o, at::ScalarType type, int64_t rows, int64_t cols, const at::Tensor* other, int64_t* ld)
    {
        int64_t mine = 0;
        const at::Tensor* const t = matrix(o, type, rows, cols, &mine);
        if (!t) return nullptr;
        if (other && mine != *ld) fine = false;
        *ld = mine;
        return t;
    }
};
void* data_or_null(const at::Tensor* t) { return t ? data(t) : nullptr; }

// Strides (n, h, w) of a tensor [N,C,S] or [N,C,H,W] whose channels are neighbours.
bool channels_last(const at::Tensor* t, int64_t* out)
{
    const int64_t n = t->dim();
    if (t->stride(1) != 1 && t->size(1) != 1) return false;
    const int64_t extent[3] = {t->size(0), n == 3 ? 1 : t->size(2), t->size(n - 1)}, stride[3] = {t->stride(0), n == 3 ? 0 : t->stride(2), t->stride(n - 1)};
    for (int i = 0; i < 3; ++i) {
        if (extent[i] > 1 && stride[i] == 0) return false;
        out[i] = extent[i] > 1 ? stride[i] : 0;
    }
    return true;
}

// What a norm's calls have in common: x and a tensor like it, the parameters' type, the descriptor but for the strides.
struct Norm {
    Tensors t;
    const at::Tensor* x = nullptr;
    at::ScalarType type, param = at::kFloat;
    int64_t C = 0;
    int32_t groups = 0;
    anr_group_norm_desc d{};

    bool init(PyObject* x_, PyObject* groups_, PyObject* act, std::initializer_list<PyObject*> parameters)
    {
        x = plain_memory(x_);
        if (!x || x->device().index() != t.s.device || (x->dim() != 3 && x->dim() != 4)) return false;
        type = x->scalar_type();
        d.dtype = type_code(type);
        if (d.dtype < 0 || !int32(groups_, &groups) || (act && !int32(act, &d.act))) return false;
        bool given = false;
        for (PyObject* const o : parameters) {
            if (absent(o)) continue;
            const at::Tensor* const v = plain_memory(o);
            if (!v || (given && v->scalar_type() != param)) return false;
            param = v->scalar_type();
            given = true;
        }
        if (param != at::kFloat && param != type) return false;
        C = x->size(1);
        d.groups = groups;
        d.param_dtype = type_code(param);
        const int64_t n = x->dim();
        d.H = 1;
        return fits(x->size(0), &d.N) && fits(C, &d.C) && (n == 3 || fits(x->size(2), &d.H)) && fits(x->size(n - 1), &d.W) && channels_last(x, d.x_stride);
    }
    const at::Tensor* vector(PyObject* o) { return t.packed(o, param, {C}); }
    const at::Tensor* statistic(PyObject* o) { return t.packed(o, at::kFloat, {x->size(0), groups}); }
};

bool run_group_norm(PyObject* const* a)
{
    Norm n;
    if ((a[9] && a[9] != Py_None) || (a[5] && !PyFloat_CheckExact(a[5])) || !n.init(a[0], a[1], a[6], {a[3], a[4]})) return false;
    const at::Tensor* const y = n.t.get(a[2], n.type, n.x->sizes());
    const at::Tensor *gamma = n.vector(a[3]), *beta = n.vector(a[4]), *mean = n.statistic(a[7]), *rstd = n.statistic(a[8]);
    if (!n.t.fine || !channels_last(y, n.d.y_stride)) return false;
    size_t need = 0;
    if (g_size(ANR_OP_GROUP_NORM, &n.d, &need) != ANR_OK) return false;
    const Workspace ws(need, n.t.s);
    return ws.here && accepted<CallNorm>(GROUP_NORM, &n.d, data(n.x), data_or_null(gamma), data_or_null(beta), a[5] ? (float)PyFloat_AS_DOUBLE(a[5]) : 1e-5f, data(y),
                                         data_or_null(mean), data_or_null(rstd), ws.ptr, ws.bytes, n.t.s.stream);
}

bool run_group_norm_backward(PyObject* const* a)
{
    Norm n;
    if ((a[11] && a[11] != Py_None) || !n.init(a[1], a[2], a[10], {a[3], a[4], a[8], a[9]})) return false;
    const at::Tensor *dy = n.t.get(a[0], n.type, n.x->sizes()), *dx = n.t.optional(a[7], n.type, n.x->sizes());
    const at::Tensor *gamma = n.vector(a[3]), *beta = n.vector(a[4]), *mean = n.statistic(a[5]), *rstd = n.statistic(a[6]), *dgamma = n.vector(a[8]), *dbeta = n.vector(a[9]);
    if (!n.t.fine || !channels_last(dy, n.d.y_stride) || !channels_last(dx ? dx : n.x, n.d.dx_stride)) return false;
    size_t need = 0;
    if (g_size(ANR_OP_GROUP_NORM_BACKWARD, &n.d, &need) != ANR_OK) return false;
    const Workspace ws(need, n.t.s);
    return ws.here && accepted<CallNormBackward>(GROUP_NORM_BACKWARD, &n.d, data(dy), data(n.x), data_or_null(gamma), data_or_null(beta), data_or_null(mean), data_or_null(rstd),
                                                 data_or_null(dx), data_or_null(dgamma), data_or_null(dbeta), ws.ptr, ws.bytes, n.t.s.stream);
}

// Strides (b, s, h) of a tensor [B,S,H,D], zeros for a packed one.
bool token_strides(const at::Tensor* t, int64_t* out)
{
    for (int i = 0; i < 3; ++i) out[i] = 0;
    if (t->is_contiguous()) return true;
    if (t->stride(3) != 1 && t->size(3) != 1) return false;
    bool all = true;
    for (int i = 0; i < 3; ++i) {
        out[i] = t->size(i) > 1 ? t->stride(i) : 0;
        all = all && out[i] == 0;
    }
    return !all || t->numel() == t->size(3);
}

bool run_rotary(PyObject* const* a)
{
    Tensors t;
    const at::Tensor *q = plain_memory(a[0]), *positions = plain_memory(a[2]), *freq = plain(a[3]);
    const bool with_k = a[1] != Py_None;
    const at::Tensor* const k = with_k ? plain_memory(a[1]) : nullptr;
    if (!q || !positions || !freq || (with_k && !k) || with_k != (a[5] != Py_None) || q->dim() != 4 || (k && k->dim() != 4) || freq->dim() != 1) return false;
    anr_rotary_desc d{};
    d.dtype = type_code(q->scalar_type());
    d.pos_type = positions->scalar_type() == at::kLong ? ANR_POS_I64 : positions->scalar_type() == at::kInt ? ANR_POS_I32 : positions->scalar_type() == at::kFloat ? ANR_POS_F32 : -1;
    if (d.dtype < 0 || d.pos_type < 0) return false;
    const at::ScalarType type = q->scalar_type();
    const int64_t B = q->size(0), S = q->size(1), H = q->size(2), D = q->size(3), Hk = k ? k->size(2) : 0;
    t.get(a[0], type, q->sizes());
    if (k) t.get(a[1], type, {B, S, Hk, D});
    const at::Tensor* const q_out = t.get(a[4], type, q->sizes());
    const at::Tensor* const k_out = k ? t.get(a[5], type, k->sizes()) : nullptr;
    if (!t.fine || !freq->is_contiguous() || freq->device().index() != t.s.device) return false;
    d.axes = 1;
    int64_t pairs = 0;
    if (absent(a[6])) {
        if (!fits(freq->size(0), &d.section[0])) return false;
        pairs = freq->size(0);
    } else {
        if (!PyTuple_CheckExact(a[6]) || PyTuple_GET_SIZE(a[6]) < 1 || PyTuple_GET_SIZE(a[6]) > 4) return false;
        d.axes = (int32_t)PyTuple_GET_SIZE(a[6]);
        for (int i = 0; i < d.axes; ++i) {
            if (!int32(PyTuple_GET_ITEM(a[6], i), &d.section[i])) return false;
            pairs += d.section[i];
        }
    }
    if (pairs != freq->size(0) || (a[7] && !int32(a[7], &d.pairing)) || (a[8] && !PyBool_Check(a[8]))) return false;
    d.inverse = a[8] == Py_True;
    const bool each = positions->dim() == 3;                // [axes,B,S], or [axes,S] for all sequences
    if ((!each && positions->dim() != 2) || positions->device().index() != t.s.device || positions->size(0) != d.axes || (each && positions->size(1) != B) ||
        positions->size(positions->dim() - 1) != S)
        return false;
    d.pos_stride[0] = positions->stride(0);
    d.pos_stride[1] = each ? positions->stride(1) : 0;
    d.pos_stride[2] = positions->stride(positions->dim() - 1);
    if (!fits(B, &d.B) || !fits(S, &d.S) || !fits(H, &d.H) || !fits(Hk, &d.Hk) || !fits(D, &d.D)) return false;
    if (!token_strides(q, d.q_stride) || !token_strides(q_out, d.q_out_stride) || (k && (!token_strides(k, d.k_stride) || !token_strides(k_out, d.k_out_stride)))) return false;
    return accepted<CallRotary>(ROTARY, &d, data(q), data_or_null(k), data(positions), data(freq), data(q_out), data_or_null(k_out), nullptr, 0, t.s.stream);
}

bool run_gated_ff(PyObject* const* a)
{
    Tensors t;
    const at::Tensor *x = plain_memory(a[0]), *first = plain_memory(a[1]);
    anr_gated_ff_desc d{};
    if (!x || !first || x->dim() != 2 || first->dim() != 2 || (a[8] && a[8] != Py_None) || absent(a[6]) != absent(a[7])) return false;
    const at::ScalarType type = x->scalar_type();
    d.dtype = type_code(type);
    d.act = ANR_ACT_SILU;
    if (d.dtype < 0 || (a[5] && !int32(a[5], &d.act))) return false;
    d.T = x->size(0);
    d.C = x->size(1);
    d.F = first->size(0);
    t.matrix(a[0], type, d.T, d.C, &d.ldx);
    const at::Tensor* const wg = t.matrix(a[1], type, d.F, d.C, &d.ldw);
    const at::Tensor* const wu = t.matrix_like(a[2], type, d.F, d.C, wg, &d.ldw);
    const at::Tensor *wd = t.matrix(a[3], type, d.C, d.F, &d.ld_down), *y = t.matrix(a[4], type, d.T, d.C, &d.ldy);
    const at::Tensor* const gate = t.matrix(a[6], type, d.T, d.F, &d.ldpre);
    const at::Tensor* const up = t.matrix_like(a[7], type, d.T, d.F, gate, &d.ldpre);
    if (!t.fine || !wu || !wd || !y) return false;
    size_t need = 0;
    if (g_size(ANR_OP_GATED_FF, &d, &need) != ANR_OK) return false;
    const Workspace ws(need, t.s);
    return ws.here &&
           accepted<CallFf>(GATED_FF, &d, data(x), data(wg), data(wu), data(wd), data(y), data_or_null(gate), data_or_null(up), ws.ptr, ws.bytes, t.s.stream);
}

bool run_gated_ff_backward(PyObject* const* a)
{
    Tensors t;
    const at::Tensor *x = plain_memory(a[1]), *first = plain_memory(a[2]);
    anr_gated_ff_desc d{};
    if (!x || !first || x->dim() != 2 || first->dim() != 2 || (a[12] && a[12] != Py_None)) return false;
    const at::ScalarType type = x->scalar_type();
    d.dtype = type_code(type);
    d.act = ANR_ACT_SILU;
    if (d.dtype < 0 || (a[11] && !int32(a[11], &d.act))) return false;
    d.T = x->size(0);
    d.C = x->size(1);
    d.F = first->size(0);
    const at::Tensor* const dy = t.matrix(a[0], type, d.T, d.C, &d.ldy);
    t.matrix(a[1], type, d.T, d.C, &d.ldx);
    const at::Tensor* const wg = t.matrix(a[2], type, d.F, d.C, &d.ldw);
    const at::Tensor* const wu = t.matrix_like(a[3], type, d.F, d.C, wg, &d.ldw);
    const at::Tensor *wd = t.matrix(a[4], type, d.C, d.F, &d.ld_down), *gate = t.matrix(a[5], type, d.T, d.F, &d.ldpre);
    const at::Tensor* const up = t.matrix_like(a[6], type, d.T, d.F, gate, &d.ldpre);
    const at::Tensor* const dx = t.matrix(a[7], type, d.T, d.C, &d.lddx);
    const at::Tensor* const dwg = t.matrix(a[8], type, d.F, d.C, &d.lddw);
    const at::Tensor* const dwu = t.matrix_like(a[9], type, d.F, d.C, dwg, &d.lddw);
    const at::Tensor* const dwd = t.matrix(a[10], type, d.C, d.F, &d.ld_ddown);
    if (!t.fine || !dy || !wu || !wd || !gate || !up) return false;
    size_t need = 0;
    if (g_size(ANR_OP_GATED_FF_BACKWARD, &d, &need) != ANR_OK) return false;
    const Workspace ws(need, t.s);
    return ws.here && accepted<CallFfBackward>(GATED_FF_BACKWARD, &d, data(dy), data(x), data(wg), data(wu), data(wd), data(gate), data(up), data_or_null(dx), data_or_null(dwg),
                                               data_or_null(dwu), data_or_null(dwd), ws.ptr, ws.bytes, t.s.stream);
}

// What the calls of a root-mean-square norm have in common: x, its type and extents, the parameters' type.
struct RmsNorm {
    Tensors t;
    const at::Tensor* x = nullptr;
    at::ScalarType type, param = at::kFloat;
    anr_rms_norm_desc d{};

    bool init(PyObject* x_, std::initializer_list<PyObject*> parameters)
    {
        x = plain_memory(x_);
        if (!x || x->dim() != 2) return false;
        type = x->scalar_type();
        d.dtype = type_code(type);
        if (d.dtype < 0) return false;
        bool given = false;
        for (PyObject* const o : parameters) {
            if (absent(o)) continue;
            const at::Tensor* const v = plain_memory(o);
            if (!v || (given && v->scalar_type() != param)) return false;
            param = v->scalar_type();
            given = true;
        }
        if (param != at::kFloat && param != type) return false;
        d.param_dtype = type_code(param);
        d.T = x->size(0);
        d.C = x->size(1);
        return matrix(x_, &d.ldx) != nullptr;
    }
    const at::Tensor* matrix(PyObject* o, int64_t* ld) { return t.matrix(o, type, d.T, d.C, ld); }
    const at::Tensor* vector(PyObject* o) { return t.packed(o, param, {d.C}); }
    const at::Tensor* statistic(PyObject* o) { return t.packed(o, at::kFloat, {d.T}); }
};

bool run_rms_norm(PyObject* const* a)
{
    RmsNorm n;
    if ((a[3] && !PyFloat_CheckExact(a[3])) || (!absent(a[5]) && absent(a[4])) || !n.init(a[0], {a[2]})) return false;
    const at::Tensor *y = n.matrix(a[1], &n.d.ldy), *residual = n.matrix(a[4], &n.d.ld_residual), *h = n.matrix(a[5], &n.d.ldh);
    const at::Tensor *gamma = n.vector(a[2]), *rstd = n.statistic(a[6]);
    return n.t.fine && y &&
           accepted<CallRmsNorm>(RMS_NORM, &n.d, data(n.x), data_or_null(residual), data_or_null(gamma), a[3] ? (float)PyFloat_AS_DOUBLE(a[3]) : 1e-6f, data_or_null(h), data(y),
                                 data_or_null(rstd), nullptr, 0, n.t.s.stream);
}

bool run_rms_norm_q8(PyObject* const* a)
{
    RmsNorm n;
    if ((a[4] && !PyFloat_CheckExact(a[4])) || (!absent(a[6]) && absent(a[5])) || !n.init(a[0], {a[3]})) return false;
    const at::Tensor *q = n.t.matrix(a[1], at::kChar, n.d.T, n.d.C, &n.d.ldy), *residual = n.matrix(a[5], &n.d.ld_residual), *h = n.matrix(a[6], &n.d.ldh);
    const at::Tensor *gamma = n.vector(a[3]), *scale = n.statistic(a[2]);
    return n.t.fine && q && scale &&
           accepted<CallRmsNorm>(RMS_NORM_Q8, &n.d, data(n.x), data_or_null(residual), data_or_null(gamma), a[4] ? (float)PyFloat_AS_DOUBLE(a[4]) : 1e-6f, data_or_null(h), data(q),
                                 data(scale), nullptr, 0, n.t.s.stream);
}

bool run_rms_norm_backward(PyObject* const* a)
{
    RmsNorm n;
    if ((a[7] && a[7] != Py_None) || !n.init(a[1], {a[2], a[5]})) return false;
    const at::Tensor *dy = n.matrix(a[0], &n.d.ldy), *dx = n.matrix(a[4], &n.d.ldh), *dh = n.matrix(a[6], &n.d.ld_residual);
    const at::Tensor *gamma = n.vector(a[2]), *rstd = n.statistic(a[3]), *dgamma = n.vector(a[5]);
    if (!n.t.fine || !dy || !rstd) return false;
    size_t need = 0;
    if (g_size(ANR_OP_RMS_NORM_BACKWARD, &n.d, &need) != ANR_OK) return false;
    const Workspace ws(need, n.t.s);
    return ws.here && accepted<CallRmsNormBackward>(RMS_NORM_BACKWARD, &n.d, data(dy), data(n.x), data_or_null(gamma), data(rstd), data_or_null(dh), data_or_null(dx),
                                                    data_or_null(dgamma), ws.ptr, ws.bytes, n.t.s.stream);
}

bool run_quantize_rows(PyObject* const* a)
{
    Tensors t;
    const at::Tensor* const x = plain_memory(a[0]);
    anr_rows_q8_desc d{};
    if (!x || x->dim() != 2) return false;
    const at::ScalarType type = x->scalar_type();
    d.dtype = type_code(type);
    if (d.dtype < 0 || (a[3] && !int32(a[3], &d.act))) return false;
    d.T = x->size(0);
    d.C = x->size(1);
    t.matrix(a[0], type, d.T, d.C, &d.ldx);
    const at::Tensor *q = t.matrix(a[1], at::kChar, d.T, d.C, &d.ldq), *up = t.matrix(a[4], type, d.T, d.C, &d.ld_up), *scale = t.packed(a[2], at::kFloat, {d.T});
    return t.fine && q && scale && accepted<CallQuantize>(QUANTIZE_ROWS, &d, data(x), data_or_null(up), data(q), data(scale), nullptr, 0, t.s.stream);
}

bool run_dequantize_rows(PyObject* const* a)
{
    Tensors t;
    const at::Tensor *q = plain_memory(a[0]), *y = plain_memory(a[2]);
    anr_rows_q8_desc d{};
    if (!q || !y || q->dim() != 2) return false;
    d.dtype = type_code(y->scalar_type());
    if (d.dtype < 0) return false;
    d.T = q->size(0);
    d.C = q->size(1);
    t.matrix(a[0], at::kChar, d.T, d.C, &d.ldq);
    t.matrix(a[2], y->scalar_type(), d.T, d.C, &d.ldx);
    const at::Tensor* const scale = t.packed(a[1], at::kFloat, {d.T});
    return t.fine && scale && accepted<Call3>(DEQUANTIZE_ROWS, &d, data(q), data(scale), data(y), nullptr, 0, t.s.stream);
}

bool run_gemm_i8(PyObject* const* a)
{
    Tensors t;
    const at::Tensor *x = plain_memory(a[0]), *w = plain_memory(a[1]), *out = plain_memory(a[4]), *bias = absent(a[5]) ? nullptr : plain_memory(a[5]);
    anr_gemm_i8_desc d{};
    if (!x || !w || !out || x->dim() != 2 || w->dim() != 2 || (a[6] && a[6] != Py_None) || (!absent(a[5]) && !bias)) return false;
    const at::ScalarType type = out->scalar_type(), kind = bias ? bias->scalar_type() : at::kFloat;
    d.dtype = type_code(type);
    d.bias_dtype = type_code(kind);
    if (d.dtype < 0 || (kind != at::kFloat && kind != type)) return false;
    d.M = x->size(0);
    d.K = x->size(1);
    d.N = w->size(0);
    t.matrix(a[0], at::kChar, d.M, d.K, &d.lda);
    t.matrix(a[1], at::kChar, d.N, d.K, &d.ldw);
    t.matrix(a[4], type, d.M, d.N, &d.ldd);
    const at::Tensor *xs = t.packed(a[2], at::kFloat, {d.M}), *ws_ = t.packed(a[3], at::kFloat, {d.N});
    if (bias) t.packed(a[5], kind, {d.N});
    if (!t.fine) return false;
    size_t need = 0;
    if (g_size(ANR_OP_GEMM_I8, &d, &need) != ANR_OK) return false;
    const Workspace ws(need, t.s);
    return ws.here && accepted<CallGemmI8>(GEMM_I8, &d, data(x), data(w), data_or_null(xs), data_or_null(ws_), data_or_null(bias), data(out), ws.ptr, ws.bytes, t.s.stream);
}

// Parameters of each operator, the required ones first, and which of them it returns.
const char* const kGemm[] = {"A", "B", "C"};
const char* const kConv[] = {"x", "w", "y", "stride", "pad", "ws", "dil", "groups", "route"};
const char* const kConvBn[] = {"x", "w", "gamma", "beta", "mean", "var", "eps", "y", "stride", "pad", "ws", "dil", "groups", "route"};
const char* const kPacked[] = {"desc", "x", "pack", "y", "ws"};
const char* const kDw[] = {"x", "w", "y", "stride", "pad", "dil"};
const char* const kScores[] = {"q", "k", "out"};
const char* const kNrm[] = {"x", "out", "ws"};
const char* const kNorm[] = {"x", "groups", "y", "gamma", "beta", "eps", "act", "mean", "rstd", "ws"};
const char* const kNormBackward[] = {"dy", "x", "groups", "gamma", "beta", "mean", "rstd", "dx", "dgamma", "dbeta", "act", "ws"};
const char* const kRotary[] = {"q", "k", "positions", "inv_freq", "q_out", "k_out", "sections", "pairing", "inverse"};
const char* const kFf[] = {"x", "w_gate", "w_up", "w_down", "y", "act", "gate", "up", "ws"};
const char* const kFfBackward[] = {"dy", "x", "w_gate", "w_up", "w_down", "gate", "up", "dx", "dw_gate", "dw_up", "dw_down", "act", "ws"};
const char* const kRmsNorm[] = {"x", "y", "gamma", "eps", "residual", "h", "rstd"};
const char* const kRmsNormBackward[] = {"dy", "x", "gamma", "rstd", "dx", "dgamma", "dh", "ws"};
const char* const kRmsNormQ8[] = {"x", "q", "scale", "gamma", "eps", "residual", "h"};
const char* const kQuantize[] = {"x", "q", "scale", "act", "up"};
const char* const kDequantize[] = {"q", "scale", "y"};
const char* const kGemmI8[] = {"a", "w", "a_scale", "w_scale", "d", "bias", "ws"};

// The parameters `result` to `last`: one of them itself, more as a tuple.
PyObject* returned(PyObject* const* a, int result, int last)
{
    if (result == last) return Py_NewRef(a[result]);
    PyObject* const tuple = PyTuple_New(last - result + 1);
    for (int i = result; tuple && i <= last; ++i) PyTuple_SET_ITEM(tuple, i - result, Py_NewRef(a[i] ? a[i] : Py_None));
    return tuple;
}

template <int OP, int N, typename Run>
PyObject* call(const char* const (&names)[N], int required, int result, int last, Run run, PyObject* const* args, Py_ssize_t n, PyObject* kwnames)
{
    PyObject* a[N];
    if (!g_python[OP]) {
        PyErr_SetString(PyExc_RuntimeError, "the operators are those of paper_2006_06762_amd.binding, which is not imported");
        return nullptr;
    }
    try {
        if (!at::impl::torch_function_mode_enabled() && arguments(names, required, args, n, kwnames, a) && run(a)) return returned(a, result, last);
    } catch (...) {
        // (memory that cannot be had: Python raises it)
    }
    if (PyErr_Occurred()) PyErr_Clear();
    return PyObject_Vectorcall(g_python[OP], args, (size_t)n, kwnames);
}

#define ANR_OPERATOR(fn, op, names, required, result, ...) ANR_OPERATOR_OF(fn, op, names, required, result, result, __VA_ARGS__)
#define ANR_OPERATOR_OF(fn, op, names, required, result, last, ...)                                        \
    PyObject* fn(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kwnames)               \
    {                                                                                             \
        return call<op>(names, required, result, last, [](PyObject* const* a) { return __VA_ARGS__; }, args, n, kwnames); \
    }
ANR_OPERATOR(py_gemm, GEMM, kGemm, 3, 2, run_gemm(a))
ANR_OPERATOR(py_conv2d, CONV2D, kConv, 3, 2, run_conv2d(a))
ANR_OPERATOR(py_conv_bn_relu, CONV_BN_RELU, kConvBn, 8, 7, run_conv_bn_relu(a))
ANR_OPERATOR(py_conv2d_packed, CONV2D_PACKED, kPacked, 4, 3, run_packed(CONV2D_PACKED, a))
ANR_OPERATOR(py_conv_bn_relu_packed, CONV_BN_RELU_PACKED, kPacked, 4, 3, run_packed(CONV_BN_RELU_PACKED, a))
ANR_OPERATOR(py_dwconv, DWCONV, kDw, 3, 2, run_dwconv(a))
ANR_OPERATOR(py_tbg, TBG, kScores, 3, 2, run_scores(TBG, a))
ANR_OPERATOR(py_tbs, TBS, kScores, 3, 2, run_scores(TBS, a))
ANR_OPERATOR(py_nrm, NRM, kNrm, 2, 1, run_nrm(a))
ANR_OPERATOR(py_group_norm, GROUP_NORM, kNorm, 3, 2, run_group_norm(a))
ANR_OPERATOR_OF(py_group_norm_backward, GROUP_NORM_BACKWARD, kNormBackward, 7, 7, 9, run_group_norm_backward(a))
ANR_OPERATOR_OF(py_rotary, ROTARY, kRotary, 6, 4, 5, run_rotary(a))
ANR_OPERATOR(py_gated_ff, GATED_FF, kFf, 5, 4, run_gated_ff(a))
ANR_OPERATOR_OF(py_gated_ff_backward, GATED_FF_BACKWARD, kFfBackward, 7, 7, 10, run_gated_ff_backward(a))
ANR_OPERATOR(py_rms_norm, RMS_NORM, kRmsNorm, 2, 1, run_rms_norm(a))
ANR_OPERATOR_OF(py_rms_norm_backward, RMS_NORM_BACKWARD, kRmsNormBackward, 4, 4, 5, run_rms_norm_backward(a))
ANR_OPERATOR_OF(py_rms_norm_q8, RMS_NORM_Q8, kRmsNormQ8, 3, 1, 2, run_rms_norm_q8(a))
ANR_OPERATOR_OF(py_quantize_rows, QUANTIZE_ROWS, kQuantize, 3, 1, 2, run_quantize_rows(a))
ANR_OPERATOR(py_dequantize_rows, DEQUANTIZE_ROWS, kDequantize, 3, 2, run_dequantize_rows(a))
ANR_OPERATOR(py_gemm_i8, GEMM_I8, kGemmI8, 5, 4, run_gemm_i8(a))
#undef ANR_OPERATOR
#undef ANR_OPERATOR_OF

// setup(functions, entries, fast_size, size): tuples in the order of the operators, entry points as integers.
PyObject* py_setup(PyObject*, PyObject* args)
{
    PyObject *functions, *entries, *fast_size, *size;
    if (!PyArg_ParseTuple(args, "O!O!OO", &PyTuple_Type, &functions, &PyTuple_Type, &entries, &fast_size, &size)) return nullptr;
    if (PyTuple_GET_SIZE(functions) != OPS || PyTuple_GET_SIZE(entries) != OPS) {
        PyErr_SetString(PyExc_ValueError, "one function and one entry point per operator");
        return nullptr;
    }
    for (int i = 0; i < OPS; ++i) {
        g_entry[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(entries, i));
        if (!g_entry[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null entry point");
            return nullptr;
        }
        Py_XSETREF(g_python[i], Py_NewRef(PyTuple_GET_ITEM(functions, i)));
    }
    g_fast_size = reinterpret_cast<CallFastSize>(PyLong_AsVoidPtr(fast_size));
    g_size = reinterpret_cast<CallSize>(PyLong_AsVoidPtr(size));
    if (!g_fast_size || !g_size) return nullptr;
    Py_RETURN_NONE;
}

PyCFunction as_cfunction(PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t, PyObject*)) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef g_methods[] = {
    {"gemm", as_cfunction(py_gemm), METH_FASTCALL | METH_KEYWORDS,
     "gemm(A, B, C)\n--\n\nC = A.B.  A [M,K] / [b,M,K], B [K,N] / [b,K,N], C [M,N] / [b,M,N]; last dim contiguous."},
    {"conv2d", as_cfunction(py_conv2d), METH_FASTCALL | METH_KEYWORDS,
     "conv2d(x, w, y, stride=(1, 1), pad=(0, 0), ws=None, dil=(1, 1), groups=1, route=0)\n--\n\n"
     "y = conv2d(x, w); x [N,C,H,W], w [K,C/groups,R,S] packed, y [N,K,OH,OW] (may be strided views).\n"
     "ws: optional workspace tensor of at least workspace_size(ANR_OP_CONV2D, desc) bytes; with fewer than\n"
     "conv2d_fast_workspace_size(desc) the kernel that conv2d_route reports runs."},
    {"conv_bn_relu", as_cfunction(py_conv_bn_relu), METH_FASTCALL | METH_KEYWORDS,
     "conv_bn_relu(x, w, gamma, beta, mean, var, eps, y, stride=(1, 1), pad=(0, 0), ws=None, dil=(1, 1), groups=1, route=0)\n--\n\n"
     "y = relu(batch norm(conv2d(x, w))) with the batch norm's vectors of K floats."},
    {"conv2d_packed", as_cfunction(py_conv2d_packed), METH_FASTCALL | METH_KEYWORDS,
     "conv2d_packed(desc, x, pack, y, ws=None)\n--\n\n"
     "conv2d with weights from conv2d_pack_weights (desc: the descriptor it returned).  x may be a strided view; one\n"
     "whose rows are no whole 16-byte units is copied first where the pack is in the patch kernel's order."},
    {"conv_bn_relu_packed", as_cfunction(py_conv_bn_relu_packed), METH_FASTCALL | METH_KEYWORDS,
     "conv_bn_relu_packed(desc, x, pack, y, ws=None)\n--\n\nconv + batch norm + ReLU with a pack made with bn=(gamma, beta, mean, var)."},
    {"dwconv", as_cfunction(py_dwconv), METH_FASTCALL | METH_KEYWORDS,
     "dwconv(x, w, y, stride=(1, 1), pad=(0, 0), dil=(1, 1))\n--\n\nDepthwise convolution: x [N,C,H,W], w [C,1,R,S] packed, y [N,C,OH,OW]."},
    {"tbg", as_cfunction(py_tbg), METH_FASTCALL | METH_KEYWORDS,
     "tbg(q, k, out)\n--\n\nout[b,h,i,j] = sum_d q[b,i,h,d] k[b,j,h,d]; q,k [B,S,H,D], out [B,H,S,S]."},
    {"tbs", as_cfunction(py_tbs), METH_FASTCALL | METH_KEYWORDS, "tbs(q, k, out)\n--\n\ntbg followed by a softmax over the last axis."},
    {"nrm", as_cfunction(py_nrm), METH_FASTCALL | METH_KEYWORDS,
     "nrm(x, out, ws=None)\n--\n\nout[b] = sqrt(sum of squares of x[b]).  x [N,M] or [b,N,M] with unit column stride, out [1] / [b]."},
    {"group_norm", as_cfunction(py_group_norm), METH_FASTCALL | METH_KEYWORDS,
     "group_norm(x, groups, y, gamma=None, beta=None, eps=1e-05, act=0, mean=None, rstd=None, ws=None)\n--\n\n"
     "y = act((x - mean) * rstd * gamma + beta) over `groups` runs of channels; x, y [N,C,S] or [N,C,H,W] channels last.\n"
     "mean, rstd: float32 [N,groups], written where given, for a backward pass."},
    {"group_norm_backward", as_cfunction(py_group_norm_backward), METH_FASTCALL | METH_KEYWORDS,
     "group_norm_backward(dy, x, groups, gamma, beta, mean, rstd, dx=None, dgamma=None, dbeta=None, act=0, ws=None)\n--\n\n"
     "Gradients of group_norm, into those of dx, dgamma and dbeta that are given, from its arguments and the mean and rstd that it wrote."},
    {"rotary", as_cfunction(py_rotary), METH_FASTCALL | METH_KEYWORDS,
     "rotary(q, k, positions, inv_freq, q_out, k_out, sections=None, pairing=0, inverse=False)\n--\n\n"
     "q_out and k_out: q [B,S,H,D] and k [B,S,Hk,D] turned by positions[axis] * inv_freq; each may be its input itself, k and k_out None.\n"
     "positions [axes,B,S] or [axes,S]; inv_freq one float for each pair of dimensions; sections: pairs of each axis (one axis: all)."},
    {"gated_ff", as_cfunction(py_gated_ff), METH_FASTCALL | METH_KEYWORDS,
     "gated_ff(x, w_gate, w_up, w_down, y, act=2, gate=None, up=None, ws=None)\n--\n\n"
     "y = (act(x.w_gate^T) * (x.w_up^T)).w_down^T; x, y [T,C], w_gate and w_up [F,C], w_down [C,F].  gate and up [T,F]: the two\n"
     "products, where a backward pass is to follow."},
    {"gated_ff_backward", as_cfunction(py_gated_ff_backward), METH_FASTCALL | METH_KEYWORDS,
     "gated_ff_backward(dy, x, w_gate, w_up, w_down, gate, up, dx=None, dw_gate=None, dw_up=None, dw_down=None, act=2, ws=None)\n--\n\n"
     "Gradients of gated_ff, into those of dx, dw_gate, dw_up and dw_down that are given, from its arguments and the gate and up that it wrote."},
    {"rms_norm", as_cfunction(py_rms_norm), METH_FASTCALL | METH_KEYWORDS,
     "rms_norm(x, y, gamma=None, eps=1e-06, residual=None, h=None, rstd=None)\n--\n\n"
     "y = h * rstd * gamma with h = x + residual and rstd = 1/sqrt(mean(h^2) + eps) over each row; x, residual, h, y [T,C].  h: where the sum goes;\n"
     "rstd: float32 [T], for a backward pass."},
    {"rms_norm_backward", as_cfunction(py_rms_norm_backward), METH_FASTCALL | METH_KEYWORDS,
     "rms_norm_backward(dy, x, gamma, rstd, dx=None, dgamma=None, dh=None, ws=None)\n--\n\n"
     "Gradients of rms_norm, into those of dx and dgamma that are given, from what it normed (its h where it had a residual) and the rstd that it\n"
     "wrote.  dh: the gradient that reaches the sum by its other way; dx is then that of x and of residual alike."},
    {"rms_norm_q8", as_cfunction(py_rms_norm_q8), METH_FASTCALL | METH_KEYWORDS,
     "rms_norm_q8(x, q, scale, gamma=None, eps=1e-06, residual=None, h=None)\n--\n\n"
     "rms_norm with its result in 8 bits: q int8 [T,C], scale float32 [T], y = q * scale."},
    {"quantize_rows", as_cfunction(py_quantize_rows), METH_FASTCALL | METH_KEYWORDS,
     "quantize_rows(x, q, scale, act=0, up=None)\n--\n\n"
     "q int8 [T,C] and scale float32 [T]: rows of act(x) * up (act(x) without up) in 8 bits, whose values are q * scale.  x and up [T,C]; for weights as\n"
     "[outputs, inputs] a scale for each output."},
    {"dequantize_rows", as_cfunction(py_dequantize_rows), METH_FASTCALL | METH_KEYWORDS,
     "dequantize_rows(q, scale, y)\n--\n\ny = q * scale; q int8 [T,C], scale float32 [T], y [T,C]."},
    {"gemm_i8", as_cfunction(py_gemm_i8), METH_FASTCALL | METH_KEYWORDS,
     "gemm_i8(a, w, a_scale, w_scale, d, bias=None, ws=None)\n--\n\n"
     "d = (a.w^T) * a_scale[:, None] * w_scale + bias; a int8 [M,K], w int8 [N,K], d [M,N] float32, float16 or bfloat16; a_scale float32 [M] and\n"
     "w_scale float32 [N], or None for ones; bias [N] of float32 or d's type."},
    {"setup", py_setup, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&g_module); }
