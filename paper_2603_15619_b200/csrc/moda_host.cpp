// Host path of the calls that a program makes once per layer or token, as a CPython extension: arguments, output tensors, the
// C entry points of libmoda_b200.so, and the autograd node of moda_attention.
//
// It serves the plain case alone: torch.Tensor (or Parameter) objects on the device, contiguous, of the documented types and
// sizes, on the current stream, with no mode, transform or tracer active.  For anything else a function returns None and the
// caller goes on with its own code (binding.py, autograd.py), which has the same checks and says what is wrong.  A call through here
// makes the same C call with the same arguments.
//
// Why: at the sizes of a decode step or of a small layer the device waits for the host.  Microseconds a call in a loop, through
// Python and ctypes -> through here: decode of one sequence over 8192 keys 15.9 -> 12.3 (10 on the device); T = 256, 2 heads, l = 4:
// forward 12.7 -> 8.5, backward 31.3 -> 20.5, moda_attention and its gradients 137 -> 86 (what is left is the engine's hand-over
// to its device thread and back).  Serving calls, host time alone: weights of the
// keys 11 -> 6.2, decode step with weights 16 -> 9.3, eviction 17 -> 5.9, shared prefix 22 -> 8.9.  Paged cache in 8 bits: write
// 10.4 -> 3.4, read 8.9 -> 3.6, selection 14.2 -> 4.8, decode step 13.5 -> 5.8.
#include <Python.h>
#include <dlfcn.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/cuda/CUDAContext.h>
#include <c10/core/DispatchKeySet.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/PyInterpreter.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <climits>
#include <initializer_list>

#include "../../include/moda.h"

namespace {

using at::Tensor;

// ---- the library: addresses from the handle that the binding has opened -----------------------------------------------
#define MODA_HOST_CALLS(X)                                                                                              \
    X(moda_attn_fwd_gqa) X(moda_attn_fwd_append) X(moda_attn_bwd_gqa) X(moda_attn_bwd_gqa_stages) X(moda_attn_bwd_gqa_slot) \
    X(moda_bwd_workspace_bytes_gqa) X(moda_depth_cache_bytes) X(moda_attn_decode) X(moda_attn_decode_varlen)            \
    X(moda_attn_decode_paged) X(moda_decode_workspace_bytes)                                                            \
    X(moda_attn_key_mass) X(moda_key_mass_workspace_bytes) X(moda_attn_decode_mass) X(moda_decode_mass_workspace_bytes) \
    X(moda_kv_evict) X(moda_attn_decode_shared) X(moda_decode_shared_workspace_bytes)                                   \
    X(moda_kv_write_e4m3) X(moda_kv_read_e4m3) X(moda_kv_select_blocks) X(moda_kv_select_workspace_bytes) \
    X(moda_attn_decode_e4m3) X(moda_decode_e4m3_workspace_bytes)
struct Library {
#define X(name) decltype(&::name) name = nullptr;
    MODA_HOST_CALLS(X)
#undef X
} lib;
PyObject* check_fn = nullptr;                                  // binding._check: raises ModaError

[[noreturn]] void fail(int rc, const char* what) {
    PyGILState_STATE gil = PyGILState_Ensure();
    PyObject* r = PyObject_CallFunction(check_fn, "is", rc, what);
    Py_XDECREF(r);
    if (r != nullptr) PyErr_Format(PyExc_RuntimeError, "%s failed: [%d]", what, rc);
    python_error e;
    e.persist();
    PyGILState_Release(gil);
    throw e;
}

struct NoGil {
    PyThreadState* state = PyEval_SaveThread();
    ~NoGil() { PyEval_RestoreThread(state); }
};

// ---- what counts as plain --------------------------------------------------------------------------------------------
// Keys of an ordinary CUDA tensor; wrappers, views that conjugate or negate, fake and batched tensors carry others.
uint64_t plain_keys() {
    static const uint64_t keys = (c10::DispatchKeySet(c10::DispatchKey::CUDA) |
                                  c10::getAutogradRelatedKeySetFromBackend(c10::BackendComponent::CUDABit) |
                                  c10::getAutocastRelatedKeySetFromBackend(c10::BackendComponent::CUDABit) |
                                  c10::DispatchKeySet(c10::DispatchKey::ADInplaceOrView)).raw_repr();
    return keys;
}
// A torch-function mode sees the torch calls of the Python form.  Not so the one of a default device (torch.set_default_device): it
// fills in a device where none is given, and these calls give one.
PyObject* device_mode = nullptr;                               // torch.utils._device.DeviceContext
bool function_mode() {
    using TLS = at::impl::PythonTorchFunctionTLS;
    if (!at::impl::torch_function_mode_enabled()) return false;
    for (int64_t i = 0; i < TLS::stack_len(); ++i)
        if (reinterpret_cast<PyObject*>(Py_TYPE(TLS::get_stack_at(i)->ptr(getPyInterpreter()))) != device_mode) return true;
    return false;
}
// No mode, functorch transform, functionalisation or tracer: but for torch-function modes their keys would be in the thread's included set.
bool plain_thread() {
    if (function_mode()) return false;
    static const uint64_t keys = (c10::DispatchKeySet(c10::DispatchKey::BackendSelect) | c10::DispatchKeySet(c10::DispatchKey::ADInplaceOrView)).raw_repr();
    return (c10::impl::tls_local_dispatch_key_set().included_.raw_repr() & ~keys) == 0;
}
const Tensor* plain(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || (t.key_set().raw_repr() & ~plain_keys()) != 0) return nullptr;
    return &t;
}
const Tensor* dense(PyObject* o, at::ScalarType type, int64_t dim) {
    const Tensor* t = plain(o);
    return t != nullptr && t->scalar_type() == type && t->dim() == dim && t->is_contiguous() ? t : nullptr;
}
// An argument that may be None: a null tensor, or a contiguous one.  False: neither.
bool optional_dense(PyObject* o, const Tensor*& t) {
    t = nullptr;
    if (o == Py_None) return true;
    t = plain(o);
    return t != nullptr && t->is_contiguous();
}
bool shape_is(const Tensor& t, std::initializer_list<int64_t> want) { return t.sizes() == at::IntArrayRef(want); }
bool int_arg(PyObject* o, int& v) {
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    const long x = PyLong_AsLongAndOverflow(o, &over);
    if (over != 0 || x < INT_MIN || x > INT_MAX) return false;
    v = int(x);
    return true;
}
bool float_arg(PyObject* o, float& v) {
    if (!PyFloat_CheckExact(o)) return false;
    v = float(PyFloat_AS_DOUBLE(o));
    return true;
}
bool small(const Tensor& t) {                                   // every extent fits the int of the C calls
    for (int64_t n : t.sizes())
        if (n > INT_MAX) return false;
    return true;
}

void* ptr(const Tensor* t) { return t != nullptr ? t->data_ptr() : nullptr; }
void* stream() { return at::cuda::getCurrentCUDAStream().stream(); }
size_t bytes_of(const Tensor& t) { return size_t(t.numel()) * t.element_size(); }
Tensor like(const Tensor& t) { return at::empty(t.sizes(), t.options().requires_grad(false)); }
Tensor fresh(std::initializer_list<int64_t> shape, at::ScalarType type, const Tensor& on) {
    return at::empty(at::IntArrayRef(shape), on.options().dtype(type).requires_grad(false));
}
// A tensor that a kernel reads or writes n elements of, where it is given.
bool holds(const Tensor* t, at::ScalarType type, int64_t n) { return t == nullptr || (t->scalar_type() == type && t->numel() >= n); }
// A given tensor's own object, or the new tensor.
PyObject* out(PyObject* given, const Tensor& made) { return given != Py_None ? Py_NewRef(given) : THPVariable_Wrap(made); }
PyObject* none() { Py_RETURN_NONE; }

// ---- attention: shapes, forward, backward ----------------------------------------------------------------------------
struct Shape { int B, T, H, Hk, d; };
bool shapes(const Tensor& Q, const Tensor& K, const Tensor& V, Shape& s) {
    if (Q.dim() != 4 || K.dim() != 4 || Q.scalar_type() != at::kBFloat16 || K.scalar_type() != at::kBFloat16 || V.scalar_type() != at::kBFloat16) return false;
    if (!small(Q) || !small(K)) return false;
    s = {int(Q.size(0)), int(Q.size(1)), int(Q.size(2)), int(K.size(2)), int(Q.size(3))};
    return K.size(0) == s.B && K.size(1) == s.T && K.size(3) == s.d && V.sizes() == K.sizes();
}
// Whether a depth cache, or its gradient, has n slots (a number that no cache has is the C call's to refuse).
bool holds_slots(const Tensor* t, const Shape& s, int n) { return t == nullptr || bytes_of(*t) >= lib.moda_depth_cache_bytes(s.B, s.T, s.Hk, s.d, n); }
bool holds_slot(const Tensor* t, const Shape& s, int slot) { return holds_slots(t, s, std::min(slot, MODA_MAX_DEPTH) + 1); }
int64_t rows(const Shape& s) { return int64_t(s.B) * s.H * s.T; }
void forward(const Shape& s, const Tensor& Q, const Tensor& K, const Tensor& V, const Tensor* depth, int l, float scale,
             const Tensor* cache, int slot, Tensor& O, Tensor& LSE) {
    if (!O.defined()) O = like(Q);
    if (!LSE.defined()) LSE = fresh({s.B, s.H, s.T}, at::kFloat, Q);
    const int rc = cache == nullptr
        ? lib.moda_attn_fwd_gqa(Q.data_ptr(), K.data_ptr(), V.data_ptr(), l > 0 ? ptr(depth) : nullptr, s.B, s.T, s.H, s.Hk, s.d, l, scale,
                                O.data_ptr(), static_cast<float*>(LSE.data_ptr()), stream())
        : lib.moda_attn_fwd_append(Q.data_ptr(), K.data_ptr(), V.data_ptr(), l > 0 ? ptr(depth) : nullptr, s.B, s.T, s.H, s.Hk, s.d, l, scale,
                                   O.data_ptr(), static_cast<float*>(LSE.data_ptr()), cache->data_ptr(), slot, stream());
    if (rc != 0) fail(rc, cache == nullptr ? "moda_attn_fwd_gqa" : "moda_attn_fwd_append");
}
// mode: moda_attn_bwd_gqa, the call with a mask, or the call with a slot
enum Mode { kWhole, kMask, kSlot };
void backward(const Shape& s, const Tensor& Q, const Tensor& K, const Tensor& V, const Tensor* depth, const Tensor& O, const Tensor& dO,
              const Tensor& LSE, int l, float scale, Mode mode, int arg, Tensor& dQ, Tensor& dK, Tensor& dV, Tensor& dcache, Tensor& ws) {
    if (!dQ.defined()) dQ = like(Q);
    if (!dK.defined()) dK = like(K);
    if (!dV.defined()) dV = like(V);
    if (l > 0 && !dcache.defined()) {
        dcache = fresh({int64_t(lib.moda_depth_cache_bytes(s.B, s.T, s.Hk, s.d, l) / 2)}, at::kBFloat16, Q);
    }
    if (!ws.defined()) ws = fresh({int64_t(lib.moda_bwd_workspace_bytes_gqa(s.B, s.T, s.H, s.Hk, s.d, l))}, at::kByte, Q);
    const void* dep = l > 0 ? ptr(depth) : nullptr;
    void* dc = l > 0 ? dcache.data_ptr() : nullptr;
    const float* lse = static_cast<const float*>(LSE.data_ptr());
    if (mode == kSlot) {
        const int rc = lib.moda_attn_bwd_gqa_slot(Q.data_ptr(), K.data_ptr(), V.data_ptr(), dep, O.data_ptr(), dO.data_ptr(), lse, s.B, s.T, s.H, s.Hk, s.d, l,
                                                  scale, dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), dcache.data_ptr(), ws.data_ptr(), bytes_of(ws), arg, stream());
        if (rc != 0) fail(rc, "moda_attn_bwd_gqa_slot");
        return;
    }
    const int rc = mode == kWhole
        ? lib.moda_attn_bwd_gqa(Q.data_ptr(), K.data_ptr(), V.data_ptr(), dep, O.data_ptr(), dO.data_ptr(), lse, s.B, s.T, s.H, s.Hk, s.d, l,
                                scale, dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), dc, ws.data_ptr(), bytes_of(ws), stream())
        : lib.moda_attn_bwd_gqa_stages(Q.data_ptr(), K.data_ptr(), V.data_ptr(), dep, O.data_ptr(), dO.data_ptr(), lse, s.B, s.T, s.H, s.Hk,
                                       s.d, l, scale, dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), dc, ws.data_ptr(), bytes_of(ws), arg,
                                       stream());
    if (rc != 0) fail(rc, mode == kWhole ? "moda_attn_bwd_gqa" : "moda_attn_bwd_gqa_stages");
}

// attn_fwd(Q, K, V, depth, l, scale, cache, slot, O, LSE) -> (O, LSE)
PyObject* attn_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int l, slot = 0;
    float scale;
    if (n != 10 || !plain_thread() || !int_arg(a[4], l) || l < 0 || !float_arg(a[5], scale) || !int_arg(a[7], slot)) return none();
    const Tensor *Q = dense(a[0], at::kBFloat16, 4), *K = dense(a[1], at::kBFloat16, 4), *V = dense(a[2], at::kBFloat16, 4);
    const Tensor *depth, *cache, *O, *LSE;
    Shape s;
    if (Q == nullptr || K == nullptr || V == nullptr || !shapes(*Q, *K, *V, s) || !optional_dense(a[3], depth) || !optional_dense(a[6], cache) ||
        !optional_dense(a[8], O) || !optional_dense(a[9], LSE)) return none();
    if (!holds(O, at::kBFloat16, Q->numel()) || !holds(LSE, at::kFloat, rows(s)) || (l > 0 && !holds_slots(depth, s, l)) || !holds_slot(cache, s, slot)) return none();
    Tensor o = O != nullptr ? *O : Tensor(), lse = LSE != nullptr ? *LSE : Tensor();
    {
        NoGil nogil;
        forward(s, *Q, *K, *V, depth, l, scale, cache, slot, o, lse);
    }
    return Py_BuildValue("NN", out(a[8], o), out(a[9], lse));
    END_HANDLE_TH_ERRORS
}

// attn_bwd(Q, K, V, depth, O, dO, LSE, l, scale, dQ, dK, dV, dcache, workspace, stages or None) -> (dQ, dK, dV, dcache); with one argument more: the one before it is a slot
PyObject* attn_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int l, arg = -1;
    float scale;
    if (n < 15 || n > 16 || !plain_thread() || !int_arg(a[7], l) || l < 0 || !float_arg(a[8], scale)) return none();
    if (a[14] != Py_None && (!int_arg(a[14], arg) || arg < 0)) return none();
    const Mode mode = n == 16 ? kSlot : a[14] == Py_None ? kWhole : kMask;
    if (mode == kSlot && (a[12] == Py_None || a[14] == Py_None)) return none();
    const Tensor *Q = dense(a[0], at::kBFloat16, 4), *K = dense(a[1], at::kBFloat16, 4), *V = dense(a[2], at::kBFloat16, 4);
    const Tensor *depth, *O, *dO, *LSE, *g[5];
    Shape s;
    if (Q == nullptr || K == nullptr || V == nullptr || !shapes(*Q, *K, *V, s) || !optional_dense(a[3], depth)) return none();
    if (!optional_dense(a[4], O) || !optional_dense(a[5], dO) || !optional_dense(a[6], LSE) || O == nullptr || dO == nullptr || LSE == nullptr) return none();
    for (int i = 0; i < 5; ++i)
        if (!optional_dense(a[9 + i], g[i])) return none();
    const int64_t nq = Q->numel(), nk = K->numel();
    if (!holds(O, at::kBFloat16, nq) || !holds(dO, at::kBFloat16, nq) || !holds(LSE, at::kFloat, rows(s)) || !holds(g[0], at::kBFloat16, nq) ||
        !holds(g[1], at::kBFloat16, nk) || !holds(g[2], at::kBFloat16, nk)) return none();
    if ((l > 0 && (!holds_slots(depth, s, l) || !holds_slots(g[3], s, l))) || (mode == kSlot && !holds_slot(g[3], s, arg))) return none();
    // no gradient cache can be made for this width or so many slots: the Python form says so
    if (l > 0 && g[3] == nullptr && lib.moda_depth_cache_bytes(s.B, s.T, s.Hk, s.d, l) == 0) return none();
    Tensor t[5];
    for (int i = 0; i < 5; ++i)
        if (g[i] != nullptr) t[i] = *g[i];
    {
        NoGil nogil;
        backward(s, *Q, *K, *V, depth, *O, *dO, *LSE, l, scale, mode, arg, t[0], t[1], t[2], t[3], t[4]);
    }
    return Py_BuildValue("NNNN", out(a[9], t[0]), out(a[10], t[1]), out(a[11], t[2]), t[3].defined() ? out(a[12], t[3]) : none());
    END_HANDLE_TH_ERRORS
}

// ---- the differentiable call ------------------------------------------------------------------------------------------
constexpr const char* kBadShapes = "K and V must be bf16 [B, T, H_kv, d] tensors matching Q's B, T and d";
void addressable(const Tensor& t) {
    TORCH_CHECK_VALUE(t.defined() && t.is_cuda(), "device (CUDA) tensors required");
    TORCH_CHECK_VALUE(t.is_contiguous(), "contiguous tensors required");
}
struct Attention : torch::autograd::Function<Attention> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const Tensor& Q_, const Tensor& K_, const Tensor& V_,
                                                  const std::optional<Tensor>& depth_, int64_t l, double scale) {
        const Tensor Q = Q_.contiguous(), K = K_.contiguous(), V = V_.contiguous(), depth = l > 0 ? *depth_ : Tensor();
        Shape s;
        TORCH_CHECK_VALUE(shapes(Q, K, V, s), kBadShapes);
        Tensor O, LSE;
        ::forward(s, Q, K, V, l > 0 ? &depth : nullptr, int(l), float(scale), nullptr, 0, O, LSE);
        ctx->save_for_backward({Q, K, V, depth, O, LSE});
        ctx->saved_data["l"] = l;
        ctx->saved_data["scale"] = scale;
        if (l > 0) ctx->saved_data["type"] = int64_t(depth.scalar_type());
        ctx->mark_non_differentiable({LSE});
        ctx->set_materialize_grads(false);                     // nothing to fill for LSE
        return {O, LSE};
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, const torch::autograd::variable_list& grads) {
        const auto saved = ctx->get_saved_variables();
        const Tensor &Q = saved[0], &K = saved[1], &V = saved[2], &depth = saved[3], &O = saved[4], &LSE = saved[5];
        const int l = int(ctx->saved_data["l"].toInt());
        const float scale = float(ctx->saved_data["scale"].toDouble());
        const Tensor dO = grads[0].defined() ? grads[0].contiguous() : at::zeros_like(O);
        // Saved-tensor hooks may hand back anything, and torch does not look at it: every tensor again, before a kernel gets its address.
        Shape s;
        for (const Tensor* t : {&Q, &K, &V, &O, &LSE, &dO}) addressable(*t);
        TORCH_CHECK_VALUE(shapes(Q, K, V, s), kBadShapes);
        TORCH_CHECK_VALUE(holds(&O, at::kBFloat16, Q.numel()) && holds(&dO, at::kBFloat16, Q.numel()),
                          "O and its gradient must be bf16 tensors of Q's size");
        TORCH_CHECK_VALUE(holds(&LSE, at::kFloat, rows(s)), "LSE must be an fp32 tensor of B H T elements");
        if (l > 0) {
            addressable(depth);
            TORCH_CHECK_VALUE(int64_t(depth.scalar_type()) == ctx->saved_data["type"].toInt(), "depth_kv has changed its type");
            TORCH_CHECK_VALUE(holds_slots(&depth, s, l), "depth_kv holds fewer than l slots");
        }
        Tensor dQ, dK, dV, dcache, ws;
        if (l > 0) {
            // the kernels write every element of slots < l; later slots of the caller's cache get no gradient
            dcache = at::empty_like(depth);
            const int64_t slots = int64_t(lib.moda_depth_cache_bytes(s.B, s.T, s.Hk, s.d, l) / 2);
            if (slots < depth.numel()) dcache.view({-1}).slice(0, slots).zero_();
        }
        ::backward(s, Q, K, V, l > 0 ? &depth : nullptr, O, dO, LSE, l, scale, kWhole, 0, dQ, dK, dV, dcache, ws);
        return {dQ, dK, dV, dcache, Tensor(), Tensor()};
    }
};

bool dual(const Tensor& t) { return t._fw_grad(0).defined(); }

// attention(Q, K, V, depth or None, l, scale) -> (O, LSE)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int l;
    float scale;
    if (n != 6 || !plain_thread() || !int_arg(a[4], l) || l < 0 || !float_arg(a[5], scale)) return none();
    const Tensor *Q = plain(a[0]), *K = plain(a[1]), *V = plain(a[2]), *depth;
    Shape s;
    if (Q == nullptr || K == nullptr || V == nullptr || !shapes(*Q, *K, *V, s) || !optional_dense(a[3], depth) || (l > 0 && (depth == nullptr || !holds_slots(depth, s, l)))) return none();
    if (dual(*Q) || dual(*K) || dual(*V) || (depth != nullptr && dual(*depth))) return none();
    const Tensor q = *Q, k = *K, v = *V;
    const std::optional<Tensor> dep = depth != nullptr ? std::optional<Tensor>(*depth) : std::nullopt;
    torch::autograd::variable_list r;
    {
        NoGil nogil;
        r = Attention::apply(q, k, v, dep, int64_t(l), PyFloat_AS_DOUBLE(a[5]));
    }
    return Py_BuildValue("NN", THPVariable_Wrap(r[0]), THPVariable_Wrap(r[1]));
    END_HANDLE_TH_ERRORS
}

// ---- decode steps -----------------------------------------------------------------------------------------------------
// decode(q, K, V, table or None, seq_lens or None, depth, T_kv, l, scale, O, LSE, workspace) -> (O, LSE): one length for all
// sequences, a length for each, or pages
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int T_kv, l;
    float scale;
    if (n != 12 || !plain_thread() || !int_arg(a[6], T_kv) || !int_arg(a[7], l) || l < 0 || !float_arg(a[8], scale)) return none();
    const Tensor *q = dense(a[0], at::kBFloat16, 3), *K = dense(a[1], at::kBFloat16, 4), *V = dense(a[2], at::kBFloat16, 4);
    if (q == nullptr || K == nullptr || V == nullptr || !small(*q) || !small(*K) || V->sizes() != K->sizes() || K->size(3) != q->size(2)) return none();
    const int B = int(q->size(0)), H = int(q->size(1)), d = int(q->size(2)), Hk = int(K->size(2));
    const bool varlen = a[4] != Py_None, paged = a[3] != Py_None;
    const Tensor *lens = nullptr, *table = nullptr, *depth = nullptr, *O, *LSE, *ws;
    if (varlen && ((lens = dense(a[4], at::kInt, 1)) == nullptr || lens->size(0) != B)) return none();
    if (paged) {
        if (!varlen || (table = dense(a[3], at::kInt, 2)) == nullptr || table->size(0) != B || !small(*table)) return none();
    } else if (K->size(0) != B) {
        return none();
    }
    if (l > 0 && ((depth = dense(a[5], at::kBFloat16, 5)) == nullptr || !shape_is(*depth, {l, B, Hk, 2, d}))) return none();
    if (!optional_dense(a[9], O) || !optional_dense(a[10], LSE) || !optional_dense(a[11], ws)) return none();
    if (!holds(O, at::kBFloat16, q->numel()) || !holds(LSE, at::kFloat, int64_t(B) * H)) return none();
    Tensor o = O != nullptr ? *O : Tensor(), lse = LSE != nullptr ? *LSE : Tensor(), w = ws != nullptr ? *ws : Tensor();
    {
        NoGil nogil;
        if (!o.defined()) o = like(*q);
        if (!lse.defined()) lse = fresh({B, H}, at::kFloat, *q);
        if (!w.defined()) w = fresh({int64_t(lib.moda_decode_workspace_bytes(B, H, d))}, at::kByte, *q);
        float* lse_p = static_cast<float*>(lse.data_ptr());
        const int* lens_p = varlen ? static_cast<const int*>(lens->data_ptr()) : nullptr;
        int rc;
        if (paged)
            rc = lib.moda_attn_decode_paged(q->data_ptr(), K->data_ptr(), V->data_ptr(), static_cast<const int*>(table->data_ptr()), lens_p,
                                            ptr(depth), B, T_kv, int(K->size(1)), int(K->size(0)), int(table->size(1)), H, Hk, d, l, scale,
                                            o.data_ptr(), lse_p, w.data_ptr(), bytes_of(w), stream());
        else if (varlen)
            rc = lib.moda_attn_decode_varlen(q->data_ptr(), K->data_ptr(), V->data_ptr(), lens_p, ptr(depth), B, T_kv, int(K->size(1)), H, Hk,
                                             d, l, scale, o.data_ptr(), lse_p, w.data_ptr(), bytes_of(w), stream());
        else
            rc = lib.moda_attn_decode(q->data_ptr(), K->data_ptr(), V->data_ptr(), ptr(depth), B, T_kv, int(K->size(1)), H, Hk, d, l, scale,
                                      o.data_ptr(), lse_p, w.data_ptr(), bytes_of(w), stream());
        if (rc != 0) fail(rc, paged ? "moda_attn_decode_paged" : varlen ? "moda_attn_decode_varlen" : "moda_attn_decode");
    }
    return Py_BuildValue("NN", out(a[9], o), out(a[10], lse));
    END_HANDLE_TH_ERRORS
}

// ---- attention weight of cached keys, eviction, shared prefix ------------------------------------------------------------
bool tensor_of(const Tensor* t, at::ScalarType type, std::initializer_list<int64_t> shape) { return t == nullptr || (t->scalar_type() == type && shape_is(*t, shape)); }
bool lens_arg(PyObject* o, int B, const Tensor*& t) {
    t = nullptr;
    return o == Py_None || ((t = dense(o, at::kInt, 1)) != nullptr && t->size(0) == B);
}
Tensor scratch(const Tensor* given, size_t bytes, const Tensor& on) {
    return given != nullptr ? *given : fresh({int64_t(std::max<size_t>(bytes, 16))}, at::kByte, on);
}
float* f32(const Tensor* t) { return static_cast<float*>(ptr(t)); }
const int* i32(const Tensor* t) { return static_cast<const int*>(ptr(t)); }

// key_mass(Q, K, LSE, scale, T_kv or None, mass_in, mass, workspace) -> mass
PyObject* key_mass(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    float scale;
    int T_kv;
    if (n != 8 || !plain_thread() || !float_arg(a[3], scale)) return none();
    const Tensor *Q = dense(a[0], at::kBFloat16, 4), *K = dense(a[1], at::kBFloat16, 4), *LSE = dense(a[2], at::kFloat, 3), *old, *mass, *ws;
    if (Q == nullptr || K == nullptr || LSE == nullptr || !small(*Q) || !small(*K)) return none();
    const int B = int(Q->size(0)), T_q = int(Q->size(1)), H = int(Q->size(2)), d = int(Q->size(3)), T_cap = int(K->size(1)), Hk = int(K->size(2));
    if (K->size(0) != B || K->size(3) != d || !shape_is(*LSE, {B, H, T_q})) return none();
    if (a[4] == Py_None) T_kv = T_cap;
    else if (!int_arg(a[4], T_kv)) return none();
    if (!optional_dense(a[5], old) || !optional_dense(a[6], mass) || !optional_dense(a[7], ws)) return none();
    if (!tensor_of(old, at::kFloat, {B, Hk, T_cap}) || !tensor_of(mass, at::kFloat, {B, Hk, T_cap})) return none();
    Tensor m = mass != nullptr ? *mass : Tensor();
    {
        NoGil nogil;
        if (!m.defined()) m = fresh({B, Hk, T_cap}, at::kFloat, *Q);
        const Tensor w = scratch(ws, ws != nullptr ? 0 : lib.moda_key_mass_workspace_bytes(B, T_q, T_kv, H, Hk, d), *Q);
        const int rc = lib.moda_attn_key_mass(Q->data_ptr(), K->data_ptr(), f32(LSE), f32(old), B, T_q, T_kv, T_cap, H, Hk, d, scale, f32(&m), w.data_ptr(),
                                              bytes_of(w), stream());
        if (rc != 0) fail(rc, "moda_attn_key_mass");
    }
    return out(a[6], m);
    END_HANDLE_TH_ERRORS
}

// What the two decode steps below have in common.
struct Step { int B, H, d, T_cap, Hk, T, l; float scale; const Tensor *q, *K, *V, *lens, *depth; };
bool step_args(PyObject* q, PyObject* K, PyObject* V, PyObject* lens, PyObject* depth, PyObject* T, PyObject* l, PyObject* scale, Step& s) {
    if (!int_arg(T, s.T) || !int_arg(l, s.l) || s.l < 0 || !float_arg(scale, s.scale)) return false;
    s.q = dense(q, at::kBFloat16, 3);
    s.K = dense(K, at::kBFloat16, 4);
    s.V = dense(V, at::kBFloat16, 4);
    if (s.q == nullptr || s.K == nullptr || s.V == nullptr || !small(*s.q) || !small(*s.K) || s.V->sizes() != s.K->sizes()) return false;
    s.B = int(s.q->size(0)), s.H = int(s.q->size(1)), s.d = int(s.q->size(2)), s.T_cap = int(s.K->size(1)), s.Hk = int(s.K->size(2));
    if (s.K->size(0) != s.B || s.K->size(3) != s.d || !lens_arg(lens, s.B, s.lens)) return false;
    s.depth = nullptr;
    return s.l == 0 || ((s.depth = dense(depth, at::kBFloat16, 5)) != nullptr && shape_is(*s.depth, {s.l, s.B, s.Hk, 2, s.d}));
}
bool step_outputs(const Step& s, PyObject* o, PyObject* lse, PyObject* work, const Tensor*& O, const Tensor*& LSE, const Tensor*& ws) {
    return optional_dense(o, O) && optional_dense(lse, LSE) && optional_dense(work, ws) && holds(O, at::kBFloat16, s.q->numel()) &&
           holds(LSE, at::kFloat, int64_t(s.B) * s.H);
}

// decode_mass(q, K, V, seq_lens or None, depth, T, l, scale, mass_in, mass, O, LSE, workspace) -> (O, LSE, mass)
PyObject* decode_mass(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Step s;
    const Tensor *old, *mass, *O, *LSE, *ws;
    if (n != 13 || !plain_thread() || !step_args(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], s) || !step_outputs(s, a[10], a[11], a[12], O, LSE, ws)) return none();
    if (!optional_dense(a[8], old) || !optional_dense(a[9], mass)) return none();
    if (!tensor_of(old, at::kFloat, {s.B, s.Hk, s.T_cap}) || !tensor_of(mass, at::kFloat, {s.B, s.Hk, s.T_cap})) return none();
    Tensor o = O != nullptr ? *O : Tensor(), lse = LSE != nullptr ? *LSE : Tensor(), m = mass != nullptr ? *mass : Tensor();
    {
        NoGil nogil;
        if (!o.defined()) o = like(*s.q);
        if (!lse.defined()) lse = fresh({s.B, s.H}, at::kFloat, *s.q);
        if (!m.defined()) m = fresh({s.B, s.Hk, s.T_cap}, at::kFloat, *s.q);
        const Tensor w = scratch(ws, ws != nullptr ? 0 : lib.moda_decode_mass_workspace_bytes(s.B, s.T, s.H, s.Hk, s.d), *s.q);
        const int rc = lib.moda_attn_decode_mass(s.q->data_ptr(), s.K->data_ptr(), s.V->data_ptr(), i32(s.lens), ptr(s.depth), f32(old), s.B, s.T, s.T_cap, s.H, s.Hk,
                                                 s.d, s.l, s.scale, o.data_ptr(), f32(&lse), f32(&m), w.data_ptr(), bytes_of(w), stream());
        if (rc != 0) fail(rc, "moda_attn_decode_mass");
    }
    return Py_BuildValue("NNN", out(a[10], o), out(a[11], lse), out(a[9], m));
    END_HANDLE_TH_ERRORS
}

// evict(K, V, mass, T, n_keep, n_recent, seq_lens or None, K_out, V_out, mass_out, index, lens_out) -> (K_out, V_out, mass_out, index, lens_out)
PyObject* evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int T, keep, recent;
    if (n != 12 || !plain_thread() || !int_arg(a[3], T) || !int_arg(a[4], keep) || !int_arg(a[5], recent) || keep < 1) return none();
    const Tensor *K = dense(a[0], at::kBFloat16, 4), *V = dense(a[1], at::kBFloat16, 4), *mass = dense(a[2], at::kFloat, 3), *lens, *g[5];
    if (K == nullptr || V == nullptr || mass == nullptr || !small(*K) || V->sizes() != K->sizes()) return none();
    const int B = int(K->size(0)), T_cap = int(K->size(1)), Hk = int(K->size(2)), d = int(K->size(3));
    if (!shape_is(*mass, {B, Hk, T_cap}) || !lens_arg(a[6], B, lens)) return none();
    for (int i = 0; i < 5; ++i)
        if (!optional_dense(a[7 + i], g[i])) return none();
    int64_t T_out = keep;
    if (g[0] != nullptr && g[0]->dim() == 4) T_out = g[0]->size(1);
    if (T_out > INT_MAX || !tensor_of(g[0], at::kBFloat16, {B, T_out, Hk, d}) || !tensor_of(g[1], at::kBFloat16, {B, T_out, Hk, d}) ||
        !tensor_of(g[2], at::kFloat, {B, Hk, T_out}) || !tensor_of(g[3], at::kInt, {B, Hk, keep}) || !tensor_of(g[4], at::kInt, {B})) return none();
    Tensor t[5];
    for (int i = 0; i < 5; ++i)
        if (g[i] != nullptr) t[i] = *g[i];
    {
        NoGil nogil;
        for (int i = 0; i < 2; ++i)
            if (!t[i].defined()) t[i] = fresh({B, T_out, Hk, d}, at::kBFloat16, *K);
        if (!t[2].defined()) t[2] = fresh({B, Hk, T_out}, at::kFloat, *K);
        if (!t[3].defined()) t[3] = fresh({B, Hk, keep}, at::kInt, *K);
        if (!t[4].defined()) t[4] = fresh({B}, at::kInt, *K);
        const int rc = lib.moda_kv_evict(K->data_ptr(), V->data_ptr(), f32(mass), i32(lens), B, T, T_cap, Hk, d, keep, recent, int(T_out), t[0].data_ptr(), t[1].data_ptr(),
                                         f32(&t[2]), static_cast<int*>(t[3].data_ptr()), static_cast<int*>(t[4].data_ptr()), stream());
        if (rc != 0) fail(rc, "moda_kv_evict");
    }
    return Py_BuildValue("NNNNN", out(a[7], t[0]), out(a[8], t[1]), out(a[9], t[2]), out(a[10], t[3]), out(a[11], t[4]));
    END_HANDLE_TH_ERRORS
}

// decode_shared(q, K_prefix, V_prefix, K, V, seq_lens or None, depth, T, l, scale, O, LSE, workspace) -> (O, LSE)
PyObject* decode_shared(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Step s;
    const Tensor *O, *LSE, *ws;
    if (n != 13 || !plain_thread() || !step_args(a[0], a[3], a[4], a[5], a[6], a[7], a[8], a[9], s) || !step_outputs(s, a[10], a[11], a[12], O, LSE, ws)) return none();
    const Tensor *Kp = dense(a[1], at::kBFloat16, 3), *Vp = dense(a[2], at::kBFloat16, 3);
    if (Kp == nullptr || Vp == nullptr || !small(*Kp) || Vp->sizes() != Kp->sizes() || Kp->size(1) != s.Hk || Kp->size(2) != s.d) return none();
    const int P = int(Kp->size(0));
    Tensor o = O != nullptr ? *O : Tensor(), lse = LSE != nullptr ? *LSE : Tensor();
    {
        NoGil nogil;
        if (!o.defined()) o = like(*s.q);
        if (!lse.defined()) lse = fresh({s.B, s.H}, at::kFloat, *s.q);
        const Tensor w = scratch(ws, ws != nullptr ? 0 : lib.moda_decode_shared_workspace_bytes(s.B, P, s.H, s.Hk, s.d), *s.q);
        const int rc = lib.moda_attn_decode_shared(s.q->data_ptr(), Kp->data_ptr(), Vp->data_ptr(), s.K->data_ptr(), s.V->data_ptr(), i32(s.lens), ptr(s.depth), s.B, P,
                                                   s.T, s.T_cap, s.H, s.Hk, s.d, s.l, s.scale, o.data_ptr(), f32(&lse), w.data_ptr(), bytes_of(w), stream());
        if (rc != 0) fail(rc, "moda_attn_decode_shared");
    }
    return Py_BuildValue("NN", out(a[10], o), out(a[11], lse));
    END_HANDLE_TH_ERRORS
}

// ---- the paged sequence cache in 8 bits ---------------------------------------------------------------------------------
// Pages, or their bounds (`per` d + `fixed` bytes a block), with the block table of a batch.
struct Paged { int page, pages, Hk, d, B, most; const Tensor *data, *table; };
bool paged_args(PyObject* data, PyObject* table, int per, int fixed, Paged& s) {
    s.data = dense(data, at::kByte, 4);
    s.table = dense(table, at::kInt, 2);
    if (s.data == nullptr || s.table == nullptr || !small(*s.data) || !small(*s.table) || s.data->size(1) > INT_MAX / 64) return false;
    const int64_t n = s.data->size(3) - fixed;
    if (n <= 0 || n % per != 0) return false;
    s.pages = int(s.data->size(0)), s.page = 64 * int(s.data->size(1)), s.Hk = int(s.data->size(2)), s.d = int(n / per);
    s.B = int(s.table->size(0)), s.most = int(s.table->size(1));
    return true;
}

// kv_write(pages, K, V, table, start or None, n_new or None, bounds or None) -> True
PyObject* kv_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Paged s;
    const Tensor *K = nullptr, *V = nullptr, *start, *count, *bounds = nullptr;
    if (n != 7 || !plain_thread() || !paged_args(a[0], a[3], 128, 512, s)) return none();
    if ((K = dense(a[1], at::kBFloat16, 4)) == nullptr || (V = dense(a[2], at::kBFloat16, 4)) == nullptr || !small(*K) || V->sizes() != K->sizes() ||
        K->size(0) != s.B || K->size(2) != s.Hk || K->size(3) != s.d || !lens_arg(a[4], s.B, start) || !lens_arg(a[5], s.B, count)) return none();
    if (a[6] != Py_None && ((bounds = dense(a[6], at::kByte, 4)) == nullptr || !shape_is(*bounds, {s.pages, s.page / 64, s.Hk, 2 * s.d + 16}))) return none();
    {
        NoGil nogil;
        const int rc = lib.moda_kv_write_e4m3(s.data->data_ptr(), ptr(bounds), K->data_ptr(), V->data_ptr(), i32(s.table), i32(start), i32(count), s.B, int(K->size(1)),
                                              s.page, s.pages, s.most, s.Hk, s.d, stream());
        if (rc != 0) fail(rc, "moda_kv_write_e4m3");
    }
    Py_RETURN_TRUE;
    END_HANDLE_TH_ERRORS
}

// kv_read(pages, table, seq_lens, T, start or None, K_out, V_out) -> (K_out, V_out), both given
PyObject* kv_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Paged s;
    int T;
    const Tensor *lens, *start, *g[2];
    if (n != 7 || !plain_thread() || !paged_args(a[0], a[1], 128, 512, s) || a[2] == Py_None || !lens_arg(a[2], s.B, lens) || !int_arg(a[3], T) ||
        !lens_arg(a[4], s.B, start)) return none();
    for (int i = 0; i < 2; ++i)
        if ((g[i] = dense(a[5 + i], at::kBFloat16, 4)) == nullptr || !shape_is(*g[i], {s.B, T, s.Hk, s.d})) return none();
    {
        NoGil nogil;
        const int rc = lib.moda_kv_read_e4m3(s.data->data_ptr(), i32(s.table), i32(lens), i32(start), s.B, T, s.page, s.pages, s.most, s.Hk, s.d, g[0]->data_ptr(),
                                             g[1]->data_ptr(), stream());
        if (rc != 0) fail(rc, "moda_kv_read_e4m3");
    }
    return Py_BuildValue("OO", a[5], a[6]);
    END_HANDLE_TH_ERRORS
}

// kv_select(q, bounds, table, seq_lens, max_seq_len, n_blocks, n_recent, index, workspace) -> index
PyObject* kv_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Paged s;
    int T, keep, recent;
    const Tensor *lens, *index, *q, *ws;
    if (n != 9 || !plain_thread() || !paged_args(a[1], a[2], 2, 16, s) || a[3] == Py_None || !lens_arg(a[3], s.B, lens) || !int_arg(a[4], T) ||
        !int_arg(a[5], keep) || !int_arg(a[6], recent) || keep < 1) return none();
    if ((q = dense(a[0], at::kBFloat16, 3)) == nullptr || !small(*q) || q->size(0) != s.B || q->size(2) != s.d || !optional_dense(a[7], index) ||
        !tensor_of(index, at::kInt, {s.B, s.Hk, keep}) || !optional_dense(a[8], ws)) return none();
    Tensor t = index != nullptr ? *index : Tensor();
    {
        NoGil nogil;
        if (!t.defined()) t = fresh({s.B, s.Hk, keep}, at::kInt, *q);
        const Tensor w = scratch(ws, ws != nullptr ? 0 : lib.moda_kv_select_workspace_bytes(s.B, T, s.Hk), *q);
        const int rc = lib.moda_kv_select_blocks(q->data_ptr(), s.data->data_ptr(), i32(s.table), i32(lens), s.B, T, s.page, s.pages, s.most, int(q->size(1)), s.Hk, s.d,
                                                 keep, recent, static_cast<int*>(t.data_ptr()), w.data_ptr(), bytes_of(w), stream());
        if (rc != 0) fail(rc, "moda_kv_select_blocks");
    }
    return out(a[7], t);
    END_HANDLE_TH_ERRORS
}

// decode_e4m3(q, pages, table, seq_lens, depth, max_seq_len, l, scale, index or None, O, LSE, workspace) -> (O, LSE)
PyObject* decode_e4m3(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Paged s;
    int T, l;
    float scale;
    const Tensor *q, *lens, *depth = nullptr, *index = nullptr, *O, *LSE, *ws;
    if (n != 12 || !plain_thread() || !paged_args(a[1], a[2], 128, 512, s) || a[3] == Py_None || !lens_arg(a[3], s.B, lens) || !int_arg(a[5], T) ||
        !int_arg(a[6], l) || l < 0 || !float_arg(a[7], scale)) return none();
    if ((q = dense(a[0], at::kBFloat16, 3)) == nullptr || !small(*q) || q->size(0) != s.B || q->size(2) != s.d) return none();
    if (l > 0 && ((depth = dense(a[4], at::kBFloat16, 5)) == nullptr || !shape_is(*depth, {l, s.B, s.Hk, 2, s.d}))) return none();
    if (a[8] != Py_None && ((index = dense(a[8], at::kInt, 3)) == nullptr || !small(*index) || index->size(0) != s.B || index->size(1) != s.Hk || index->size(2) < 1)) return none();
    const int H = int(q->size(1));
    if (!optional_dense(a[9], O) || !optional_dense(a[10], LSE) || !optional_dense(a[11], ws) || !holds(O, at::kBFloat16, q->numel()) ||
        !holds(LSE, at::kFloat, int64_t(s.B) * H)) return none();
    Tensor o = O != nullptr ? *O : Tensor(), lse = LSE != nullptr ? *LSE : Tensor();
    {
        NoGil nogil;
        if (!o.defined()) o = like(*q);
        if (!lse.defined()) lse = fresh({s.B, H}, at::kFloat, *q);
        const Tensor w = scratch(ws, ws != nullptr ? 0 : lib.moda_decode_e4m3_workspace_bytes(s.B, H, s.Hk, s.d), *q);
        const int rc = lib.moda_attn_decode_e4m3(q->data_ptr(), s.data->data_ptr(), i32(s.table), i32(lens), i32(index), index != nullptr ? int(index->size(2)) : 0, ptr(depth),
                                                 s.B, T, s.page, s.pages, s.most, H, s.Hk, s.d, l, scale, o.data_ptr(), f32(&lse), w.data_ptr(), bytes_of(w), stream());
        if (rc != 0) fail(rc, "moda_attn_decode_e4m3");
    }
    return Py_BuildValue("NN", out(a[9], o), out(a[10], lse));
    END_HANDLE_TH_ERRORS
}

// ---- module -----------------------------------------------------------------------------------------------------------
// bind(handle of libmoda_b200.so, check, DeviceContext): must come first
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 3) return PyErr_Format(PyExc_TypeError, "bind(handle, check, device_mode)");
    void* handle = PyLong_AsVoidPtr(a[0]);
    if (PyErr_Occurred()) return nullptr;
#define X(name)                                                                                            \
    lib.name = reinterpret_cast<decltype(&::name)>(dlsym(handle, #name));                                  \
    if (lib.name == nullptr) return PyErr_Format(PyExc_ImportError, "libmoda_b200.so has no %s", #name);
    MODA_HOST_CALLS(X)
#undef X
    Py_XSETREF(check_fn, Py_NewRef(a[1]));
    Py_XSETREF(device_mode, Py_NewRef(a[2]));
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f))
PyMethodDef methods[] = {
    {"bind", FAST(bind), METH_FASTCALL, nullptr},         {"attn_fwd", FAST(attn_fwd), METH_FASTCALL, nullptr},
    {"attn_bwd", FAST(attn_bwd), METH_FASTCALL, nullptr}, {"attention", FAST(attention), METH_FASTCALL, nullptr},
    {"decode", FAST(decode), METH_FASTCALL, nullptr},     {"key_mass", FAST(key_mass), METH_FASTCALL, nullptr},
    {"decode_mass", FAST(decode_mass), METH_FASTCALL, nullptr}, {"evict", FAST(evict), METH_FASTCALL, nullptr},
    {"decode_shared", FAST(decode_shared), METH_FASTCALL, nullptr}, {"kv_write", FAST(kv_write), METH_FASTCALL, nullptr},
    {"kv_read", FAST(kv_read), METH_FASTCALL, nullptr},   {"kv_select", FAST(kv_select), METH_FASTCALL, nullptr},
    {"decode_e4m3", FAST(decode_e4m3), METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() { return PyModule_Create(&module); }
