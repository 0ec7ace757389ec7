// The differentiable functions of autograd.py as native autograd nodes.
//
// What bounds a training step on a small batch is the host: on 256 samples of 64 rows on average the kernels of a step take
// 44 us, and through torch.autograd.Function the step took 105, since the backward of a Python function is entered on the
// engine's thread with the interpreter's lock to be handed over, and everything around the three launches is Python.  Here
// both directions are C++; the entry points of libjfa.so are called by the addresses that the ctypes binding has loaded.
//
// Only plain calls come here (see autograd.py): anything that the checks below do not find in order is answered with None, and
// the Python function, which raises what is to be raised, takes it.
#include <pybind11/functional.h>
#include <torch/extension.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <unordered_set>

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

// C ABI of include/jfa.h
using Forward = int (*)(const void *, const void *, const void *, const int64_t *, int64_t, int64_t, int, int, void *, float *, void *);
using Backward = int (*)(const void *, const void *, const void *, const void *, const void *, const float *, const int64_t *, int64_t, int64_t,
                         int, int, void *, void *, void *, float *, void *);
using ForwardCross = int (*)(const void *, const void *, const void *, const int64_t *, const int64_t *, int64_t, int64_t, int64_t, int, int,
                             void *, float *, void *);
using BackwardCross = int (*)(const void *, const void *, const void *, const void *, const void *, const float *, const int64_t *,
                              const int64_t *, int64_t, int64_t, int64_t, int, int, void *, void *, void *, float *, void *);

using ToDense = int (*)(const void *, const int64_t *, int64_t, int64_t, int64_t, uint32_t, void *, void *);
using ToJagged = int (*)(const void *, const int64_t *, int64_t, int64_t, int64_t, void *, void *);
using Product = int (*)(const void *, const void *, const int64_t *, int64_t, int64_t, int, int, void *, void *);
using Softmax = int (*)(const void *, const int64_t *, int64_t, int64_t, int, void *, void *);
using SoftmaxBackward = int (*)(const void *, const void *, const int64_t *, int64_t, int64_t, int, void *, void *);

using Linear = int (*)(const void *, const void *, const void *, const float *, const int64_t *, int64_t, int64_t, int64_t, int, int, float, const float *, void *,
                       float *, void *, size_t, void *);
using LinearBackward = int (*)(const void *, const void *, const void *, const void *, const float *, const int64_t *, int64_t, int64_t, int64_t, int, int, float,
                               const float *, const float *, void *, void *, void *, float *, void *, size_t, void *);
using LinearStep = int (*)(const void *, const void *, const void *, const float *, int64_t, int, int, float, const float *, void *, float *, void *);
using LinearWorkspace = size_t (*)(int64_t, int64_t, int64_t, int, int, int);
using Norm = int (*)(const void *, const void *, const void *, const int64_t *, int64_t, int64_t, int64_t, int64_t, float, void *, float *, float *, void *);
using NormBackward = int (*)(const void *, const void *, const void *, const float *, const float *, const int64_t *, int64_t, int64_t, int64_t, int64_t, void *,
                             void *, void *, void *, size_t, void *);
using Embed = int (*)(const void *, const void *, int, const int64_t *, int64_t, int64_t, int64_t, int64_t, float, void *, void *);
using EmbedBackward = int (*)(const void *, const void *, int, const int64_t *, int64_t, int64_t, int64_t, int64_t, float, void *, void *, size_t, void *);
using RowsWorkspace = size_t (*)(int64_t, int64_t, int64_t);

struct Library {   // [0]: bf16, [1]: fp32
    Linear linear[2];
    LinearBackward linear_backward[2];
    LinearStep linear_step[2];
    LinearWorkspace linear_workspace;
    Norm norm[2];
    NormBackward norm_backward[2];
    Embed embedding[2];
    EmbedBackward embedding_backward[2];
    RowsWorkspace norm_workspace, embedding_workspace;
    PyObject *parameter = nullptr;   // torch.nn.Parameter
    Forward forward[2], forward_causal[2];
    Backward backward[2], backward_causal[2];
    ForwardCross forward_cross[2];
    BackwardCross backward_cross[2];
    ToDense to_dense;
    ToJagged to_jagged;
    Product dense_bmm, jagged_bmm;
    Softmax softmax;
    SoftmaxBackward softmax_backward;
    PyObject *check = nullptr;   // binding._check: raises JfaError for a status that is not JFA_OK
    PyObject *pointer = nullptr;   // binding._ptr: raises AssertionError for a tensor that is not contiguous or not on the GPU
};
Library lib;

struct Refused {};   // the call is the Python function's

void *stream() { return c10::hip::getCurrentHIPStream().stream(); }

// In a backward, on the engine's thread: the error that a Python function raises for this argument.
void raise_from(PyObject *function, pybind11::object argument) {
    PyObject *r = PyObject_CallFunctionObjArgs(function, argument.ptr(), nullptr);
    Py_XDECREF(r);
    if (r) throw std::runtime_error("jfa backward failed");
    python_error e;
    e.persist();
    throw std::move(e);
}
void check_backward(int status) {
    if (status == 0) return;
    pybind11::gil_scoped_acquire gil;
    raise_from(lib.check, pybind11::int_(status));
}

bool plain(const Tensor &t) { return t.defined() && t.is_cuda() && t.is_contiguous(); }
bool plain_offsets(const Tensor &t) { return plain(t) && t.dim() == 1 && t.scalar_type() == at::kLong; }
int kind(const Tensor &q) {
    if (q.scalar_type() == at::kBFloat16) return 0;
    if (q.scalar_type() == at::kFloat) return 1;
    throw Refused{};
}
// What the graph gives back for a saved tensor is any tensor that a hook has made of it: it has to be what the kernels take it for.
// (The engine has made dout one of the output's size and type; a hook of the node comes after that.)
void check_on_gpu(const Tensor &t) {
    if (plain(t)) return;
    pybind11::gil_scoped_acquire gil;
    raise_from(lib.pointer, pybind11::cast(t));
}
int check_dout(const Tensor &dout) {
    check_on_gpu(dout);
    TORCH_CHECK(dout.dim() == 3 && (dout.scalar_type() == at::kBFloat16 || dout.scalar_type() == at::kFloat),
                "jagged attention, backward: a gradient of ", dout.sizes(), " ", dout.scalar_type());
    return dout.scalar_type() == at::kFloat;
}
void check_saved(const Tensor &t, at::IntArrayRef sizes, at::ScalarType type, const Tensor &dout) {
    check_on_gpu(t);
    TORCH_CHECK(t.sizes() == sizes && t.scalar_type() == type && t.device() == dout.device(), "jagged attention, backward: a tensor of ", sizes, " ",
                type, " on ", dout.device(), " was saved, ", t.sizes(), " ", t.scalar_type(), " on ", t.device(), " came back");
}
float *floats(const Tensor &t) { return static_cast<float *>(t.data_ptr()); }
const int64_t *longs(const Tensor &t) { return static_cast<const int64_t *>(t.data_ptr()); }
Tensor statistics(const Tensor &q, int64_t planes) { return at::empty({planes, q.size(1), q.size(0)}, q.options().dtype(at::kFloat)); }

struct SelfAttention : torch::autograd::Function<SelfAttention> {
    static Tensor forward(AutogradContext *ctx, const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &offsets, int64_t max_len, bool causal) {
        const int f32 = kind(q);
        const Tensor out = at::empty_like(q), lse = at::empty({q.size(1), q.size(0)}, q.options().dtype(at::kFloat));
        const Forward fn = (causal ? lib.forward_causal : lib.forward)[f32];
        int status;
        {
            pybind11::gil_scoped_release nogil;
            status = fn(q.data_ptr(), k.data_ptr(), v.data_ptr(), longs(offsets), offsets.numel() - 1, max_len, (int)q.size(1), (int)q.size(2),
                        out.data_ptr(), floats(lse), stream());
        }
        if (status != 0) throw Refused{};   // the Python function meets the same error and reports it
        ctx->save_for_backward({q, k, v, out, lse, offsets});
        ctx->saved_data["call"] = std::vector<int64_t>{max_len, causal, offsets.numel()};
        return out;
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads) {
        const variable_list saved = ctx->get_saved_variables();
        const Tensor &q = saved[0], &k = saved[1], &v = saved[2], &out = saved[3], &lse = saved[4], &offsets = saved[5];
        const Tensor dout = grads[0].contiguous();
        const std::vector<int64_t> call = ctx->saved_data["call"].toIntVector();   // max_len, causal, offsets' length
        const int f32 = check_dout(dout);
        for (const Tensor *t : {&q, &k, &v, &out}) check_saved(*t, dout.sizes(), dout.scalar_type(), dout);
        check_saved(lse, {dout.size(1), dout.size(0)}, at::kFloat, dout);
        check_saved(offsets, call[2], at::kLong, dout);
        const Tensor dq = at::empty_like(q), dk = at::empty_like(q), dv = at::empty_like(q), stats = statistics(q, f32 ? 1 : 2);
        const Backward fn = (call[1] ? lib.backward_causal : lib.backward)[f32];
        check_backward(fn(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), dout.data_ptr(), floats(lse), longs(offsets), offsets.numel() - 1,
                          call[0], (int)q.size(1), (int)q.size(2), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                          floats(stats), stream()));
        return {dq, dk, dv, Tensor(), Tensor(), Tensor()};
    }
};

struct CrossAttention : torch::autograd::Function<CrossAttention> {
    static Tensor forward(AutogradContext *ctx, const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &offsets_q, const Tensor &offsets_kv,
                          int64_t max_len_q, int64_t max_len_kv) {
        const int f32 = kind(q);
        const Tensor out = at::empty_like(q), lse = at::empty({q.size(1), q.size(0)}, q.options().dtype(at::kFloat));
        int status;
        {
            pybind11::gil_scoped_release nogil;
            status = lib.forward_cross[f32](q.data_ptr(), k.data_ptr(), v.data_ptr(), longs(offsets_q), longs(offsets_kv), offsets_q.numel() - 1,
                                            max_len_q, max_len_kv, (int)q.size(1), (int)q.size(2), out.data_ptr(), floats(lse), stream());
        }
        if (status != 0) throw Refused{};
        ctx->save_for_backward({q, k, v, out, lse, offsets_q, offsets_kv});
        ctx->saved_data["call"] = std::vector<int64_t>{max_len_q, max_len_kv, offsets_q.numel(), k.size(0)};
        return out;
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads) {
        const variable_list saved = ctx->get_saved_variables();
        const Tensor &q = saved[0], &k = saved[1], &v = saved[2], &out = saved[3], &lse = saved[4], &offsets_q = saved[5], &offsets_kv = saved[6];
        const Tensor dout = grads[0].contiguous();
        const std::vector<int64_t> call = ctx->saved_data["call"].toIntVector();   // max_len_q, max_len_kv, offsets' length, rows of k
        const int f32 = check_dout(dout);
        for (const Tensor *t : {&q, &out}) check_saved(*t, dout.sizes(), dout.scalar_type(), dout);
        for (const Tensor *t : {&k, &v}) check_saved(*t, {call[3], dout.size(1), dout.size(2)}, dout.scalar_type(), dout);
        check_saved(lse, {dout.size(1), dout.size(0)}, at::kFloat, dout);
        for (const Tensor *t : {&offsets_q, &offsets_kv}) check_saved(*t, call[2], at::kLong, dout);
        const Tensor dq = at::empty_like(q), dk = at::empty_like(k), dv = at::empty_like(v), stats = statistics(q, f32 ? 1 : 2);
        check_backward(lib.backward_cross[f32](q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), dout.data_ptr(), floats(lse), longs(offsets_q),
                                               longs(offsets_kv), offsets_q.numel() - 1, call[0], call[1], (int)q.size(1), (int)q.size(2), dq.data_ptr(), dk.data_ptr(),
                                               dv.data_ptr(), floats(stats), stream()));
        return {dq, dk, dv, Tensor(), Tensor(), Tensor(), Tensor()};
    }
};

std::optional<Tensor> self_attention(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &offsets, int64_t max_len, bool causal) {
    if (!plain(q) || !plain(k) || !plain(v) || !plain_offsets(offsets) || q.dim() != 3 || k.sizes() != q.sizes() || v.sizes() != q.sizes() ||
        k.scalar_type() != q.scalar_type() || v.scalar_type() != q.scalar_type())
        return std::nullopt;
    try {
        return SelfAttention::apply(q, k, v, offsets, max_len, causal);
    } catch (const Refused &) {
        return std::nullopt;
    }
}

std::optional<Tensor> cross_attention(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &offsets_q, const Tensor &offsets_kv,
                                      int64_t max_len_q, int64_t max_len_kv) {
    if (!plain(q) || !plain(k) || !plain(v) || !plain_offsets(offsets_q) || !plain_offsets(offsets_kv) || q.dim() != 3 || k.dim() != 3 ||
        k.sizes() != v.sizes() || k.size(1) != q.size(1) || k.size(2) != q.size(2) || k.scalar_type() != q.scalar_type() ||
        v.scalar_type() != q.scalar_type() || offsets_q.numel() != offsets_kv.numel())
        return std::nullopt;
    try {
        return CrossAttention::apply(q, k, v, offsets_q, offsets_kv, max_len_q, max_len_kv);
    } catch (const Refused &) {
        return std::nullopt;
    }
}

// ---- the binding's calls without gradients, results allocated here ----
// What bounds a call on a small batch is the host again: the ctypes call and the Python around it took 7.5 us, twice a small batch's
// kernel; from here a call takes 4.4 (four bf16 samples of up to 64 rows; fp32, where the kernel takes longer, 5.4).  The functions take the arguments as the interpreter has them; whatever
// is not exactly what they expect, and whatever goes wrong, is answered with None: the Python function takes the call and raises what there is to raise.
const Tensor *exact_tensor(PyObject *o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const Tensor &t = THPVariable_Unpack(o);
    using c10::DispatchKey;
    // tensors that stand for others (function transforms, fake and functional tensors) have one of these keys
    constexpr c10::DispatchKeySet stands_for_others({DispatchKey::Python, DispatchKey::Functionalize, DispatchKey::FuncTorchBatched,
                                                     DispatchKey::FuncTorchGradWrapper, DispatchKey::BatchedNestedTensor, DispatchKey::Conjugate,
                                                     DispatchKey::Negative, DispatchKey::ZeroTensor});
    return t.key_set().has_any(stands_for_others) || !plain(t) ? nullptr : &t;
}
bool as_int64(PyObject *o, int64_t *x) {
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    *x = PyLong_AsLongLongAndOverflow(o, &overflow);
    return overflow == 0;
}
bool nobody_listens() {   // no function mode, dispatch mode, function transform or tracer is to see the allocations
    using c10::DispatchKey;
    constexpr c10::DispatchKeySet modes({DispatchKey::Python, DispatchKey::PythonTLSSnapshot, DispatchKey::FuncTorchDynamicLayerFrontMode,
                                         DispatchKey::FuncTorchVmapMode, DispatchKey::Functionalize});
    return !c10::impl::tls_local_dispatch_key_set().included_.has_any(modes) && !torch::jit::tracer::isTracing() && !at::impl::torch_function_mode_enabled();
}
// (q, k, v, offsets, max_len, causal), or with offsets_kv, max_len_q, max_len_kv for cross attention
template <bool kCross> PyObject *forward_call(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    int64_t max_len = 0, max_len_kv = 0;
    const Tensor *q, *k, *v, *offsets, *offsets_kv = nullptr;
    if (n_args != (kCross ? 7 : 6) || !nobody_listens() || !(q = exact_tensor(args[0])) || !(k = exact_tensor(args[1])) || !(v = exact_tensor(args[2])) ||
        !(offsets = exact_tensor(args[3])) || (kCross && !(offsets_kv = exact_tensor(args[4]))) || !as_int64(args[kCross ? 5 : 4], &max_len) ||
        (kCross && !as_int64(args[6], &max_len_kv)) || (!kCross && !PyBool_Check(args[5])))
        Py_RETURN_NONE;
    const at::ScalarType type = q->scalar_type();
    const bool shapes = q->dim() == 3 && k->dim() == 3 && k->sizes() == v->sizes() &&
                        (kCross ? k->size(1) == q->size(1) && k->size(2) == q->size(2) && offsets_kv->numel() == offsets->numel() : k->sizes() == q->sizes());
    if (!shapes || (type != at::kBFloat16 && type != at::kFloat) || k->scalar_type() != type || v->scalar_type() != type || !plain_offsets(*offsets) ||
        (kCross && !plain_offsets(*offsets_kv)))
        Py_RETURN_NONE;
    const int f32 = type == at::kFloat;
    Tensor out, lse;
    int status;
    {
        pybind11::gil_scoped_release nogil;
        out = at::empty(q->sizes(), q->options());
        lse = at::empty({q->size(1), q->size(0)}, q->options().dtype(at::kFloat));
        const int64_t B = offsets->numel() - 1;
        const int H = (int)q->size(1), D = (int)q->size(2);
        if constexpr (kCross)
            status = lib.forward_cross[f32](q->data_ptr(), k->data_ptr(), v->data_ptr(), longs(*offsets), longs(*offsets_kv), B, max_len, max_len_kv, H, D,
                                            out.data_ptr(), floats(lse), stream());
        else
            status = (args[5] == Py_True ? lib.forward_causal : lib.forward)[f32](q->data_ptr(), k->data_ptr(), v->data_ptr(), longs(*offsets), B, max_len, H, D,
                                                                                 out.data_ptr(), floats(lse), stream());
    }
    if (status != 0) Py_RETURN_NONE;
    PyObject *pair = PyTuple_New(2);
    if (!pair) return nullptr;
    PyTuple_SET_ITEM(pair, 0, THPVariable_Wrap(std::move(out)));
    PyTuple_SET_ITEM(pair, 1, THPVariable_Wrap(std::move(lse)));
    return pair;
    END_HANDLE_TH_ERRORS
}
// (values, offsets, max_len): rows past a sample's end become zeros
PyObject *to_dense_call(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    int64_t max_len = 0;
    const Tensor *values, *offsets;
    if (n_args != 3 || !nobody_listens() || !(values = exact_tensor(args[0])) || !(offsets = exact_tensor(args[1])) || !as_int64(args[2], &max_len) ||
        max_len < 0 || values->dim() < 1 || !plain_offsets(*offsets) || offsets->numel() < 1)
        Py_RETURN_NONE;
    std::vector<int64_t> sizes{offsets->numel() - 1, max_len};
    int64_t row_bytes = (int64_t)values->element_size();
    for (int64_t d = 1; d < values->dim(); ++d) {
        sizes.push_back(values->size(d));
        row_bytes *= values->size(d);
    }
    Tensor dense;
    int status;
    {
        pybind11::gil_scoped_release nogil;
        dense = at::empty(sizes, values->options());
        status = lib.to_dense(values->data_ptr(), longs(*offsets), sizes[0], max_len, row_bytes, 0, dense.data_ptr(), stream());
    }
    if (status != 0) Py_RETURN_NONE;
    return THPVariable_Wrap(std::move(dense));
    END_HANDLE_TH_ERRORS
}
// (dense, offsets, values): values, filled
PyObject *to_jagged_call(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    const Tensor *dense, *offsets, *values;
    if (n_args != 3 || !nobody_listens() || !(dense = exact_tensor(args[0])) || !(offsets = exact_tensor(args[1])) || !(values = exact_tensor(args[2])) ||
        dense->dim() < 2 || values->dim() < 1 || !plain_offsets(*offsets) || offsets->numel() - 1 != dense->size(0))
        Py_RETURN_NONE;
    int64_t row_bytes = (int64_t)dense->element_size(), values_row = (int64_t)values->element_size();
    for (int64_t d = 2; d < dense->dim(); ++d) row_bytes *= dense->size(d);
    for (int64_t d = 1; d < values->dim(); ++d) values_row *= values->size(d);
    if (row_bytes != values_row) Py_RETURN_NONE;
    int status;
    {
        pybind11::gil_scoped_release nogil;
        status = lib.to_jagged(dense->data_ptr(), longs(*offsets), dense->size(0), dense->size(1), row_bytes, values->data_ptr(), stream());
    }
    if (status != 0) Py_RETURN_NONE;
    Py_INCREF(args[2]);
    return args[2];
    END_HANDLE_TH_ERRORS
}
// The feature operators on bf16: (x, w or y, offsets, max_len), the softmax (x, offsets, max_len)
enum class Feature { kDenseBmm, kJaggedBmm, kSoftmax, kSoftmaxBackward };
template <Feature kOp> PyObject *feature_call(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    constexpr int kTensors = kOp == Feature::kSoftmax ? 1 : 2;
    int64_t max_len = 0;
    const Tensor *a, *b = nullptr, *offsets;
    if (n_args != kTensors + 2 || !nobody_listens() || !(a = exact_tensor(args[0])) || (kTensors == 2 && !(b = exact_tensor(args[1]))) ||
        !(offsets = exact_tensor(args[kTensors])) || !as_int64(args[kTensors + 1], &max_len) || !plain_offsets(*offsets) || offsets->numel() < 1 ||
        a->dim() != 2 || a->scalar_type() != at::kBFloat16 || (b && b->scalar_type() != at::kBFloat16))
        Py_RETURN_NONE;
    const int64_t B = offsets->numel() - 1, n = a->size(0), D = a->size(1);
    if constexpr (kOp == Feature::kDenseBmm)
        if (b->dim() != 3 || b->size(0) != B || b->size(1) != D) Py_RETURN_NONE;
    if constexpr (kOp == Feature::kJaggedBmm)
        if (b->dim() != 2 || b->size(0) != n) Py_RETURN_NONE;
    if constexpr (kOp == Feature::kSoftmaxBackward)
        if (b->sizes() != a->sizes()) Py_RETURN_NONE;
    if (D > 128 || (b && b->size(-1) > 128)) Py_RETURN_NONE;
    Tensor out;
    int status;
    {
        pybind11::gil_scoped_release nogil;
        if constexpr (kOp == Feature::kDenseBmm || kOp == Feature::kJaggedBmm) {
            const int T = (int)b->size(-1);
            constexpr bool kDense = kOp == Feature::kDenseBmm;
            out = kDense ? at::empty({n, T}, a->options()) : at::empty({B, D, T}, a->options());
            status = (kDense ? lib.dense_bmm : lib.jagged_bmm)(a->data_ptr(), b->data_ptr(), longs(*offsets), B, max_len, (int)D, T, out.data_ptr(), stream());
        } else {
            out = at::empty(a->sizes(), a->options());
            if constexpr (kOp == Feature::kSoftmax)
                status = lib.softmax(a->data_ptr(), longs(*offsets), B, max_len, (int)D, out.data_ptr(), stream());
            else
                status = lib.softmax_backward(a->data_ptr(), b->data_ptr(), longs(*offsets), B, max_len, (int)D, out.data_ptr(), stream());
        }
    }
    if (status != 0) Py_RETURN_NONE;
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// In a backward: whether a graph is being captured that gradients would leave.  Autograd runs a node, and what adds up a leaf's gradient, on the
// stream that was current when it was made, and makes that stream wait for the one that the gradient comes from.  A leaf whose
// gradient has been asked for on another stream by a graph that is still alive keeps that graph's node; captured, the wait draws the other stream
// into the capture, which then cannot be ended (the process ends instead).
bool gradients_leave_capture() {
    if (c10::hip::currentStreamCaptureStatusMayInitCtx() == c10::hip::CaptureStatus::None) return false;
    const c10::StreamId here = c10::hip::getCurrentHIPStream().id();
    const std::shared_ptr<torch::autograd::Node> node = torch::autograd::get_current_node();
    if (!node) return false;
    std::unordered_set<torch::autograd::Node *> seen{node.get()};
    std::vector<torch::autograd::Node *> todo{node.get()};
    while (!todo.empty()) {
        torch::autograd::Node *const at = todo.back();
        todo.pop_back();
        const auto stream = at->stream();
        if (stream && stream->id() != here) return true;
        for (const torch::autograd::Edge &e : at->next_edges())
            if (e.function && seen.insert(e.function.get()).second) todo.push_back(e.function.get());
    }
    return false;
}


// ---- linear attention, layer norm, embedding lookup ----
// Functions of autograd.py: graphs are made here, and where there is none to be made the result alone.  What is not an ordinary call is answered
// with None as above.
using Maybe = std::optional<Tensor>;

void check_capture() {
    TORCH_CHECK(!gradients_leave_capture(),
                "A backward pass is being captured into a graph while the gradients of its leaves belong to another stream: an earlier graph of the same leaves is "
                "still alive.  Let go of that graph's results first, or run it on the stream of the capture.");
}
// A saved tensor as it comes back (see check_saved()).
void check_back(const Tensor &t, at::IntArrayRef sizes, at::ScalarType type, c10::Device device) {
    check_on_gpu(t);
    TORCH_CHECK(t.sizes() == sizes && t.scalar_type() == type && t.device() == device, "backward: a tensor of ", sizes, " ", type, " on ", device, " was saved, ", t.sizes(),
                " ", t.scalar_type(), " on ", t.device(), " came back");
}
void check_call(int status, bool in_backward) {   // in a forward the Python function meets the same error and reports it
    if (status == 0) return;
    if (!in_backward) throw Refused{};
    check_backward(status);
}
const void *data(const Maybe &t) { return t && t->defined() ? t->data_ptr() : nullptr; }
const float *floats_or_null(const Maybe &t) { return static_cast<const float *>(data(t)); }
const int64_t *longs_or_null(const Maybe &t) { return static_cast<const int64_t *>(data(t)); }
int64_t samples(const Maybe &offsets) { return offsets && offsets->defined() ? offsets->numel() - 1 : 0; }
Tensor bytes(size_t n, const Tensor &like) { return n ? at::empty({(int64_t)n}, like.options().dtype(at::kByte)) : Tensor(); }
void *place(const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
bool wants_gradient(std::initializer_list<const Tensor *> tensors) {
    if (!at::GradMode::is_enabled()) return false;
    for (const Tensor *t : tensors)
        if (t && t->requires_grad()) return true;
    return false;
}
Maybe maybe(const Tensor *t) { return t ? Maybe(*t) : Maybe(); }

// A backward's results: where a graph of the backward is being made, going through them to what they were computed from is an error.  (Left as they are they
// would count as constants.)
variable_list once(variable_list gradients, const variable_list &from) {
    if (at::GradMode::is_enabled())
        torch::autograd::set_history(gradients, std::make_shared<torch::autograd::Error>("the gradients of this operator cannot be differentiated again",
                                                                                         torch::autograd::collect_next_edges(from)));
    return gradients;
}

// (q, k, v, log_decay, offsets, max_len, scale, initial_state) -> out, and the final state if wanted
std::pair<Tensor, Tensor> linear_call(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &log_decay, const Tensor &offsets, int64_t max_len, double scale,
                                      const Maybe &initial, bool want_state) {
    const int H = (int)q.size(1), D = (int)q.size(2);
    const int64_t B = offsets.numel() - 1;
    const Tensor out = at::empty(q.sizes(), q.options());
    const Tensor final_state = want_state ? at::empty({B, H, D, D}, q.options().dtype(at::kFloat)) : Tensor();
    const size_t need = lib.linear_workspace(B, q.size(0), max_len, H, D, 0);
    const Tensor workspace = bytes(need, q);
    check_call(lib.linear[kind(q)](q.data_ptr(), k.data_ptr(), v.data_ptr(), floats(log_decay), longs(offsets), B, q.size(0), max_len, H, D, (float)scale, floats_or_null(initial),
                                   out.data_ptr(), static_cast<float *>(place(final_state)), place(workspace), need, stream()), false);
    return {out, final_state};
}
struct LinearAttention : torch::autograd::Function<LinearAttention> {
    static variable_list forward(AutogradContext *ctx, const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &log_decay, const Tensor &offsets, int64_t max_len,
                                 double scale, const Maybe &initial, bool want_state) {
        const auto [out, final_state] = linear_call(q, k, v, log_decay, offsets, max_len, scale, initial, want_state);
        ctx->save_for_backward({q, k, v, log_decay, offsets, initial ? *initial : Tensor()});
        ctx->saved_data["call"] = std::vector<int64_t>{max_len, offsets.numel(), q.size(0), q.size(1), q.size(2), (int64_t)q.scalar_type(), initial && initial->requires_grad(),
                                                       initial.has_value()};
        ctx->saved_data["scale"] = scale;
        ctx->set_materialize_grads(false);
        return want_state ? variable_list{out, final_state} : variable_list{out};
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads) {
        check_capture();
        const variable_list saved = ctx->get_saved_variables();
        const std::vector<int64_t> call = ctx->saved_data["call"].toIntVector();
        const int64_t max_len = call[0], B = call[1] - 1;
        const int H = (int)call[3], D = (int)call[4];
        const at::ScalarType type = (at::ScalarType)call[5];
        const Tensor &q = saved[0], &k = saved[1], &v = saved[2], &log_decay = saved[3], &offsets = saved[4];
        check_on_gpu(q);
        const c10::Device device = q.device();
        for (const Tensor *t : {&q, &k, &v}) check_back(*t, {call[2], H, D}, type, device);
        check_back(log_decay, {H}, at::kFloat, device);
        check_back(offsets, {call[1]}, at::kLong, device);
        if (call[7]) check_back(saved[5], {B, H, D, D}, at::kFloat, device);
        const Tensor dout = grads[0].defined() ? grads[0].contiguous() : at::zeros_like(q);
        check_back(dout, {call[2], H, D}, type, device);
        const Tensor dfinal = grads.size() > 1 && grads[1].defined() ? grads[1].contiguous() : Tensor();
        if (dfinal.defined()) check_back(dfinal, {B, H, D, D}, at::kFloat, device);
        const Tensor dq = at::empty(q.sizes(), q.options()), dk = at::empty(q.sizes(), q.options()), dv = at::empty(q.sizes(), q.options());
        const Tensor dinitial = call[6] ? at::empty({B, H, D, D}, q.options().dtype(at::kFloat)) : Tensor();
        const size_t need = lib.linear_workspace(B, q.size(0), max_len, H, D, 1);
        const Tensor workspace = bytes(need, q);
        check_call(lib.linear_backward[type == at::kFloat](q.data_ptr(), k.data_ptr(), v.data_ptr(), dout.data_ptr(), floats(log_decay), longs(offsets), B, q.size(0), max_len, H, D,
                                                           (float)ctx->saved_data["scale"].toDouble(), static_cast<float *>(place(saved[5])), static_cast<float *>(place(dfinal)),
                                                           dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), static_cast<float *>(place(dinitial)), place(workspace), need, stream()),
                   true);
        return once({dq, dk, dv, Tensor(), Tensor(), Tensor(), Tensor(), dinitial, Tensor()}, {q, k, v, saved[5], grads[0], dfinal});
    }
};

// (x, weight, bias, offsets, eps) -> y, and mean and rstd [2, rows, reps] if wanted
struct NormSizes { int64_t rows, reps, N; };
std::pair<Tensor, Tensor> norm_call(const Tensor &x, const Maybe &weight, const Maybe &bias, const Maybe &offsets, double eps, const NormSizes &n, bool want_statistics) {
    const Tensor y = at::empty(x.sizes(), x.options());
    const Tensor statistics = want_statistics ? at::empty({2, n.rows, n.reps}, x.options().dtype(at::kFloat)) : Tensor();
    float *const mean = static_cast<float *>(place(statistics)), *const rstd = mean ? mean + n.rows * n.reps : nullptr;
    check_call(lib.norm[kind(x)](x.data_ptr(), data(weight), data(bias), longs_or_null(offsets), samples(offsets), n.rows, n.reps, n.N, (float)eps, y.data_ptr(), mean, rstd,
                                 stream()), false);
    return {y, statistics};
}
struct LayerNorm : torch::autograd::Function<LayerNorm> {
    static Tensor forward(AutogradContext *ctx, const Tensor &x, const Maybe &weight, const Maybe &bias, const Maybe &offsets, double eps, int64_t rows, int64_t reps, int64_t N) {
        const auto [y, statistics] = norm_call(x, weight, bias, offsets, eps, {rows, reps, N}, true);
        ctx->save_for_backward({x, weight ? *weight : Tensor(), statistics, offsets ? *offsets : Tensor()});
        ctx->saved_data["call"] = std::vector<int64_t>{rows, reps, N, (int64_t)x.scalar_type(), weight.has_value(), offsets ? offsets->numel() : -1,
                                                       weight && weight->requires_grad(), bias && bias->requires_grad()};
        ctx->saved_data["sizes"] = x.sizes().vec();
        ctx->saved_data["shape"] = weight ? weight->sizes().vec() : bias ? bias->sizes().vec() : std::vector<int64_t>{N};
        return y;
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads) {
        check_capture();
        const variable_list saved = ctx->get_saved_variables();
        const std::vector<int64_t> call = ctx->saved_data["call"].toIntVector(), sizes = ctx->saved_data["sizes"].toIntVector(), shape = ctx->saved_data["shape"].toIntVector();
        const Tensor &x = saved[0], &weight = saved[1], &statistics = saved[2], &offsets = saved[3];
        const int64_t rows = call[0], reps = call[1], N = call[2];
        const at::ScalarType type = (at::ScalarType)call[3];
        check_on_gpu(x);
        check_back(x, sizes, type, x.device());
        if (call[4]) check_back(weight, shape, type, x.device());
        check_back(statistics, {2, rows, reps}, at::kFloat, x.device());
        if (call[5] >= 0) check_back(offsets, {call[5]}, at::kLong, x.device());
        const Tensor dy = grads[0].contiguous();
        check_back(dy, sizes, type, x.device());
        const Tensor dx = at::empty(sizes, x.options());
        const Tensor dweight = call[6] ? at::empty(shape, x.options()) : Tensor(), dbias = call[7] ? at::empty(shape, x.options()) : Tensor();
        const size_t need = call[6] || call[7] ? lib.norm_workspace(rows, reps, N) : 0;
        const Tensor workspace = bytes(need, x);
        const float *const mean = floats(statistics);
        check_call(lib.norm_backward[type == at::kFloat](x.data_ptr(), place(weight), dy.data_ptr(), mean, mean + rows * reps, static_cast<int64_t *>(place(offsets)),
                                                         call[5] >= 0 ? call[5] - 1 : 0, rows, reps, N, dx.data_ptr(), place(dweight), place(dbias), place(workspace), need, stream()),
                   true);
        return once({dx, dweight, dbias, Tensor(), Tensor(), Tensor(), Tensor(), Tensor()}, {x, weight, dy});
    }
};

Tensor embedding_of(const Tensor &table, const Tensor &ids, const Maybe &offsets, double scale) {
    std::vector<int64_t> sizes = table.sizes().vec();
    sizes[0] = ids.numel();
    const Tensor out = at::empty(sizes, table.options());
    const int64_t V = table.size(0);
    check_call(lib.embedding[kind(table)](table.data_ptr(), ids.data_ptr(), (int)ids.element_size(), longs_or_null(offsets), samples(offsets), ids.numel(), V,
                                          V ? table.numel() / V : 0, (float)scale, out.data_ptr(), stream()), false);
    return out;
}
struct Embedding : torch::autograd::Function<Embedding> {
    static Tensor forward(AutogradContext *ctx, const Tensor &table, const Tensor &ids, const Maybe &offsets, double scale) {
        const Tensor out = embedding_of(table, ids, offsets, scale);
        ctx->save_for_backward({ids, offsets ? *offsets : Tensor()});
        ctx->saved_data["call"] = std::vector<int64_t>{ids.numel(), (int64_t)ids.scalar_type(), offsets ? offsets->numel() : -1, (int64_t)table.scalar_type()};
        ctx->saved_data["sizes"] = table.sizes().vec();
        ctx->saved_data["scale"] = scale;
        return out;
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads) {
        check_capture();
        const variable_list saved = ctx->get_saved_variables();
        const std::vector<int64_t> call = ctx->saved_data["call"].toIntVector(), sizes = ctx->saved_data["sizes"].toIntVector();
        const Tensor &ids = saved[0], &offsets = saved[1], dout = grads[0].contiguous();
        const at::ScalarType type = (at::ScalarType)call[3];
        std::vector<int64_t> out_sizes = sizes;
        out_sizes[0] = call[0];
        check_on_gpu(dout);
        check_back(dout, out_sizes, type, dout.device());
        check_back(ids, {call[0]}, (at::ScalarType)call[1], dout.device());
        if (call[2] >= 0) check_back(offsets, {call[2]}, at::kLong, dout.device());
        const Tensor dtable = at::empty(sizes, dout.options());
        const int64_t V = sizes[0], N = dtable.numel() / V;
        const size_t need = lib.embedding_workspace(call[0], V, N);
        const Tensor workspace = bytes(need, dout);
        check_call(lib.embedding_backward[type == at::kFloat](dout.data_ptr(), ids.data_ptr(), (int)ids.element_size(), static_cast<int64_t *>(place(offsets)),
                                                              call[2] >= 0 ? call[2] - 1 : 0, call[0], V, N, (float)ctx->saved_data["scale"].toDouble(), dtable.data_ptr(),
                                                              place(workspace), need, stream()),
                   true);
        return once({dtable, Tensor(), Tensor(), Tensor()}, {dout});
    }
};

// The arguments as the interpreter has them: a tensor (a parameter, too), or None where that may be; on the current device.
bool tensor_of(PyObject *o, const Tensor **t, bool may_be_none = false) {
    *t = nullptr;
    if (o == Py_None) return may_be_none;
    if (!THPVariable_CheckExact(o) && (PyObject *)Py_TYPE(o) != lib.parameter) return false;
    const Tensor &x = THPVariable_Unpack(o);
    using c10::DispatchKey;
    constexpr c10::DispatchKeySet stands_for_others({DispatchKey::Python, DispatchKey::Functionalize, DispatchKey::FuncTorchBatched, DispatchKey::FuncTorchGradWrapper,
                                                     DispatchKey::BatchedNestedTensor, DispatchKey::Conjugate, DispatchKey::Negative, DispatchKey::ZeroTensor});
    if (x.key_set().has_any(stands_for_others) || !plain(x) || x.device().index() != c10::hip::current_device()) return false;
    *t = &x;
    return true;
}
bool double_of(PyObject *o, double *x) {
    if (!PyFloat_CheckExact(o)) return false;
    *x = PyFloat_AS_DOUBLE(o);
    return true;
}
bool known_type(const Tensor &t) { return t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kFloat; }
bool offsets_fit(const Tensor *t) { return !t || (t->dim() == 1 && t->scalar_type() == at::kLong && t->numel() >= 1); }
bool states_fit(const Tensor *t, int64_t B, const Tensor &q) {
    return !t || (t->scalar_type() == at::kFloat && t->sizes() == at::IntArrayRef({B, q.size(1), q.size(2), q.size(2)}));
}
bool rows_fit(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &log_decay) {
    return known_type(q) && q.dim() == 3 && q.size(0) > 0 && q.size(1) < (1 << 30) && q.size(2) <= 128 && k.sizes() == q.sizes() && v.sizes() == q.sizes() && k.scalar_type() == q.scalar_type() &&
           v.scalar_type() == q.scalar_type() && log_decay.scalar_type() == at::kFloat && log_decay.dim() == 1 && log_decay.size(0) == q.size(1) && !log_decay.requires_grad();
}
// (q, k, v, log_decay, offsets, max_len, scale, initial_state, return_state): out, or (out, final state)
PyObject *linear_attention_call(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    const Tensor *q, *k, *v, *log_decay, *offsets, *initial;
    int64_t max_len = 0;
    double scale = 0.0;
    if (n_args != 9 || !nobody_listens() || !tensor_of(args[0], &q) || !tensor_of(args[1], &k) || !tensor_of(args[2], &v) || !tensor_of(args[3], &log_decay) ||
        !tensor_of(args[4], &offsets) || !as_int64(args[5], &max_len) || !double_of(args[6], &scale) || !tensor_of(args[7], &initial, true) || !PyBool_Check(args[8]) ||
        !offsets_fit(offsets) || !rows_fit(*q, *k, *v, *log_decay) || !states_fit(initial, offsets->numel() - 1, *q))
        Py_RETURN_NONE;
    const bool want_state = args[8] == Py_True;
    Tensor out, final_state;
    try {
        pybind11::gil_scoped_release nogil;
        if (wants_gradient({q, k, v, initial})) {
            const variable_list results = LinearAttention::apply(*q, *k, *v, *log_decay, *offsets, max_len, scale, maybe(initial), want_state);
            out = results[0];
            if (want_state) final_state = results[1];
        } else
            std::tie(out, final_state) = linear_call(*q, *k, *v, *log_decay, *offsets, max_len, scale, maybe(initial), want_state);
    } catch (const Refused &) {
        Py_RETURN_NONE;
    }
    if (!want_state) return THPVariable_Wrap(std::move(out));
    PyObject *pair = PyTuple_New(2);
    if (!pair) return nullptr;
    PyTuple_SET_ITEM(pair, 0, THPVariable_Wrap(std::move(out)));
    PyTuple_SET_ITEM(pair, 1, THPVariable_Wrap(std::move(final_state)));
    return pair;
    END_HANDLE_TH_ERRORS
}
// (q, k, v, log_decay, state, scale, new_state): out
PyObject *linear_step_call(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    const Tensor *q, *k, *v, *log_decay, *state, *new_state;
    double scale = 0.0;
    if (n_args != 7 || !nobody_listens() || !tensor_of(args[0], &q) || !tensor_of(args[1], &k) || !tensor_of(args[2], &v) || !tensor_of(args[3], &log_decay) ||
        !tensor_of(args[4], &state) || !double_of(args[5], &scale) || !tensor_of(args[6], &new_state) || !rows_fit(*q, *k, *v, *log_decay) || !states_fit(state, q->size(0), *q) ||
        !states_fit(new_state, q->size(0), *q))
        Py_RETURN_NONE;
    Tensor out;
    int status;
    {
        pybind11::gil_scoped_release nogil;
        out = at::empty(q->sizes(), q->options());
        status = lib.linear_step[kind(*q)](q->data_ptr(), k->data_ptr(), v->data_ptr(), floats(*log_decay), q->size(0), (int)q->size(1), (int)q->size(2), (float)scale, floats(*state),
                                           out.data_ptr(), floats(*new_state), stream());
    }
    if (status != 0) Py_RETURN_NONE;
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}
// (x, weight, bias, offsets, eps): y
PyObject *layer_norm_call(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    const Tensor *x, *weight, *bias, *offsets;
    double eps = 0.0;
    if (n_args != 5 || !nobody_listens() || !tensor_of(args[0], &x) || !tensor_of(args[1], &weight, true) || !tensor_of(args[2], &bias, true) ||
        !tensor_of(args[3], &offsets, true) || !double_of(args[4], &eps) || !known_type(*x) || x->dim() < 2 || !offsets_fit(offsets))
        Py_RETURN_NONE;
    const Tensor *const first = weight ? weight : bias;
    const at::IntArrayRef shape = first ? first->sizes() : x->sizes().slice(x->dim() - 1);
    if (shape.empty() || (int64_t)shape.size() >= x->dim() || x->sizes().slice(x->dim() - shape.size()) != shape) Py_RETURN_NONE;
    for (const Tensor *t : {weight, bias})
        if (t && (t->sizes() != shape || t->scalar_type() != x->scalar_type())) Py_RETURN_NONE;
    NormSizes n{x->size(0), 1, 1};
    for (const int64_t d : shape) n.N *= d;
    for (int64_t d = 1; d < x->dim() - (int64_t)shape.size(); ++d) n.reps *= x->size(d);
    Tensor y;
    try {
        pybind11::gil_scoped_release nogil;
        if (wants_gradient({x, weight, bias})) y = LayerNorm::apply(*x, maybe(weight), maybe(bias), maybe(offsets), eps, n.rows, n.reps, n.N);
        else y = norm_call(*x, maybe(weight), maybe(bias), maybe(offsets), eps, n, false).first;
    } catch (const Refused &) {
        Py_RETURN_NONE;
    }
    return THPVariable_Wrap(std::move(y));
    END_HANDLE_TH_ERRORS
}
// (table, ids, offsets, scale): out
PyObject *embedding_call(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    const Tensor *table, *ids, *offsets;
    double scale = 0.0;
    if (n_args != 4 || !nobody_listens() || !tensor_of(args[0], &table) || !tensor_of(args[1], &ids) || !tensor_of(args[2], &offsets, true) || !double_of(args[3], &scale) ||
        !known_type(*table) || table->dim() < 1 || ids->dim() != 1 || (ids->scalar_type() != at::kLong && ids->scalar_type() != at::kInt) || !offsets_fit(offsets))
        Py_RETURN_NONE;
    Tensor out;
    try {
        pybind11::gil_scoped_release nogil;
        out = wants_gradient({table}) ? Embedding::apply(*table, *ids, maybe(offsets), scale) : embedding_of(*table, *ids, maybe(offsets), scale);
    } catch (const Refused &) {
        Py_RETURN_NONE;
    }
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}
#define JFA_CALL(name, function) {name, (PyCFunction)(void (*)())function, METH_FASTCALL, nullptr}
PyMethodDef calls[] = {JFA_CALL("forward", forward_call<false>),
                       JFA_CALL("forward_cross", forward_call<true>),
                       JFA_CALL("to_dense", to_dense_call),
                       JFA_CALL("to_jagged", to_jagged_call),
                       JFA_CALL("dense_bmm", feature_call<Feature::kDenseBmm>),
                       JFA_CALL("jagged_bmm", feature_call<Feature::kJaggedBmm>),
                       JFA_CALL("softmax", feature_call<Feature::kSoftmax>),
                       JFA_CALL("softmax_backward", feature_call<Feature::kSoftmaxBackward>),
                       JFA_CALL("linear_attention", linear_attention_call),
                       JFA_CALL("linear_step", linear_step_call),
                       JFA_CALL("layer_norm", layer_norm_call),
                       JFA_CALL("embedding", embedding_call),
                       {nullptr, nullptr, 0, nullptr}};
#undef JFA_CALL

// entry: name of an entry point -> its address
void bind_library(const std::function<int64_t(const std::string &)> &entry, pybind11::object check, pybind11::object pointer, pybind11::object parameter) {
    const char *suffix[2] = {"", "_f32"};
    auto at = [&](const char *name, int i) { return (uintptr_t)entry(std::string(name) + suffix[i]); };
    for (int i = 0; i < 2; ++i) {
        lib.forward[i] = reinterpret_cast<Forward>(at("jfa_forward", i));
        lib.forward_causal[i] = reinterpret_cast<Forward>(at("jfa_forward_causal", i));
        lib.backward[i] = reinterpret_cast<Backward>(at("jfa_backward", i));
        lib.backward_causal[i] = reinterpret_cast<Backward>(at("jfa_backward_causal", i));
        lib.forward_cross[i] = reinterpret_cast<ForwardCross>(at("jfa_forward_cross", i));
        lib.backward_cross[i] = reinterpret_cast<BackwardCross>(at("jfa_backward_cross", i));
        lib.linear[i] = reinterpret_cast<Linear>(at("jfa_linear_attention", i));
        lib.linear_backward[i] = reinterpret_cast<LinearBackward>(at("jfa_linear_attention_backward", i));
        lib.linear_step[i] = reinterpret_cast<LinearStep>(at("jfa_linear_attention_step", i));
        lib.norm[i] = reinterpret_cast<Norm>(at("jfa_layer_norm", i));
        lib.norm_backward[i] = reinterpret_cast<NormBackward>(at("jfa_layer_norm_backward", i));
        lib.embedding[i] = reinterpret_cast<Embed>(at("jfa_embedding", i));
        lib.embedding_backward[i] = reinterpret_cast<EmbedBackward>(at("jfa_embedding_backward", i));
    }
    auto plain_entry = [&](const char *name) { return (uintptr_t)entry(name); };
    lib.to_dense = reinterpret_cast<ToDense>(plain_entry("jfa_jagged_to_dense"));
    lib.to_jagged = reinterpret_cast<ToJagged>(plain_entry("jfa_dense_to_jagged"));
    lib.dense_bmm = reinterpret_cast<Product>(plain_entry("jfa_jagged_dense_bmm"));
    lib.jagged_bmm = reinterpret_cast<Product>(plain_entry("jfa_jagged_jagged_bmm"));
    lib.softmax = reinterpret_cast<Softmax>(plain_entry("jfa_jagged_softmax"));
    lib.softmax_backward = reinterpret_cast<SoftmaxBackward>(plain_entry("jfa_jagged_softmax_backward"));
    lib.linear_workspace = reinterpret_cast<LinearWorkspace>(plain_entry("jfa_linear_attention_workspace_bytes"));
    lib.norm_workspace = reinterpret_cast<RowsWorkspace>(plain_entry("jfa_layer_norm_workspace_bytes"));
    lib.embedding_workspace = reinterpret_cast<RowsWorkspace>(plain_entry("jfa_embedding_workspace_bytes"));
    lib.parameter = parameter.release().ptr();
    lib.check = check.release().ptr();   // kept for the life of the process
    lib.pointer = pointer.release().ptr();
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
    m.def("bind_library", &bind_library);
    m.def("self_attention", &self_attention);
    m.def("cross_attention", &cross_attention);
    m.def("gradients_leave_capture", &gradients_leave_capture);
    if (PyModule_AddFunctions(m.ptr(), calls) != 0) throw pybind11::error_already_set();
}
