"""Jagged flash attention as differentiable torch functions of q, k and v (paper Section 2.2: the operators have a
forward and a backward so that they can be trained through).

Argument marshalling only: the forward of each function is the library's forward entry point, its backward the
library's backward entry point on the tensors the forward saved; nothing is computed here, and a missing library
raises as everywhere in the binding.  Ordinary calls go through autograd nodes in C++ (csrc/jfa_autograd.cpp), which a training
step on a small batch spends half as much host time in; the torch.autograd.Function classes below are the same for the rest.

    out = jagged_flash_attention(q, k, v, offsets, max_len)                      # self attention, causal=True for the causal variant
    out = jagged_flash_cross_attention(q, k, v, offsets_q, offsets_kv, max_len_q, max_len_kv)
    out = jagged_linear_attention(q, k, v, log_decay, offsets, max_len)              # a decay for each head; states in and out if wanted
    y = jagged_layer_norm(x, weight, bias, offsets)                                  # rows of any shape that ends in weight's
    x = jagged_embedding(table, ids, offsets, scale)                                 # a row of the table for each id

q, k, v: [rows, H, D] bf16 or fp32 on the GPU, contiguous; offsets: int64 [B + 1] on the GPU.  Gradients flow to q, k
and v (and to x, weight, bias, the table and the states); offsets, ids, decays and the length bounds are not differentiable.
Rows behind offsets[B] are nobody's: they are not read, and results and gradients hold anything there.
"""
import ctypes
import importlib.util
import threading
import warnings

import torch
from torch.autograd import forward_ad

from . import binding
from .build import native_path

__all__ = ["jagged_flash_attention", "jagged_flash_cross_attention", "jagged_linear_attention", "jagged_layer_norm", "jagged_embedding"]


class _SelfAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, offsets, max_len, causal):
        out, lse = binding.jfa_forward(q, k, v, offsets, max_len, causal=causal)
        ctx.save_for_backward(q, k, v, out, lse, offsets)
        ctx.max_len, ctx.causal = max_len, causal
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, out, lse, offsets = ctx.saved_tensors
        dq, dk, dv, _ = binding.jfa_backward(q, k, v, out, dout.contiguous(), lse, offsets, ctx.max_len, causal=ctx.causal)
        return dq, dk, dv, None, None, None


class _CrossAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, offsets_q, offsets_kv, max_len_q, max_len_kv):
        out, lse = binding.jfa_forward_cross(q, k, v, offsets_q, offsets_kv, max_len_q, max_len_kv)
        ctx.save_for_backward(q, k, v, out, lse, offsets_q, offsets_kv)
        ctx.max_len_q, ctx.max_len_kv = max_len_q, max_len_kv
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, out, lse, offsets_q, offsets_kv = ctx.saved_tensors
        dq, dk, dv, _ = binding.jfa_backward_cross(q, k, v, out, dout.contiguous(), lse, offsets_q, offsets_kv,
                                                   ctx.max_len_q, ctx.max_len_kv)
        return dq, dk, dv, None, None, None, None


def _check_capture():
    """In a backward: refuses a capture that would end the process (see gradients_leave_capture in csrc/jfa_autograd.cpp)."""
    if torch.cuda.is_current_stream_capturing():
        if _native is None:
            _load_native()
        if _native is not False and _native.gradients_leave_capture():
            raise RuntimeError("A backward pass is being captured into a graph while the gradients of its leaves belong to another stream: an earlier graph of the "
                               "same leaves is still alive.  Let go of that graph's results first, or run it on the stream of the capture.")


class _Once(torch.autograd.Function):
    @staticmethod
    def forward(ctx, n, *tensors):
        return tuple(t.detach() for t in tensors[:n])

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("the gradients of this operator cannot be differentiated again")


def _once(gradients, *of):
    """A backward's results: where a graph of the backward is being made, going through them to what they were computed from is an error.  (Left as they are
    they would count as constants.)"""
    if not torch.is_grad_enabled():
        return gradients
    wanted = [g for g in gradients if g is not None]
    results = iter(_Once.apply(len(wanted), *wanted, *(t for t in of if t is not None)))
    return tuple(None if g is None else next(results) for g in gradients)


class _LinearAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, log_decay, offsets, max_len, scale, initial_state, return_state):
        out, final_state = binding.jfa_linear_attention(q, k, v, log_decay, offsets, max_len, scale, initial_state, return_state=return_state)
        ctx.save_for_backward(q, k, v, log_decay, offsets, initial_state)
        ctx.max_len, ctx.scale = max_len, scale
        return (out, final_state) if return_state else out

    @staticmethod
    def backward(ctx, dout, dfinal_state=None):
        _check_capture()
        q, k, v, log_decay, offsets, initial_state = ctx.saved_tensors
        dq, dk, dv, dinitial = binding.jfa_linear_attention_backward(
            q, k, v, dout.contiguous(), log_decay, offsets, ctx.max_len, ctx.scale, initial_state,
            None if dfinal_state is None else dfinal_state.contiguous(), return_dstate=ctx.needs_input_grad[7])
        return _once((dq, dk, dv, None, None, None, None, dinitial, None), q, k, v, initial_state, dout, dfinal_state)


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, offsets, eps):
        y, mean, rstd = binding.jfa_layer_norm(x, weight, bias, offsets, eps, statistics=any(ctx.needs_input_grad))
        ctx.save_for_backward(x, weight, mean, rstd, offsets)
        ctx.shape = next((t.shape for t in (weight, bias) if t is not None), x.shape[-1:])
        return y

    @staticmethod
    def backward(ctx, dy):
        _check_capture()
        x, weight, mean, rstd, offsets = ctx.saved_tensors
        dx, dweight, dbias = binding.jfa_layer_norm_backward(x, weight, dy.contiguous(), mean, rstd, offsets, normalized_shape=ctx.shape,
                                                             want_dweight=ctx.needs_input_grad[1], want_dbias=ctx.needs_input_grad[2])
        return _once((dx, dweight, dbias, None, None), x, weight, dy)


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, ids, offsets, scale):
        ctx.save_for_backward(ids, offsets)
        ctx.V, ctx.scale = table.shape[0], scale
        return binding.jfa_embedding(table, ids, offsets, scale)

    @staticmethod
    def backward(ctx, dout):
        _check_capture()
        ids, offsets = ctx.saved_tensors
        return _once((binding.jfa_embedding_backward(dout.contiguous(), ids, ctx.V, offsets, ctx.scale), None, None, None), dout)


_native = None   # the C++ nodes; False where they have not been built for this torch
_loading = threading.Lock()
_PLAIN = (torch.Tensor, torch.nn.Parameter)


def _load_native():
    global _native
    with _loading:   # several threads may make their first call at once
        if _native is not None:
            return
        try:
            spec = importlib.util.spec_from_file_location(__package__ + "._native", native_path(torch.__version__))
            nodes = importlib.util.module_from_spec(spec)
            spec.loader.exec_module(nodes)
        except ImportError as e:
            warnings.warn(f"The C++ autograd nodes are not there, the Python functions do their work more slowly ({e}).  "
                          "They are built by `python -m paper_2409_15373_amd.build`.")
            _native = False
            return
        lib = binding.load()
        nodes.bind_library(lambda name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value, binding._check, binding._ptr,
                           torch.nn.Parameter)
        _native = nodes


def _ordinary(*tensors) -> bool:
    """Whether a call may pass torch.autograd.Function by: tracers, function transforms, forward mode and tensor subclasses have to see it."""
    if torch.compiler.is_compiling():
        return False
    if _native is None:
        _load_native()
    return (_native is not False and all(type(t) in _PLAIN for t in tensors) and torch._C._get_tracing_state() is None
            and not torch._C._are_functorch_transforms_active() and forward_ad._current_level < 0)


def _nodes():
    """The C++ functions, None where a call is not theirs whatever its arguments (they look at those themselves)."""
    if torch.compiler.is_compiling() or forward_ad._current_level >= 0:
        return None
    if _native is None:
        _load_native()
    return _native or None


def jagged_flash_attention(q, k, v, offsets, max_len: int, causal: bool = False):
    """softmax(Q K^T / sqrt(D)) V per sample and head over the jagged rows that `offsets` delimits (Section 2.1)."""
    max_len, causal = int(max_len), bool(causal)
    if _ordinary(q, k, v, offsets):
        out = _native.self_attention(q, k, v, offsets, max_len, causal)
        if out is not None:   # None: not in order, the function below says what is wrong
            return out
    return _SelfAttention.apply(q, k, v, offsets, max_len, causal)


def jagged_flash_cross_attention(q, k, v, offsets_q, offsets_kv, max_len_q: int, max_len_kv: int):
    """The queries of sample b (rows of offsets_q) attend to its keys and values (rows of offsets_kv)."""
    max_len_q, max_len_kv = int(max_len_q), int(max_len_kv)
    if _ordinary(q, k, v, offsets_q, offsets_kv):
        out = _native.cross_attention(q, k, v, offsets_q, offsets_kv, max_len_q, max_len_kv)
        if out is not None:
            return out
    return _CrossAttention.apply(q, k, v, offsets_q, offsets_kv, max_len_q, max_len_kv)


def jagged_linear_attention(q, k, v, log_decay, offsets, max_len: int, scale=None, initial_state=None, return_state: bool = False):
    """out_i = scale q_i S_i with S_i = exp(log_decay) S_(i-1) + k_i^T v_i per sample and head; q, k, v as for jagged_flash_attention,
    log_decay fp32 [H], scale 1 / sqrt(D) if not given.  initial_state: fp32 [B, H, D, D], zeros if not given; return_state: the samples'
    final states too, as a second result.  Gradients flow to the states as well, not to log_decay.
    Of this and the following functions the gradients cannot be differentiated again."""
    if log_decay.requires_grad and torch.is_grad_enabled():
        raise ValueError("jagged_linear_attention: log_decay is not differentiable")
    args = (q, k, v, log_decay, offsets, int(max_len), q.shape[-1] ** -0.5 if scale is None else float(scale), initial_state, bool(return_state))
    if (nodes := _nodes()) and (result := nodes.linear_attention(*args)) is not None:   # None: not in order, the function below says what is wrong
        return result
    return _LinearAttention.apply(*args)


def jagged_layer_norm(x, weight=None, bias=None, offsets=None, eps: float = 1e-5):
    """Layer norm over the last dimensions of x [rows, ...], those of weight and bias (without either the last one).  offsets: of
    the rows only the first offsets[B] are there."""
    if (nodes := _nodes()) and (y := nodes.layer_norm(x, weight, bias, offsets, float(eps))) is not None:
        return y
    return _LayerNorm.apply(x, weight, bias, offsets, float(eps))


def jagged_embedding(table, ids, offsets=None, scale: float = 1.0):
    """scale table[ids] for table [V, ...] and ids [rows] (int64 or int32), zeros for an id outside the table.  offsets: of the
    rows only the first offsets[B] are there."""
    if (nodes := _nodes()) and (out := nodes.embedding(table, ids, offsets, float(scale))) is not None:
        return out
    return _Embedding.apply(table, ids, offsets, float(scale))
