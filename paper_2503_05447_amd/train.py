"""Binding of the training operators declared in include/lsm_train.h: routing of tokens to experts, the experts of many tokens,
losses over a large vocabulary, each with its backward pass.

Argument marshalling only, as in binding.py: every operator runs in the HIP kernels of liblsm_hip.so on ``stream``
(default: torch's current stream) without synchronising.  Every tensor begins at a multiple of 16 bytes.
"""
import ctypes
import functools
from operator import index

import torch

from .binding import LsmError, _alloc_on, _ptr, _raw_stream_calls, _stream_handle, library
from .block import _dtype


class _RouteParams(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32)] + [(n, ctypes.c_int32) for n in ("n", "E", "top_k", "dtype", "renormalise")]


class _ExpertsParams(ctypes.Structure):
    _fields_ = ([("struct_size", ctypes.c_uint32)] + [(n, ctypes.c_int32) for n in ("n", "D", "F", "E", "top_k", "dtype", "reserved")]
                + [("x_stride", ctypes.c_int64), ("dy_stride", ctypes.c_int64)])


class _VocabParams(ctypes.Structure):
    _fields_ = ([("struct_size", ctypes.c_uint32)] + [(n, ctypes.c_int32) for n in ("n", "D", "V", "K", "dtype")]
                + [("temperature", ctypes.c_float), ("reserved", ctypes.c_int32), ("x_stride", ctypes.c_int64)])


def _current_device():
    device = _raw_stream_calls()[1]
    return device() if device is not None else torch.cuda.current_device()


def _sized(params, sizes):
    """A parameter block of `sizes`, by reference; ctypes itself would cut a number off at 32 bits."""
    p = params(ctypes.sizeof(params), *sizes)
    if any(getattr(p, f) != s for (f, t), s in zip(params._fields_[1:], sizes) if t is not ctypes.c_float):
        raise ValueError("a size is beyond the 32 bits (strides: 64) that the library takes: %s" % (sizes,))
    return ctypes.byref(p)


# Parameter blocks by reference, kept by the numbers in them (sizes only, no pointers), and the workspaces they ask for.
@functools.lru_cache(maxsize=256)
def _route_params(*sizes):
    p = _sized(_RouteParams, sizes)
    return p, library().lsm_moe_plan_workspace_bytes(p)


@functools.lru_cache(maxsize=256)
def _experts_params(*sizes):
    p = _sized(_ExpertsParams, sizes)
    return p, library().lsm_moe_experts_workspace_bytes(p), library().lsm_moe_experts_bwd_workspace_bytes(p)


@functools.lru_cache(maxsize=256)
def _vocab_params(*sizes):
    p = _sized(_VocabParams, sizes)
    return p, library().lsm_vocab_loss_workspace_bytes(p), library().lsm_vocab_loss_bwd_workspace_bytes(p)


def _device(t, name):
    """Number of the device that a call's first tensor is on; the launches go to the current one."""
    if not t.is_cuda:
        raise ValueError("%s: need a device tensor, got one on %s" % (name, t.device))
    dev, current = t.get_device(), _current_device()
    if dev != current and dev >= 0:
        raise ValueError("%s is on cuda:%d, the current device is cuda:%d" % (name, dev, current))
    return dev


def _check(t, shape, dtype, dev, name):
    """A call's marshalling is most of its time for a few tokens: what is asked is asked in one line."""
    if t is not None and (t.dtype != dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous()):
        raise ValueError("%s: need a contiguous tensor %s of %s on device %d, got %s %s on %s"
                         % (name, tuple(shape), dtype, dev, tuple(t.shape), t.dtype, t.device))


def _workspace(workspace, need, like):
    """The caller's workspace, or a new one beside `like` (None where none is needed)."""
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=like.device) if need else None
    if workspace.get_device() != like.get_device() or not workspace.is_contiguous():
        raise ValueError("workspace: need a contiguous tensor on %s, got one on %s" % (like.device, workspace.device))
    return workspace


def _bytes(workspace):
    return 0 if workspace is None else workspace.numel() * workspace.element_size()


def _rows(t, dev, name):
    """Elements between the rows of a [n, D] tensor that is dense along D."""
    if t.dim() != 2 or t.get_device() != dev or t.stride(1) != 1 and t.shape[1] != 1:
        raise ValueError("%s: need a [n,D] tensor, dense along D, on device %d, got %s with strides %s on %s"
                         % (name, dev, tuple(t.shape), t.stride(), t.device))
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _done(rc, name):
    if rc != 0:
        raise LsmError(rc, name)


def lsm_moe_route(logits, top_k, renormalise=True, stream=None):
    """weights, chosen = the top_k experts of each row of logits [n,E] (float32 or bfloat16), by falling logit, equal ones by index.

    weights [n,top_k] float32: the softmax over all experts, with ``renormalise`` divided by its sum over the chosen ones;
    chosen [n,top_k] int32.  An expert of -inf or NaN is never chosen: where too few are left the expert is -1 and the weight 0
    (a row of -inf: padding, no expert at all).  E at most 256, top_k at most 16."""
    if logits.dim() != 2:
        raise ValueError("logits: need [n,E], got %s" % (tuple(logits.shape),))
    n, E = logits.shape
    dt, k = _dtype(logits, "logits"), index(top_k)
    _check(logits, (n, E), logits.dtype, _device(logits, "logits"), "logits")
    p, _ = _route_params(n, E, k, dt, 1 if renormalise else 0)
    with _alloc_on(stream):
        weights = torch.empty((n, max(k, 0)), dtype=torch.float32, device=logits.device)
        chosen = torch.empty_like(weights, dtype=torch.int32)
    _done(library().lsm_moe_route(p, _ptr(logits), _ptr(weights), _ptr(chosen), _stream_handle(stream)), "lsm_moe_route")
    return weights, chosen


def lsm_moe_route_bwd(logits, chosen, d_weights, renormalise=True, stream=None):
    """d_logits [n,E] (the logits' type) of L = <weights, d_weights>, from the logits and the experts that lsm_moe_route chose;
    d_weights [n,top_k] float32, not used where there is no expert."""
    if logits.dim() != 2 or chosen.dim() != 2:
        raise ValueError("need logits [n,E], chosen [n,top_k], got %s, %s" % (tuple(logits.shape), tuple(chosen.shape)))
    n, E = logits.shape
    k = chosen.shape[1]
    dt = _dtype(logits, "logits")
    dev = _device(logits, "logits")
    _check(logits, (n, E), logits.dtype, dev, "logits")
    _check(chosen, (n, k), torch.int32, dev, "chosen")
    _check(d_weights, (n, k), torch.float32, dev, "d_weights")
    p, _ = _route_params(n, E, k, dt, 1 if renormalise else 0)
    with _alloc_on(stream):
        d_logits = torch.empty_like(logits)
    _done(library().lsm_moe_route_bwd(p, _ptr(logits), _ptr(chosen), _ptr(d_weights), _ptr(d_logits), _stream_handle(stream)),
          "lsm_moe_route_bwd")
    return d_logits


def lsm_moe_plan(chosen, E, workspace=None, stream=None):
    """offsets, order, place: the (token, expert) pairs of chosen [n,top_k] int32 sorted by expert, as the experts' operators take
    them (int32, [E+1], [n top_k], [n,top_k]).  The pairs t top_k + j of expert e are order[offsets[e]:offsets[e+1]], rising; place
    is where each pair went.  A pair whose expert is outside [0, E) is left out: its place, and what is behind offsets[E] in
    order, is -1."""
    if chosen.dim() != 2:
        raise ValueError("chosen: need [n,top_k], got %s" % (tuple(chosen.shape),))
    n, k = chosen.shape
    E = index(E)
    _check(chosen, (n, k), torch.int32, _device(chosen, "chosen"), "chosen")
    p, need = _route_params(n, E, k, 0, 0)
    with _alloc_on(stream):
        workspace = _workspace(workspace, need, chosen)
        offsets = torch.empty(max(E, 0) + 1, dtype=torch.int32, device=chosen.device)
        order = torch.empty(n * k, dtype=torch.int32, device=chosen.device)
        place = torch.empty_like(chosen)
    _done(library().lsm_moe_plan(p, _ptr(chosen), _ptr(offsets), _ptr(order), _ptr(place), _ptr(workspace), _bytes(workspace),
                                 _stream_handle(stream)), "lsm_moe_plan")
    return offsets, order, place


def _experts(x, weights, plan, w_gate_up, w_down, d_y):
    if x.dim() != 2 or weights.dim() != 2 or w_down.dim() != 3:
        raise ValueError("need x [n,D], weights [n,top_k], w_gate_up [E,2F,D], w_down [E,D,F], got %s" %
                         ", ".join(str(tuple(t.shape)) for t in (x, weights, w_gate_up, w_down)))
    n, D = x.shape
    E, _, F = w_down.shape
    k = weights.shape[1]
    dt = _dtype(x, "x")
    offsets, order, place = plan
    dev, dtype = _device(x, "x"), x.dtype
    _check(weights, (n, k), torch.float32, dev, "weights")
    _check(offsets, (E + 1,), torch.int32, dev, "offsets")
    _check(order, (n * k,), torch.int32, dev, "order")
    _check(place, (n, k), torch.int32, dev, "place")
    _check(w_gate_up, (E, 2 * F, D), dtype, dev, "w_gate_up")
    _check(w_down, (E, D, F), dtype, dev, "w_down")
    stride = _rows(x, dev, "x")
    if d_y is not None and (d_y.dtype != x.dtype or d_y.shape != x.shape):
        raise ValueError("d_y: need %s %s, got %s %s" % (tuple(x.shape), x.dtype, tuple(d_y.shape), d_y.dtype))
    return _experts_params(n, D, F, E, k, dt, 0, stride, D if d_y is None else _rows(d_y, dev, "d_y"))


def lsm_moe_experts(x, weights, plan, w_gate_up, w_down, residual=None, y=None, workspace=None, stream=None):
    """y [n,D] = residual + sum_j weights[t,j] Wd_e (silu(Wg_e x_t) * (Wu_e x_t)) over the pairs of ``plan`` (lsm_moe_plan), for
    any number of tokens (lsm_moe_step, with the routing in it, is the faster form for a decode step of up to about 100).

    x [n,D] float32 or bfloat16, dense along D (rows may be further apart, by multiples of 8 elements); weights [n,top_k] float32;
    w_gate_up [E,2F,D] (F rows of the gate, F rows of the factor), w_down [E,D,F], residual [n,D] or None of x's type; D and F
    multiples of 8, E at most 256, top_k at most 16."""
    p, need, _ = _experts(x, weights, plan, w_gate_up, w_down, None)
    dev = x.get_device()
    _check(residual, x.shape, x.dtype, dev, "residual")
    with _alloc_on(stream):
        workspace = _workspace(workspace, need, x)
        if y is None:
            y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        else:
            _check(y, x.shape, x.dtype, dev, "y")
    _done(library().lsm_moe_experts(p, _ptr(x), _ptr(weights), *map(_ptr, plan), _ptr(w_gate_up), _ptr(w_down), _ptr(residual), _ptr(y),
                                    _ptr(workspace), _bytes(workspace), _stream_handle(stream)), "lsm_moe_experts")
    return y


def lsm_moe_experts_bwd(x, weights, plan, w_gate_up, w_down, d_y, weight_grads=True, workspace=None, stream=None):
    """Gradients of L = <y, d_y>: a dict with dx [n,D] (through the experts; the residual's gradient is d_y), d_weights [n,top_k]
    float32, d_w_gate_up and d_w_down (None without ``weight_grads``).  Nothing is saved by the forward call.  d_y like x, dense
    along D; the other arguments as in lsm_moe_experts."""
    if d_y is None:
        raise ValueError("d_y is required")
    p, _, need = _experts(x, weights, plan, w_gate_up, w_down, d_y)
    with _alloc_on(stream):
        workspace = _workspace(workspace, need, x)
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        d_weights = torch.empty_like(weights)
        d_gate_up, d_down = (torch.empty_like(w_gate_up), torch.empty_like(w_down)) if weight_grads else (None, None)
    _done(library().lsm_moe_experts_bwd(p, _ptr(x), _ptr(weights), *map(_ptr, plan), _ptr(w_gate_up), _ptr(w_down), _ptr(d_y), _ptr(dx),
                                        _ptr(d_weights), _ptr(d_gate_up), _ptr(d_down), _ptr(workspace), _bytes(workspace),
                                        _stream_handle(stream)), "lsm_moe_experts_bwd")
    return dict(dx=dx, d_weights=d_weights, d_w_gate_up=d_gate_up, d_w_down=d_down)


def _vocab(x, w, index_, teacher, temperature):
    if x.dim() != 2 or w.dim() != 2:
        raise ValueError("need x [n,D], w [V,D], got %s, %s" % (tuple(x.shape), tuple(w.shape)))
    n, D = x.shape
    V = w.shape[0]
    dt = _dtype(x, "x")
    dev = _device(x, "x")
    _check(w, (V, D), x.dtype, dev, "w")
    K = 0
    if teacher is None:
        _check(index_, (n,), torch.int32, dev, "target")
    else:
        if index_.dim() != 2:
            raise ValueError("index: need [n,K], got %s" % (tuple(index_.shape),))
        K = index_.shape[1]
        if K == 0:
            raise ValueError("index: need at least one entry a token")
        _check(index_, (n, K), torch.int32, dev, "index")
        _check(teacher, (n, K), torch.float32, dev, "teacher")
    return _vocab_params(n, D, V, K, dt, float(temperature), 0, _rows(x, dev, "x"))


def _vocab_fwd(x, w, index_, teacher, temperature, workspace, stream, name):
    p, need, _ = _vocab(x, w, index_, teacher, temperature)
    with _alloc_on(stream):
        workspace = _workspace(workspace, need, x)
        loss = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
        lse = torch.empty_like(loss)
    _done(library().lsm_vocab_loss(p, _ptr(x), _ptr(w), _ptr(index_), _ptr(teacher), _ptr(loss), _ptr(lse), _ptr(workspace),
                                   _bytes(workspace), _stream_handle(stream)), name)
    return loss, lse


def _vocab_bwd(x, w, index_, teacher, lse, d_loss, temperature, weight_grad, workspace, stream, name):
    p, _, need = _vocab(x, w, index_, teacher, temperature)
    _check(lse, (x.shape[0],), torch.float32, x.get_device(), "lse")
    _check(d_loss, (x.shape[0],), torch.float32, x.get_device(), "d_loss")
    with _alloc_on(stream):
        workspace = _workspace(workspace, need, x)
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        dw = torch.empty_like(w) if weight_grad else None
    _done(library().lsm_vocab_loss_bwd(p, _ptr(x), _ptr(w), _ptr(index_), _ptr(teacher), _ptr(lse), _ptr(d_loss), _ptr(dx), _ptr(dw),
                                       _ptr(workspace), _bytes(workspace), _stream_handle(stream)), name)
    return dict(dx=dx, dw=dw)


def lsm_linear_cross_entropy(x, w, target, temperature=1.0, workspace=None, stream=None):
    """loss, lse [n] float32 of the softmax over z = x w^T / temperature:   lse = log sum_v exp(z_v),   loss = lse - z_target.

    x [n,D] float32 or bfloat16, dense along D (rows may be further apart, by multiples of 8 elements), w [V,D] of its type, target
    [n] int32; D a multiple of 8.  The logits are never kept.  A token whose target is outside [0, V) (-100, say) is left out: loss and
    lse are 0."""
    return _vocab_fwd(x, w, target, None, temperature, workspace, stream, "lsm_linear_cross_entropy")


def lsm_linear_cross_entropy_bwd(x, w, target, lse, d_loss, temperature=1.0, weight_grad=True, workspace=None, stream=None):
    """Gradients of L = <loss, d_loss> with the lse of the forward call: a dict with dx [n,D] (0 for tokens left out) and dw [V,D]
    (None without ``weight_grad``); d_loss [n] float32 (1 / tokens for a mean)."""
    return _vocab_bwd(x, w, target, None, lse, d_loss, temperature, weight_grad, workspace, stream, "lsm_linear_cross_entropy_bwd")


def lsm_linear_distill(x, w, index, teacher, temperature=1.0, workspace=None, stream=None):
    """loss, lse [n] float32: the divergence of softmax(x w^T / temperature) from a teacher of whom each token's K best logits are known.

    index [n,K] int32 and teacher [n,K] float32: tokens and logits, in any order, K at most 256; p = softmax(teacher / temperature) over
    a token's entries, loss = sum_j p_j (log p_j - log softmax(x w^T / temperature)[index_j]).  An entry whose index is outside [0, V) or
    whose logit is -inf or NaN does not count, entries of the same index each count with their own p; a token without any is left out (loss
    and lse 0).  x, w as in lsm_linear_cross_entropy."""
    if teacher is None:
        raise ValueError("teacher is required")
    return _vocab_fwd(x, w, index, teacher, temperature, workspace, stream, "lsm_linear_distill")


def lsm_linear_distill_bwd(x, w, index, teacher, lse, d_loss, temperature=1.0, weight_grad=True, workspace=None, stream=None):
    """Gradients of L = <loss, d_loss> with the lse of the forward call: a dict with dx [n,D] and dw [V,D] (None without
    ``weight_grad``)."""
    if teacher is None:
        raise ValueError("teacher is required")
    return _vocab_bwd(x, w, index, teacher, lse, d_loss, temperature, weight_grad, workspace, stream, "lsm_linear_distill_bwd")
