"""Binding of the operators around the token mixer declared in include/lsm_block.h: norm and rotation of queries and keys,
a mixture-of-experts layer for a few tokens, one step of a beam search.

Argument marshalling only, as in binding.py: every operator runs in the HIP kernels of liblsm_hip.so on ``stream``
(default: torch's current stream) without synchronising.  Every tensor begins at a multiple of 16 bytes, as torch allocates
them; a view that begins elsewhere (a row of a [steps, B] table of positions) is refused, and copied by the caller.
"""
import ctypes
import functools
from operator import index

import torch

from .binding import (DTYPE_BF16, DTYPE_F32, LAYOUT_BHTD, LAYOUT_BTHD, LsmError, _alloc_on, _check, _ptr, _stream_handle,
                      library)

NORM_NONE, NORM_RMS, NORM_L2 = 0, 1, 2
ROT_HALVES, ROT_PAIRS = 0, 1

_ERR_SHAPE, _ERR_ALIGN = -2, -4  # of lsm_status
_DTYPES = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}


class _QkParams(ctypes.Structure):
    _fields_ = ([("struct_size", ctypes.c_uint32)]
                + [(n, ctypes.c_int32) for n in ("B", "T", "H_q", "H_k", "d", "dtype", "norm", "rotation", "rot_dim", "n_pos")]
                + [(n, ctypes.c_float) for n in ("eps", "q_scale", "k_scale")] + [("reserved", ctypes.c_int32)]
                + [(n, ctypes.c_int64 * 3) for n in ("q", "k", "q_out", "k_out", "dq", "dk")])


def _dtype(t, name):
    try:
        return _DTYPES[t.dtype]
    except KeyError:
        raise ValueError("%s must be float32 or bfloat16" % name) from None


def _heads(shape, stride, layout, name):
    """(B, T, H, d), (batch, head, token strides) of a [B,H,T,d], [B,T,H,d] or, for one token, [B,H,d] tensor."""
    if len(shape) not in (3, 4) or stride[-1] != 1:
        raise ValueError("%s: need 3 or 4 axes, the last one dense, got %s with strides %s" % (name, tuple(shape), tuple(stride)))
    if len(shape) == 3:
        return (shape[0], 1, shape[1], shape[2]), (stride[0], stride[1], 0)
    if layout == LAYOUT_BTHD:
        return tuple(shape), (stride[0], stride[2], stride[1])
    return (shape[0], shape[2], shape[1], shape[3]), tuple(stride[:3])


def _shape_of(sizes, layout, dim):
    B, T, H, d = sizes
    return (B, H, d) if dim == 3 else (B, T, H, d) if layout == LAYOUT_BTHD else (B, H, T, d)


def _dense(shape):
    stride, n = [], 1
    for s in reversed(shape):
        stride.insert(0, n)
        n *= s
    return tuple(stride)


# What follows from shapes and strides alone is worked out once and kept (sizes only, no pointers): a decoded token's call costs
# little more than its marshalling.  4 sequences, 16 heads: 14 -> 11 us a call.  Every number comes in as a Python one, here and in
# the caches below: a tensor of one element would be found again by its identity, whatever it holds by then.
@functools.lru_cache(maxsize=256)
def _qk_plan(q, k, given, grads, table, dtype, norm, rotation, eps, q_scale, k_scale, layout, out_layout):
    """Parameter block by reference, its workspace's size, shapes of q's and k's results (None where they are given), of the
    positions and of a weight.  q, k, and the pairs given (tensors to write to) and grads (of the results; backward): (shape,
    strides) or None; the results are the outputs or, with grads, the inputs' gradients."""
    sizes, strides = {}, dict(q=(0, 0, 0), k=(0, 0, 0), q_out=(0, 0, 0), k_out=(0, 0, 0), dq=(0, 0, 0), dk=(0, 0, 0))
    sizes["q"], strides["q"] = _heads(*q, layout, "q")
    dim = len(q[0])
    if k is not None:
        sizes["k"], strides["k"] = _heads(*k, layout, "k")
        a, b = sizes["q"], sizes["k"]
        if len(k[0]) != dim or (a[0], a[1], a[3]) != (b[0], b[1], b[3]):
            raise ValueError("q and k differ in more than their heads: %s, %s" % (tuple(q[0]), tuple(k[0])))
    result = ("dq", "dk") if grads is not None else ("q_out", "k_out")
    new = [None, None]
    for i, n in enumerate("qk"):
        if n not in sizes:
            if given[i] is not None or (grads is not None and grads[i] is not None):
                raise ValueError("a tensor for %s without %s" % (n, n))
            continue
        if grads is not None:
            if grads[i] is None:
                raise ValueError("d_%s_out is required" % n)
            got, strides[n + "_out"] = _heads(*grads[i], out_layout, "d_%s_out" % n)
            if got != sizes[n] or len(grads[i][0]) != dim:
                raise ValueError("d_%s_out: need %s, got %s" % (n, _shape_of(sizes[n], out_layout, dim), tuple(grads[i][0])))
        order = layout if grads is not None else out_layout
        shape = _shape_of(sizes[n], order, dim)
        if given[i] is None:
            new[i] = shape
            strides[result[i]] = _heads(shape, _dense(shape), order, result[i])[1]
        else:
            got, strides[result[i]] = _heads(*given[i], order, result[i])
            if got != sizes[n] or len(given[i][0]) != dim:
                raise ValueError("%s: need %s, got %s" % (result[i], shape, tuple(given[i][0])))
    B, T, H, d = sizes["q"]
    n_pos, rot = (0, 0) if table is None else table
    p = ctypes.byref(_QkParams(ctypes.sizeof(_QkParams), B, T, H, sizes["k"][2] if k is not None else 0, d, dtype, norm, rotation,
                               rot, n_pos, eps, q_scale, k_scale, 0, *[(ctypes.c_int64 * 3)(*s) for s in strides.values()]))
    need = library().lsm_qk_norm_rope_bwd_workspace_bytes(p) if grads is not None else 0
    return p, need, new[0], new[1], (B,) if dim == 3 else (B, T), (d,)


def _form(t, like, name):
    """(shape, strides) of a device tensor of q's type, None for None."""
    if t is None:
        return None
    if t.dtype != like.dtype or not t.is_cuda:
        raise ValueError("%s: need a device tensor of %s, got %s on %s" % (name, like.dtype, t.dtype, t.device))
    return t.shape, t.stride()


def _qk_tables(cos_sin, positions, q_weight, k_weight, k, pos_shape, w_shape):
    if cos_sin is not None:
        _check(cos_sin, cos_sin.shape, torch.float32, "cos_sin")
    _check(positions, pos_shape, torch.int32, "positions")
    _check(q_weight, w_shape, torch.float32, "q_weight")
    _check(k_weight, w_shape, torch.float32, "k_weight")
    if k is None and k_weight is not None:
        raise ValueError("k_weight without k")


def _workspace(workspace, need, like):
    """The caller's workspace, or a new one beside `like`."""
    if workspace is None:
        return torch.empty(max(need, 256), dtype=torch.uint8, device=like.device)
    _check(workspace, workspace.shape, workspace.dtype, "workspace")
    return workspace


def _table(cos_sin):
    if cos_sin is None:
        return None
    if cos_sin.dim() != 2:
        raise ValueError("cos_sin: need [n_pos, rot_dim], got %s" % (tuple(cos_sin.shape),))
    return cos_sin.shape


def lsm_qk_norm_rope(q, k=None, cos_sin=None, positions=None, q_weight=None, k_weight=None, norm=NORM_RMS, eps=1e-6,
                     rotation=ROT_HALVES, q_scale=1.0, k_scale=1.0, layout=LAYOUT_BHTD, out_layout=None, q_out=None,
                     k_out=None, stream=None):
    """q_out, k_out = scale * rotation(weight * normalised row), for every head of every token.

    q [B,H_q,T,d], k [B,H_k,T,d] (or None) in ``layout``, float32 or bfloat16, dense along d only: slices of a fused
    projection go in as they stand; [B,H,d] for one token.  d 64, 128 or 256; H_k may differ from H_q.
    norm: NORM_RMS (mean of squares), NORM_L2 (sum of squares: unit rows, what the delta rule expects of keys) or
    NORM_NONE.  q_weight, k_weight: [d] float32 or None.
    cos_sin: [n_pos, rot_dim] float32, rot_dim/2 cosines and then rot_dim/2 sines a position, or None (no rotation); the
    first rot_dim features (a multiple of 16) are rotated, as pairs (i, i + rot_dim/2) or, with ROT_PAIRS, (2i, 2i + 1).
    positions: [B,T] int32 (for q of 3 axes [B]); None: 0..T-1 in every sequence.  A position outside the table makes that
    token's rows NaN.
    out_layout: order of the results (default ``layout``); q_out, k_out: tensors to write to (q, k themselves in ``layout``
    too)."""
    layout = index(layout)
    p, _, q_new, k_new, pos_shape, w_shape = _qk_plan(
        _form(q, q, "q"), _form(k, q, "k"), (_form(q_out, q, "q_out"), _form(k_out, q, "k_out")), None, _table(cos_sin), _dtype(q, "q"),
        index(norm), index(rotation), float(eps), float(q_scale), float(k_scale), layout, layout if out_layout is None else index(out_layout))
    _qk_tables(cos_sin, positions, q_weight, k_weight, k, pos_shape, w_shape)
    with _alloc_on(stream):
        if q_new is not None:
            q_out = torch.empty(q_new, dtype=q.dtype, device=q.device)
        if k_new is not None:
            k_out = torch.empty(k_new, dtype=q.dtype, device=q.device)
    rc = library().lsm_qk_norm_rope(p, _ptr(q), _ptr(k), _ptr(q_weight), _ptr(k_weight), _ptr(cos_sin), _ptr(positions),
                                    _ptr(q_out), _ptr(k_out), _stream_handle(stream))
    if rc != 0:
        raise LsmError(rc, "lsm_qk_norm_rope")
    return q_out, k_out


def lsm_qk_norm_rope_bwd(q, k, d_q_out, d_k_out, cos_sin=None, positions=None, q_weight=None, k_weight=None, norm=NORM_RMS,
                         eps=1e-6, rotation=ROT_HALVES, q_scale=1.0, k_scale=1.0, layout=LAYOUT_BHTD, out_layout=None,
                         dq=None, dk=None, workspace=None, stream=None):
    """Gradients of L = <q_out, d_q_out> + <k_out, d_k_out>: a dict with dq, dk (like q and k, dense, or written to the
    tensors given: slices of a fused projection's gradient) and d_q_weight, d_k_weight ([d] float32; None where there is no
    weight).  The other arguments as in lsm_qk_norm_rope; d_q_out, d_k_out in ``out_layout``, dense along d only."""
    if d_q_out is None:
        raise ValueError("d_q_out is required")
    layout = index(layout)
    p, need, q_new, k_new, pos_shape, w_shape = _qk_plan(
        _form(q, q, "q"), _form(k, q, "k"), (_form(dq, q, "dq"), _form(dk, q, "dk")),
        (_form(d_q_out, q, "d_q_out"), _form(d_k_out, q, "d_k_out")), _table(cos_sin), _dtype(q, "q"),
        index(norm), index(rotation), float(eps), float(q_scale), float(k_scale), layout, layout if out_layout is None else index(out_layout))
    _qk_tables(cos_sin, positions, q_weight, k_weight, k, pos_shape, w_shape)
    with _alloc_on(stream):
        if q_new is not None:
            dq = torch.empty(q_new, dtype=q.dtype, device=q.device)
        if k_new is not None:
            dk = torch.empty(k_new, dtype=q.dtype, device=q.device)
        workspace = _workspace(workspace, need, q)
        dqw = None if q_weight is None else torch.empty(w_shape, dtype=torch.float32, device=q.device)
        dkw = None if k_weight is None else torch.empty(w_shape, dtype=torch.float32, device=q.device)
    rc = library().lsm_qk_norm_rope_bwd(p, _ptr(q), _ptr(k), _ptr(q_weight), _ptr(k_weight), _ptr(cos_sin), _ptr(positions),
                                        _ptr(d_q_out), _ptr(d_k_out), _ptr(dq), _ptr(dk), _ptr(dqw), _ptr(dkw),
                                        _ptr(workspace), workspace.numel(), _stream_handle(stream))
    if rc != 0:
        raise LsmError(rc, "lsm_qk_norm_rope_bwd")
    return dict(dq=dq, dk=dk, d_q_weight=dqw, d_k_weight=dkw)


class _MoeParams(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32)] + [(n, ctypes.c_int32) for n in ("n", "D", "F", "E", "top_k", "dtype", "renormalise")]


@functools.lru_cache(maxsize=256)
def _moe_params(*sizes):
    """Parameter block by reference, and the workspace it asks for."""
    p = ctypes.byref(_MoeParams(ctypes.sizeof(_MoeParams), *sizes))
    return p, library().lsm_moe_step_workspace_bytes(p)


def lsm_moe_step(x, router, w_gate_up, w_down, top_k, renormalise=True, residual=None, y=None, workspace=None, stream=None):
    """y = residual + the mixture of experts of each row of x, for up to 128 tokens (the form for decoding).

    x [n,D], router [E,D], w_gate_up [E,2F,D] (F rows of the gate, F rows of the factor), w_down [E,D,F], residual [n,D] or
    None, all float32 or all bfloat16; D and F multiples of 8, E at most 256, top_k at most 16.  A token goes to the top_k
    experts of largest router output (equal ones by index), weighted by the softmax over all experts, with ``renormalise``
    divided by its sum over the chosen ones: sum_e w_e Wd_e (silu(Wg_e x) * (Wu_e x))."""
    if x.dim() != 2 or router.dim() != 2 or w_down.dim() != 3:
        raise ValueError("need x [n,D], router [E,D], w_gate_up [E,2F,D], w_down [E,D,F], got %s" %
                         ", ".join(str(tuple(t.shape)) for t in (x, router, w_gate_up, w_down)))
    n, D = x.shape
    E, F = router.shape[0], w_down.shape[2]
    dt, dtype = _dtype(x, "x"), x.dtype
    _check(x, (n, D), dtype, "x")
    _check(router, (E, D), dtype, "router")
    _check(w_gate_up, (E, 2 * F, D), dtype, "w_gate_up")
    _check(w_down, (E, D, F), dtype, "w_down")
    _check(residual, (n, D), dtype, "residual")
    p, need = _moe_params(n, D, F, E, index(top_k), dt, 1 if renormalise else 0)
    with _alloc_on(stream):
        workspace = _workspace(workspace, need, x)
        if y is None:
            y = torch.empty_like(x)
        else:
            _check(y, (n, D), dtype, "y")
    rc = library().lsm_moe_step(p, _ptr(x), _ptr(router), _ptr(w_gate_up), _ptr(w_down), _ptr(residual), _ptr(y), _ptr(workspace),
                                workspace.numel(), _stream_handle(stream))
    if rc != 0:
        raise LsmError(rc, "lsm_moe_step")
    return y


class _BeamParams(ctypes.Structure):
    _fields_ = ([("struct_size", ctypes.c_uint32)] + [(n, ctypes.c_int32) for n in ("B", "K", "V", "n_out", "dtype", "eos", "reserved")]
                + [("row_stride", ctypes.c_int64)])


@functools.lru_cache(maxsize=256)
def _beam_params(*sizes):
    """Parameter block by reference, and the workspace it asks for."""
    p = ctypes.byref(_BeamParams(ctypes.sizeof(_BeamParams), *sizes))
    return p, library().lsm_beam_select_workspace_bytes(p)


def lsm_beam_select(logits, scores, n_out=None, finished=None, eos=None, workspace=None, stream=None):
    """scores, parent, token, finished = the n_out (default K, at most 32) best of K x V candidates of each sequence.

    logits [B,K,V] float32 or bfloat16 (dense along V, rows evenly spaced: a padded vocabulary's slice goes in as it is),
    scores [B,K] float32 log-probabilities of the beams so far (-inf: no such beam).  Candidate (k, t) has
    scores[k] + log_softmax(logits[k])[t]; a beam marked in ``finished`` ([B,K] bool; needs eos) offers only eos, at its
    score.  Results [B,n_out], best first, equal scores by rising k V + t: float32 scores, int32 parents and tokens, and with
    an ``eos`` whether the beam has ended (bool), else None.  A NaN logit counts as -inf."""
    if not logits.is_cuda or logits.dim() != 3 or logits.stride(2) != 1 or (logits.shape[0] > 1 and logits.shape[1] > 1
                                                                          and logits.stride(0) != logits.shape[1] * logits.stride(1)):
        raise ValueError("logits: need a [B,K,V] device tensor, dense along V, its rows evenly spaced, got %s with strides %s on %s"
                         % (tuple(logits.shape), logits.stride(), logits.device))
    B, K, V = logits.shape
    dt = _dtype(logits, "logits")
    _check(scores, (B, K), torch.float32, "scores")
    if finished is not None and eos is None:
        raise ValueError("finished needs eos")
    _check(finished, (B, K), torch.bool, "finished")
    n_out = K if n_out is None else index(n_out)
    row = logits.stride(1) if K > 1 else logits.stride(0) if B > 1 else V
    p, need = _beam_params(B, K, V, n_out, dt, -1 if eos is None else index(eos), 0, row)
    with _alloc_on(stream):
        workspace = _workspace(workspace, need, logits)
        out = torch.empty((B, max(n_out, 0)), dtype=torch.float32, device=logits.device)
        parent = torch.empty_like(out, dtype=torch.int32)
        token = torch.empty_like(out, dtype=torch.int32)
        ended = None if eos is None else torch.empty_like(out, dtype=torch.bool)
    rc = library().lsm_beam_select(p, _ptr(logits), _ptr(scores), _ptr(finished), _ptr(out), _ptr(parent), _ptr(token), _ptr(ended),
                                   _ptr(workspace), workspace.numel(), _stream_handle(stream))
    if rc != 0:
        raise LsmError(rc, "lsm_beam_select")
    return out, parent, token, ended


_MAX_STATES = 64


def lsm_state_reorder(states, parent, stream=None):
    """In place: row b K + i of every tensor in ``states`` (one tensor or a list; first axis B K, or [B,K,...]; dense, rows of
    whole 4 bytes) becomes its row b K + parent[b,i].  parent [B,K] int32, as lsm_beam_select returns it for n_out = K; a value
    outside [0, K) fills its row with 0xff bytes (NaN).  Beams that stay are not touched; 64 tensors a launch, none of which
    shares memory with another or with parent."""
    states = [states] if isinstance(states, torch.Tensor) else list(states)
    if parent.dim() != 2:
        raise ValueError("parent: need [B,K], got %s" % (tuple(parent.shape),))
    _check(parent, parent.shape, torch.int32, "parent")
    B, K = parent.shape
    at, size = [], []
    for t in states:  # all of them before the first launch: nothing is moved if one is refused
        if not t.is_cuda or not t.is_contiguous() or t.dim() == 0 or t.numel() == 0 or not (
                t.shape[0] == B * K or (t.dim() > 1 and t.shape[:2] == (B, K))):
            raise ValueError("states: need contiguous device tensors of %d rows, got %s on %s" % (B * K, tuple(t.shape), t.device))
        at.append(t.data_ptr())
        size.append(t.numel() // (B * K) * t.element_size())
        if size[-1] % 4 or at[-1] % 16:
            raise LsmError(_ERR_SHAPE if size[-1] % 4 else _ERR_ALIGN, "lsm_state_reorder")
    if len(at) > _MAX_STATES:  # of one launch's the library sees it itself
        places = sorted(zip(at, size))
        if any(a + n * B * K > b for (a, n), (b, _) in zip(places, places[1:])):
            raise LsmError(_ERR_SHAPE, "lsm_state_reorder")
    for i in range(0, len(at), _MAX_STATES):
        n = min(_MAX_STATES, len(at) - i)
        rc = library().lsm_state_reorder((ctypes.c_void_p * n)(*at[i:i + n]), (ctypes.c_size_t * n)(*size[i:i + n]), n, _ptr(parent),
                                         B, K, _stream_handle(stream))
        if rc != 0:
            raise LsmError(rc, "lsm_state_reorder")
