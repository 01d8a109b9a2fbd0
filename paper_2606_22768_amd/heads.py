"""Queries and keys normed head by head and rotated by their positions, and the
gradients: the C calls fgd_rotate_heads* and tensor-level calls on top of
them.

    q, k = rotate_heads(q, k, positions, freqs, q_weight, k_weight)
    dq, dk, dq_weight, dk_weight = rotate_heads_grads(dq, dk, q, k, positions, freqs, q_weight, k_weight)

with q, k the projection's own (the call's inputs) in both.
"""

from __future__ import annotations

import ctypes

from . import DTYPES, FGD_BF16, FGD_F32, _check, _dev, _stream, lib
from .mx4 import _check_workspace, _current, _dtype_code, _on, _on_gpu

_I64 = ctypes.c_int64


class fgd_heads(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32), ("batch", ctypes.c_int32),
                ("q_heads", ctypes.c_int32), ("k_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("tokens", ctypes.c_int64),
                ("position_stride", ctypes.c_int64), ("weight_stride", ctypes.c_int64), ("eps", ctypes.c_float),
                ("weight_dtype", ctypes.c_int32)]

    def __init__(self, dtype=FGD_F32, batch=1, q_heads=0, k_heads=0, head_dim=0, rot_dim=0, interleaved=0, tokens=0,
                 position_stride=0, weight_stride=0, eps=0.0, weight_dtype=FGD_F32):
        super().__init__(ctypes.sizeof(fgd_heads), DTYPES.get(dtype, dtype), batch, q_heads, k_heads, head_dim, rot_dim,
                         interleaved, tokens, position_stride, weight_stride, eps,
                         DTYPES.get(weight_dtype, weight_dtype))


# --------------------------------------------------------------- raw C ABI

def _strides(s):
    """Strides of batch, token and head as the C call takes them."""
    return None if s is None else (_I64 * 3)(*s)


def fgd_rotate_heads(sizes, q, q_strides, k, k_strides, positions, freqs, q_weight, k_weight, q_out, q_out_strides,
                     k_out, k_out_strides, stream=None):
    _check(lib.fgd_rotate_heads(ctypes.byref(sizes), _dev(q), _strides(q_strides), _dev(k), _strides(k_strides),
                                _dev(positions), _dev(freqs), _dev(q_weight), _dev(k_weight), _dev(q_out),
                                _strides(q_out_strides), _dev(k_out), _strides(k_out_strides), _stream(stream)),
           "fgd_rotate_heads")


def fgd_rotate_heads_grads(sizes, dq, dq_strides, dk, dk_strides, q, q_strides, k, k_strides, positions, freqs,
                           q_weight, k_weight, q_grad, q_grad_strides, k_grad, k_grad_strides, q_weight_grad,
                           k_weight_grad, workspace, workspace_bytes, stream=None):
    _check(lib.fgd_rotate_heads_grads(ctypes.byref(sizes), _dev(dq), _strides(dq_strides), _dev(dk),
                                      _strides(dk_strides), _dev(q), _strides(q_strides), _dev(k), _strides(k_strides),
                                      _dev(positions), _dev(freqs), _dev(q_weight), _dev(k_weight), _dev(q_grad),
                                      _strides(q_grad_strides), _dev(k_grad), _strides(k_grad_strides),
                                      _dev(q_weight_grad), _dev(k_weight_grad), _dev(workspace), workspace_bytes,
                                      _stream(stream)), "fgd_rotate_heads_grads")


def fgd_rotate_heads_grads_workspace_size(sizes) -> int:
    n = _I64()
    _check(lib.fgd_rotate_heads_grads_workspace_size(ctypes.byref(sizes), ctypes.byref(n)),
           "fgd_rotate_heads_grads_workspace_size")
    return n.value


# ----------------------------------------------------------- tensor level

# What the checks of a call found, by the types, shapes, strides and devices
# of its tensors and its settings: a program's next call of the same sizes is
# spared them (rotate_heads of 64 tokens: 10 us of host time for 18).
_PLANS = {}


def _form(t):
    """What a call's checks can depend on of a tensor (or None)."""
    return None if t is None else (t.shape, t.stride(), t.dtype, t.device)


def _known(key):
    """The plan of a call, if it has one and its device is the current one."""
    import torch

    plan = _PLANS.get(key)
    return plan if plan is not None and plan[0] == torch.cuda.current_device() else None


def _keep(key, *plan):
    if len(_PLANS) >= 1024:
        _PLANS.clear()
    _PLANS[key] = plan


def _array(name, t, dtype, device):
    """A contiguous tensor of `dtype` on `device`."""
    import torch

    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor, got {type(t).__name__}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name}: expected a tensor on {device}, got {t.device}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")


def _heads(name, t, like=None):
    """(batch, tokens, heads, dim) of a tensor of heads, which has the type,
    device and axes of `like`."""
    code = _dtype_code(t, name)
    if t.dim() not in (3, 4):
        raise ValueError(f"{name}: expected [tokens][heads][dim] or [batch][tokens][heads][dim], got shape "
                         f"{tuple(t.shape)}")
    if t.shape[-1] > 1 and t.numel() and t.stride(-1) != 1:
        raise ValueError(f"{name}: heads must be contiguous")
    if like is not None:
        if t.dtype != like.dtype:
            raise TypeError(f"{name}: expected {like.dtype}, got {t.dtype}")
        if t.device != like.device:
            raise ValueError(f"{name}: expected a tensor on {like.device}, got {t.device}")
        if t.shape[:-2] != like.shape[:-2] or t.shape[-1] != like.shape[-1]:
            raise ValueError(f"{name}: expected shape {(*like.shape[:-2], 'heads', like.shape[-1])}, got "
                             f"{tuple(t.shape)}")
    return code, (t.shape[0] if t.dim() == 4 else 1), *t.shape[-3:]


def _axes(t):
    """Strides of batch, token and head."""
    return None if t is None else (t.stride(0) if t.dim() == 4 else 0, t.stride(-3), t.stride(-2))


def _sizes(q, k, positions, freqs, q_weight, k_weight, eps, interleaved):
    """The call's sizes, after the checks of what both directions share."""
    import torch

    if q is None:
        raise TypeError("q: expected a torch tensor, got None")
    code, batch, tokens, heads, dim = _heads("q", q)
    device = q.device
    k_heads = 0 if k is None else _heads("k", k, q)[3]
    if k is None and k_weight is not None:
        raise ValueError("k_weight: there are no keys")
    rot = pstride = 0
    if freqs is not None:
        _array("freqs", freqs, torch.float64, device)
        if freqs.dim() != 1:
            raise ValueError(f"freqs: expected shape [rotated elements / 2], got {tuple(freqs.shape)}")
        rot = 2 * freqs.shape[0]
        _array("positions", positions, torch.int32, device)
        if tuple(positions.shape) == (tokens,):
            pass
        elif q.dim() == 4 and tuple(positions.shape) == (batch, tokens):
            pstride = tokens
        else:
            raise ValueError(f"positions: expected shape [{tokens}]{f' or [{batch}][{tokens}]' if q.dim() == 4 else ''}"
                             f", got {tuple(positions.shape)}")
    wcode, wstride = None, None
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is None:
            continue
        c = _dtype_code(w, name)
        _array(name, w, w.dtype, device)
        if tuple(w.shape) == (dim,):
            stride = 0
        elif q.dim() == 4 and tuple(w.shape) == (batch, dim):
            stride = dim
        else:
            raise ValueError(f"{name}: expected shape [{dim}]{f' or [{batch}][{dim}]' if q.dim() == 4 else ''}, got "
                             f"{tuple(w.shape)}")
        if wcode not in (None, c) or wstride not in (None, stride):
            raise ValueError("q_weight and k_weight must have one type and shape")
        wcode, wstride = c, stride
    return fgd_heads(code, batch, heads, k_heads, dim, rot, int(bool(interleaved)), tokens, pstride, wstride or 0,
                     float(eps), FGD_F32 if wcode is None else wcode)


def _like(name, t, of):
    """`t` as an output in the place of `of`, new if there is none."""
    import torch

    if of is None:
        if t is not None:
            raise ValueError(f"{name}: there are no keys")
        return None
    if t is None:
        return torch.empty(of.shape, dtype=of.dtype, device=of.device)
    _heads(name, t, of)
    if t.shape != of.shape:
        raise ValueError(f"{name}: expected shape {tuple(of.shape)}, got {tuple(t.shape)}")
    return t


def rotate_heads(q, k, positions, freqs, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, q_out=None,
                 k_out=None, stream=None):
    """(q', k'): q [T][heads][D] and k (or None) [T][its heads][D], float32 or
    bfloat16, or both with a batch's axis before (every worker's), heads
    contiguous: each head over the root of its mean square plus eps and times
    its weight (float32 or bfloat16 [D], or [batch][D]; None: no norm), then
    its first 2 len(freqs) elements turned by positions (int32 [T], or
    [batch][T]) times freqs (float64; None: no rotation), in pairs (i, i +
    len(freqs)), or (2 i, 2 i + 1) if `interleaved`.  q_out and k_out may be q
    and k themselves."""
    import torch

    plain = q_out is None and k_out is None and stream is None and type(eps) is float and type(interleaved) is bool
    if plain:
        try:
            key = (_form(q), _form(k), _form(positions), _form(freqs), _form(q_weight), _form(k_weight), eps,
                   interleaved, "rotate")
            plan = _known(key)
        except AttributeError:  # no tensors: the checks say so
            key = plan = None
        if plan is not None:
            index, sizes, qs, ks, qos, kos = plan
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
            k_out = None if k is None else torch.empty_like(k, memory_format=torch.contiguous_format)
            _check(lib.fgd_rotate_heads(ctypes.byref(sizes), q.data_ptr(), qs, _at(k), ks, _at(positions), _at(freqs),
                                        _at(q_weight), _at(k_weight), q_out.data_ptr(), qos, _at(k_out), kos,
                                        _current(index)), "fgd_rotate_heads")
            return q_out, k_out
    sizes = _sizes(q, k, positions, freqs, q_weight, k_weight, eps, interleaved)
    _on_gpu("q", q, None)
    with _on(q.device, stream):
        q_out, k_out = _like("q_out", q_out, q), _like("k_out", k_out, k)
        fgd_rotate_heads(sizes, q, _axes(q), k, _axes(k), positions, freqs, q_weight, k_weight, q_out, _axes(q_out),
                         k_out, _axes(k_out), _current(q.device))
    if plain and key is not None:
        _keep(key, q.device.index, sizes, *(_strides(_axes(t)) for t in (q, k, q_out, k_out)))
    return q_out, k_out


def _at(t):
    """A tensor's address, without a check of its device."""
    return None if t is None else t.data_ptr()


def rotate_heads_grads(dq, dk, q, k, positions, freqs, q_weight=None, k_weight=None, eps=1e-6, interleaved=False,
                       workspace=None, stream=None):
    """The gradients (of q, of k, of q_weight, of k_weight) of rotate_heads(q,
    k, ...) from those of its outputs; the weights' in float32, of shared ones
    the sum over the batch.  None in the place of what there is not; q and k
    may be None where they have no weight.  The workspace (a uint8 device
    tensor of fgd_rotate_heads_grads_workspace_size bytes) is allocated when
    not given."""
    import torch

    plain = workspace is None and stream is None and type(eps) is float and type(interleaved) is bool
    if plain:
        try:
            key = (_form(dq), _form(dk), _form(q), _form(k), _form(positions), _form(freqs), _form(q_weight),
                   _form(k_weight), eps, interleaved, "grads")
            plan = _known(key)
        except AttributeError:
            key = plan = None
        if plan is not None:
            index, sizes, need, strides = plan
            q_grad = torch.empty_like(dq, memory_format=torch.contiguous_format)
            k_grad = None if dk is None else torch.empty_like(dk, memory_format=torch.contiguous_format)
            wq = None if q_weight is None else torch.empty_like(q_weight, dtype=torch.float32)
            wk = None if k_weight is None else torch.empty_like(k_weight, dtype=torch.float32)
            work = dq.new_empty(need, dtype=torch.uint8) if need else None
            _check(lib.fgd_rotate_heads_grads(ctypes.byref(sizes), dq.data_ptr(), strides[0], _at(dk), strides[1],
                                              _at(q), strides[2], _at(k), strides[3], _at(positions), _at(freqs),
                                              _at(q_weight), _at(k_weight), q_grad.data_ptr(), strides[4], _at(k_grad),
                                              strides[5], _at(wq), _at(wk), _at(work), need, _current(index)),
                   "fgd_rotate_heads_grads")
            return q_grad, k_grad, wq, wk
    sizes = _sizes(dq, dk, positions, freqs, q_weight, k_weight, eps, interleaved)
    for name, x, dy, w in (("q", q, dq, q_weight), ("k", k, dk, k_weight)):
        if x is None and w is not None:
            raise TypeError(f"{name}: expected a torch tensor, got None")
        if x is not None and dy is not None:
            _heads(name, x, dy)
            if x.shape != dy.shape:
                raise ValueError(f"{name}: expected shape {tuple(dy.shape)}, got {tuple(x.shape)}")
    need = fgd_rotate_heads_grads_workspace_size(sizes)
    need = 0 if q_weight is None and k_weight is None else need
    if workspace is not None:
        _check_workspace(workspace, need, dq.device)
    _on_gpu("dq", dq, None)
    with _on(dq.device, stream):
        q_grad, k_grad = _like("", None, dq), _like("", None, dk)
        wq, wk = (None if w is None else torch.empty(w.shape, dtype=torch.float32, device=dq.device)
                  for w in (q_weight, k_weight))
        if workspace is None and need:
            workspace = torch.empty(need, dtype=torch.uint8, device=dq.device)
        fgd_rotate_heads_grads(sizes, dq, _axes(dq), dk, _axes(dk), q, _axes(q), k, _axes(k), positions, freqs, q_weight,
                               k_weight, q_grad, _axes(q_grad), k_grad, _axes(k_grad), wq, wk, workspace,
                               0 if workspace is None else workspace.numel() * workspace.element_size(),
                               _current(dq.device))
    if plain and key is not None:
        _keep(key, dq.device.index, sizes, need, tuple(_strides(_axes(t)) for t in (dq, dk, q, k, q_grad, k_grad)))
    return q_grad, k_grad, wq, wk
