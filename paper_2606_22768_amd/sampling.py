"""Sampling one token per row of logits: the C call fgd_sample and the
tensor-level sample()."""

from __future__ import annotations

import ctypes

from . import DTYPES, FGD_BF16, FGD_F32, _check, _dev, _stream, lib
from .mx4 import _check_workspace, _current, _on


class fgd_sampling(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("temperature", ctypes.c_float),
                ("temperature_rows", ctypes.c_void_p), ("top_p", ctypes.c_float), ("min_p", ctypes.c_float),
                ("top_p_rows", ctypes.c_void_p), ("min_p_rows", ctypes.c_void_p), ("top_k", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("top_k_rows", ctypes.c_void_p)]


# --------------------------------------------------------------- raw C ABI

def fgd_sample_workspace_size(dtype, num_rows, vocab) -> int:
    n = ctypes.c_int64()
    _check(lib.fgd_sample_workspace_size(DTYPES.get(dtype, dtype), int(num_rows), int(vocab), ctypes.byref(n)),
           "fgd_sample_workspace_size")
    return n.value


def fgd_sample(logits, dtype, num_rows, vocab, ldk, uniform, settings, tokens_out, probs_out=None, workspace=None,
               workspace_bytes=0, stream=None):
    """The C call; `settings` is an fgd_sampling structure."""
    _check(lib.fgd_sample(_dev(logits), DTYPES.get(dtype, dtype), int(num_rows), int(vocab), int(ldk), _dev(uniform),
                          None if settings is None else ctypes.byref(settings), _dev(tokens_out), _dev(probs_out),
                          _dev(workspace), int(workspace_bytes), _stream(stream)), "fgd_sample")


# ----------------------------------------------------------- tensor level

def sample(logits, uniform, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, vocab=None, tokens_out=None,
           probs_out=None, workspace=None, stream=None):
    """One token per row of logits [rows][ldk] (float32 or bfloat16, rows
    contiguous) from uniform [rows] (float32 in [0, 1)); returns (tokens
    int32 [rows], their probabilities among the kept tokens float32 [rows]).
    temperature, top_k, top_p and min_p are numbers, or tensors [rows]
    (float32; int32 for top_k) on the logits' GPU; what they mean, and what
    becomes of rows with nothing left or a NaN, stands at fgd_sample in
    fgd.h.  `vocab` is the number of logits of a row that count (all)."""
    import torch

    if not isinstance(logits, torch.Tensor):
        raise TypeError(f"logits: expected a torch tensor, got {type(logits).__name__}")
    if logits.dtype == torch.float32:
        dtype = FGD_F32
    elif logits.dtype == torch.bfloat16:
        dtype = FGD_BF16
    else:
        raise TypeError(f"logits: expected float32 or bfloat16, got {logits.dtype}")
    if logits.dim() != 2:
        raise ValueError(f"logits: expected [rows][vocab], got shape {tuple(logits.shape)}")
    U, width = logits.shape
    V = width if vocab is None else int(vocab)
    if V > width:
        raise ValueError(f"vocab: {V} is above the {width} logits of a row")
    if width > 1 and logits.stride(1) != 1:
        raise ValueError("logits: rows must be contiguous")
    ldk = logits.stride(0) if U > 1 else max(width, 1)
    if U > 1 and ldk < V:
        raise ValueError("logits: rows must not overlap")
    dev = logits.device
    s = fgd_sampling(ctypes.sizeof(fgd_sampling))
    if type(temperature) is float:
        s.temperature = temperature
    else:
        s.temperature, s.temperature_rows = _setting(temperature, "temperature", torch.float32, U, dev)
    if type(top_k) is int:
        s.top_k = _top_k(top_k)
    else:
        s.top_k, s.top_k_rows = _setting(top_k, "top_k", torch.int32, U, dev)
    if type(top_p) is float:
        s.top_p = top_p
    else:
        s.top_p, s.top_p_rows = _setting(top_p, "top_p", torch.float32, U, dev)
    if type(min_p) is float:
        s.min_p = min_p
    else:
        s.min_p, s.min_p_rows = _setting(min_p, "min_p", torch.float32, U, dev)
    _rows(uniform, "uniform", torch.float32, U, dev)
    if tokens_out is not None:
        _rows(tokens_out, "tokens_out", torch.int32, U, dev)
    if probs_out is not None:
        _rows(probs_out, "probs_out", torch.float32, U, dev)
    need = fgd_sample_workspace_size(dtype, U, V)
    if workspace is not None:
        _check_workspace(workspace, need, dev)
    if dev.type != "cuda":
        raise ValueError(f"logits: expected a tensor on a GPU, got {dev}")
    with _on(dev, stream):
        tokens_out = torch.empty(U, dtype=torch.int32, device=dev) if tokens_out is None else tokens_out
        probs_out = torch.empty(U, dtype=torch.float32, device=dev) if probs_out is None else probs_out
        if workspace is None and need:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        fgd_sample(logits, dtype, U, V, ldk, uniform, s, tokens_out, probs_out, workspace,
                   0 if workspace is None else workspace.numel() * workspace.element_size(), _current(dev))
    return tokens_out, probs_out


def _setting(v, name, dtype, rows, device):
    """(scalar, device address or None) of a number or a tensor of one value per row."""
    import torch

    if isinstance(v, torch.Tensor):
        _rows(v, name, dtype, rows, device)
        return 0, v.data_ptr() or None
    return (_top_k(int(v)) if dtype == torch.int32 else float(v)), None


def _top_k(k):
    """k in the C type's range: a number above every vocabulary keeps all
    tokens, as one that is not above 0 does."""
    return min(max(k, 0), 0x7fffffff)


def _rows(t, name, dtype, rows, device):
    """A tensor of one `dtype` value per row, contiguous, on `device`."""
    import torch

    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor, got {type(t).__name__}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.dim() != 1 or t.shape[0] != rows:
        raise ValueError(f"{name}: expected shape [{rows}], got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if t.device != device:
        raise ValueError(f"{name}: expected a tensor on the logits' device {device}, got {t.device}")
