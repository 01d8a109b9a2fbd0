"""Matrices in microscaled 4-bit floating point and products of them: the C
calls fgd_mx4_* and tensor-level calls on top of them.

A quantised matrix (Mx4) holds 17 bytes for every 32 elements of a row.  Its
blocks run along its rows, the axis a product sums over; a transposed view
is quantised along the other axis of the stored matrix, as a layer's
gradients need it:

    w4 = mx4_quantize(w)                  # w [N][K], or [M][N][K]: every worker's
    y = mx4_linear(x, w4)                 # x [T][K] -> y [T][N]
    dx, dw = mx4_linear_grads(dy, x, mx4_quantize(w.mT))

A call that is given a stream runs on it, and the tensors that it allocates
belong to that stream, as under torch.cuda.stream; before another stream uses
them, it has to wait.
"""

from __future__ import annotations

import contextlib
import ctypes

from . import DTYPES, FGD_BF16, FGD_F32, _check, _dev, _stream, lib

_I64 = ctypes.c_int64


# --------------------------------------------------------------- raw C ABI

def fgd_mx4_size(batch, rows, cols):
    """(bytes of the codes, bytes of the scales)."""
    if batch > 0x7fffffff:  # ctypes would take its lower 32 bits
        raise ValueError(f"batch: {batch} is above 2^31 - 1")
    c, s = _I64(), _I64()
    _check(lib.fgd_mx4_size(int(batch), int(rows), int(cols), ctypes.byref(c), ctypes.byref(s)), "fgd_mx4_size")
    return c.value, s.value


def fgd_mx4_quantize(x, dtype, batch, rows, cols, batch_stride, row_stride, col_stride, codes, scales, stream=None):
    _check(lib.fgd_mx4_quantize(_dev(x), DTYPES.get(dtype, dtype), batch, rows, cols, batch_stride, row_stride,
                                col_stride, _dev(codes), _dev(scales), _stream(stream)), "fgd_mx4_quantize")


def fgd_mx4_quantize_both(x, dtype, batch, rows, cols, batch_stride, row_stride, codes, scales, t_codes, t_scales,
                          stream=None):
    _check(lib.fgd_mx4_quantize_both(_dev(x), DTYPES.get(dtype, dtype), batch, rows, cols, batch_stride, row_stride,
                                     _dev(codes), _dev(scales), _dev(t_codes), _dev(t_scales), _stream(stream)),
           "fgd_mx4_quantize_both")


def fgd_mx4_dequantize(codes, scales, batch, rows, cols, out, dtype, batch_stride, row_stride, stream=None):
    _check(lib.fgd_mx4_dequantize(_dev(codes), _dev(scales), batch, rows, cols, _dev(out), DTYPES.get(dtype, dtype),
                                  batch_stride, row_stride, _stream(stream)), "fgd_mx4_dequantize")


def fgd_mx4_matmul(a_codes, a_scales, w_codes, w_scales, batch, m, n, k, out, out_dtype, out_batch_stride,
                   out_row_stride, stream=None):
    _check(lib.fgd_mx4_matmul(_dev(a_codes), _dev(a_scales), _dev(w_codes), _dev(w_scales), batch, m, n, k,
                              _dev(out), DTYPES.get(out_dtype, out_dtype), out_batch_stride, out_row_stride,
                              _stream(stream)), "fgd_mx4_matmul")


def fgd_mx4_linear(x, x_dtype, x_batch_stride, x_row_stride, w_codes, w_scales, batch, tokens, n, k, out, out_dtype,
                   out_batch_stride, out_row_stride, workspace, workspace_bytes, stream=None):
    _check(lib.fgd_mx4_linear(_dev(x), DTYPES.get(x_dtype, x_dtype), x_batch_stride, x_row_stride, _dev(w_codes),
                              _dev(w_scales), batch, tokens, n, k, _dev(out), DTYPES.get(out_dtype, out_dtype),
                              out_batch_stride, out_row_stride, _dev(workspace), workspace_bytes, _stream(stream)),
           "fgd_mx4_linear")


def fgd_mx4_linear_workspace_size(batch, tokens, k) -> int:
    n = _I64()
    _check(lib.fgd_mx4_linear_workspace_size(int(batch), int(tokens), int(k), ctypes.byref(n)),
           "fgd_mx4_linear_workspace_size")
    return n.value


def fgd_mx4_linear_grads(dy, dy_dtype, dy_batch_stride, dy_row_stride, x, x_dtype, x_batch_stride, x_row_stride,
                         wt_codes, wt_scales, batch, tokens, n, k, dx, dx_dtype, dx_batch_stride, dx_row_stride, dw,
                         dw_dtype, dw_batch_stride, dw_row_stride, workspace, workspace_bytes, stream=None):
    _check(lib.fgd_mx4_linear_grads(_dev(dy), DTYPES.get(dy_dtype, dy_dtype), dy_batch_stride, dy_row_stride, _dev(x),
                                    DTYPES.get(x_dtype, x_dtype), x_batch_stride, x_row_stride, _dev(wt_codes),
                                    _dev(wt_scales), batch, tokens, n, k, _dev(dx), DTYPES.get(dx_dtype, dx_dtype),
                                    dx_batch_stride, dx_row_stride, _dev(dw), DTYPES.get(dw_dtype, dw_dtype),
                                    dw_batch_stride, dw_row_stride, _dev(workspace), workspace_bytes,
                                    _stream(stream)), "fgd_mx4_linear_grads")


def fgd_mx4_linear_grads_workspace_size(batch, tokens, n, k) -> int:
    size = _I64()
    _check(lib.fgd_mx4_linear_grads_workspace_size(int(batch), int(tokens), int(n), int(k), ctypes.byref(size)),
           "fgd_mx4_linear_grads_workspace_size")
    return size.value


# ----------------------------------------------------------- tensor level

class Mx4:
    """A matrix [rows][cols], or a batch of them, in microscaled 4-bit
    floating point: the device arrays `codes` and `scales` (uint8, laid out
    as fgd.h says) and the sizes.  `batch` is None for a single matrix.
    Made from arrays that were kept (a checkpoint's), these are checked: the
    kernels read as many bytes as the sizes say."""

    __slots__ = ("codes", "scales", "batch", "rows", "cols")

    def __init__(self, codes, scales, batch, rows, cols):
        import torch

        need = fgd_mx4_size(1 if batch is None else batch, rows, cols)
        for name, t, size in (("codes", codes, need[0]), ("scales", scales, need[1])):
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name}: expected a torch tensor, got {type(t).__name__}")
            if t.dtype != torch.uint8:
                raise TypeError(f"{name}: expected uint8, got {t.dtype}")
            if t.numel() != size:
                raise ValueError(f"{name}: expected {size} bytes, got {t.numel()}")
            if not t.is_contiguous():
                raise ValueError(f"{name}: must be contiguous")
        if scales.device != codes.device:
            raise ValueError(f"scales: expected a tensor on {codes.device}, got {scales.device}")
        self.codes, self.scales, self.batch, self.rows, self.cols = codes, scales, batch, rows, cols

    @property
    def shape(self):
        return (self.rows, self.cols) if self.batch is None else (self.batch, self.rows, self.cols)

    @property
    def device(self):
        return self.codes.device

    @property
    def nbytes(self):
        return self.codes.numel() + self.scales.numel()

    def __repr__(self):
        return f"Mx4(shape={self.shape}, device={self.device})"


def _dtype_code(t, name):
    import torch

    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor, got {type(t).__name__}")
    if t.dtype == torch.float32:
        return FGD_F32
    if t.dtype == torch.bfloat16:
        return FGD_BF16
    raise TypeError(f"{name}: expected float32 or bfloat16, got {t.dtype}")


def _matrix(t, name):
    """(dtype code, batch or None, rows, cols, batch stride, row stride, col stride)."""
    code = _dtype_code(t, name)
    if t.dim() == 2:
        return (code, None, *t.shape, 0, *t.stride())
    if t.dim() == 3:
        return (code, *t.shape, *t.stride())
    raise ValueError(f"{name}: expected [rows][cols] or [batch][rows][cols], got shape {tuple(t.shape)}")


def _on_gpu(name, t, device):
    if t.device.type != "cuda" or (device is not None and t.device != device):
        raise ValueError(f"{name}: expected a tensor on {'a GPU' if device is None else device}, got {t.device}")


_HERE = contextlib.nullcontext()


def _on(device, stream=None):
    """A context in which `device` and the stream (torch's current one when
    none is given) are current, so that what a call allocates in it belongs to
    the stream that uses it."""
    import torch

    if stream is None:
        return _HERE if torch.cuda.current_device() == device.index else torch.cuda.device(device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(_stream(stream), device)
    if stream.device != device:
        raise ValueError(f"stream: expected a stream of {device}, got one of {stream.device}")
    return torch.cuda.stream(stream)


def _current(device):
    """torch's current stream on `device`, a torch device or its number (which
    spares torch a search for the current one, which takes longer than the rest
    of a call)."""
    import torch

    index = device if type(device) is int else device.index
    try:
        return torch._C._cuda_getCurrentRawStream(index)  # 0.1 us; the stream's object takes 1.1
    except AttributeError:  # a torch without it
        return torch.cuda.current_stream(index).cuda_stream


def _is_mx4(q, name):
    if not isinstance(q, Mx4):
        raise TypeError(f"{name}: expected an Mx4 matrix (mx4_quantize), got {type(q).__name__}")
    return q


def _output_dtype(out, dtype, shape, device):
    """torch's dtype of the output tensor, which is checked if there is one."""
    import torch

    if out is None:
        t = {"f32": torch.float32, "bf16": torch.bfloat16}.get(dtype, dtype)
        if t not in (torch.float32, torch.bfloat16):
            raise TypeError(f"dtype: expected 'f32' or 'bf16', got {dtype!r}")
        return t
    _dtype_code(out, "out")
    if tuple(out.shape) != tuple(shape):
        raise ValueError(f"out: expected shape {tuple(shape)}, got {tuple(out.shape)}")
    _on_gpu("out", out, device)
    if out.shape[-1] > 1 and out.stride(-1) != 1:
        raise ValueError("out: rows must be contiguous")
    return out.dtype


def _output(out, t, shape, device):
    """The output tensor, new if there is none, and its dtype code and strides."""
    import torch

    if out is None:
        out = torch.empty(shape, dtype=t, device=device)
    return out, FGD_F32 if t == torch.float32 else FGD_BF16, (out.stride(0) if out.dim() == 3 else 0), out.stride(-2)


def _packed(n, batch, rows, cols, device):
    import torch

    cb, sb = fgd_mx4_size(n, rows, cols)
    q = Mx4.__new__(Mx4)  # what it is given needs no check
    q.codes = torch.empty(cb, dtype=torch.uint8, device=device)
    q.scales = torch.empty(sb, dtype=torch.uint8, device=device)
    q.batch, q.rows, q.cols = batch, rows, cols
    return q


def mx4_quantize(x, stream=None) -> Mx4:
    """x [rows][cols] or [batch][rows][cols], float32 or bfloat16, its rows or
    its columns contiguous (a transposed view is quantised along the stored
    matrix's columns)."""
    code, batch, rows, cols, bs, rs, cs = _matrix(x, "x")
    if x.numel() and rs != 1 and cs != 1:
        if cols == 1:
            cs = 1  # a single element per row: its column stride is never used
        elif rows == 1:
            rs = 1
        else:
            raise ValueError("x: its rows or its columns must be contiguous")
    _on_gpu("x", x, None)
    n = 1 if batch is None else batch
    with _on(x.device, stream):
        q = _packed(n, batch, rows, cols, x.device)
        fgd_mx4_quantize(x, code, n, rows, cols, bs, rs, cs, q.codes, q.scales, _current(x.device))
    return q


def mx4_quantize_both(x, stream=None):
    """(mx4_quantize(x), mx4_quantize(x.mT)) from one reading of x: what a
    matrix needs that takes part in a layer's product and in its gradients."""
    code, batch, rows, cols, bs, rs, cs = _matrix(x, "x")
    if cols > 1 and x.numel() and cs != 1:
        if rs != 1 and rows > 1:  # a single row's elements are columns of their own
            raise ValueError("x: its rows or its columns must be contiguous")
        t, q = mx4_quantize_both(x.mT, stream)
        return q, t
    _on_gpu("x", x, None)
    n = 1 if batch is None else batch
    with _on(x.device, stream):
        q, t = _packed(n, batch, rows, cols, x.device), _packed(n, batch, cols, rows, x.device)
        fgd_mx4_quantize_both(x, code, n, rows, cols, bs, rs, q.codes, q.scales, t.codes, t.scales,
                              _current(x.device))
    return q, t


def mx4_dequantize(q, dtype="f32", out=None, stream=None):
    """The values of q, as a tensor of `dtype` ("f32", "bf16" or torch's) or
    into `out`."""
    _is_mx4(q, "q")
    t = _output_dtype(out, dtype, q.shape, q.device)
    _on_gpu("q", q, None)
    with _on(q.device, stream):
        out, code, bs, rs = _output(out, t, q.shape, q.device)
        fgd_mx4_dequantize(q.codes, q.scales, 1 if q.batch is None else q.batch, q.rows, q.cols, out, code, bs, rs,
                           _current(q.device))
    return out


def mx4_matmul(a, w, dtype="bf16", out=None, stream=None):
    """a [..][m][k] times w [..][n][k], transposed: [..][m][n] of `dtype`, or
    into `out`.  Both are Mx4, with the same batch."""
    _is_mx4(a, "a")
    _is_mx4(w, "w")
    if a.cols != w.cols or a.batch != w.batch:
        raise ValueError(f"a and w must share their batch and columns, got {a.shape} and {w.shape}")
    if a.device != w.device:
        raise ValueError(f"a and w must be on one GPU, got {a.device} and {w.device}")
    shape = (a.rows, w.rows) if a.batch is None else (a.batch, a.rows, w.rows)
    t = _output_dtype(out, dtype, shape, a.device)
    _on_gpu("a", a, None)
    with _on(a.device, stream):
        out, code, bs, rs = _output(out, t, shape, a.device)
        fgd_mx4_matmul(a.codes, a.scales, w.codes, w.scales, 1 if a.batch is None else a.batch, a.rows, w.rows,
                       a.cols, out, code, bs, rs, _current(a.device))
    return out


def mx4_linear(x, w, dtype=None, out=None, workspace=None, stream=None):
    """x [..][T][K] (float32 or bfloat16, rows contiguous) through a layer
    with 4-bit weights w [..][N][K]: quantises x and returns [..][T][N] of
    x's dtype, of `dtype`, or into `out`.  The workspace (a uint8 device
    tensor of fgd_mx4_linear_workspace_size bytes) is allocated when not
    given."""
    import torch

    code, batch, rows, cols, bs, rs, cs = _matrix(x, "x")
    _is_mx4(w, "w")
    if cols != w.cols or batch != w.batch:
        raise ValueError(f"x and w must share their batch and columns, got {tuple(x.shape)} and {w.shape}")
    if cols > 1 and x.numel() and cs != 1:
        raise ValueError("x: rows must be contiguous")
    _on_gpu("x", x, w.device)
    n = 1 if batch is None else batch
    shape = (rows, w.rows) if batch is None else (batch, rows, w.rows)
    t = _output_dtype(out, x.dtype if dtype is None else dtype, shape, x.device)
    need = fgd_mx4_linear_workspace_size(n, rows, cols)
    if workspace is not None:
        _check_workspace(workspace, need, x.device)
    with _on(x.device, stream):
        out, ocode, obs, ors = _output(out, t, shape, x.device)
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
        fgd_mx4_linear(x, code, bs, rs, w.codes, w.scales, n, rows, w.rows, cols, out, ocode, obs, ors, workspace,
                       workspace.numel() * workspace.element_size(), _current(x.device))
    return out


def _check_workspace(t, need, device):
    import torch

    if not isinstance(t, torch.Tensor):
        raise TypeError(f"workspace: expected a torch tensor, got {type(t).__name__}")
    if t.numel() * t.element_size() < need:
        raise ValueError(f"workspace: needs at least {need} bytes, got {t.numel() * t.element_size()}")
    if not t.is_contiguous():
        raise ValueError("workspace: must be contiguous")
    _on_gpu("workspace", t, device)


def mx4_linear_grads(dy, x, w_t, dx_dtype=None, dw_dtype="f32", stream=None):
    """The gradients of y = x w^T from 4-bit products, each operand quantised
    along the axis its product sums over (the rounding itself is passed
    through): dx [..][T][K] = dy w in dy's dtype (or dx_dtype) and dw
    [..][N][K] = dy^T x in dw_dtype.  dy [..][T][N]; x [..][T][K], or
    mx4_quantize(x.mT) kept from the forward pass; w_t = mx4_quantize(w.mT)."""
    import torch

    _is_mx4(w_t, "w_t")
    code, batch, T, N, bs, rs, cs = _matrix(dy, "dy")
    dx_dtype = dy.dtype if dx_dtype is None else dx_dtype
    if isinstance(x, Mx4):
        x_t = x
        if x_t.rows != w_t.rows:
            raise ValueError(f"x: expected {w_t.rows} rows of its transpose, got shape {x_t.shape}")
    else:
        xcode, _, _, K, xbs, xrs, xcs = _matrix(x, "x")
        if x.shape[:-1] != dy.shape[:-1] or K != w_t.rows:
            raise ValueError(f"x: expected shape {(*dy.shape[:-1], w_t.rows)}, got {tuple(x.shape)}")
        if (cs == 1 or N == 1) and (xcs == 1 or K == 1):  # one call
            if w_t.cols != N or w_t.batch != batch:
                raise ValueError(f"dy and w_t must share their batch and columns, got {tuple(dy.shape)} and "
                                 f"{w_t.shape}")
            device = w_t.device
            _on_gpu("dy", dy, device)
            _on_gpu("x", x, device)
            dims = () if batch is None else (batch,)
            dx_t = _output_dtype(None, dx_dtype, None, device)
            dw_t = _output_dtype(None, dw_dtype, None, device)
            n = 1 if batch is None else batch
            need = fgd_mx4_linear_grads_workspace_size(n, T, N, K)
            with _on(device, stream):
                dx, dxcode, dxbs, dxrs = _output(None, dx_t, (*dims, T, K), device)
                dw, dwcode, dwbs, dwrs = _output(None, dw_t, (*dims, N, K), device)
                workspace = torch.empty(need, dtype=torch.uint8, device=device)
                fgd_mx4_linear_grads(dy, code, bs, rs, x, xcode, xbs, xrs, w_t.codes, w_t.scales, n, T, N, K, dx,
                                     dxcode, dxbs, dxrs, dw, dwcode, dwbs, dwrs, workspace, need, _current(device))
            return dx, dw
        x_t = mx4_quantize(x.mT, stream)
    dy4, dy_t = mx4_quantize_both(dy, stream)
    dx = mx4_matmul(dy4, w_t, dx_dtype, stream=stream)
    dw = mx4_matmul(dy_t, x_t, dw_dtype, stream=stream)
    return dx, dw
