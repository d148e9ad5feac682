"""Microscaled 4-bit (MX) operands and layers (include/bcpnn.h): argument marshalling only.

A Matrix is a matrix in blocks of 32 values along its rows, each with one power-of-two scale and a
4-bit code per value, in a device buffer as the matrix instructions read it.  quantize makes one,
dequantize gives its values, product multiplies two; Layer is a BCPNN layer for inference on 4-bit
weights.  The functions enqueue on PyTorch's current stream of the tensors' device and wait for
nothing; a Layer enqueues on the stream it was made on, whose device its tensors are on.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import numpy as np
import torch

from . import bcpnn
from .bcpnn import _check, _dev_ptr, _host, lib

DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}

# Small calls are bound by the host (a launch takes 3 us of it), so the checks build no objects, and the
# current stream and device come as the numbers that they are (a torch.cuda.Stream costs 1.8 us) where this
# torch has them so.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                      lambda device: torch.cuda.current_stream(device).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)

_forward, _readout, _predict = lib.bcpnn_mx_forward, lib.bcpnn_mx_readout, lib.bcpnn_mx_predict
_quantize, _dequantize, _product = lib.bcpnn_mx_quantize, lib.bcpnn_mx_dequantize, lib.bcpnn_mx_product
_operand_bytes, _product_bytes = lib.bcpnn_mx_bytes, lib.bcpnn_mx_product_bytes


def _bytes(rows: int, cols: int) -> int:
    n = _operand_bytes(rows, cols)
    if n < 0:
        raise ValueError(f"matrix sizes {rows} x {cols} out of range")
    return n


class Matrix:
    """An MX operand [rows][cols]: its sizes and its buffer (uint8, as long as bcpnn_mx_bytes says)."""
    __slots__ = ("rows", "cols", "data")

    def __init__(self, rows: int, cols: int, data: torch.Tensor):
        _dev_ptr(data, "data", torch.uint8, (_bytes(rows, cols),))
        self.rows, self.cols, self.data = rows, cols, data

    @property
    def shape(self):
        return self.rows, self.cols

    @classmethod
    def empty(cls, rows: int, cols: int, device="cuda") -> "Matrix":
        m = cls.__new__(cls)
        m.rows, m.cols = rows, cols
        m.data = torch.empty(_bytes(rows, cols), dtype=torch.uint8, device=device)
        return m


def _check_matrix(t, name, shape=None):
    """Dtype code of a 2-D CUDA tensor whose rows are contiguous."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    code = DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, float16 or bfloat16, got {t.dtype}")
    if t.dim() != 2 or (shape is not None and t.shape != shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {shape or 'two dimensions'}")
    if t.stride(1) != 1 and t.shape[1] > 1:
        raise ValueError(f"{name} must have contiguous rows")
    return code


def _row_stride(t):
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _operand(m, name, device, rows, cols):
    if not isinstance(m, Matrix):
        raise TypeError(f"{name} must be a Matrix")
    if m.rows != rows or m.cols != cols:
        raise ValueError(f"{name} has shape {m.shape}, expected {(rows, cols)}")
    if m.data.get_device() != device:
        raise ValueError(f"{name} is on {m.data.device}, expected cuda:{device}")
    return m.data.data_ptr()


def _call(fn, device, *args):
    """fn(*args, PyTorch's current stream of `device`) with the device current."""
    if device == _current_device():
        _check(fn(*args, _raw_stream(device)))
    else:
        with torch.cuda.device(device):
            _check(fn(*args, _raw_stream(device)))


def _ptr(t, name, dtype, shape, device):
    """_dev_ptr of a tensor on a layer's device: its kernels run there, whichever device is current."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.get_device() != device:
        raise (ValueError if getattr(t, "is_cuda", False) else TypeError)(f"{name} must be a tensor on cuda:{device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {shape}")
    return t.data_ptr()


def quantize(x: torch.Tensor, rows: bool = True, columns: bool = False, out=None):
    """The Matrix of x (float32, float16 or bfloat16, contiguous rows) with blocks along its rows, the
    Matrix of its transpose (blocks along its columns), or, with both asked for, the pair of them from
    one read of x.  out: the Matrix (or pair) to write instead of new ones."""
    if not (rows or columns):
        raise ValueError("rows or columns must be asked for")
    code = _check_matrix(x, "x")
    r, c = x.shape
    device = x.get_device()
    by_row = by_col = pr = pc = None
    if out is None:
        if rows:
            by_row = Matrix.empty(r, c, x.device)
            pr = by_row.data.data_ptr()
        if columns:
            by_col = Matrix.empty(c, r, x.device)
            pc = by_col.data.data_ptr()
    else:
        by_row, by_col = out if rows and columns else (out, None) if rows else (None, out)
        if rows:
            pr = _operand(by_row, "out", device, r, c)
        if columns:
            pc = _operand(by_col, "out", device, c, r)
    _call(_quantize, device, x.data_ptr(), code, r, c, _row_stride(x), pr, pc)
    return (by_row, by_col) if rows and columns else by_row if rows else by_col


def dequantize(m: Matrix, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None):
    """The values of m [rows][cols] as dtype, or in `out`."""
    if not isinstance(m, Matrix):
        raise TypeError("m must be a Matrix")
    if out is None:
        out = torch.empty((m.rows, m.cols), dtype=dtype, device=m.data.device)
    code = _check_matrix(out, "out", (m.rows, m.cols))
    device = out.get_device()
    _call(_dequantize, device, _operand(m, "m", device, m.rows, m.cols), m.rows, m.cols,
          out.data_ptr(), code, _row_stride(out))
    return out


def product(a: Matrix, b: Matrix, bias: Optional[torch.Tensor] = None, alpha: float = 1.0,
            beta: float = 0.0, out: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.float32):
    """alpha a b^T + beta out + bias: [a.rows][b.rows] of dtype, or in `out` (which beta needs).  bias:
    float32 [b.rows].  The gradients of c = product(a, b) for g = dL/dc, with every matrix
    quantised by row (r) or by column (c): product(g_r, b_c) for a, product(g_c, a_c) for b."""
    if not isinstance(a, Matrix) or not isinstance(b, Matrix):
        raise TypeError("a and b must be Matrices")
    m, n, k = a.rows, b.rows, a.cols
    device = a.data.get_device()
    pb = _operand(b, "b", device, n, k)
    if out is None:
        if beta != 0.0:
            raise ValueError("beta needs out")
        out = torch.empty((m, n), dtype=dtype, device=a.data.device)
    code = _check_matrix(out, "out", (m, n))
    pbias = None
    if bias is not None:
        pbias = _dev_ptr(bias, "bias", torch.float32, (n,))
    if out.get_device() != device or (bias is not None and bias.get_device() != device):
        raise ValueError(f"out and bias must be on cuda:{device}")
    work, size = None, _product_bytes(m, n, k)
    if size > 0:
        work = torch.empty(size, dtype=torch.uint8, device=a.data.device)
    _call(_product, device, a.data.data_ptr(), pb, m, n, k, alpha, beta, pbias, out.data_ptr(), code,
          _row_stride(out), None if work is None else work.data_ptr())
    return out


class Layer:
    """A BCPNN layer for inference on 4-bit weights and inputs (one bcpnn_mx), from the dense weights
    w [N_in][N_out] and biases b [N_out] on the GPU (work of the current stream on them is waited for);
    `of` makes it from a trained bcpnn.Layer."""

    def __init__(self, cfg: bcpnn.Config, mask: Optional[np.ndarray], w: torch.Tensor, b: torch.Tensor,
                 stream=None):
        n_in, n_out = cfg.in_hcu * cfg.in_mcu, cfg.out_hcu * cfg.out_mcu
        pw, pb = _dev_ptr(w, "w", torch.float32, (n_in, n_out)), _dev_ptr(b, "b", torch.float32, (n_out,))
        current = torch.cuda.current_stream(None if w is None else w.device)
        stream = current if stream is None else stream
        for t in (w, b):
            if t is not None and t.get_device() != stream.device_index:
                raise ValueError(f"w and b must be on the stream's device, cuda:{stream.device_index}")
        if stream.cuda_stream != current.cuda_stream:
            stream.wait_stream(current)
        keep = None if mask is None else _host(mask, np.uint8, (cfg.in_hcu, cfg.out_hcu))
        h = ctypes.c_void_p()
        with torch.cuda.device(stream.device_index):
            _check(lib.bcpnn_mx_create(ctypes.byref(cfg), None if keep is None else keep.ctypes.data, pw, pb,
                                       ctypes.c_void_p(stream.cuda_stream), ctypes.byref(h)))
        self._own(cfg, stream, h)

    @classmethod
    def of(cls, layer: bcpnn.Layer) -> "Layer":
        """The present weights, biases and mask of `layer`, on its stream."""
        h = ctypes.c_void_p()
        with torch.cuda.device(layer.stream.device_index):
            _check(lib.bcpnn_mx_from_layer(layer._h, ctypes.byref(h)))
        self = cls.__new__(cls)
        self._own(layer.cfg, layer.stream, h)
        return self

    def _own(self, cfg, stream, h):
        self.cfg, self.stream, self.device, self._h = cfg, stream, stream.device_index, h
        self.n_in, self.n_out = cfg.in_hcu * cfg.in_mcu, cfg.out_hcu * cfg.out_mcu

    def close(self):
        if getattr(self, "_h", None):
            lib.bcpnn_mx_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def forward(self, x, y, s=None):
        """y (and s, the support) [B][N_out] of x [B][N_in]."""
        B, device = x.shape[0], self.device
        if device != _current_device():
            with torch.cuda.device(device):
                return self.forward(x, y, s)
        _check(_forward(self._h, _ptr(x, "x", torch.float32, (B, self.n_in), device), B,
                        _ptr(y, "y", torch.float32, (B, self.n_out), device),
                        _ptr(s, "s", torch.float32, (B, self.n_out), device)))

    def readout(self, x, winner):
        """winner [B][out_hcu]: the MCU of the largest support."""
        B, device = x.shape[0], self.device
        if device != _current_device():
            with torch.cuda.device(device):
                return self.readout(x, winner)
        _check(_readout(self._h, _ptr(x, "x", torch.float32, (B, self.n_in), device), B,
                        _ptr(winner, "winner", torch.int32, (B, self.cfg.out_hcu), device)))

    def predict_with(self, readout, x, y, winner):
        """winner [B]: the argmax of the 4-bit layer `readout` over this layer's activities of x
        [B][N_in], as many rows per launch as the workspace y [rows][N_out] has."""
        B, rows, device = x.shape[0], y.shape[0], self.device
        if device != _current_device():
            with torch.cuda.device(device):
                return self.predict_with(readout, x, y, winner)
        _check(_predict(self._h, readout._h, _ptr(x, "x", torch.float32, (B, self.n_in), device), B,
                        _ptr(y, "y", torch.float32, (rows, self.n_out), device), rows,
                        _ptr(winner, "winner", torch.int32, (B,), device)))
