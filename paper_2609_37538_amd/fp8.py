"""ctypes binding of matrices in 8-bit floating point (include/avsg_fp8.h): the
same entry points, argument marshalling only, and wrappers that take torch
tensors.

:class:`Fp8` is a matrix or a batch of them in this form, made by
:func:`fp8_quantize` or from codes and scales that a program has;
:func:`fp8_matmul` multiplies activations by weights.  The wrappers run on the
current stream of their tensors' GPU and raise ValueError for tensors the kernels
do not take.  There is no backward pass: with gradients enabled they raise
ValueError for tensors that require one.
"""
from __future__ import annotations

import ctypes

from . import latent as _L
from .avsg import _P, _vp
from .latent import _check, _i32, _i64, _need, _plain_type

AVSG_FP8_BLOCK = 128


class AvsgFp8(ctypes.Structure):
    _fields_ = [("d_codes", _P), ("d_scales", _P), ("code_stride", _i64), ("code_batch_stride", _i64),
                ("scale_stride", _i64), ("scale_batch_stride", _i64), ("block_rows", _i32)]


_lib = None


def load():
    """The library with the signatures of this module's entry points."""
    global _lib
    if _lib is not None:
        return _lib
    lib = _L.load()
    ptr = ctypes.POINTER
    for name, args in (
            ("avsg_fp8_quantize", [_P, _i32, _i32, _i64, _i64, _i64, _i64, ptr(AvsgFp8), _P]),
            ("avsg_fp8_dequantize", [ptr(AvsgFp8), _i32, _i64, _i64, _P, _i32, _i64, _i64, _P]),
            ("avsg_fp8_matmul", [ptr(AvsgFp8), ptr(AvsgFp8), _i32, _i64, _i64, _i64, _P, _i32, _i64, _i64, _P])):
        f = getattr(lib, name)
        f.restype, f.argtypes = _i32, args
    _lib = lib
    return lib


# ---------------------------------------------------------------------------
# entry points, same names as the C ABI
# ---------------------------------------------------------------------------
def avsg_fp8_quantize(d_x: int, dtype: int, batch: int, rows: int, cols: int, x_stride: int, x_batch_stride: int, out: AvsgFp8,
                      stream: int = 0) -> None:
    _check(load().avsg_fp8_quantize(_vp(d_x), dtype, batch, rows, cols, x_stride, x_batch_stride, out, _vp(stream)), "avsg_fp8_quantize")


def avsg_fp8_dequantize(x: AvsgFp8, batch: int, rows: int, cols: int, d_out: int, dtype: int, out_stride: int, out_batch_stride: int,
                        stream: int = 0) -> None:
    _check(load().avsg_fp8_dequantize(x, batch, rows, cols, _vp(d_out), dtype, out_stride, out_batch_stride, _vp(stream)),
           "avsg_fp8_dequantize")


def avsg_fp8_matmul(a: AvsgFp8, b: AvsgFp8, batch: int, m: int, n: int, k: int, d_out: int, out_type: int, out_stride: int,
                    out_batch_stride: int, stream: int = 0) -> None:
    _check(load().avsg_fp8_matmul(a, b, batch, m, n, k, _vp(d_out), out_type, out_stride, out_batch_stride, _vp(stream)), "avsg_fp8_matmul")


# ---------------------------------------------------------------------------
# wrappers
# ---------------------------------------------------------------------------
def _torch():
    torch = _L._torch()
    load()
    return torch


def _strides(x):
    """Strides of a tensor, 0 for dimensions of one entry, which do not matter."""
    return [0 if n <= 1 else s for s, n in zip(x.stride(), x.shape)]


class Fp8:
    """A matrix or a batch of them in 8-bit floating point: codes float8_e4m3fn [..., R, K] and float32
    scales, [..., R, K/128] (rows=1, of activations) or [..., R/128, K/128] (rows=128, of weights), counts
    of blocks rounded up; K a multiple of 16."""

    __slots__ = ("codes", "scales", "rows", "_view")

    def __init__(self, codes, scales, rows: int = 1):
        torch = _torch()
        _need(rows in (1, AVSG_FP8_BLOCK), f"rows must be 1 or {AVSG_FP8_BLOCK}")
        _need(codes.dtype is torch.float8_e4m3fn and scales.dtype is torch.float32 and codes.is_cuda and codes.device == scales.device,
              "codes must be a float8_e4m3fn and scales a float32 tensor on one GPU")
        for x in (codes, scales):
            if x.requires_grad:
                _L._no_gradient("codes and scales")
        shape = codes.shape
        _need(len(shape) in (2, 3) and shape[-1] % 16 == 0, "codes must be [..., R, K] with K a multiple of 16")
        _need(scales.shape == (*shape[:-2], -(-shape[-2] // rows), -(-shape[-1] // AVSG_FP8_BLOCK)),
              "codes and scales must belong together: a scale for each block")
        self.codes, self.scales, self.rows, self._view = codes, scales, rows, None

    @property
    def shape(self):
        """Of the matrix it stands for."""
        return tuple(self.codes.shape)

    @property
    def device(self):
        return self.codes.device

    def transpose(self, i: int, j: int) -> "Fp8":
        """With two leading dimensions exchanged (the columns stay in place; blocks of 128 rows too)."""
        n = self.codes.dim()
        _need(i % n != n - 1 and j % n != n - 1, "columns cannot be exchanged: blocks lie along them")
        if i % n == j % n:
            return self
        _need(self.rows == 1, "rows in blocks of 128 cannot be exchanged")
        return _fp8(self.codes.transpose(i, j), self.scales.transpose(i, j), 1)

    def _c(self) -> AvsgFp8:
        """The matrix as the library takes it; made once, for codes and scales do not move."""
        view = self._view
        if view is None:
            codes, scales = self.codes, self.scales
            at, c, s = codes.data_ptr(), _strides(codes), _strides(scales)
            if 0 in codes.shape:
                c = s = [0] * len(c)
            else:
                _need(c[-1] == 1 and s[-1] in (0, 1) and not at & 15 and not any(st & 15 for st in c[:-1]),
                      "rows of codes must be contiguous and 16-byte aligned, and a row's scales contiguous")
            view = AvsgFp8(at, scales.data_ptr(), c[-2], c[0] if len(c) == 3 else 0, s[-2], s[0] if len(s) == 3 else 0, self.rows)
            self._view = view
        return view


def _fp8(codes, scales, rows) -> Fp8:
    """An Fp8 of tensors that need no checks."""
    m = Fp8.__new__(Fp8)
    m.codes, m.scales, m.rows, m._view = codes, scales, rows, None
    return m


def _plain(x, dtype, what):
    """(address, row stride, batch stride) of a plain [..., R, K] whose rows are 16-byte aligned."""
    st, unit = _strides(x), 8 if dtype == _L.AVSG_BF16 else 4
    if 0 in x.shape:
        return x.data_ptr(), 0, 0
    _need(st[-1] == 1 and not x.data_ptr() & 15 and not any(s % unit for s in st[:-1]), f"{what}: rows must be contiguous and 16-byte aligned")
    return x.data_ptr(), st[-2], st[0] if len(st) == 3 else 0


def fp8_quantize(x, rows: int = 1) -> Fp8:
    """8-bit form of x, [R][K] or [A][R][K] with K a multiple of 16, in bfloat16 or float32: a scale for each
    128 columns of a row (rows=1) or for each block of 128 x 128 (rows=128)."""
    torch = _torch()
    dtype, shape, dev = _plain_type(x, "x"), x.shape, x.device
    _need(len(shape) in (2, 3) and shape[-1] % 16 == 0, "x must be [..., R, K] with K a multiple of 16")
    _need(rows in (1, AVSG_FP8_BLOCK), f"rows must be 1 or {AVSG_FP8_BLOCK}")
    at, stride, batch_stride = _plain(x, dtype, "x")
    codes = torch.empty(shape, dtype=torch.float8_e4m3fn, device=dev)
    scales = torch.empty((*shape[:-2], -(-shape[-2] // rows), -(-shape[-1] // AVSG_FP8_BLOCK)), dtype=torch.float32, device=dev)
    m = _fp8(codes, scales, rows)
    batch = shape[0] if len(shape) == 3 else 1
    _L._run(_lib.avsg_fp8_quantize, "avsg_fp8_quantize", dev.index, at, dtype, batch, shape[-2], shape[-1], stride, batch_stride, m._c())
    return m


def fp8_dequantize(m: Fp8, dtype=None):
    """The values that an Fp8 stands for, in bfloat16 (the default) or float32."""
    shape, dev = m.shape, m.device
    out = _L._t.empty(shape, dtype=dtype or _L._t.bfloat16, device=dev)
    kind = _plain_type(out, "dtype")
    at, stride, batch_stride = _plain(out, kind, "out")
    _L._run(_lib.avsg_fp8_dequantize, "avsg_fp8_dequantize", dev.index, m._c(), shape[0] if len(shape) == 3 else 1, shape[-2], shape[-1], at,
            kind, stride, batch_stride)
    return out


def fp8_matmul(a: Fp8, b: Fp8, out=None, dtype=None):
    """a b^T for a [M][K] with scales per row and b [N][K] with scales per 128 x 128, or for batches of both;
    `out` ([M][N] or [batch][M][N], bfloat16 or float32, rows contiguous) or a new tensor of `dtype` (bfloat16)."""
    sa, sb, dev = a.codes.shape, b.codes.shape, a.codes.device
    three = len(sa) == 3
    if len(sa) != len(sb) or sa[-1] != sb[-1] or dev != b.codes.device or (three and sa[0] != sb[0]):
        raise ValueError("a and b must have the same dimensions, batch, columns and GPU")
    if a.rows != 1 or b.rows != AVSG_FP8_BLOCK:
        raise ValueError("a must have a scale per 128 columns of a row (rows=1), b per 128 x 128 (rows=128)")
    shape = (*sa[:-1], sb[-2])
    if out is None:
        out = _L._t.empty(shape, dtype=dtype or _L._t.bfloat16, device=dev)
    st = out.stride()
    if out.shape != shape or out.device != dev or (shape[-1] > 1 and st[-1] != 1):
        raise ValueError(f"out must be {shape} on {dev} with contiguous rows")
    kind = _plain_type(out, "out")
    _L._run(_lib.avsg_fp8_matmul, "avsg_fp8_matmul", dev.index, a._c(), b._c(), sa[0] if three else 1, shape[-2], shape[-1], sa[-1],
            out.data_ptr(), kind, st[-2], st[0] if three else 0)
    return out
