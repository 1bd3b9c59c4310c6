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
    """Strides of a tensor, 0 for dimensions of one entry, which do not matter, and of tensors without entries."""
    if 0 in x.shape:
        return (0,) * x.dim()
    return tuple(0 if n == 1 else s for s, n in zip(x.stride(), x.shape))


class Fp8:
    """A matrix or a batch of them in 8-bit floating point: codes float8_e4m3fn [..., R, K] and float32
    scales, [..., R, K/128] (rows=1, of activations) or [..., R/128, K/128] (rows=128, of weights), counts
    of blocks rounded up; K a multiple of 16."""

    # Small calls cost more time on the host than on the GPU, so what fp8_quantize makes is one allocation
    # (codes, then scales), and its tensors are made where they are asked for.
    __slots__ = ("device", "rows", "_shape", "_codes", "_scales", "_base", "_code_strides", "_scale_strides", "_view")

    def __init__(self, codes, scales, rows: int = 1):
        torch = _torch()
        _need(rows in (1, AVSG_FP8_BLOCK), f"rows must be 1 or {AVSG_FP8_BLOCK}")
        _need(codes.dtype is torch.float8_e4m3fn and scales.dtype is torch.float32 and codes.is_cuda and codes.device == scales.device,
              "codes must be a float8_e4m3fn and scales a float32 tensor on one GPU")
        for x in (codes, scales):
            if x.requires_grad:
                _L._no_gradient("codes and scales")
        shape = tuple(codes.shape)
        _need(len(shape) in (2, 3) and shape[-1] % 16 == 0, "codes must be [..., R, K] with K a multiple of 16")
        _need(scales.shape == (*shape[:-2], -(-shape[-2] // rows), -(-shape[-1] // AVSG_FP8_BLOCK)),
              "codes and scales must belong together: a scale for each block")
        self.device, self.rows, self._shape = codes.device, rows, shape
        self._codes, self._scales, self._base, self._view = codes, scales, None, None

    @property
    def shape(self):
        """Of the matrix it stands for."""
        return self._shape

    @property
    def codes(self):
        if self._codes is None:
            flat = self._base[:self._code_bytes()].view(_L._t.float8_e4m3fn)
            self._codes = flat.as_strided(self._shape, (*self._code_strides, 1))
        return self._codes

    @property
    def scales(self):
        if self._scales is None:
            shape = (*self._shape[:-2], -(-self._shape[-2] // self.rows), -(-self._shape[-1] // AVSG_FP8_BLOCK))
            flat = self._base[self._code_bytes():].view(_L._t.float32)
            self._scales = flat.as_strided(shape, (*self._scale_strides, 1))
        return self._scales

    def _code_bytes(self) -> int:
        n = 1
        for size in self._shape:
            n *= size
        return n

    def transpose(self, i: int, j: int) -> "Fp8":
        """With two leading dimensions exchanged (the columns stay in place; blocks of 128 rows too)."""
        n = len(self._shape)
        _need(i % n != n - 1 and j % n != n - 1, "columns cannot be exchanged: blocks lie along them")
        if i % n == j % n:
            return self
        _need(self.rows == 1, "rows in blocks of 128 cannot be exchanged")
        if self._base is None:
            return Fp8(self._codes.transpose(i, j), self._scales.transpose(i, j))
        s, c, b = self._shape, self._code_strides, self._scale_strides
        return _fp8(self.device, self._base, 1, (s[1], s[0], s[2]), (c[1], c[0]), (b[1], b[0]))

    def _c(self) -> AvsgFp8:
        """The matrix as the library takes it; made once, for codes and scales do not move."""
        view = self._view
        if view is not None:
            return view
        if self._base is not None:
            at, c, s = self._base.data_ptr(), self._code_strides, self._scale_strides
            scales_at = at + self._code_bytes()
            view = (AvsgFp8(at, scales_at, c[0], 0, s[0], 0, self.rows) if len(c) == 1
                    else AvsgFp8(at, scales_at, c[1], c[0], s[1], s[0], self.rows))
        else:
            at, c, s = self._codes.data_ptr(), _strides(self._codes), _strides(self._scales)
            if self._codes.numel():
                # (one scale that stands for several blocks of a row does not lie where the kernels read the others')
                _need(c[-1] == 1 and (s[-1] == 1 or self._scales.shape[-1] == 1) and not at & 15 and not any(st & 15 for st in c[:-1]),
                      "rows of codes must be contiguous and 16-byte aligned, and a row's scales contiguous")
            view = AvsgFp8(at, self._scales.data_ptr(), c[-2], c[0] if len(c) == 3 else 0, s[-2], s[0] if len(s) == 3 else 0, self.rows)
        self._view = view
        return view


def _fp8(device, base, rows, shape, code_strides, scale_strides) -> Fp8:
    """An Fp8 in one allocation: the codes, then the scales."""
    m = Fp8.__new__(Fp8)
    m.device, m.rows, m._base, m._shape, m._code_strides, m._scale_strides = device, rows, base, shape, code_strides, scale_strides
    m._codes = m._scales = m._view = None
    return m


def _plain(x, dtype, what):
    """(address, row stride, batch stride) of a plain [..., R, K] whose rows are 16-byte aligned."""
    at, shape = x.data_ptr(), x.shape
    if x.is_contiguous() and not at & 15:
        # (rows are of multiples of 16 entries)
        return at, shape[-1], shape[-2] * shape[-1]
    st, mask = _strides(x), 7 if dtype == _L.AVSG_BF16 else 3
    if 0 in shape:
        return at, 0, 0
    _need(st[-1] == 1 and not at & 15 and not any(s & mask for s in st[:-1]), f"{what}: rows must be contiguous and 16-byte aligned")
    return at, st[-2], st[0] if len(st) == 3 else 0


def fp8_quantize(x, rows: int = 1) -> Fp8:
    """8-bit form of x, [R][K] or [A][R][K] with K a multiple of 16, in bfloat16 or float32: a scale for each
    128 columns of a row (rows=1) or for each block of 128 x 128 (rows=128)."""
    torch = _torch() if _lib is None or _L._t is None else _L._t
    dtype, shape, dev = _plain_type(x, "x"), tuple(x.shape), x.device
    _need(len(shape) in (2, 3) and shape[-1] % 16 == 0, "x must be [..., R, K] with K a multiple of 16")
    at, stride, batch_stride = _plain(x, dtype, "x")
    batch, r, k = shape if len(shape) == 3 else (1, *shape)
    if rows == 1:
        down = r
    else:
        _need(rows == AVSG_FP8_BLOCK, f"rows must be 1 or {AVSG_FP8_BLOCK}")
        down = -(-r // AVSG_FP8_BLOCK)
    across = -(-k // AVSG_FP8_BLOCK)
    base = torch.empty(batch * (r * k + 4 * down * across), dtype=torch.uint8, device=dev)
    m = _fp8(dev, base, rows, shape, (k,) if len(shape) == 2 else (r * k, k), (across,) if len(shape) == 2 else (down * across, across))
    _L._run(_lib.avsg_fp8_quantize, "avsg_fp8_quantize", dev.index, at, dtype, batch, r, k, stride, batch_stride, m._c())
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
    sa, sb, dev = a._shape, b._shape, a.device
    three = len(sa) == 3
    if len(sa) != len(sb) or sa[-1] != sb[-1] or dev != b.device or (three and sa[0] != sb[0]):
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
    if not out.is_contiguous():
        _L._outputs("out", sa[0] if three else 1, st[0], shape[-2], st[-2], shape[-1])
    _L._run(_lib.avsg_fp8_matmul, "avsg_fp8_matmul", dev.index, a._c(), b._c(), sa[0] if three else 1, shape[-2], shape[-1], sa[-1],
            out.data_ptr(), kind, st[-2], st[0] if three else 0)
    return out
