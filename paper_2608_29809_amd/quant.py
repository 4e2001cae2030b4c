"""8-bit operators on PyTorch tensors: block quantisation, the product of
block-scaled matrices, the 8-bit cache of keys and values with the attention
that reads it, and int8 rows with their product.  Argument checks and allocation only; every
computation is a call into libregioncache.so.

    w = quantize(weight, 128)                 # a scale for each 128 x 128 tile
    a = quantize(x)                           # a scale for each row and 128 columns
    y = qgemm(a, w, bias, gelu=True)          # bfloat16 or float32

    cache = QuantCache.alloc(batch, heads, tokens)
    qcache_store(cache, active, k, v)         # fresh rows of the active tokens
    o = qcache_attention(cache, active, q)    # active queries over all keys

    w = quantize_int8(weight)                 # a scale for each output channel
    y = igemm(quantize_int8(x), w, bias)      # and for each token

Values are e4m3 and scales powers of two, held as the byte e of 2^(e - 127), or
int8 with a float32 scale for each row (those of the last two).
Calls go to the current stream of their tensors' device.
"""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional

import torch

from . import abi
from .runtime import ActiveSet

__all__ = ["QuantMatrix", "QuantCache", "IntMatrix", "quantize", "qgemm", "qcache_store", "qcache_attention", "quantize_int8",
           "igemm"]

HEAD_DIM = 72
BLOCK = 128      # columns (and a weight's rows) that share a scale
KEY_BLOCK = 64   # tokens of a cache block
_DTYPES = {torch.float32: abi.RC_F32, torch.bfloat16: abi.RC_BF16}
_F8, _U8, _F32, _I8 = torch.float8_e4m3fn, torch.uint8, torch.float32, torch.int8
_SCALE = 1.0 / math.sqrt(HEAD_DIM)

# The kernels of small calls take 3 to 7 us, a launch 3.2, so the host's time is a
# call's time: torch.cuda.current_stream would add 2.8 us, current_device 0.2, sizes
# as a tuple 0.35 to each torch.empty.  The quick lookups are private names of
# PyTorch; where they are missing the public ones serve.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
# (0.8 us for a tensor of the current device, torch.empty 1.3.  Results are made past Python's
# dispatch, so modes that replace or watch torch.empty do not see them, and past the filling
# of new memory that deterministic algorithms ask for: kernels write all of a result.)
_empty_strided = getattr(getattr(getattr(torch._C, "_dynamo", None), "guards", None), "_empty_strided_cuda", None)
# Tells autograd that kernels write tensors (one or a tuple): a graph that saved one fails
# in its backward pass instead of using other values.
_written = torch.autograd.graph.increment_version
_grad_enabled = torch.is_grad_enabled


def _empty(rows: int, cols: int, dtype: torch.dtype, index: int) -> torch.Tensor:
    """A new [rows][cols] tensor on GPU `index`."""
    if _empty_strided is not None and index == _current_device():
        return _empty_strided((rows, cols), (cols, 1), dtype)
    return torch.empty(rows, cols, dtype=dtype, device=index)


def _dtype(t: torch.Tensor, what: str) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise ValueError(f"{what} is {t.dtype}, not float32 or bfloat16")
    return d


def _on_gpu(first: torch.Tensor, *others: Optional[torch.Tensor]) -> int:
    """Index of the one GPU that holds the tensors."""
    if not first.is_cuda:
        raise ValueError(f"the tensors must be on the GPU, not on {first.device}")
    index = first.get_device()
    for t in others:
        if t is not None and t.get_device() != index:
            raise ValueError(f"tensors on {first.device} and {t.device}")
    return index


def _call(f, index: int, *args):
    """f(*args, stream) with GPU `index` current and its current stream."""
    if index == _current_device():
        f(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            f(*args, _raw_stream(index))


def _no_gradient(name: str) -> ValueError:
    """Of a tensor through which autograd would expect a gradient: the operators have none."""
    return ValueError(f"{name} has no gradient: call it under torch.no_grad() or with detached tensors")


def _ld(t: torch.Tensor, rows: int, cols: int, what: str) -> int:
    """Elements between the rows of a [rows][cols] tensor whose rows are contiguous."""
    if t.shape != (rows, cols):
        raise ValueError(f"{what} is {tuple(t.shape)}, not [{rows}, {cols}]")
    if t.is_contiguous():
        return cols
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{what}: the values of a row must be contiguous")
    return ld if rows > 1 else max(cols, ld)


class _InMemory:
    """Tensors `data` and `scales` with a C structure of their addresses and
    sizes, made once: where the tensors were given other memory since (set_,
    resize_, .data) it is refused."""

    __slots__ = ("_data", "_scales", "_struct", "_at_data", "_at_scales")

    def _hold(self, data: torch.Tensor, scales: torch.Tensor, kind, *sizes) -> None:
        self._data, self._scales = data, scales
        self._at_data, self._at_scales = at_data, at_scales = data.data_ptr(), scales.data_ptr()
        self._struct = kind(at_data, at_scales, *sizes)

    data = property(lambda self: self._data)
    scales = property(lambda self: self._scales)

    def struct(self):
        if self._data.data_ptr() != self._at_data or self._scales.data_ptr() != self._at_scales:
            raise ValueError(f"the memory of a {type(self).__name__}'s tensors was exchanged or resized")
        return self._struct


class QuantMatrix(_InMemory):
    """A matrix in 8 bits: `data` float8_e4m3fn [rows, cols], `scales` uint8
    [column blocks, row blocks rounded up to 16], block_rows 1 or 128.  Views
    of rows are given as data[:n] with the same scales."""

    __slots__ = ("_block_rows",)

    def __init__(self, data: torch.Tensor, scales: torch.Tensor, block_rows: int):
        if data.dtype != _F8 or data.dim() != 2:
            raise ValueError("data must be float8_e4m3fn [rows, cols]")
        if scales.dtype != _U8 or scales.dim() != 2 or not (scales.is_contiguous() or scales.stride(1) == 1):
            raise ValueError("scales must be uint8 [column blocks, row blocks] with contiguous rows")
        if block_rows != 1 and block_rows != BLOCK:
            raise ValueError(f"block_rows {block_rows} is not 1 or {BLOCK}")
        (rows, cols), (col_blocks, row_blocks) = data.shape, scales.shape
        if rows >> 31 or col_blocks != -(-cols // BLOCK) or row_blocks < -(-rows // block_rows) or row_blocks % 16:
            raise ValueError(f"scales {tuple(scales.shape)} do not cover data {tuple(data.shape)} (row blocks padded to 16)")
        _on_gpu(data, scales)
        ld = cols if data.is_contiguous() else _ld(data, rows, cols, "data")
        self._block_rows = block_rows
        self._hold(data, scales, abi.rc_qmat, ld, rows, cols, row_blocks if col_blocks == 1 else scales.stride(0), block_rows)

    block_rows = property(lambda self: self._block_rows)

    @classmethod
    def alloc(cls, rows: int, cols: int, block_rows: int = 1, device="cuda") -> "QuantMatrix":
        if block_rows != 1 and block_rows != BLOCK:
            raise ValueError(f"block_rows {block_rows} is not 1 or {BLOCK}")
        if rows >> 31 or cols >> 31:
            raise ValueError(f"{rows} x {cols} is too large")
        m = cls.__new__(cls)
        row_blocks = -(-rows // block_rows)
        row_blocks += -row_blocks % 16
        m._block_rows = block_rows
        m._hold(torch.empty(rows, cols, dtype=_F8, device=device), torch.empty(-(-cols // BLOCK), row_blocks, dtype=_U8, device=device),
                abi.rc_qmat, cols, rows, cols, row_blocks, block_rows)
        return m


class IntMatrix(_InMemory):
    """A matrix in int8 with a scale for each row: `data` int8 [rows, cols],
    `scales` float32 [rows].  Views of rows are given as data[:n], scales[:n]."""

    __slots__ = ()

    def __init__(self, data: torch.Tensor, scales: torch.Tensor):
        shape = data.shape
        if data.dtype != _I8 or len(shape) != 2:
            raise ValueError("data must be int8 [rows, cols]")
        rows, cols = shape
        if scales.dtype != _F32 or scales.dim() != 1 or scales.numel() != rows or not scales.is_contiguous():
            raise ValueError(f"scales must be contiguous float32 [{rows}]")
        if rows >> 31 or cols >> 31:
            raise ValueError(f"{rows} x {cols} is too large")
        _on_gpu(data, scales)
        self._hold(data, scales, abi.rc_imat, cols if data.is_contiguous() else _ld(data, rows, cols, "data"), rows, cols)

    @classmethod
    def alloc(cls, rows: int, cols: int, device="cuda") -> "IntMatrix":
        if rows >> 31 or cols >> 31:
            raise ValueError(f"{rows} x {cols} is too large")
        return cls._of(torch.empty(rows, cols, dtype=_I8, device=device), torch.empty(rows, dtype=_F32, device=device), rows, cols)

    @classmethod
    def _new(cls, rows: int, cols: int, index: int) -> "IntMatrix":
        if _empty_strided is None or index != _current_device():
            return cls.alloc(rows, cols, index)
        return cls._of(_empty_strided((rows, cols), (cols, 1), _I8), _empty_strided((rows,), (1,), _F32), rows, cols)

    @classmethod
    def _of(cls, data: torch.Tensor, scales: torch.Tensor, rows: int, cols: int) -> "IntMatrix":
        m = cls.__new__(cls)
        m._hold(data, scales, abi.rc_imat, cols, rows, cols)
        return m


class QuantCache(_InMemory):
    """Keys and values of `batch` chains in 8 bits: `data` float8_e4m3fn
    [batch, heads, blocks, 2, 64, 72] (a block's 64 keys, then its values) and
    `scales` uint8 [batch, heads, blocks, 2].  Chains may be any multiple of
    16 bytes apart; within a chain the cache is contiguous."""

    __slots__ = ("batch", "heads", "tokens")

    def __init__(self, data: torch.Tensor, scales: torch.Tensor):
        if data.dtype != _F8 or data.dim() != 6:
            raise ValueError(f"data must be float8_e4m3fn [batch, heads, blocks, 2, {KEY_BLOCK}, {HEAD_DIM}]")
        batch, heads, blocks, two, tokens, dim = data.shape
        if two != 2 or tokens != KEY_BLOCK or dim != HEAD_DIM:
            raise ValueError(f"data must be float8_e4m3fn [batch, heads, blocks, 2, {KEY_BLOCK}, {HEAD_DIM}]")
        if scales.dtype != _U8 or scales.shape != (batch, heads, blocks, 2):
            raise ValueError("scales must be uint8 [batch, heads, blocks, 2]")
        if not (batch and heads and blocks):
            raise ValueError("the cache is empty")
        if not (data.is_contiguous() or data[0].is_contiguous()) or not (scales.is_contiguous() or scales[0].is_contiguous()):
            raise ValueError("a chain of the cache must be contiguous")
        _on_gpu(data, scales)
        self.batch, self.heads, self.tokens = batch, heads, blocks * KEY_BLOCK
        self._hold(data, scales, abi.rc_qcache, data.stride(0), scales.stride(0), batch, heads, self.tokens)

    @classmethod
    def alloc(cls, batch: int, heads: int, tokens: int, device="cuda") -> "QuantCache":
        """A cache of zeros."""
        if tokens <= 0 or tokens % KEY_BLOCK:
            raise ValueError(f"tokens {tokens} is not a positive multiple of {KEY_BLOCK}")
        shape = (batch, heads, tokens // KEY_BLOCK, 2)
        return cls(torch.zeros(shape + (KEY_BLOCK, HEAD_DIM), dtype=torch.uint8, device=device).view(torch.float8_e4m3fn),
                   torch.zeros(shape, dtype=torch.uint8, device=device))


def quantize(x: torch.Tensor, block_rows: int = 1, out: Optional[QuantMatrix] = None) -> QuantMatrix:
    """x [rows, cols] float32 or bfloat16, cols a multiple of 16, in 8 bits
    with a scale for each row and 128 columns (block_rows 1) or each 128 x 128
    tile (128)."""
    dtype = _dtype(x, "x")
    if x.dim() != 2:
        raise ValueError(f"x is {tuple(x.shape)}, not [rows, cols]")
    rows, cols = x.shape
    ldx = cols if x.is_contiguous() else _ld(x, rows, cols, "x")
    given = out is not None
    if not given:
        index = _on_gpu(x)
        out = QuantMatrix.alloc(rows, cols, block_rows, x.device)
    else:
        index = _on_gpu(x, out._data)
        if (out._struct.rows, out._struct.cols) != x.shape or out.block_rows != block_rows:
            raise ValueError("out has another shape or other blocks")
    if rows:
        _call(abi.rc_quantize, index, x.data_ptr(), dtype, ldx, C.byref(out.struct()))
        if given:
            _written((out._data, out._scales))
    return out


def qgemm(a: QuantMatrix, w: QuantMatrix, bias: Optional[torch.Tensor] = None, gelu: bool = False,
          dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """act(a w^T + bias): a [m, k] with block_rows 1, w [n, k] with block_rows
    128, bias float32 [n]; the result [m, n] in dtype (or in out)."""
    A, W = a.struct(), w.struct()
    m, n = A.rows, W.rows
    if bias is not None and (bias.dtype != torch.float32 or bias.shape != (n,) or not bias.is_contiguous()):
        raise ValueError(f"bias must be contiguous float32 [{n}]")
    given = out is not None
    if not given:
        if dtype not in _DTYPES:
            raise ValueError(f"dtype {dtype} is not float32 or bfloat16")
        out, ldo = torch.empty(m, n, dtype=dtype, device=a._data.device), n
    else:
        ldo = _ld(out, m, n, "out")
    index = _on_gpu(a._data, w._data, bias, out)
    if m:
        _call(abi.rc_qgemm, index, C.byref(A), C.byref(W), None if bias is None else bias.data_ptr(), 1 if gelu else 0,
              out.data_ptr(), _dtype(out, "out"), ldo)
        if given:
            _written(out)
    return out


def quantize_int8(x: torch.Tensor, out: Optional[IntMatrix] = None) -> IntMatrix:
    """x [rows, cols] float32 or bfloat16, cols a multiple of 16, in int8 with a
    scale for each row: a weight's output channels, an activation's tokens.  A
    row that holds a value that is not finite gets the scale NaN.  Nothing of the
    result has a gradient."""
    dtype = _dtype(x, "x")
    shape = x.shape
    if len(shape) != 2:
        raise ValueError(f"x is {tuple(shape)}, not [rows, cols]")
    rows, cols = shape
    ldx = cols if x.is_contiguous() else _ld(x, rows, cols, "x")
    given = out is not None
    if not given:
        index = _on_gpu(x)
        if rows >> 31 or cols >> 31:
            raise ValueError(f"{rows} x {cols} is too large")
        out = IntMatrix._new(rows, cols, index)
    else:
        index = _on_gpu(x, out._data)
        if (out._struct.rows, out._struct.cols) != shape:
            raise ValueError("out has another shape")
    if rows:
        _call(abi.rc_quantize_int8, index, x.data_ptr(), dtype, ldx, C.byref(out.struct()))
        if given:
            _written((out._data, out._scales))
    return out


def igemm(a: IntMatrix, w: IntMatrix, bias: Optional[torch.Tensor] = None, gelu: bool = False,
          dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """act(a w^T + bias): a [m, k], w [n, k], bias float32 [n]; the result [m, n]
    in dtype (or in out).  The sum over k is exact.  There is no gradient: tensors
    that require one are refused where they are recorded."""
    if _grad_enabled() and (a._scales.requires_grad or w._scales.requires_grad or bias is not None and bias.requires_grad
                            or out is not None and out.requires_grad):
        raise _no_gradient("igemm")
    A, W = a.struct(), w.struct()
    m, n = A.rows, W.rows
    if bias is not None and (bias.dtype != _F32 or bias.shape != (n,) or not bias.is_contiguous()):
        raise ValueError(f"bias must be contiguous float32 [{n}]")
    given = out is not None
    if not given:
        code = _DTYPES.get(dtype)
        if code is None:
            raise ValueError(f"dtype {dtype} is not float32 or bfloat16")
        index = _on_gpu(a._data, w._data, bias)
        out, ldo = _empty(m, n, dtype, index), n
    else:
        ldo, code = _ld(out, m, n, "out"), _dtype(out, "out")
        index = _on_gpu(a._data, w._data, bias, out)
    if m:
        _call(abi.rc_igemm, index, C.byref(A), C.byref(W), None if bias is None else bias.data_ptr(), 1 if gelu else 0,
              out.data_ptr(), code, ldo)
        if given:
            _written(out)
    return out


def qcache_store(cache: QuantCache, active: ActiveSet, k: torch.Tensor, v: torch.Tensor) -> None:
    """Merge the fresh keys and values of the active tokens into the cache:
    k, v [active tokens, heads * 72] float32 or bfloat16 with one row stride
    (views of one product's output will do)."""
    dtype, cols, rows = _dtype(k, "k"), cache.heads * HEAD_DIM, active.total
    ld = _ld(k, rows, cols, "k")
    if v.dtype != k.dtype or _ld(v, rows, cols, "v") != ld:
        raise ValueError("k and v must have one type and row stride")
    index = _on_gpu(cache._data, k, v, active.idx, active.offsets)
    if rows:
        _call(abi.rc_qcache_store, index, C.byref(cache.struct()), C.byref(active.struct()), k.data_ptr(), v.data_ptr(), dtype, ld)
        _written((cache._data, cache._scales))


def qcache_attention(cache: QuantCache, rows: ActiveSet, q: torch.Tensor, scale: Optional[float] = None,
                     key_len: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of the query rows (chains as in `rows`; its tokens are not
    read) over the first key_len[b] keys (default: all) of their chain.
    q [rows, heads * 72] bfloat16; scale defaults to 1/sqrt(72); key_len int32
    [batch] on the GPU; rows of a chain without keys are 0."""
    cols, total = cache.heads * HEAD_DIM, rows.total
    if q.dtype != torch.bfloat16:
        raise ValueError(f"q is {q.dtype}, not bfloat16")
    ldq = cols if q.shape == (total, cols) and q.is_contiguous() else _ld(q, total, cols, "q")
    if key_len is not None and (key_len.dtype != torch.int32 or key_len.shape != (cache.batch,) or not key_len.is_contiguous()):
        raise ValueError(f"key_len must be contiguous int32 [{cache.batch}]")
    given = out is not None
    if not given:
        out = torch.empty(total, cols, dtype=torch.bfloat16, device=q.device)
    elif out.dtype != torch.bfloat16:
        raise ValueError(f"out is {out.dtype}, not bfloat16")
    ldo = _ld(out, total, cols, "out")
    index = _on_gpu(cache._data, q, out, key_len, rows.offsets)
    if total:
        c, s = cache.struct(), rows.struct()
        nbytes = abi.rc_qcache_attention_scratch_bytes(C.byref(c), C.byref(s))
        scratch = torch.empty(nbytes, dtype=_U8, device=q.device) if nbytes else None
        _call(abi.rc_qcache_attention, index, C.byref(c), C.byref(s), None if key_len is None else key_len.data_ptr(),
              q.data_ptr(), ldq, _SCALE if scale is None else float(scale), out.data_ptr(), ldo,
              scratch.data_ptr() if nbytes else None, nbytes)
        if given:
            _written(out)
    return out
