"""8-bit operators on PyTorch tensors: block quantisation, the product of
block-scaled matrices, and the 8-bit cache of keys and values with the
attention that reads it.  Argument checks and allocation only; every
computation is a call into libregioncache.so.

    w = quantize(weight, 128)                 # a scale for each 128 x 128 tile
    a = quantize(x)                           # a scale for each row and 128 columns
    y = qgemm(a, w, bias, gelu=True)          # bfloat16 or float32

    cache = QuantCache.alloc(batch, heads, tokens)
    qcache_store(cache, active, k, v)         # fresh rows of the active tokens
    o = qcache_attention(cache, active, q)    # active queries over all keys

Values are e4m3 and scales powers of two, held as the byte e of 2^(e - 127).
Calls go to the current stream of their tensors' device.
"""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional

import torch

from . import abi
from .runtime import ActiveSet

__all__ = ["QuantMatrix", "QuantCache", "quantize", "qgemm", "qcache_store", "qcache_attention"]

HEAD_DIM = 72
BLOCK = 128      # columns (and a weight's rows) that share a scale
KEY_BLOCK = 64   # tokens of a cache block
_DTYPES = {torch.float32: abi.RC_F32, torch.bfloat16: abi.RC_BF16}
_F8, _U8 = torch.float8_e4m3fn, torch.uint8
_SCALE = 1.0 / math.sqrt(HEAD_DIM)

# The kernels of small calls take 3 to 7 us, a launch 3.2, so the host's time is a
# call's time: torch.cuda.current_stream would add 2.8 us, current_device 0.2, sizes
# as a tuple 0.35 to each torch.empty.  The quick lookups are private names of
# PyTorch; where they are missing the public ones serve.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


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


class QuantMatrix:
    """A matrix in 8 bits: `data` float8_e4m3fn [rows, cols], `scales` uint8
    [column blocks, row blocks rounded up to 16], block_rows 1 or 128.  Views
    of rows are given as data[:n] with the same scales."""

    __slots__ = ("_data", "_scales", "_block_rows", "_struct")

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
        self._data, self._scales, self._block_rows = data, scales, block_rows
        self._struct = abi.rc_qmat(data.data_ptr(), scales.data_ptr(), ld, rows, cols,
                                   row_blocks if col_blocks == 1 else scales.stride(0), block_rows)

    # (read-only: the C structure is made once)
    data = property(lambda self: self._data)
    scales = property(lambda self: self._scales)
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
        m._data = data = torch.empty(rows, cols, dtype=_F8, device=device)
        m._scales = scales = torch.empty(-(-cols // BLOCK), row_blocks, dtype=_U8, device=device)
        m._block_rows = block_rows
        m._struct = abi.rc_qmat(data.data_ptr(), scales.data_ptr(), cols, rows, cols, row_blocks, block_rows)
        return m

    def struct(self) -> abi.rc_qmat:
        return self._struct


class QuantCache:
    """Keys and values of `batch` chains in 8 bits: `data` float8_e4m3fn
    [batch, heads, blocks, 2, 64, 72] (a block's 64 keys, then its values) and
    `scales` uint8 [batch, heads, blocks, 2].  Chains may be any multiple of
    16 bytes apart; within a chain the cache is contiguous."""

    __slots__ = ("_data", "_scales", "_struct", "batch", "heads", "tokens")

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
        self._data, self._scales = data, scales
        self.batch, self.heads, self.tokens = batch, heads, blocks * KEY_BLOCK
        self._struct = abi.rc_qcache(data.data_ptr(), scales.data_ptr(), data.stride(0), scales.stride(0), batch, heads,
                                     self.tokens)

    # (read-only: the C structure is made once)
    data = property(lambda self: self._data)
    scales = property(lambda self: self._scales)

    @classmethod
    def alloc(cls, batch: int, heads: int, tokens: int, device="cuda") -> "QuantCache":
        """A cache of zeros."""
        if tokens <= 0 or tokens % KEY_BLOCK:
            raise ValueError(f"tokens {tokens} is not a positive multiple of {KEY_BLOCK}")
        shape = (batch, heads, tokens // KEY_BLOCK, 2)
        return cls(torch.zeros(shape + (KEY_BLOCK, HEAD_DIM), dtype=torch.uint8, device=device).view(torch.float8_e4m3fn),
                   torch.zeros(shape, dtype=torch.uint8, device=device))

    def struct(self) -> abi.rc_qcache:
        return self._struct


def quantize(x: torch.Tensor, block_rows: int = 1, out: Optional[QuantMatrix] = None) -> QuantMatrix:
    """x [rows, cols] float32 or bfloat16, cols a multiple of 16, in 8 bits
    with a scale for each row and 128 columns (block_rows 1) or each 128 x 128
    tile (128)."""
    dtype = _dtype(x, "x")
    if x.dim() != 2:
        raise ValueError(f"x is {tuple(x.shape)}, not [rows, cols]")
    rows, cols = x.shape
    ldx = cols if x.is_contiguous() else _ld(x, rows, cols, "x")
    if out is None:
        index = _on_gpu(x)
        out = QuantMatrix.alloc(rows, cols, block_rows, x.device)
    else:
        index = _on_gpu(x, out.data)
        if out.data.shape != x.shape or out.block_rows != block_rows:
            raise ValueError("out has another shape or other blocks")
    if rows:
        _call(abi.rc_quantize, index, x.data_ptr(), dtype, ldx, C.byref(out._struct))
    return out


def qgemm(a: QuantMatrix, w: QuantMatrix, bias: Optional[torch.Tensor] = None, gelu: bool = False,
          dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """act(a w^T + bias): a [m, k] with block_rows 1, w [n, k] with block_rows
    128, bias float32 [n]; the result [m, n] in dtype (or in out)."""
    A, W = a._struct, w._struct
    m, n = A.rows, W.rows
    if bias is not None and (bias.dtype != torch.float32 or bias.shape != (n,) or not bias.is_contiguous()):
        raise ValueError(f"bias must be contiguous float32 [{n}]")
    if out is None:
        if dtype not in _DTYPES:
            raise ValueError(f"dtype {dtype} is not float32 or bfloat16")
        out, ldo = torch.empty(m, n, dtype=dtype, device=a.data.device), n
    else:
        ldo = _ld(out, m, n, "out")
    index = _on_gpu(a.data, w.data, bias, out)
    if m:
        _call(abi.rc_qgemm, index, C.byref(A), C.byref(W), None if bias is None else bias.data_ptr(), 1 if gelu else 0,
              out.data_ptr(), _dtype(out, "out"), ldo)
    return out


def qcache_store(cache: QuantCache, active: ActiveSet, k: torch.Tensor, v: torch.Tensor) -> None:
    """Merge the fresh keys and values of the active tokens into the cache:
    k, v [active tokens, heads * 72] float32 or bfloat16 with one row stride
    (views of one product's output will do)."""
    dtype, cols, rows = _dtype(k, "k"), cache.heads * HEAD_DIM, active.total
    ld = _ld(k, rows, cols, "k")
    if v.dtype != k.dtype or _ld(v, rows, cols, "v") != ld:
        raise ValueError("k and v must have one type and row stride")
    index = _on_gpu(cache.data, k, v, active.idx, active.offsets)
    if rows:
        _call(abi.rc_qcache_store, index, C.byref(cache._struct), C.byref(active.struct()), k.data_ptr(), v.data_ptr(), dtype, ld)


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
    if out is None:
        out = torch.empty(total, cols, dtype=torch.bfloat16, device=q.device)
    elif out.dtype != torch.bfloat16:
        raise ValueError(f"out is {out.dtype}, not bfloat16")
    ldo = _ld(out, total, cols, "out")
    index = _on_gpu(cache.data, q, out, key_len, rows.offsets)
    if total:
        c, s = cache._struct, rows.struct()
        nbytes = abi.rc_qcache_attention_scratch_bytes(C.byref(c), C.byref(s))
        scratch = torch.empty(nbytes, dtype=_U8, device=q.device) if nbytes else None
        _call(abi.rc_qcache_attention, index, C.byref(c), C.byref(s), None if key_len is None else key_len.data_ptr(),
              q.data_ptr(), ldq, _SCALE if scale is None else float(scale), out.data_ptr(), ldo,
              scratch.data_ptr() if nbytes else None, nbytes)
    return out
