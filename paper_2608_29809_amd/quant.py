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
_SCALE = 1.0 / math.sqrt(HEAD_DIM)


_raw_stream = torch._C._cuda_getCurrentRawStream  # (torch.cuda.current_stream takes 2.8 us of a call's 9)


def _dtype(t: torch.Tensor, what: str) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise ValueError(f"{what} is {t.dtype}, not float32 or bfloat16")
    return d


def _on_gpu(first: torch.Tensor, *others: Optional[torch.Tensor]) -> torch.device:
    """The one GPU that holds the tensors."""
    dev = first.device
    if dev.type != "cuda":
        raise ValueError(f"the tensors must be on the GPU, not on {dev}")
    for t in others:
        if t is not None and t.device != dev:
            raise ValueError(f"tensors on {dev} and {t.device}")
    return dev


def _call(f, device: torch.device, *args):
    """f(*args, stream) with `device` current and its current stream."""
    index = device.index
    if index == torch.cuda.current_device():
        f(*args, _raw_stream(index))
    else:
        with torch.cuda.device(device):
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

    __slots__ = ("data", "scales", "block_rows")

    def __init__(self, data: torch.Tensor, scales: torch.Tensor, block_rows: int):
        if data.dtype != torch.float8_e4m3fn or data.dim() != 2:
            raise ValueError("data must be float8_e4m3fn [rows, cols]")
        if scales.dtype != torch.uint8 or scales.dim() != 2 or (scales.stride(1) != 1 and scales.shape[1] > 1):
            raise ValueError("scales must be uint8 [column blocks, row blocks] with contiguous rows")
        if block_rows != 1 and block_rows != BLOCK:
            raise ValueError(f"block_rows {block_rows} is not 1 or {BLOCK}")
        (rows, cols), (col_blocks, row_blocks) = data.shape, scales.shape
        if col_blocks != -(-cols // BLOCK) or row_blocks < -(-rows // block_rows) or row_blocks % 16:
            raise ValueError(f"scales {tuple(scales.shape)} do not cover data {tuple(data.shape)} (row blocks padded to 16)")
        _on_gpu(data, scales)
        self.data, self.scales, self.block_rows = data, scales, block_rows

    @classmethod
    def alloc(cls, rows: int, cols: int, block_rows: int = 1, device="cuda") -> "QuantMatrix":
        if block_rows != 1 and block_rows != BLOCK:
            raise ValueError(f"block_rows {block_rows} is not 1 or {BLOCK}")
        m = cls.__new__(cls)
        row_blocks = -(-rows // block_rows)
        m.data = torch.empty((rows, cols), dtype=torch.float8_e4m3fn, device=device)
        m.scales = torch.empty((-(-cols // BLOCK), row_blocks + -row_blocks % 16), dtype=torch.uint8, device=device)
        m.block_rows = block_rows
        return m

    def struct(self) -> abi.rc_qmat:
        rows, cols = self.data.shape
        col_blocks, row_blocks = self.scales.shape
        scale_ld = row_blocks if col_blocks == 1 else self.scales.stride(0)
        return abi.rc_qmat(self.data.data_ptr(), self.scales.data_ptr(), _ld(self.data, rows, cols, "data"), rows, cols,
                           scale_ld, self.block_rows)


class QuantCache:
    """Keys and values of `batch` chains in 8 bits: `data` float8_e4m3fn
    [batch, heads, blocks, 2, 64, 72] (a block's 64 keys, then its values) and
    `scales` uint8 [batch, heads, blocks, 2].  Chains may be any multiple of
    16 bytes apart; within a chain the cache is contiguous."""

    __slots__ = ("data", "scales", "batch", "heads", "tokens")

    def __init__(self, data: torch.Tensor, scales: torch.Tensor):
        shape = data.shape
        if data.dtype != torch.float8_e4m3fn or len(shape) != 6 or shape[3:] != (2, KEY_BLOCK, HEAD_DIM):
            raise ValueError(f"data must be float8_e4m3fn [batch, heads, blocks, 2, {KEY_BLOCK}, {HEAD_DIM}]")
        if scales.dtype != torch.uint8 or scales.shape != shape[:4]:
            raise ValueError("scales must be uint8 [batch, heads, blocks, 2]")
        batch, heads, blocks = shape[:3]
        if not (batch and heads and blocks):
            raise ValueError("the cache is empty")
        if not (data.is_contiguous() or data[0].is_contiguous()) or not (scales.is_contiguous() or scales[0].is_contiguous()):
            raise ValueError("a chain of the cache must be contiguous")
        _on_gpu(data, scales)
        self.data, self.scales = data, scales
        self.batch, self.heads, self.tokens = batch, heads, blocks * KEY_BLOCK

    @classmethod
    def alloc(cls, batch: int, heads: int, tokens: int, device="cuda") -> "QuantCache":
        """A cache of zeros."""
        if tokens <= 0 or tokens % KEY_BLOCK:
            raise ValueError(f"tokens {tokens} is not a positive multiple of {KEY_BLOCK}")
        shape = (batch, heads, tokens // KEY_BLOCK, 2)
        return cls(torch.zeros(shape + (KEY_BLOCK, HEAD_DIM), dtype=torch.uint8, device=device).view(torch.float8_e4m3fn),
                   torch.zeros(shape, dtype=torch.uint8, device=device))

    def struct(self) -> abi.rc_qcache:
        return abi.rc_qcache(self.data.data_ptr(), self.scales.data_ptr(), self.data.stride(0), self.scales.stride(0),
                             self.batch, self.heads, self.tokens)


def quantize(x: torch.Tensor, block_rows: int = 1, out: Optional[QuantMatrix] = None) -> QuantMatrix:
    """x [rows, cols] float32 or bfloat16, cols a multiple of 16, in 8 bits
    with a scale for each row and 128 columns (block_rows 1) or each 128 x 128
    tile (128)."""
    dtype = _dtype(x, "x")
    if x.dim() != 2:
        raise ValueError(f"x is {tuple(x.shape)}, not [rows, cols]")
    rows, cols = x.shape
    ldx = _ld(x, rows, cols, "x")
    if out is None:
        dev = _on_gpu(x)
        out = QuantMatrix.alloc(rows, cols, block_rows, dev)
    else:
        dev = _on_gpu(x, out.data)
        if out.data.shape != x.shape or out.block_rows != block_rows:
            raise ValueError("out has another shape or other blocks")
    if rows:
        _call(abi.rc_quantize, dev, x.data_ptr(), dtype, ldx, C.byref(out.struct()))
    return out


def qgemm(a: QuantMatrix, w: QuantMatrix, bias: Optional[torch.Tensor] = None, gelu: bool = False,
          dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """act(a w^T + bias): a [m, k] with block_rows 1, w [n, k] with block_rows
    128, bias float32 [n]; the result [m, n] in dtype (or in out)."""
    m, n = a.data.shape[0], w.data.shape[0]
    if bias is not None and (bias.dtype != torch.float32 or bias.shape != (n,) or not bias.is_contiguous()):
        raise ValueError(f"bias must be contiguous float32 [{n}]")
    if out is None:
        if dtype not in _DTYPES:
            raise ValueError(f"dtype {dtype} is not float32 or bfloat16")
        out = torch.empty((m, n), dtype=dtype, device=a.data.device)
    ldo = _ld(out, m, n, "out")
    dev = _on_gpu(a.data, w.data, bias, out)
    if m:
        _call(abi.rc_qgemm, dev, C.byref(a.struct()), C.byref(w.struct()), None if bias is None else bias.data_ptr(),
              1 if gelu else 0, out.data_ptr(), _dtype(out, "out"), ldo)
    return out


def qcache_store(cache: QuantCache, active: ActiveSet, k: torch.Tensor, v: torch.Tensor) -> None:
    """Merge the fresh keys and values of the active tokens into the cache:
    k, v [active tokens, heads * 72] float32 or bfloat16 with one row stride
    (views of one product's output will do)."""
    dtype, cols, rows = _dtype(k, "k"), cache.heads * HEAD_DIM, active.total
    ld = _ld(k, rows, cols, "k")
    if v.dtype != k.dtype or _ld(v, rows, cols, "v") != ld:
        raise ValueError("k and v must have one type and row stride")
    dev = _on_gpu(cache.data, k, v, active.idx, active.offsets)
    if rows:
        _call(abi.rc_qcache_store, dev, C.byref(cache.struct()), C.byref(active.struct()), k.data_ptr(), v.data_ptr(), dtype, ld)


def qcache_attention(cache: QuantCache, rows: ActiveSet, q: torch.Tensor, scale: Optional[float] = None,
                     key_len: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of the query rows (chains as in `rows`; its tokens are not
    read) over the first key_len[b] keys (default: all) of their chain.
    q [rows, heads * 72] bfloat16; scale defaults to 1/sqrt(72); key_len int32
    [batch] on the GPU; rows of a chain without keys are 0."""
    cols, total = cache.heads * HEAD_DIM, rows.total
    if q.dtype != torch.bfloat16:
        raise ValueError(f"q is {q.dtype}, not bfloat16")
    ldq = _ld(q, total, cols, "q")
    if key_len is not None and (key_len.dtype != torch.int32 or key_len.shape != (cache.batch,) or not key_len.is_contiguous()):
        raise ValueError(f"key_len must be contiguous int32 [{cache.batch}]")
    if out is None:
        out = torch.empty((total, cols), dtype=torch.bfloat16, device=q.device)
    elif out.dtype != torch.bfloat16:
        raise ValueError(f"out is {out.dtype}, not bfloat16")
    ldo = _ld(out, total, cols, "out")
    dev = _on_gpu(cache.data, q, out, key_len, rows.offsets)
    if total:
        c, s = cache.struct(), rows.struct()
        nbytes = abi.rc_qcache_attention_scratch_bytes(C.byref(c), C.byref(s))
        scratch = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
        _call(abi.rc_qcache_attention, dev, C.byref(c), C.byref(s), None if key_len is None else key_len.data_ptr(),
              q.data_ptr(), ldq, _SCALE if scale is None else float(scale), out.data_ptr(), ldo,
              scratch.data_ptr() if nbytes else None, nbytes)
    return out
