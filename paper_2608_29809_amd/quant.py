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


def _need(ok: bool, msg: str):
    if not ok:
        raise ValueError(msg)


def _dtype(t: torch.Tensor, what: str) -> int:
    _need(t.dtype in _DTYPES, f"{what} is {t.dtype}, not float32 or bfloat16")
    return _DTYPES[t.dtype]


def _on_gpu(first: torch.Tensor, *others: Optional[torch.Tensor]):
    _need(first.is_cuda, "the tensors must be on the GPU")
    for t in others:
        _need(t is None or t.device == first.device, f"tensors on {first.device} and {t.device if t is not None else None}")


def _call(f, device: torch.device, *args):
    """f(*args, stream) with `device` current and its current stream."""
    if device.index == torch.cuda.current_device():
        f(*args, torch.cuda.current_stream().cuda_stream)
    else:
        with torch.cuda.device(device):
            f(*args, torch.cuda.current_stream().cuda_stream)


def _rows(t: torch.Tensor, cols: int, what: str):
    """A [rows][cols] tensor whose rows are contiguous."""
    _need(t.dim() == 2 and t.shape[1] == cols, f"{what} is {tuple(t.shape)}, not [rows, {cols}]")
    _need(t.stride(1) == 1 or cols == 1, f"{what}: the values of a row must be contiguous")
    return t.stride(0) if t.shape[0] > 1 else max(cols, t.stride(0))


class QuantMatrix:
    """A matrix in 8 bits: `data` float8_e4m3fn [rows, cols], `scales` uint8
    [column blocks, row blocks rounded up to 16], block_rows 1 or 128.  Views
    of rows are given as data[:n] with the same scales."""

    __slots__ = ("data", "scales", "block_rows")

    def __init__(self, data: torch.Tensor, scales: torch.Tensor, block_rows: int):
        _need(data.dim() == 2 and data.dtype == torch.float8_e4m3fn, "data must be float8_e4m3fn [rows, cols]")
        _need(scales.dim() == 2 and scales.dtype == torch.uint8 and scales.stride(1) == 1, "scales must be uint8 rows")
        _need(block_rows in (1, BLOCK), f"block_rows {block_rows} is not 1 or {BLOCK}")
        _need(scales.shape[0] == -(-data.shape[1] // BLOCK) and scales.shape[1] >= -(-data.shape[0] // block_rows),
              f"scales {tuple(scales.shape)} do not cover data {tuple(data.shape)}")
        _on_gpu(data, scales)
        self.data, self.scales, self.block_rows = data, scales, block_rows

    @classmethod
    def alloc(cls, rows: int, cols: int, block_rows: int = 1, device="cuda") -> "QuantMatrix":
        data = torch.empty((rows, cols), dtype=torch.float8_e4m3fn, device=device)
        row_blocks = -(-rows // max(block_rows, 1))
        scales = torch.empty((-(-cols // BLOCK), row_blocks + -row_blocks % 16), dtype=torch.uint8, device=device)
        return cls(data, scales, block_rows)

    def struct(self) -> abi.rc_qmat:
        rows, cols = self.data.shape
        ld = _rows(self.data, cols, "data")
        scale_ld = self.scales.stride(0) if self.scales.shape[0] > 1 else self.scales.shape[1]
        return abi.rc_qmat(self.data.data_ptr(), self.scales.data_ptr(), ld, rows, cols, scale_ld, self.block_rows)


class QuantCache:
    """Keys and values of `batch` chains in 8 bits: `data` float8_e4m3fn
    [batch, heads, blocks, 2, 64, 72] (a block's 64 keys, then its values) and
    `scales` uint8 [batch, heads, blocks, 2].  Chains may be any multiple of
    16 bytes apart; within a chain the cache is contiguous."""

    __slots__ = ("data", "scales", "batch", "heads", "tokens")

    def __init__(self, data: torch.Tensor, scales: torch.Tensor):
        _need(data.dim() == 6 and tuple(data.shape[3:]) == (2, KEY_BLOCK, HEAD_DIM) and data.dtype == torch.float8_e4m3fn,
              f"data must be float8_e4m3fn [batch, heads, blocks, 2, {KEY_BLOCK}, {HEAD_DIM}]")
        _need(scales.dtype == torch.uint8 and scales.shape == data.shape[:4], "scales must be uint8 [batch, heads, blocks, 2]")
        _need(data.numel() > 0, "the cache is empty")
        _need(data[0].is_contiguous() and scales[0].is_contiguous(), "a chain of the cache must be contiguous")
        _on_gpu(data, scales)
        self.data, self.scales = data, scales
        self.batch, self.heads, self.tokens = data.shape[0], data.shape[1], data.shape[2] * KEY_BLOCK

    @classmethod
    def alloc(cls, batch: int, heads: int, tokens: int, device="cuda") -> "QuantCache":
        """A cache of zeros."""
        _need(tokens > 0 and tokens % KEY_BLOCK == 0, f"tokens {tokens} is not a positive multiple of {KEY_BLOCK}")
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
    _need(x.dim() == 2, f"x is {tuple(x.shape)}, not [rows, cols]")
    ldx = _rows(x, x.shape[1], "x")
    if out is None:
        out = QuantMatrix.alloc(x.shape[0], x.shape[1], block_rows, x.device)
    _need(out.data.shape == x.shape and out.block_rows == block_rows, "out has another shape or other blocks")
    _on_gpu(x, out.data)
    if x.shape[0]:
        _call(abi.rc_quantize, x.device, x.data_ptr(), dtype, ldx, C.byref(out.struct()))
    return out


def qgemm(a: QuantMatrix, w: QuantMatrix, bias: Optional[torch.Tensor] = None, gelu: bool = False,
          dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """act(a w^T + bias): a [m, k] with block_rows 1, w [n, k] with block_rows
    128, bias float32 [n]; the result [m, n] in dtype (or in out)."""
    m, n = a.data.shape[0], w.data.shape[0]
    _need(bias is None or (bias.dtype == torch.float32 and tuple(bias.shape) == (n,) and bias.is_contiguous()),
          f"bias must be contiguous float32 [{n}]")
    if out is None:
        _need(dtype in _DTYPES, f"dtype {dtype} is not float32 or bfloat16")
        out = torch.empty((m, n), dtype=dtype, device=a.data.device)
    _need(out.shape == (m, n), f"out is {tuple(out.shape)}, not [{m}, {n}]")
    ldo = _rows(out, n, "out")
    _on_gpu(a.data, w.data, bias, out)
    if m:
        _call(abi.rc_qgemm, out.device, C.byref(a.struct()), C.byref(w.struct()), None if bias is None else bias.data_ptr(),
              1 if gelu else 0, out.data_ptr(), _dtype(out, "out"), ldo)
    return out


def qcache_store(cache: QuantCache, active: ActiveSet, k: torch.Tensor, v: torch.Tensor) -> None:
    """Merge the fresh keys and values of the active tokens into the cache:
    k, v [active tokens, heads * 72] float32 or bfloat16 with one row stride
    (views of one product's output will do)."""
    dtype, cols = _dtype(k, "k"), cache.heads * HEAD_DIM
    ld = _rows(k, cols, "k")
    _need(v.dtype == k.dtype and v.shape == k.shape and _rows(v, cols, "v") == ld, "k and v must be alike")
    _need(k.shape[0] == active.total, f"{k.shape[0]} rows for {active.total} active tokens")
    _on_gpu(cache.data, k, v, active.idx, active.offsets)
    if active.total:
        _call(abi.rc_qcache_store, cache.data.device, C.byref(cache.struct()), C.byref(active.struct()), k.data_ptr(),
              v.data_ptr(), dtype, ld)


def qcache_attention(cache: QuantCache, rows: ActiveSet, q: torch.Tensor, scale: Optional[float] = None,
                     key_len: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of the query rows (chains as in `rows`; its tokens are not
    read) over the first key_len[b] keys (default: all) of their chain.
    q [rows, heads * 72] bfloat16; scale defaults to 1/sqrt(72); key_len int32
    [batch] on the GPU; rows of a chain without keys are 0."""
    cols = cache.heads * HEAD_DIM
    _need(q.dtype == torch.bfloat16, f"q is {q.dtype}, not bfloat16")
    ldq = _rows(q, cols, "q")
    _need(q.shape[0] == rows.total, f"{q.shape[0]} rows for {rows.total} in the set")
    _need(key_len is None or (key_len.dtype == torch.int32 and tuple(key_len.shape) == (cache.batch,) and
                              key_len.is_contiguous()), f"key_len must be contiguous int32 [{cache.batch}]")
    if out is None:
        out = torch.empty((q.shape[0], cols), dtype=torch.bfloat16, device=q.device)
    _need(out.dtype == torch.bfloat16 and out.shape == q.shape, f"out must be bfloat16 {tuple(q.shape)}")
    ldo = _rows(out, cols, "out")
    _on_gpu(cache.data, q, out, key_len, rows.offsets)
    if rows.total:
        c, s = cache.struct(), rows.struct()
        nbytes = abi.rc_qcache_attention_scratch_bytes(C.byref(c), C.byref(s))
        scratch = torch.empty(nbytes, dtype=torch.uint8, device=q.device) if nbytes else None
        _call(abi.rc_qcache_attention, q.device, C.byref(c), C.byref(s), None if key_len is None else key_len.data_ptr(),
              q.data_ptr(), ldq, 1.0 / math.sqrt(HEAD_DIM) if scale is None else float(scale), out.data_ptr(), ldo,
              scratch.data_ptr() if nbytes else None, nbytes)
    return out
