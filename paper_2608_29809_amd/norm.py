"""Norms before and after a block on PyTorch tensors, fused with what stands
beside them: the modulation of the normalised rows, their quantisation for the
next product, and the gated residual update.  Argument checks and allocation
only; every computation is a call into libregioncache.so.

    a = norm_modulate(x, Norm("layer"), scale, shift, dtype=torch.int8)    # what the block takes
    h = ...                                                                # what it makes of it
    a = residual_norm(x, h, gate, post=Norm("rms", weight=w),              # x <- x + gate post(h), and
                      pre=Norm("layer"), scale=scale2, shift=shift2)       # what the next block takes

scale, shift and gate are one vector, or one for each chain with the chains'
row ranges in `rows`.  Results are bfloat16 or float32 tensors, for dtype
torch.float8_e4m3fn a QuantMatrix and for torch.int8 an IntMatrix.  Calls go to
the current stream of their tensors' device.  There are no gradients: where they
are recorded, tensors that require one are refused; a norm's weights are constants.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Union

import torch

from . import abi
from .quant import _DTYPES, _F8, _F32, _I8, IntMatrix, QuantMatrix, _call, _dtype, _empty, _grad_enabled, _ld, _no_gradient, _on_gpu, _written
from .runtime import ActiveSet

__all__ = ["Norm", "norm_modulate", "residual_norm"]

_KINDS = {"layer": abi.RC_NORM_LAYER, "rms": abi.RC_NORM_RMS}
Result = Union[torch.Tensor, QuantMatrix, IntMatrix]


class Norm:
    """LayerNorm ("layer") or RMS norm ("rms") of rows, with weight and bias
    (float32 [cols]) or without.  Both are held as they lie in memory now:
    changes in place are seen, another tensor put in their place is not, and
    where that memory is resized the norm is refused."""

    __slots__ = ("_kind", "_eps", "_cols", "_index", "_weight", "_bias", "_struct", "_address")

    def __init__(self, kind: str = "layer", eps: float = 1e-6, weight: Optional[torch.Tensor] = None,
                 bias: Optional[torch.Tensor] = None):
        code = _KINDS.get(kind)
        if code is None:
            raise ValueError(f"norm {kind!r} is not 'layer' or 'rms'")
        cols = index = at_weight = at_bias = held_weight = held_bias = None
        if weight is not None:
            cols, index, at_weight, held_weight = self._hold(weight, "weight")
        if bias is not None:
            cols_bias, index_bias, at_bias, held_bias = self._hold(bias, "bias")
            if weight is not None and cols != cols_bias:
                raise ValueError(f"weight and bias have {cols} and {cols_bias} values")
            if weight is not None and index != index_bias:
                raise ValueError(f"weight and bias are on {weight.device} and {bias.device}")
            cols, index = cols_bias, index_bias
        self._kind, self._eps, self._cols, self._index, self._weight, self._bias = kind, eps, cols, index, held_weight, held_bias
        self._struct = abi.rc_norm(code, eps, at_weight, at_bias)
        self._address = C.addressof(self._struct)

    @staticmethod
    def _hold(t: torch.Tensor, what: str):
        """Its width, device, address, and memory: a storage, where that lies and its bytes (a tensor may be given other memory)."""
        if t.dtype != _F32 or t.dim() != 1 or not t.is_contiguous():
            raise ValueError(f"{what} must be contiguous float32 [cols]")
        memory = t.untyped_storage()
        return t.shape[0], t.get_device(), t.data_ptr(), (memory, memory.data_ptr(), memory.nbytes())

    def _tensor(self, held, address) -> Optional[torch.Tensor]:
        if held is None:
            return None
        _intact(held, "a norm's weights")
        memory, start, _ = held
        return torch.empty(0, dtype=_F32, device=memory.device).set_(memory, max(0, (address or 0) - start) // 4, (self._cols,))

    # (read-only: the C structure is made once)
    kind = property(lambda self: self._kind)
    eps = property(lambda self: self._eps)
    weight = property(lambda self: self._tensor(self._weight, self._struct.weight))
    bias = property(lambda self: self._tensor(self._bias, self._struct.bias))


def _intact(held, what: str) -> None:
    """Refuses memory that was moved, freed or cut since it was held."""
    memory, start, size = held
    if memory.data_ptr() != start or memory.nbytes() != size:
        raise ValueError(f"the memory of {what} was resized")


def _vector(t: torch.Tensor, cols: int, rows: Optional[ActiveSet], index: int, what: str):
    """Address and chain stride of [cols] or [chains, cols] float32 vectors."""
    if t.dtype != _F32:
        raise ValueError(f"{what} is {t.dtype}, not float32")
    if t.get_device() != index:
        raise ValueError(f"{what} is on {t.device}, x on cuda:{index}")
    shape, strides = t.shape, t.stride()
    chains = len(shape) == 2
    if len(shape) == 0 or shape[-1] != cols or (shape[0] != (1 if rows is None else rows.batch) if chains else len(shape) != 1):
        raise ValueError(f"{what} is {tuple(shape)}, not [{cols}] or [{1 if rows is None else rows.batch}, {cols}]")
    if strides[-1] != 1 and cols > 1:
        raise ValueError(f"{what}: the values of a vector must be contiguous")
    return t.data_ptr(), strides[0] if chains and shape[0] > 1 else 0


def _norm(norm: Norm, cols: int, index: int, what: str) -> int:
    """Address of the norm's C structure."""
    if norm._cols is not None:
        if norm._cols != cols:
            raise ValueError(f"{what} has weights of {norm._cols} values, x {cols}")
        if norm._index != index:
            raise ValueError(f"the weights of {what} are on {'the CPU' if norm._index < 0 else f'cuda:{norm._index}'}, x on cuda:{index}")
        if norm._weight is not None:
            _intact(norm._weight, f"the weight of {what}")
        if norm._bias is not None:
            _intact(norm._bias, f"the bias of {what}")
    return norm._address


def _run(x, h, gate, post, residual_scale, pre, scale, shift, rows, dtype, out):
    written = () if h is None else (x,)
    if out is not None:
        written += (out,) if isinstance(out, torch.Tensor) else (out._data, out._scales)
    if _grad_enabled() and (x.requires_grad or h is not None and h.requires_grad or gate is not None and gate.requires_grad
                            or scale is not None and scale.requires_grad or shift is not None and shift.requires_grad
                            or written and written[-1].requires_grad):
        raise _no_gradient("norm_modulate" if h is None else "residual_norm")
    shape = x.shape
    if len(shape) != 2:
        raise ValueError(f"x is {tuple(shape)}, not [rows, cols]")
    n, cols = shape
    if n >> 31 or cols >> 31:
        raise ValueError(f"{n} x {cols} is too large")
    x_dtype, ldx = _dtype(x, "x"), cols if x.is_contiguous() else _ld(x, n, cols, "x")
    if h is None:
        index = _on_gpu(x)
        ph = ldh = h_dtype = pgate = sgate = ppost = 0
    else:
        index = _on_gpu(x, h)
        ph, ldh, h_dtype = h.data_ptr(), _ld(h, n, cols, "h"), _dtype(h, "h")
        pgate, sgate = (0, 0) if gate is None else _vector(gate, cols, rows, index, "gate")
        ppost = 0 if post is None else _norm(post, cols, index, "post")
    ppre = pscale = sscale = pshift = sshift = pout = ldo = out_dtype = e4m3 = int8 = 0
    if pre is not None:
        ppre = _norm(pre, cols, index, "the norm")
        if scale is not None:
            pscale, sscale = _vector(scale, cols, rows, index, "scale")
        if shift is not None:
            pshift, sshift = _vector(shift, cols, rows, index, "shift")
        if out is None:
            if dtype in _DTYPES:
                out_dtype, ldo = _DTYPES[dtype], cols
                out = _empty(n, cols, dtype, index)
                pout = out.data_ptr()
            elif dtype == _I8:
                out = IntMatrix._new(n, cols, index)
                int8 = C.addressof(out.struct())
            elif dtype == _F8:
                out = QuantMatrix.alloc(n, cols, 1, x.device)
                e4m3 = C.addressof(out.struct())
            else:
                raise ValueError(f"dtype {dtype} is not float32, bfloat16, float8_e4m3fn or int8")
        elif isinstance(out, IntMatrix):
            _on_gpu(x, out._data)
            int8 = C.addressof(out.struct())
        elif isinstance(out, QuantMatrix):
            _on_gpu(x, out._data)
            e4m3 = C.addressof(out.struct())
        else:
            _on_gpu(x, out)
            pout, ldo, out_dtype = out.data_ptr(), _ld(out, n, cols, "out"), _dtype(out, "out")
    elif scale is not None or shift is not None or out is not None:
        raise ValueError("scale, shift or out without a norm before the next block (pre)")
    chains = None
    if rows is not None:
        if rows.total != n:
            raise ValueError(f"the chains have {rows.total} rows, x {n}")
        if rows.offsets.get_device() != index:
            raise ValueError(f"the chains' offsets are on {rows.offsets.device}, x on cuda:{index}")
        chains = rows.struct()
    if n:
        _call(abi.rc_residual_norm, index, abi.norm_args(
            n, cols, x.data_ptr(), ldx, ph, ldh, x_dtype, h_dtype, ppost, ppre, residual_scale, sgate, sscale, sshift, pgate, pscale, pshift,
            0 if chains is None else C.addressof(chains), pout, ldo, out_dtype, e4m3, int8))
        if written:
            _written(written)
    return out


def norm_modulate(x: torch.Tensor, norm: Norm, scale: Optional[torch.Tensor] = None, shift: Optional[torch.Tensor] = None,
                  rows: Optional[ActiveSet] = None, dtype: torch.dtype = torch.bfloat16, out: Optional[Result] = None) -> Result:
    """norm(x) (1 + scale) + shift of rows x [rows, cols] float32 or bfloat16,
    cols to 16384, in dtype or in out, which may be x.  scale, shift: float32
    [cols] or [chains, cols], chains' row ranges as in `rows` (its tokens are not
    read)."""
    if norm is None:
        raise ValueError("norm is None")
    return _run(x, None, None, None, 1.0, norm, scale, shift, rows, dtype, out)


def residual_norm(x: torch.Tensor, h: torch.Tensor, gate: Optional[torch.Tensor] = None, post: Optional[Norm] = None,
                  residual_scale: float = 1.0, pre: Optional[Norm] = None, scale: Optional[torch.Tensor] = None,
                  shift: Optional[torch.Tensor] = None, rows: Optional[ActiveSet] = None, dtype: torch.dtype = torch.bfloat16,
                  out: Optional[Result] = None) -> Optional[Result]:
    """x <- residual_scale x + gate post(h) in place, and with `pre` the result
    pre(x) (1 + scale) + shift of the new x as norm_modulate would give it (of
    its float32 values, before they are rounded to x's type).  x, h [rows, cols]
    float32 or bfloat16; x, h and out do not overlap; gate like scale and shift."""
    if h is None:
        raise ValueError("h is None")
    return _run(x, h, gate, post, residual_scale, pre, scale, shift, rows, dtype, out)
