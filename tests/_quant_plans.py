"""The library's choices of tiles and key ranges for the 8-bit operators (host code)."""
from __future__ import annotations

import ctypes as C

EPI = {"store": 0, "gelu": 1, "gelu8": 2, "resid": 3}


class _Tile(C.Structure):
    _fields_ = [("bm", C.c_int), ("bn", C.c_int)]


class _Attn(C.Structure):
    _fields_ = [("qh", C.c_int), ("splits", C.c_int), ("workgroups", C.c_longlong)]


def product_tile(m, n, k, epi="store", large=True):
    """(rows, columns) of a workgroup's tile; large: the results allow the largest tiles (8-bit, or bfloat16 with n and
    the rows' distance multiples of 8)."""
    from paper_2608_29809_amd import abi
    f = abi.LIB._ZN2rc10plan_qgemmEiiiNS_8QGemmEpiEb
    f.restype, f.argtypes = _Tile, [C.c_int] * 4 + [C.c_bool]
    p = f(m, n, k, EPI[epi], large)
    return p.bm, p.bn


def attention(counts, heads, tokens):
    """(32-query halves per wave, 0: the kernel for few queries; key ranges) for chains of `counts` query rows."""
    from paper_2608_29809_amd import abi
    f = abi.LIB._ZN2rc15plan_qattentionEPKiiii
    f.restype, f.argtypes = _Attn, [C.POINTER(C.c_int)] + [C.c_int] * 3
    offs = [0]
    for n in counts:
        offs.append(offs[-1] + int(n))
    p = f((C.c_int * len(offs))(*offs), len(counts), heads, tokens)
    return p.qh, p.splits
