"""Plain forms of the 8-bit operators in float64 NumPy, from their definitions."""
from __future__ import annotations

import numpy as np

# every e4m3 number by its code: 4 exponent bits (bias 7), 3 of mantissa, codes 127 and 255 NaN
_c = np.arange(256)
_e, _m = (_c >> 3) & 15, _c & 7
E4M3 = np.where(_e == 0, _m * 2.0 ** -9, (8 + _m) * 2.0 ** (_e - 10.0)) * np.where(_c & 128, -1.0, 1.0)
E4M3[[127, 255]] = np.nan


def scale_byte(amax) -> np.ndarray:
    """The least e >= 1 with amax <= 448 * 2^(e - 127)."""
    amax = np.asarray(amax, np.float64)
    e = np.ones(amax.shape, np.int64)
    for _ in range(300):
        e += amax > 448.0 * 2.0 ** (e - 127.0)
    return e


def round_e4m3(y) -> np.ndarray:
    """Nearest e4m3 number (|y| <= 448), ties to the even code; not finite: NaN."""
    y = np.asarray(y, np.float64)
    grid = E4M3[:127]
    a = np.where(np.isfinite(y), np.abs(y), 0.0)
    hi = np.clip(np.searchsorted(grid, a), 1, 126)
    lo = hi - 1
    up = (grid[hi] - a < a - grid[lo]) | ((grid[hi] - a == a - grid[lo]) & (hi % 2 == 0))
    q = np.copysign(grid[np.where(up, hi, lo)], y)
    return np.where(np.isfinite(y), q, np.nan)


def amax_finite(x, axis):
    return np.max(np.where(np.isfinite(x), np.abs(x), 0.0), axis=axis)


def quantize(x, tile):
    """Values (e4m3 numbers) and scale bytes [column blocks][row blocks]."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    padded = np.pad(x, ((0, -rows % tile), (0, -cols % 128)))
    e = scale_byte(amax_finite(padded.reshape(-1, tile, padded.shape[1] // 128, 128), (1, 3)).T)
    f = np.repeat(np.repeat(2.0 ** (127.0 - e).T, tile, 0)[:rows], 128, 1)[:, :cols]
    return round_e4m3(x * f), e


def dequantize(q, e, tile):
    f = 2.0 ** (np.asarray(e, np.float64) - 127.0)
    f = np.repeat(np.repeat(f.T, tile, 0)[:q.shape[0]], 128, 1)[:, :q.shape[1]]
    return np.asarray(q, np.float64) * f


def gelu(y):
    return 0.5 * y * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (y + 0.044715 * y ** 3)))


def store(data, scales, per_chain, k, v):
    """data [B][H][blocks][2][64][72] values, scales bytes: both changed in place."""
    r = 0
    heads = data.shape[1]
    for b, toks in enumerate(per_chain):
        for blk in sorted({int(t) // 64 for t in toks}):
            at = [(r + i, int(t) % 64) for i, t in enumerate(toks) if t // 64 == blk]
            for which, rows in ((0, k), (1, v)):
                for h in range(heads):
                    w = data[b, h, blk, which] * 2.0 ** (scales[b, h, blk, which] - 127.0)
                    for src, dst in at:
                        w[dst] = rows[src, h * 72:(h + 1) * 72]
                    e = scale_byte(amax_finite(w, None))
                    data[b, h, blk, which] = round_e4m3(w * 2.0 ** (127.0 - e))
                    scales[b, h, blk, which] = e
        r += len(toks)


def attention(data, scales, offsets, key_len, q, scale):
    """Output and the weighted mean of |v| [rows][heads * 72] (what rounding errors are measured against)."""
    heads = data.shape[1]
    o, mean_abs = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(len(offsets) - 1):
        n = int(key_len[b])
        rows = slice(offsets[b], offsets[b + 1])
        if n == 0 or offsets[b] == offsets[b + 1]:
            continue
        for h in range(heads):
            blocks = data[b, h] * (2.0 ** (scales[b, h].astype(np.float64) - 127.0))[..., None, None]
            kk, vv = blocks[:, 0].reshape(-1, 72)[:n], blocks[:, 1].reshape(-1, 72)[:n]
            c = slice(h * 72, (h + 1) * 72)
            s = q[rows, c] @ kk.T * scale
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            o[rows, c] = p @ vv
            mean_abs[rows, c] = p @ np.abs(vv)
    return o, mean_abs
