"""Attention inputs in which every tile of keys decides some row.

A query is aimed at two keys of different tiles: both have the same logit, far above
all others, so the row is the mean of their values.  A tile left out, taken twice or
read with another tile's scales moves a row by far more than roundings do.  Keys have
the same distribution in every tile, but scale bytes that differ from tile to tile."""
from __future__ import annotations

import torch

SCALE = 72 ** -0.5


def cache(batch, heads, tokens, seed, spread, device):
    """Codes [batch][heads][tiles][2][64][72] as float8, scale bytes [batch][heads][tiles][2].  spread: value scales over
    a range of 2^7, else of 2."""
    gen = torch.Generator(device).manual_seed(seed)
    tiles = tokens // 64
    x = torch.randn((batch, heads, tiles, 2, 64, 72), generator=gen, device=device) * 100.0
    t = torch.arange(tiles, device=device) + 2 * torch.arange(heads, device=device)[:, None]
    less = (3 * t) % 5
    x[:, :, :, 0] *= torch.exp2(-less.float())[..., None, None]
    e = torch.empty((batch, heads, tiles, 2), dtype=torch.uint8, device=device)
    e[..., 0] = (120 + less).to(torch.uint8)
    e[..., 1] = (118 + (5 * t) % 7 if spread else 120 + t % 2).to(torch.uint8)
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn), e  # (beyond 464 a value would become NaN)


def values(codes, e):
    """Keys and values [batch][2][heads][tokens][72] in float64."""
    v = codes.double() * torch.exp2(e.double() - 127.0)[..., None, None]
    return v.permute(0, 3, 1, 2, 4, 5).flatten(3, 4)


def pairs(keys, tiles=None):
    """Pairs of keys, the first and last key of every tile (or of those given) among them."""
    n = -(-keys // 64)
    out = []
    for t in range(n) if tiles is None else tiles:
        other = (t + n // 2 + (n > 2)) % n
        at = min(64 * other + (17 * t + 5) % 64, keys - 1)
        for a in (64 * t, min(64 * t + 63, keys - 1)):
            out.append((a, at if at != a else a - 1 if a else a + 1))
    return out


def queries(k, aim, level):
    """bfloat16 queries [rows][72] with logit `level` at both keys of aim [rows][2]; k [tokens][72] float64."""
    ab = k[aim]                                            # [rows][2][72]
    gram = (ab[:, :, None] * ab[:, None]).sum(-1)
    det = gram[:, 0, 0] * gram[:, 1, 1] - gram[:, 0, 1] ** 2
    x = torch.stack([gram[:, 1, 1] - gram[:, 0, 1], gram[:, 0, 0] - gram[:, 0, 1]], 1) / det[:, None] * (level / SCALE)
    return (x[..., None] * ab).sum(1).to(torch.bfloat16)


def weights(q, k, keys):
    """Softmax weights [rows][keys] in float64."""
    return torch.softmax(q.double() @ k[:keys].t() * SCALE, -1)


def bound(o, mean_abs):
    """The result rounded once, 2^-8 |o|; rounded probabilities, 2^-8 (mean |v| + |o|); scores' errors below 2^-13, 2^-12 of
    mean |v|."""
    return 2.0 ** -8 * (2 * o.abs() + mean_abs) + 2.0 ** -12 * mean_abs
