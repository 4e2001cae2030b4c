"""Sizes at which the 8-bit operators' kernels pass from one buffer, tile or key range to the next, against plain forms."""
import numpy as np
import pytest
import torch

import _quant_plans as P
import _quant_ref as R
from test_quant_gpu import KERNELS, Q, check_attention, dev, matrix, product, random_cache, rnd, rows_set  # noqa: F401  (Q: a fixture)

pytestmark = pytest.mark.gpu


def dequantized(q, e, tile):
    return torch.from_numpy(R.dequantize(q, e, tile)).cuda()


@pytest.mark.parametrize("gelu", [False, True])
def test_product_of_two_steps_a_tile(Q, gelu):
    """256 columns of K in 256 x 256 tiles, four of them per workgroup: the bias of each tile is its own.  The bound is
    that of the other products: 2^-16 of the sum of magnitudes (1.13 of it behind GELU, and 2^-19 of the value), and the
    result's rounding, 2^-8 of it."""
    m, n, k = 8100, 8136, 256
    assert P.product_tile(m, n, k, "gelu" if gelu else "store") == (256, 256)
    a, ea, w, ew = product(m, n, k, seed=31)
    bias = rnd(torch.float32, n, seed=32, std=50.0)  # (far apart from column to column)
    y = Q.qgemm(matrix(Q, a, ea, 1), matrix(Q, w, ew, 128), dev(bias), gelu=gelu).double()
    av, wv, bv = dequantized(a, ea, 1), dequantized(w, ew, 128), torch.from_numpy(bias).cuda()
    ref, tol = av @ wv.t() + bv, 2.0 ** -16 * (av.abs() @ wv.abs().t() + bv.abs())
    if gelu:
        ref = 0.5 * ref * (1.0 + torch.tanh((2.0 / np.pi) ** 0.5 * (ref + 0.044715 * ref ** 3)))
        tol = 1.13 * tol + 2.0 ** -19 * ref.abs()
    tol += 2.0 ** -8 * ref.abs() + 1e-38
    assert ((y - ref).abs() <= tol).all()


def put(cache, v, e):
    """Values and scale bytes into the cache."""
    cache.data.copy_(torch.from_numpy(v).float().to(torch.float8_e4m3fn))
    cache.scales.copy_(torch.from_numpy(e).to(torch.uint8))


@pytest.mark.parametrize("heads,tokens,rows", KERNELS)
@pytest.mark.parametrize("share", [0.5, 1.0])
def test_attention_scores_beyond_float32(Q, heads, tokens, rows, share):
    """Finite queries and keys whose product is below the least float32, in whole key ranges: such keys have no weight
    beside keys with logits near -720 (whose float32 error is below 2^-13, 2^-12 of mean |v| in the result), and where
    there are no others the row is 0."""
    nb = tokens // 64
    far = np.arange(nb) < max(1, round(nb * share)) if nb > 1 else np.array([share == 1.0])
    cache, v, e, *_ = random_cache(Q, 1, heads, nb, seed=rows)
    v[:, :, far, 0], e[:, :, far, 0] = 0.0, 230
    v[:, :, far, 0, :, 0] = -448.0      # times 2^103
    v[:, :, ~far, 0, :, 0] = -192.0     # times 2^-35
    e[:, :, ~far, 0] = 92
    put(cache, v, e)
    q = rnd(torch.bfloat16, rows, heads * 72, seed=1, std=3e8)
    q[:, ::72] = 2.0 ** 40
    o = Q.qcache_attention(cache, rows_set([rows]), dev(q, torch.bfloat16))
    if share == 1.0:
        assert (o == 0).all()
    else:
        check_attention(o, v, e, [rows], [tokens], q)
