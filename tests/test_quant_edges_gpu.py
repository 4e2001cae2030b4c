"""Sizes at which the 8-bit operators' kernels pass from one buffer, tile or key range to the next, against plain forms."""
import numpy as np
import pytest
import torch

import _quant_plans as P
import _quant_ref as R
from test_quant_gpu import Q, dev, matrix, product, rnd  # noqa: F401  (Q: a fixture)

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
