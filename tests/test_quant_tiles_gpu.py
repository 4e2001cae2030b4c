"""Products in every tile that the library chooses among: those that the other tests' sizes do not reach, and the steps
with 8-bit weights at the row counts whose epilogues (8-bit GELU results, residual and hidden state) take each tile."""
import numpy as np
import pytest
import torch

import _quant_ref as R
from test_quant_gpu import Q, check_product, dev, matrix, product, rnd  # noqa: F401  (Q: a fixture)
from test_quant_step_gpu import Case, slot_values

pytestmark = pytest.mark.gpu

# m, n, k, GELU, float32 results
PRODUCTS = [
    (723, 1152, 4608, True, False), (723, 1152, 4608, True, True),    # 64 x 64
    (301, 2304, 400, False, True), (301, 2304, 400, True, True),      # 64 x 128, whole vectors of float32
    (301, 2304, 400, False, False),
    (1501, 4608, 272, False, True), (1501, 4608, 272, True, True),    # 128 x 128 likewise
    (3, 40, 65536, False, False), (70, 200, 65536, True, True),       # the longest sum
    (1501, 1160, 65536, False, False),
]
# chains alike, active tokens of each: 128 x 128 tiles for the GELU results (1000, 1405 and 3650 rows), 64 x 128 and
# 128 x 128 for the residual (1405 and 2000; 3650 and 4000); chains and the last tile end inside a tile
STEPS = [(2, 500), (5, 281), (5, 400), (5, 730), (5, 800)]


@pytest.mark.parametrize("m,n,k,gelu,f32", PRODUCTS)
def test_products_of_other_tiles(Q, m, n, k, gelu, f32):
    a, ea, w, ew = product(m, n, k, seed=m + k)
    bias = rnd(torch.float32, n, seed=9)
    dt = torch.float32 if f32 else torch.bfloat16
    buf = torch.full((m + 2, n + 8), 77.0, dtype=dt, device="cuda")
    Q.qgemm(matrix(Q, a, ea, 1, 32), matrix(Q, w, ew, 128, 16), dev(bias), gelu=gelu, out=buf[:m, :n])
    check_product(buf[:m, :n], a, ea, w, ew, bias, gelu, f32)
    assert (buf[:, n:] == 77.0).all() and (buf[m:] == 77.0).all()


@pytest.fixture(scope="module")
def case():
    """Five chains alike on a grid of 1024 tokens, 8-bit weights."""
    c = Case(B=5, layers=1, grid=(32, 32))
    c.txt[:], c.lat[:] = c.txt[0], c.lat[0]
    c.tkv, c.latent = c.model.prepare_text(c.model.to_storage(c.txt)), torch.from_numpy(c.lat).cuda()
    c.model.quantize_weights()
    return c


@pytest.mark.parametrize("chains,active", STEPS)
def test_region_steps_of_other_tiles(case, chains, active):
    """The first chain against the oracle, the others equal to it."""
    from paper_2608_29809_amd.runtime import ActiveSet
    s, m = case.s, case.model
    tkv = m.prepare_text(m.to_storage(case.txt[:chains]))
    x = case.latent[:chains].contiguous()
    cache, out = m.alloc_cache(chains, 1, bits=8), torch.empty_like(x)
    m.build_cache(cache, 0, x, 500, 450, tkv, latent_out=out)
    before = [slot_values(cache, 0, 0)[0]]
    h = cache.H(0, 0, 0).clone()
    idx = np.sort(np.random.default_rng(active).choice(s.tokens, active, replace=False))
    m.reuse_step(cache, 0, ActiveSet.from_lists([idx] * chains), x, 300, 250, tkv, latent_out=out)
    case.check(cache, 0, 300, [idx], True, before)
    rest = np.setdiff1d(np.arange(s.tokens), idx)
    assert torch.equal(cache.H(0, 0, 0)[rest], h[rest])
    for b in range(1, chains):
        assert torch.equal(cache.H(b, 0, 0), cache.H(0, 0, 0)) and torch.equal(out[b], out[0])
        assert torch.equal(cache.quant(0, 0).data[b].view(torch.uint8), cache.quant(0, 0).data[0].view(torch.uint8))


def test_dense_step_of_1024_px():
    """4096 rows of one chain: every block against the oracle."""
    c = Case(B=1, layers=1, grid=(64, 64))
    c.model.quantize_weights()
    cache, out = c.model.alloc_cache(1, 1, bits=8), torch.empty_like(c.latent)
    c.model.build_cache(cache, 0, c.latent, 500, 450, c.tkv, latent_out=out)
    c.check(cache, 0, 500, [np.arange(c.s.tokens)], True)
    assert torch.isfinite(out).all()
