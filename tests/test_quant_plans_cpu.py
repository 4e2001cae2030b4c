"""What the GPU tests of the 8-bit operators reach: every tile of the products and every kernel of the attention, by
the library's own choice; and what its aimed queries would notice."""
import pytest
import torch

import _quant_aimed as A
import _quant_plans as P
from test_quant_aimed_gpu import CASES, LONG_FEW
from test_quant_gpu import LARGE, SIZES
from test_quant_tiles_gpu import PRODUCTS, STEPS

SMALL = [(16, 16), (32, 32), (64, 32), (64, 64), (64, 128), (128, 128)]
BIG = [(192, 256), (256, 256)]


def test_products_of_the_tests_reach_every_tile():
    """Every tile that has an epilogue, with every type of its results."""
    seen = set()
    for m, n, k in SIZES:
        epi = "gelu" if m % 2 else "store"
        seen |= {(P.product_tile(m, n, k, epi, n % 8 == 0), epi, "bf16"), (P.product_tile(m, n, k, epi, False), epi, "f32")}
    for m, n, k, _ in LARGE:
        seen |= {(P.product_tile(m, n, k, epi), epi, "bf16") for epi in ("store", "gelu")}
    for m, n, k, gelu, f32 in PRODUCTS:
        epi = "gelu" if gelu else "store"
        seen.add((P.product_tile(m, n, k, epi, not f32), epi, "f32" if f32 else "bf16"))
    rows = [chains * active for chains, active in STEPS] + [4096] + [29, 70, 93, 512, 8000, 10240]  # (the other steps')
    for m in rows:
        seen |= {(P.product_tile(m, 4608, 1152, "gelu8"), "gelu8", "e4m3"), (P.product_tile(m, 1152, 4608, "resid"), "resid", "f32")}
    want = {(t, epi, out) for t in SMALL for epi in ("store", "gelu") for out in ("bf16", "f32")}
    want |= {(t, epi, "bf16") for t in BIG for epi in ("store", "gelu")}
    want |= {(t, "gelu8", "e4m3") for t in SMALL[4:] + BIG} | {(t, "resid", "f32") for t in SMALL[2:] + BIG}
    assert seen == want


def test_attention_cases_reach_every_kernel():
    seen = {}
    for heads, tokens, counts, keys in CASES:
        qh, splits = P.attention(counts, heads, tokens)
        tiles = -(-max(keys) // 64) // splits
        seen.setdefault((qh, splits > 1), []).append(tiles)
    assert set(seen) == {(qh, s) for qh in (0, 1, 2) for s in (False, True)}
    for qh in (1, 2):  # ranges of more than 64 tiles
        assert max(seen[qh, False] + seen[qh, True]) > 64
    heads, tokens, rows = LONG_FEW
    qh, splits = P.attention([rows], heads, tokens)
    assert qh == 0 and splits == 16 and tokens // 64 // splits // 8 > 64  # (of each of eight waves)


@pytest.mark.parametrize("spread", [True, False])
def test_aimed_queries_notice_a_wrong_tile(spread):
    """A tile left out, taken twice, or with a neighbour's scale of its keys or values, planted in the plain form."""
    tokens, keys = 2048, 2021
    codes, e = A.cache(1, 1, tokens, 7, spread, "cpu")
    k, v = A.values(codes, e)[0, :, 0]
    aim = torch.tensor(A.pairs(keys))
    q = A.queries(k, aim, 36.0)
    s = q.double() @ k[:keys].t() * A.SCALE
    p = torch.softmax(s, -1)
    ref, mean_abs = p @ v[:keys], p @ v[:keys].abs()
    both = p.gather(1, aim)
    assert (both > 0.2).all() and (both.sum(1) > 0.9).all()
    w, tiles = torch.exp(s - 36.0), -(-keys // 64)

    def noticed(w, v):
        o = (w @ v[:keys]) / w.sum(1, keepdim=True)
        return ((o - ref).abs() > A.bound(ref, mean_abs)).any()

    assert not noticed(w, v)
    for t in range(tiles):
        c = slice(64 * t, min(64 * t + 64, keys))
        for times in (0.0, 2.0):
            other = w.clone()
            other[:, c] *= times
            assert noticed(other, v), (t, times)
        for near in (t - 1, t + 1):
            if 0 <= near < tiles:
                f = torch.exp2(e[0, 0, near].double() - e[0, 0, t].double())
                other = w.clone()
                other[:, c] = torch.exp(s[:, c] * f[0] - 36.0)
                assert noticed(other, v), (t, near, "keys")
                other = v.clone()
                other[c] *= f[1]
                assert noticed(w, other), (t, near, "values")
