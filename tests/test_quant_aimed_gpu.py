"""Attention over the 8-bit cache with queries aimed at the keys of every tile."""
import pytest
import torch

import _quant_aimed as A
from test_quant_gpu import KERNELS, Q, rows_set  # noqa: F401  (Q: a fixture)

pytestmark = pytest.mark.gpu

# heads, tokens, query rows of the chains, key lengths: every kernel and split; several chains, and more than travel in
# the arguments (heads x splits a multiple of eight, and not); more than 64 tiles (one register of scale bytes) in a range
# of the kernels for one and for two query halves per wave
MANY = tuple(1024 - 13 * b for b in range(20))
CASES = [(h, t, (r,), (t - 27,)) for h, t, r in KERNELS] + [
    (2, 4096, (70, 0, 300, 5), (4096, 4096, 2500, 65)),
    (2, 1024, (300,) * 12 + (0, 700) + (130,) * 6, MANY),
    (16, 1024, (300,) * 20, MANY),
    (16, 1024, (900,) * 20, MANY),
    (16, 5120, (10000,), (5101,)),
    (4, 16384, (16384,), (16380,)),
]
LONG_FEW = (1, 1 << 20, 16)  # more than 64 tiles in a wave's share of a range


def run(Q, codes, e, counts, keys, level, aims):
    """Rows of chain b, head h aimed at the pairs of aims[b] in turn, in as many calls as they take; all against float64."""
    batch, heads = codes.shape[:2]
    cache = Q.QuantCache(codes, e)
    kv = A.values(codes, e)
    kl = torch.tensor(keys, dtype=torch.int32, device="cuda")
    calls = max(-(-len(a) // n) for a, n in zip(aims, counts) if n)
    well = []
    for call in range(calls):
        q = torch.zeros((sum(counts), heads * 72), dtype=torch.bfloat16, device="cuda")
        aimed = {}
        r0 = 0
        for b, n in enumerate(counts):
            for h in range(heads if n else 0):
                aim = torch.tensor(aims[b], device="cuda")[(torch.arange(n, device="cuda") + call * n + 5 * h) % len(aims[b])]
                aimed[b, h] = aim
                q[r0:r0 + n, h * 72:(h + 1) * 72] = A.queries(kv[b, 0, h], aim, level)
            r0 += n
        o = Q.qcache_attention(cache, rows_set(counts), q, key_len=kl).double()
        r0 = 0
        for b, n in enumerate(counts):
            for h in range(heads if n else 0):
                c = slice(h * 72, (h + 1) * 72)
                v = kv[b, 1, h, :keys[b]]
                p = A.weights(q[r0:r0 + n, c], kv[b, 0, h], keys[b])
                both = p.gather(1, aimed[b, h])
                well.append((both > 0.2).all(1) & (both.sum(1) > 0.9))
                ref, mean_abs = p @ v, p @ v.abs()
                err = (o[r0:r0 + n, c] - ref).abs()
                assert (err <= A.bound(ref, mean_abs)).all(), (b, h, (err / A.bound(ref, mean_abs)).max().item())
            r0 += n
    # the inputs are what they are meant to be (in the tail of 10^7 products a third key comes near)
    assert torch.cat(well).double().mean() > 0.9


@pytest.mark.parametrize("spread", [True, False])
@pytest.mark.parametrize("level", [36.0, 75.0])  # 75: the sums leave their range and the kernels start again
@pytest.mark.parametrize("heads,tokens,counts,keys", CASES)
def test_attention_aimed_at_every_tile(Q, heads, tokens, counts, keys, level, spread):
    codes, e = A.cache(len(counts), heads, tokens, 7, spread, "cuda")
    run(Q, codes, e, counts, keys, level, [A.pairs(n) for n in keys])


def test_few_queries_aimed_at_a_long_cache(Q):
    """Tiles on both sides of each wave's reload of scale bytes, in every range."""
    heads, tokens, rows = LONG_FEW
    codes, e = A.cache(1, heads, tokens, 8, False, "cuda")
    tiles = tokens // 64
    near = [s * tiles // 16 + 8 * i + w for s in range(16) for w in range(8) for i in (63, 64)]
    run(Q, codes, e, (rows,), (tokens,), 36.0, [A.pairs(tokens, near)])
