"""8-bit operators on the GPU against plain forms in float64.

Quantised values and scale bytes are equal to the plain form's.  Products:
bfloat16 results are rounded once (2^-8 of the value) after sums whose
128-product parts keep 17 bits of their largest term (2^-16 of the sum of
magnitudes); float32 results have one rounding per instruction of 32 products
and at most 32 inside it, (K/32 + 32) 2^-24 of the sum of magnitudes.
Attention: the result is rounded once, 2^-8 |o|; the rounded probabilities,
2^-8 each, change the weighted mean by at most 2^-8 (mean |v| + |o|); float32
scores of up to 100 are off by 2^-17, which is 2^-12 of mean |v| with room."""
import numpy as np
import pytest
import torch

import _quant_ref as R

pytestmark = pytest.mark.gpu

NAN8 = 0x7F


@pytest.fixture(scope="module")
def Q():
    from paper_2608_29809_amd import quant
    return quant


def active(per_chain):
    from paper_2608_29809_amd.runtime import ActiveSet
    return ActiveSet.from_lists([np.asarray(p, np.int32) for p in per_chain])


def rows_set(counts):
    return active([np.zeros(c, np.int32) for c in counts])


def dev(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def np64(t):
    return t.detach().cpu().double().numpy()


def codes(t):
    """float8 tensor -> float64 values."""
    return t.detach().cpu().float().double().numpy()


def as_f8(values):
    """e4m3 values -> float8 tensor on the GPU (exact)."""
    return torch.from_numpy(np.ascontiguousarray(values)).float().to(torch.float8_e4m3fn).cuda()


def rnd(dtype, *shape, seed, std=1.0):
    x = np.random.default_rng(seed).standard_normal(shape) * std
    return torch.from_numpy(x).to(dtype).double().numpy()  # values that the type holds


# ------------------------------------------------------------------ quantisation

@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 16), (3, 128), (17, 48), (130, 1072), (723, 1152), (257, 144)])
def test_quantize(Q, rows, cols, dtype, tile):
    x = rnd(dtype, rows, cols, seed=rows + cols)
    x *= 10.0 ** np.random.default_rng(3).uniform(-6, 6, (rows, 1)).round()
    x = torch.from_numpy(x).to(dtype).double().numpy()
    m = Q.quantize(dev(x, dtype), tile)
    q, e = R.quantize(x, tile)
    np.testing.assert_array_equal(codes(m.data), q)
    np.testing.assert_array_equal(m.scales[:, :e.shape[1]].cpu().numpy(), e)


@pytest.mark.parametrize("tile", [1, 128])
def test_quantize_special_values(Q, tile):
    """Zeros, borders of the scale's choice, infinities, NaN, subnormals, the largest floats, one kind per row."""
    x = np.zeros((9, 128))
    x[1, 5], x[1, 6] = 448.0, 1.0                        # fits exactly
    x[2, 5], x[2, 6] = np.nextafter(np.float32(448.0), np.float32(500.0)), -1.0  # just does not
    x[3, :4] = [np.inf, -np.inf, np.nan, 3.0]
    x[4, :3] = [1e-40, -1e-42, 0.0]
    x[5, :3] = [3.4028234e38, -1.0, 1e30]
    x[6] = R.E4M3[:128] * 2.0 ** 20                      # every code (the last is NaN)
    x[7] = (np.concatenate([R.E4M3[:126] + R.E4M3[1:127], [896.0, 896.0]]) / 2)  # ties
    x[8] = -x[7]
    x = x.astype(np.float32).astype(np.float64)
    m = Q.quantize(dev(x), tile)
    q, e = R.quantize(x, tile)
    np.testing.assert_array_equal(codes(m.data), q)
    np.testing.assert_array_equal(m.scales[:, :e.shape[1]].cpu().numpy(), e)


def test_quantize_strides(Q):
    """Rows apart in the input and in the output; what lies between is left as it was."""
    x = rnd(torch.bfloat16, 37, 208, seed=1)
    src = torch.full((37, 256), 7.0, dtype=torch.bfloat16, device="cuda")
    src[:, :208] = dev(x, torch.bfloat16)
    data = torch.full((40, 240), 0x55, dtype=torch.uint8, device="cuda")
    scales = torch.full((2, 64), 0x55, dtype=torch.uint8, device="cuda")
    out = Q.QuantMatrix(data.view(torch.float8_e4m3fn)[:37, :208], scales, 1)
    Q.quantize(src[:, :208], 1, out)
    q, e = R.quantize(x, 1)
    np.testing.assert_array_equal(codes(out.data), q)
    np.testing.assert_array_equal(scales[:, :37].cpu().numpy(), e)
    assert (data[:, 208:] == 0x55).all() and (data[37:] == 0x55).all() and (scales[:, 37:] == 0x55).all()


# ------------------------------------------------------------------ product

def product(m, n, k, seed):
    a, ea = R.quantize(rnd(torch.float32, m, k, seed=seed) * 10.0 ** np.random.default_rng(seed).uniform(-2, 2, (m, 1)), 1)
    w, ew = R.quantize(rnd(torch.float32, n, k, seed=seed + 1, std=0.02), 128)
    return a, ea, w, ew


def matrix(Q, q, e, tile, gap=0):
    """A QuantMatrix whose rows are `gap` bytes apart, with NaN codes between and behind them."""
    rows, cols = q.shape
    buf = torch.full((rows + 3, cols + gap), NAN8, dtype=torch.uint8, device="cuda")
    buf[:rows, :cols] = as_f8(q).view(torch.uint8)
    s = torch.full((e.shape[0], e.shape[1] + -e.shape[1] % 16 + gap), 0xFF, dtype=torch.uint8, device="cuda")
    s[:, :e.shape[1]] = torch.from_numpy(e).to(torch.uint8).cuda()
    return Q.QuantMatrix(buf.view(torch.float8_e4m3fn)[:rows, :cols], s, tile)


def check_product(y, a, ea, w, ew, bias, gelu, f32):
    av, wv = R.dequantize(a, ea, 1), R.dequantize(w, ew, 128)
    ref, mag = av @ wv.T, np.abs(av) @ np.abs(wv).T
    if bias is not None:
        ref, mag = ref + bias, mag + np.abs(bias)
    tol = mag * ((a.shape[1] / 32 + 32) * 2.0 ** -24 if f32 else 2.0 ** -16)
    if gelu:
        # slope at most 1.13; the function itself to 2^-19 of its value
        ref, tol = R.gelu(ref), 1.13 * tol + 2.0 ** -19 * np.abs(ref)
    tol = tol + (2.0 ** -23 if f32 else 2.0 ** -8) * np.abs(ref) + 1e-38
    err = np.abs(np64(y) - ref)
    assert (err <= tol).all(), (err / tol).max()


SIZES = [(1, 4608, 1152), (1, 1, 16), (2, 7, 48), (5, 130, 128), (17, 16, 400), (128, 128, 256), (129, 144, 4608),
         (33, 1152, 1152), (219, 1000, 1072), (723, 300, 1152), (64, 4608, 144), (300, 257, 640),
         (600, 1150, 1040), (777, 2300, 272), (2999, 2050, 400), (200, 1152, 640), (199, 1101, 1008)]


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_qgemm(Q, m, n, k, f32):
    a, ea, w, ew = product(m, n, k, seed=m + n + k)
    bias = rnd(torch.float32, n, seed=9) if n % 2 == 0 else None
    gelu = m % 2 == 1
    y = Q.qgemm(matrix(Q, a, ea, 1), matrix(Q, w, ew, 128), None if bias is None else dev(bias), gelu=gelu,
                dtype=torch.float32 if f32 else torch.bfloat16)
    check_product(y, a, ea, w, ew, bias, gelu, f32)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("ldo", [56, 53])
@pytest.mark.parametrize("m", [3, 70])
def test_qgemm_strides(Q, m, ldo, f32):
    """Rows apart in all three matrices, NaN codes between the operands' rows; the result's gaps stay."""
    n, k = 50, 176
    a, ea, w, ew = product(m, n, k, seed=5)
    dt = torch.float32 if f32 else torch.bfloat16
    buf = torch.full((m + 2, ldo), 77.0, dtype=dt, device="cuda")
    Q.qgemm(matrix(Q, a, ea, 1, 32), matrix(Q, w, ew, 128, 48), out=buf[:m, :n])
    check_product(buf[:m, :n], a, ea, w, ew, None, False, f32)
    assert (buf[:, n:] == 77.0).all() and (buf[m:] == 77.0).all()


@pytest.mark.parametrize("m", [4, 150])
@pytest.mark.parametrize("f32", [False, True])
def test_qgemm_nan_stays_in_its_row_and_column(Q, m, f32):
    a, ea, w, ew = product(m, 40, 256, seed=6)
    a[2, 100], w[33, 7] = np.nan, np.nan
    y = np64(Q.qgemm(matrix(Q, a, ea, 1), matrix(Q, w, ew, 128), dtype=torch.float32 if f32 else torch.bfloat16))
    bad = np.zeros(y.shape, bool)
    bad[2], bad[:, 33] = True, True
    np.testing.assert_array_equal(np.isnan(y), bad)


# 256 x 256 tiles in one round of workgroups, 128 x 128, 256 x 256 in two rounds, 192 x 256 in one and two; some into gaps
LARGE = [(3001, 4360, 640, 4360), (4500, 6000, 384, 6016), (5700, 5000, 640, 5016), (2300, 4600, 896, 4600), (4100, 4600, 1152, 4616)]


@pytest.mark.parametrize("m,n,k,ldo", LARGE)
def test_qgemm_large(Q, m, n, k, ldo):
    a, ea, w, ew = product(m, n, k, seed=m)
    bias = rnd(torch.float32, n, seed=9)
    buf = torch.full((m + 2, ldo), 77.0, dtype=torch.bfloat16, device="cuda")
    A, W = matrix(Q, a, ea, 1, 32), matrix(Q, w, ew, 128, 16)  # (NaN codes between and behind the rows)
    for gelu in (False, True):
        Q.qgemm(A, W, dev(bias), gelu=gelu, out=buf[:m, :n])
        check_product(buf[:m, :n], a, ea, w, ew, bias, gelu, False)
    Q.qgemm(A, W, out=buf[:m, :n])
    check_product(buf[:m, :n], a, ea, w, ew, None, False, False)
    assert torch.equal(Q.qgemm(A, W), buf[:m, :n])  # (the same again)
    assert (buf[:, n:] == 77.0).all() and (buf[m:] == 77.0).all()


@pytest.mark.parametrize("m,n,k,_", [LARGE[0], LARGE[3]])
def test_qgemm_large_nan_stays_in_its_row_and_column(Q, m, n, k, _):
    a, ea, w, ew = product(m, n, k, seed=6)
    a[2, 100], a[m - 1, k - 1], w[33, 7], w[n - 1, 0] = np.nan, np.nan, np.nan, np.nan
    y = Q.qgemm(matrix(Q, a, ea, 1), matrix(Q, w, ew, 128))
    bad = torch.zeros(y.shape, dtype=torch.bool, device="cuda")
    bad[[2, m - 1]], bad[:, [33, n - 1]] = True, True
    assert torch.equal(torch.isnan(y), bad)


@pytest.mark.parametrize("tile,m,n,k", [(1, 5, 48, 300), (1, 130, 64, 1152), (128, 5, 200, 384)])
def test_qgemm_scale_views(Q, tile, m, n, k):
    """Scales that are the last columns of a wider tensor, whose memory ends with them."""
    k -= k % 16
    a, ea, w, ew = product(m, n, k, seed=11)
    A, W = matrix(Q, a, ea, 1), matrix(Q, w, ew, 128)
    X = A if tile == 1 else W
    wide = torch.full((X.scales.shape[0], 16 + X.scales.shape[1]), 0xFF, dtype=torch.uint8, device="cuda")
    wide[:, 16:] = X.scales
    X = Q.QuantMatrix(X.data, wide[:, 16:], tile)
    y = Q.qgemm(X, W) if tile == 1 else Q.qgemm(A, X)
    check_product(y, a, ea, w, ew, None, False, False)


def test_qgemm_scales_far_apart(Q):
    """Blocks of one sum whose scales differ by 2^60, the large ones cancelling."""
    a, ea, w, ew = product(40, 48, 384, seed=7)
    a[:, 256:], w[:, 256:] = a[:, 128:256], -w[:, 128:256]
    ea[1] += 60
    ea[2], ew[2] = ea[1], ew[1]
    for f32 in (False, True):
        y = Q.qgemm(matrix(Q, a, ea, 1), matrix(Q, w, ew, 128), dtype=torch.float32 if f32 else torch.bfloat16)
        check_product(y, a, ea, w, ew, None, False, f32)


# ------------------------------------------------------------------ cache

def random_cache(Q, batch, heads, blocks, seed, gap=0):
    """A cache with chains `gap` bytes apart, and its values and scale bytes."""
    rng = np.random.default_rng(seed)
    e = rng.integers(118, 131, (batch, heads, blocks, 2))
    v = R.round_e4m3(rng.standard_normal((batch, heads, blocks, 2, 64, 72)) * 100.0)
    n, ns = heads * blocks * 2 * 64 * 72, heads * blocks * 2
    data = torch.full((batch, n + gap), 0x5A, dtype=torch.uint8, device="cuda")
    scales = torch.full((batch, ns + gap), 0x5A, dtype=torch.uint8, device="cuda")
    data[:, :n] = as_f8(v).view(torch.uint8).view(batch, n)
    scales[:, :ns] = torch.from_numpy(e.reshape(batch, ns)).to(torch.uint8).cuda()
    cache = Q.QuantCache(data[:, :n].view(torch.float8_e4m3fn).unflatten(1, (heads, blocks, 2, 64, 72)),
                         scales[:, :ns].unflatten(1, (heads, blocks, 2)))
    return cache, v, e, data, scales


CHAINS = [
    [[5]],
    [[0, 63, 64, 127, 128]],
    [list(range(192))],
    [[], list(range(60, 70)), [191]],
    [list(range(64, 128)), [1, 2, 3, 100, 190, 191]],
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("per_chain", CHAINS)
def test_store(Q, per_chain, dtype):
    batch, heads, rows = len(per_chain), 3, sum(map(len, per_chain))
    cache, v, e, data, scales = random_cache(Q, batch, heads, 3, seed=rows, gap=48)
    std = np.where(np.arange(rows) % 3 == 0, 30.0, 0.5)[:, None]  # some rows raise their block's scale
    kn, vn = (rnd(torch.float32, rows, heads * 72, seed=s) * std for s in (1, 2))
    both = torch.zeros((rows, 2 * heads * 72 + 8), dtype=dtype, device="cuda")
    both[:, :heads * 72], both[:, heads * 72:2 * heads * 72] = dev(kn, dtype), dev(vn, dtype)
    kt, vt = both[:, :heads * 72], both[:, heads * 72:2 * heads * 72]
    Q.qcache_store(cache, active(per_chain), kt, vt)
    R.store(v, e, per_chain, np64(kt), np64(vt))
    np.testing.assert_array_equal(codes(cache.data), v)
    np.testing.assert_array_equal(cache.scales.cpu().numpy(), e)
    assert (data[:, -48:] == 0x5A).all() and (scales[:, -48:] == 0x5A).all()


def test_store_into_zeroed_cache_and_special_values(Q):
    cache = Q.QuantCache.alloc(1, 2, 128)
    k = rnd(torch.float32, 2, 144, seed=1)
    k[0, 3], k[1, 80] = np.inf, np.nan
    v = np.zeros((2, 144))
    Q.qcache_store(cache, active([[7, 70]]), dev(k), dev(v))
    val, e = np.zeros((1, 2, 2, 2, 64, 72)), np.zeros((1, 2, 2, 2), np.int64)
    R.store(val, e, [[7, 70]], np64(dev(k)), v)
    np.testing.assert_array_equal(codes(cache.data), val)
    np.testing.assert_array_equal(cache.scales.cpu().numpy(), e)


def test_store_again_changes_nothing(Q):
    per = [[3, 9, 64, 100]]
    cache, *_ = random_cache(Q, 1, 2, 2, seed=4)
    k, v = dev(rnd(torch.float32, 4, 144, seed=1, std=40.0)), dev(rnd(torch.float32, 4, 144, seed=2))
    Q.qcache_store(cache, active(per), k, v)
    once = cache.data.view(torch.uint8).clone(), cache.scales.clone()
    Q.qcache_store(cache, active(per), k, v)
    assert torch.equal(cache.data.view(torch.uint8), once[0]) and torch.equal(cache.scales, once[1])


def test_store_long_list(Q):
    """Searches of a list longer than one round of probes, by 20 chains (more than travel in the arguments)."""
    rng = np.random.default_rng(0)
    per = [np.sort(rng.choice(8192, int(n), replace=False)).astype(np.int32) for n in rng.integers(0, 300, 19)]
    per.append(np.sort(rng.choice(8192, 5000, replace=False)).astype(np.int32))
    rows = sum(map(len, per))
    cache, v, e, *_ = random_cache(Q, 20, 1, 128, seed=2)
    k, vv = dev(rnd(torch.float32, rows, 72, seed=3)), dev(rnd(torch.float32, rows, 72, seed=4))
    Q.qcache_store(cache, active(per), k, vv)
    R.store(v, e, per, np64(k), np64(vv))
    np.testing.assert_array_equal(codes(cache.data), v)
    np.testing.assert_array_equal(cache.scales.cpu().numpy(), e)


# ------------------------------------------------------------------ attention

def check_attention(o, v, e, counts, key_len, q, scale=72 ** -0.5):
    offsets = np.concatenate([[0], np.cumsum(counts)])
    ref, mean_abs = R.attention(v, e, offsets, key_len, q, scale)
    tol = 2.0 ** -8 * (2 * np.abs(ref) + mean_abs) + 2.0 ** -12 * mean_abs
    err = np.abs(np64(o) - ref)
    assert np.isfinite(err).all()
    assert (err <= tol).all(), (err / np.maximum(tol, 1e-300)).max()


def attention_case(Q, heads, tokens, counts, key_len=None, seed=0, std=0.3, gap=0):
    cache, v, e, data, scales = random_cache(Q, len(counts), heads, tokens // 64, seed, gap)
    e[..., 0] = 122  # keys of standard deviation 3
    cache.scales[..., 0] = 122
    q = rnd(torch.bfloat16, sum(counts), heads * 72, seed=seed + 1, std=std)
    kl = None if key_len is None else torch.tensor(key_len, dtype=torch.int32, device="cuda")
    o = Q.qcache_attention(cache, rows_set(counts), dev(q, torch.bfloat16), key_len=kl)
    check_attention(o, v, e, counts, [tokens] * len(counts) if key_len is None else np.clip(key_len, 0, tokens), q)


@pytest.mark.parametrize("tokens", [64, 128, 192, 1024])
@pytest.mark.parametrize("rows", [1, 31, 33, 129, 300])
def test_attention(Q, rows, tokens):
    attention_case(Q, 2, tokens, [rows], seed=rows + tokens)


@pytest.mark.parametrize("key_len", [0, 1, 31, 32, 33, 63, 64, 65, 191, 192, 1000, -5])
def test_attention_key_lengths(Q, key_len):
    attention_case(Q, 2, 192, [40], [key_len], seed=3)


def test_attention_ragged_chains(Q):
    attention_case(Q, 3, 512, [0, 1, 200, 64, 3, 129], [512, 77, 300, 0, 512, 1], seed=5, gap=64)


def test_attention_many_chains(Q):
    """More chains than travel in the arguments."""
    rng = np.random.default_rng(2)
    attention_case(Q, 1, 128, list(rng.integers(0, 9, 25)), list(rng.integers(0, 129, 25)), seed=6)


def test_attention_long_cache_one_query(Q):
    attention_case(Q, 2, 16384, [1], [16201], seed=7)


def test_attention_many_rows(Q):
    attention_case(Q, 4, 640, [2100, 1300], [640, 600], seed=8)


@pytest.mark.parametrize("rows", [1, 200])
@pytest.mark.parametrize("std", [20.0, 60.0])
def test_attention_large_logits(Q, rows, std):
    """Logits of hundreds to a thousand: one key takes nearly all weight.  (Scores off by 2^-23 of their size move a
    probability by up to 2^-13 here, inside the tolerance's 2^-12.)"""
    attention_case(Q, 1, 512, [rows], seed=9, std=std)


# heads, tokens, rows: few queries without and with split keys, one and two query halves per wave likewise
KERNELS = [(1, 256, 1), (1, 256, 70), (2, 4096, 5), (4, 192, 5000), (2, 4096, 1000), (9, 256, 7200), (16, 1856, 1300)]


@pytest.mark.parametrize("heads,tokens,rows", KERNELS)
def test_attention_kernels(Q, heads, tokens, rows):
    attention_case(Q, heads, tokens, [rows], [tokens - 27], seed=rows)


@pytest.mark.parametrize("heads,tokens,rows", KERNELS)
@pytest.mark.parametrize("level", [-1.0, 1.0])
def test_attention_logits_far_from_zero(Q, heads, tokens, rows, level):
    """Every logit of a query near -450, or +450: nothing may under- or overflow."""
    cache, v, e, *_ = random_cache(Q, 1, heads, tokens // 64, seed=1)
    v[:, :, :, 0, :, 0], e[..., 0] = 128.0, 120
    cache.data[:, :, :, 0, :, 0] = torch.full((1, heads, tokens // 64, 64), 128.0, device="cuda").to(torch.float8_e4m3fn)
    cache.scales[..., 0] = 120
    q = rnd(torch.bfloat16, rows, heads * 72, seed=2, std=0.5)
    q[:, ::72] = 3840.0 * level
    o = Q.qcache_attention(cache, rows_set([rows]), dev(q, torch.bfloat16))
    check_attention(o, v, e, [rows], [tokens], q)


@pytest.mark.parametrize("heads,tokens,rows", KERNELS)
def test_attention_large_values(Q, heads, tokens, rows):
    """Values near the largest float beside large weights: only their weighted mean is finite."""
    cache, v, e, *_ = random_cache(Q, 1, heads, tokens // 64, seed=1)
    e[..., 0], e[..., 1] = 122, 240  # values up to 448 * 2^113 = 4.6e36
    cache.scales.copy_(torch.from_numpy(e).to(torch.uint8))
    q = rnd(torch.bfloat16, rows, heads * 72, seed=2, std=0.3)
    o = Q.qcache_attention(cache, rows_set([rows]), dev(q, torch.bfloat16))
    check_attention(o, v, e, [rows], [tokens], q)


@pytest.mark.parametrize("heads,rows", [(2, 1), (2, 33), (2, 150), (4, 5000), (9, 7200)])
@pytest.mark.parametrize("key_len", [0, 1, 70, 128, 200])
def test_attention_ignores_what_lies_behind_the_keys(Q, heads, rows, key_len):
    """NaN codes and scale bytes of 255 behind key_len."""
    cache, v, e, *_ = random_cache(Q, 1, heads, 4, seed=key_len)
    e[..., 0] = 122
    cache.scales[..., 0] = 122
    raw = cache.data.view(torch.uint8)
    for blk in range(4):
        n = max(0, min(64, key_len - 64 * blk))
        raw[:, :, blk, :, n:] = NAN8
        v[:, :, blk, :, n:] = 0.0
        if n == 0:
            cache.scales[:, :, blk] = 255
    q = rnd(torch.bfloat16, rows, heads * 72, seed=3, std=0.3)
    o = Q.qcache_attention(cache, rows_set([rows]), dev(q, torch.bfloat16),
                           key_len=torch.tensor([key_len], dtype=torch.int32, device="cuda"))
    check_attention(o, v, e, [rows], [key_len], q)


@pytest.mark.parametrize("counts", [[4, 6], [9000, 2300]])
def test_attention_nan_stays_in_its_chain_head_and_row(Q, counts):
    cache, v, e, *_ = random_cache(Q, 2, 2, 2, seed=1)
    rows, last = sum(counts), counts[0] + 3
    q = rnd(torch.bfloat16, rows, 144, seed=2, std=0.05)
    q[last, 3] = np.nan                    # a row of chain 1, head 0
    cache.data[0, 1, 1, 1, 5, 8] = float("nan")  # chain 0, head 1: dim 8 of every row
    o = np64(Q.qcache_attention(cache, rows_set(counts), dev(q, torch.bfloat16)))
    bad = np.zeros((rows, 144), bool)
    bad[last, :72], bad[:counts[0], 72 + 8] = True, True
    np.testing.assert_array_equal(np.isnan(o), bad)


@pytest.mark.parametrize("scale", [0.0, 1.0, -0.1])
def test_attention_scale_and_strides(Q, scale):
    """Other softmax scales; query and result rows apart, gaps and later rows left as they were."""
    cache, v, e, *_ = random_cache(Q, 1, 1, 3, seed=2)
    e[..., 0] = 120
    cache.scales[..., 0] = 120
    q = rnd(torch.bfloat16, 50, 72, seed=3, std=0.2)
    qb = torch.full((50, 96), float("nan"), dtype=torch.bfloat16, device="cuda")
    qb[:, :72] = dev(q, torch.bfloat16)
    ob = torch.full((53, 88), 5.0, dtype=torch.bfloat16, device="cuda")
    Q.qcache_attention(cache, rows_set([50]), qb[:, :72], scale=scale, out=ob[:50, :72])
    check_attention(ob[:50, :72], v, e, [50], [192], q, scale)
    assert (ob[:, 72:] == 5.0).all() and (ob[50:] == 5.0).all()


# ------------------------------------------------------------------ together

def pipeline(Q, x, w, bias, cache, act):
    qkv = Q.qgemm(Q.quantize(x), w, bias)
    c = cache.heads * 72
    Q.qcache_store(cache, act, qkv[:, c:2 * c], qkv[:, 2 * c:])
    return qkv, Q.qcache_attention(cache, act, qkv[:, :c])


def pipeline_inputs(Q, seed):
    heads, c = 16, 1152
    cache, v, e, *_ = random_cache(Q, 2, heads, 4, seed)
    e -= 7  # values of standard deviation near 1
    cache.scales.copy_(torch.from_numpy(e).to(torch.uint8))
    per = [sorted(np.random.default_rng(seed).choice(256, 60, replace=False).tolist()), list(range(100, 117))]
    x = rnd(torch.bfloat16, 77, c, seed=seed + 1)
    w, bias = rnd(torch.bfloat16, 3 * c, c, seed=seed + 2, std=0.03), rnd(torch.float32, 3 * c, seed=seed + 3, std=0.1)
    return cache, v, e, per, x, w, bias


def test_operators_together(Q):
    """Projection, merge and attention of a region: each against the plain form on what the one before gave."""
    cache, v, e, per, x, w, bias = pipeline_inputs(Q, 11)
    wq = Q.quantize(dev(w, torch.bfloat16), 128)
    qkv, o = pipeline(Q, dev(x, torch.bfloat16), wq, dev(bias), cache, active(per))
    check_product(qkv, *R.quantize(x, 1), *R.quantize(w, 128), bias, False, False)
    y = np64(qkv)
    R.store(v, e, per, y[:, 1152:2304], y[:, 2304:])
    np.testing.assert_array_equal(codes(cache.data), v)
    np.testing.assert_array_equal(cache.scales.cpu().numpy(), e)
    check_attention(o, v, e, [60, 17], [256, 256], y[:, :1152])


def test_captured_and_replayed(Q):
    """The same run captured into a graph and replayed on new inputs, with eager work between the replays."""
    cache, v, e, per, x, w, bias = pipeline_inputs(Q, 12)
    wq, bt, act = Q.quantize(dev(w, torch.bfloat16), 128), dev(bias), active(per)
    first = cache.data.view(torch.uint8).clone(), cache.scales.clone()
    xs = [dev(rnd(torch.bfloat16, 77, 1152, seed=s), torch.bfloat16) for s in (1, 2, 3)]
    x_in = xs[0].clone()

    def reset():
        cache.data.view(torch.uint8).copy_(first[0])
        cache.scales.copy_(first[1])

    pipeline(Q, x_in, wq, bt, cache, act)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qkv, o = pipeline(Q, x_in, wq, bt, cache, act)
    for x_new in xs:
        reset()
        want = [t.clone() for t in pipeline(Q, x_new, wq, bt, cache, act)]
        state = cache.data.view(torch.uint8).clone()
        reset()
        x_in.copy_(x_new)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(qkv, want[0]) and torch.equal(o, want[1])
        assert torch.equal(cache.data.view(torch.uint8), state)


def test_two_streams_at_once(Q):
    """Runs that overlap on two streams give what they give alone."""
    sets = [pipeline_inputs(Q, s) for s in (13, 14)]
    args = [(dev(x, torch.bfloat16), Q.quantize(dev(w, torch.bfloat16), 128), dev(b), c, active(per))
            for c, _, _, per, x, w, b in sets]
    want = []
    for a in args:
        keep = a[3].data.view(torch.uint8).clone(), a[3].scales.clone()
        want.append([t.clone() for t in pipeline(Q, *a)])
        a[3].data.view(torch.uint8).copy_(keep[0])
        a[3].scales.copy_(keep[1])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in args]
    got = []
    for s, a in zip(streams, args):
        with torch.cuda.stream(s):
            got.append(pipeline(Q, *a))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


# ------------------------------------------------------------------ offsets beyond 32 bits

def test_quantize_beyond_32_bits(Q):
    """4.3e9 values: the last row, and the block before the last of a tile."""
    rows, cols = 1 << 18, 16384
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    last = rnd(torch.bfloat16, 1, cols, seed=3)
    x[-1] = dev(last, torch.bfloat16)[0]
    for tile in (1, 128):
        m = Q.quantize(x, tile)
        block = np.zeros((128, cols))
        block[-1] = last[0]
        q, e = R.quantize(block, tile)
        np.testing.assert_array_equal(codes(m.data[-128:]), q)
        used = rows // tile
        np.testing.assert_array_equal(m.scales[:, used - 128 // tile:used].cpu().numpy(), e)
        assert (m.data[:-1].view(torch.int64) == 0).all()
        del m


def test_qgemm_beyond_32_bits(Q):
    """2.4e9 results, of two steps of K per tile."""
    m, n, k = 40000, 60001 // 8 * 8, 256
    a, ea, w, ew = product(m, n, k, seed=21)
    y = Q.qgemm(matrix(Q, a, ea, 1), matrix(Q, w, ew, 128))
    rows = np.concatenate([[0, 255, 256, m - 1], np.random.default_rng(1).integers(0, m, 20)])
    check_product(y[torch.from_numpy(rows).cuda()], a[rows], ea[:, rows], w, ew, None, False, False)
    assert torch.isfinite(y.view(-1)[::7].float()).all()


def test_cache_beyond_32_bits(Q):
    """A cache of 4.8 GB, zeros but for its last block: its keys' weight is 1 each, the last ones' about e^14."""
    heads, tokens = 2, 1 << 24
    cache = Q.QuantCache.alloc(1, heads, tokens)
    per = [list(range(tokens - 64, tokens))]
    q = rnd(torch.bfloat16, 1, heads * 72, seed=1)
    unit = q.reshape(heads, 72) / (q.reshape(heads, 72) ** 2).sum(1, keepdims=True)
    k = np.repeat((unit * 14.0 * 72 ** 0.5).reshape(1, -1), 64, 0) * np.linspace(0.9, 1.0, 64)[:, None]
    v = rnd(torch.bfloat16, 64, heads * 72, seed=2)
    Q.qcache_store(cache, active(per), dev(k, torch.bfloat16), dev(v, torch.bfloat16))
    o = np64(Q.qcache_attention(cache, rows_set([1]), dev(q, torch.bfloat16)))
    assert (cache.data[0, :, :-1, :, 0].view(torch.uint8) == 0).all()
    K, V = (codes(cache.data[0, :, -1, i]) * 2.0 ** (cache.scales[0, :, -1, i].cpu().numpy().astype(float) - 127)[:, None, None]
            for i in (0, 1))
    p = np.exp(72 ** -0.5 * np.einsum("htd,hd->ht", K, q.reshape(heads, 72)))
    den = p.sum(1) + (tokens - 64)
    ref, mean_abs = (np.einsum("ht,htd->hd", p, x) / den[:, None] for x in (V, np.abs(V)))
    # the probabilities and the result rounded, 2^-9 each; sums of 4096 steps per wave, 2^-12
    tol = 2.0 ** -8 * (2 * np.abs(ref) + mean_abs) + 2.0 ** -12 * mean_abs
    assert (np.abs(o.reshape(heads, 72) - ref) <= tol).all()


def test_empty_calls(Q):
    m = Q.quantize(torch.empty((0, 32), dtype=torch.bfloat16, device="cuda"))
    w = Q.quantize(torch.ones((5, 32), device="cuda"), 128)
    assert tuple(Q.qgemm(m, w).shape) == (0, 5)
    cache = Q.QuantCache.alloc(2, 1, 64)
    none = rows_set([0, 0])
    empty = torch.empty((0, 72), dtype=torch.bfloat16, device="cuda")
    Q.qcache_store(cache, none, empty, empty)
    assert tuple(Q.qcache_attention(cache, none, empty).shape) == (0, 72)
    assert (cache.data.view(torch.uint8) == 0).all()
