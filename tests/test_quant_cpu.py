"""Host-side checks of the 8-bit operators: refusals before any launch (a call
that would pass is made only where there is no GPU), scratch sizes, and the
plain forms that the GPU tests compare with."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import _quant_ref as R
from paper_2608_29809_amd import abi, quant

NO_GPU = torch.cuda.device_count() == 0
FAKE = 1 << 20  # aligned, never dereferenced


def qmat(**over):
    d = dict(data=FAKE, scales=FAKE, ld=256, rows=40, cols=256, scale_ld=48, block_rows=1)
    d.update(over)
    return abi.rc_qmat(*[d[f] for f, _ in abi.rc_qmat._fields_])


def qcache(**over):
    d = dict(data=FAKE, scales=FAKE, chain_stride=4 * 128 * 144, scale_stride=16, batch=2, heads=4, tokens=128)
    d.update(over)
    return abi.rc_qcache(*[d[f] for f, _ in abi.rc_qcache._fields_])


def aset(offs, idx=FAKE, offsets=FAKE, batch=None):
    h = (C.c_int32 * len(offs))(*offs)
    a = abi.rc_active_set(idx, offsets, C.cast(h, C.POINTER(C.c_int32)), len(offs) - 1 if batch is None else batch)
    a.keep = h
    return a


@pytest.mark.parametrize("over,status", [
    (dict(data=None), -1), (dict(scales=None), -1), (dict(data=FAKE + 8), -3), (dict(scales=FAKE + 1), -3),
    (dict(cols=250), -8), (dict(cols=0), -2), (dict(cols=1 << 17, ld=1 << 17), -8), (dict(ld=240), -2),
    (dict(ld=264), -3), (dict(rows=-1), -2), (dict(scale_ld=32), -2), (dict(scale_ld=44), -3),
    (dict(block_rows=64), -8), (dict(rows=1 << 30, scale_ld=1 << 30), -2),
])
def test_matrix_refusals(over, status):
    bad, a, w = qmat(**over), qmat(), qmat(block_rows=128)
    assert abi.LIB.rc_quantize(FAKE, abi.RC_BF16, 256, C.byref(bad), None) == status
    assert abi.rc_last_error()
    if over.get("block_rows", 1) == 1:
        assert abi.LIB.rc_qgemm(C.byref(bad), C.byref(w), None, 0, FAKE, 1, 40, None) in (status, -2)
    if "scale_ld" not in over:
        over = dict(block_rows=128, **{k: v for k, v in over.items() if k != "block_rows"})
        assert abi.LIB.rc_qgemm(C.byref(a), C.byref(qmat(**over)), None, 0, FAKE, 1, 1 << 31, None) < 0


def test_quantize_refusals():
    f, m = abi.LIB.rc_quantize, qmat()
    assert f(FAKE, 2, 256, C.byref(m), None) == -1
    assert f(FAKE, abi.RC_BF16, 248, C.byref(m), None) == -2
    assert f(FAKE, abi.RC_BF16, 260, C.byref(m), None) == -3
    assert f(None, abi.RC_BF16, 256, C.byref(m), None) == -1
    assert f(FAKE + 8, abi.RC_BF16, 256, C.byref(m), None) == -3
    assert f(FAKE, abi.RC_BF16, 256, None, None) == -1
    assert f(None, abi.RC_F32, 256, C.byref(qmat(rows=0, data=None, scales=None)), None) == 0  # nothing to do
    if NO_GPU:
        assert f(FAKE, abi.RC_F32, 260, C.byref(m), None) == -6


def test_qgemm_refusals():
    def call(a=None, w=None, bias=FAKE, gelu=0, out=FAKE, dt=1, ldo=40):
        a, w = a or qmat(), w or qmat(block_rows=128)
        return abi.LIB.rc_qgemm(C.byref(a), C.byref(w), bias, gelu, out, dt, ldo, None)

    assert call(a=qmat(block_rows=128)) == -8
    assert call(w=qmat()) == -8
    assert call(w=qmat(block_rows=128, cols=128)) == -2
    assert call(w=qmat(block_rows=128, rows=0)) == -2
    assert call(gelu=2) == -1
    assert call(dt=2) == -1
    assert call(ldo=39) == -2
    assert call(out=None) == -1
    assert call(out=FAKE + 4) == -3
    assert call(bias=FAKE + 2) == -3
    assert call(a=qmat(rows=1 << 24, scale_ld=1 << 24), w=qmat(block_rows=128, rows=1 << 20, scale_ld=1 << 13),
                ldo=1 << 20) == -2
    assert call(a=qmat(rows=0)) == 0
    if NO_GPU:
        assert call() == -6


@pytest.mark.parametrize("over,status", [
    (dict(data=None), -1), (dict(scales=None), -1), (dict(data=FAKE + 4), -3), (dict(scales=FAKE + 2), -3),
    (dict(batch=0), -2), (dict(heads=0), -2), (dict(heads=2000), -2), (dict(tokens=100), -8), (dict(tokens=0), -8),
    (dict(tokens=1 << 25, chain_stride=1 << 40, scale_stride=1 << 30), -8), (dict(chain_stride=4 * 128 * 144 - 16), -2),
    (dict(scale_stride=15), -2), (dict(chain_stride=4 * 128 * 144 + 8), -3),
])
def test_cache_refusals(over, status):
    c, a = qcache(**over), aset([0, 5, 9])
    assert abi.LIB.rc_qcache_store(C.byref(c), C.byref(a), FAKE, FAKE, 0, 288, None) == status
    assert abi.LIB.rc_qcache_attention(C.byref(c), C.byref(a), None, FAKE, 288, 0.1, FAKE, 288, FAKE, 1 << 40, None) == status
    assert abi.rc_qcache_attention_scratch_bytes(C.byref(c), C.byref(a)) == 0


def test_store_refusals():
    def call(a, k=FAKE, v=FAKE, dt=0, ld=288):
        return abi.LIB.rc_qcache_store(C.byref(qcache()), C.byref(a), k, v, dt, ld, None)

    good = aset([0, 5, 9])
    assert call(aset([0, 5])) == -2                    # batch
    assert call(aset([0, 5, 3])) == -4                 # not monotone
    assert call(aset([1, 5, 9])) == -4
    assert call(aset([0, 129, 129])) == -4             # more rows than tokens
    assert call(aset([0, 5, 9], offsets=None)) == -1
    assert call(aset([0, 5, 9], idx=None)) == -1
    assert call(good, k=None) == -1 and call(good, v=None) == -1
    assert call(good, k=FAKE + 8) == -3
    assert call(good, dt=3) == -1
    assert call(good, ld=284) == -2
    assert call(good, ld=290) == -3
    assert call(good, dt=1, ld=292) == -3
    assert call(aset([0, 0, 0], idx=None, offsets=None), k=None, v=None) == 0
    assert abi.LIB.rc_qcache_store(None, C.byref(good), FAKE, FAKE, 0, 288, None) == -1
    assert abi.LIB.rc_qcache_store(C.byref(qcache()), None, FAKE, FAKE, 0, 288, None) == -1
    if NO_GPU:
        assert call(good) == -6


def test_attention_refusals():
    def call(a, key_len=None, q=FAKE, ldq=288, scale=0.1, out=FAKE, ldo=288, scratch=FAKE, nbytes=1 << 40, c=None):
        return abi.LIB.rc_qcache_attention(C.byref(c or qcache()), C.byref(a), key_len, q, ldq, scale, out, ldo, scratch,
                                           nbytes, None)

    good = aset([0, 5, 9], idx=None)
    assert call(aset([0, 5])) == -2
    assert call(aset([0, 5, 3])) == -4
    assert call(aset([0, 5, 1 << 25])) == -4
    assert call(aset([0, 1 << 24, 1 << 25])) == -2      # in all
    assert call(good, ldq=280) == -2 and call(good, ldo=280) == -2
    assert call(good, ldq=290) == -3 and call(good, ldo=292) == -3
    assert call(good, scale=math.inf) == -1 and call(good, scale=math.nan) == -1
    assert call(good, q=None) == -1 and call(good, out=None) == -1
    assert call(good, q=FAKE + 8) == -3 and call(good, key_len=FAKE + 2) == -3
    need = abi.rc_qcache_attention_scratch_bytes(C.byref(qcache()), C.byref(good))
    if need:
        assert call(good, nbytes=need - 1) == -5
        assert call(good, scratch=None) == -1
        assert call(good, scratch=FAKE + 4) == -3
    big, a1 = qcache(batch=1, tokens=16384), aset([0, 1], idx=None)
    assert abi.rc_qcache_attention_scratch_bytes(C.byref(big), C.byref(a1)) > 0  # one query: the keys are split
    assert call(a1, c=big, nbytes=0) == -5
    assert call(aset([0, 0, 0], idx=None, offsets=None), q=None, out=None, scratch=None, nbytes=0) == 0
    if NO_GPU:
        assert call(good) == -6


# ------------------------------------------------------------------ steps on an 8-bit pool

def make_ctx(dtype=abi.RC_BF16, layers=2, grid=(32, 32)):
    L = (abi.rc_layer_weights * layers)()
    for i in range(layers):
        for f in abi.LAYER_FIELDS:
            setattr(L[i], f, FAKE)
    w = abi.rc_weights()
    w.layers = C.cast(L, C.POINTER(abi.rc_layer_weights))
    for f in abi.GLOBAL_FIELDS:
        setattr(w, f, FAKE)
    cfg = abi.rc_model_config(1152, 16, 72, 4608, layers, 120, 4096, *grid, 4, 2, 8, dtype, 0, 1e-6)
    ctx = C.c_void_p()
    assert abi.LIB.rc_create(C.byref(cfg), C.byref(w), C.byref(ctx)) == 0
    return ctx, L


def step_io(**over):
    d = dict(input=FAKE, t_vec=None, timestep=500, timestep_next=450, text_kv=FAKE, delta_cols_host=None,
             n_delta=0, maps=None, latent_out=FAKE, text_valid=None, guided=0, guidance_scale=0.0)
    d.update(over)
    return abi.rc_step_io(*[d[f] for f, _ in abi.rc_step_io._fields_])


def test_pool_sizes_and_offsets():
    ctx, keep = make_ctx()
    N, C_, L = 1024, 1152, 2
    scales = 16 * (N // 64) * 2
    slot = 2 * N * C_ + scales + 2 * N * C_
    assert scales % 256 == 0 and abi.rc_quant_cache_bytes(ctx, 3, 5) == 3 * 5 * L * slot + 3 * 6 * 4 * 64 * 64 * 4
    view = abi.rc_cache_view(FAKE, abi.rc_quant_cache_bytes(ctx, 3, 5), 3, 5)
    d, sc, h = C.c_size_t(), C.c_size_t(), C.c_size_t()
    abi.rc_quant_cache_offsets(ctx, C.byref(view), 2, 4, 1, C.byref(d), C.byref(sc), C.byref(h))
    base = ((2 * 5 + 4) * L + 1) * slot
    assert (d.value, sc.value, h.value) == (base, base + 2 * N * C_, base + 2 * N * C_ + scales)
    abi.rc_quant_cache_latent_offset(ctx, C.byref(view), 1, 5, C.byref(d))
    assert d.value == 3 * 5 * L * slot + (6 + 5) * 4 * 64 * 64 * 4
    with pytest.raises(abi.RcError):
        abi.rc_quant_cache_offsets(ctx, C.byref(view), 3, 0, 0, C.byref(d), None, None)
    assert abi.rc_quant_workspace_bytes(ctx, 500, 1) > abi.rc_workspace_bytes(ctx, 500, 1)
    assert abi.rc_quant_cache_bytes(ctx, 0, 5) == 0 and abi.rc_quant_workspace_bytes(ctx, 5, 0) == 0
    f32, keep2 = make_ctx(abi.RC_F32)
    assert abi.rc_quant_cache_bytes(f32, 1, 1) == 0 and abi.rc_quant_workspace_bytes(f32, 1, 1) == 0
    abi.rc_destroy(ctx)
    abi.rc_destroy(f32)


def test_quant_step_refusals():
    ctx, keep = make_ctx()
    nb, ws = abi.rc_quant_cache_bytes(ctx, 2, 4), abi.rc_quant_workspace_bytes(ctx, 2048, 2)
    view, a, io = abi.rc_cache_view(FAKE, nb, 2, 4), aset([0, 10, 20]), step_io()
    build, step = abi.LIB.rc_build_cache_quant, abi.LIB.rc_reuse_step_quant
    fuse = abi.RC_FUSE_UPDATE
    assert build(None, C.byref(view), 0, C.byref(io), FAKE, ws, None) == -1
    assert build(ctx, C.byref(view), 4, C.byref(io), FAKE, ws, None) == -2
    assert build(ctx, C.byref(abi.rc_cache_view(FAKE, nb - 1, 2, 4)), 0, C.byref(io), FAKE, ws, None) == -5
    assert build(ctx, C.byref(view), 0, C.byref(step_io(timestep=1000)), FAKE, ws, None) == -1
    assert step(ctx, C.byref(view), 1, C.byref(a), C.byref(io), 0, FAKE, ws, None) == -8       # not in place
    assert step(ctx, C.byref(view), 1, C.byref(a), C.byref(io), fuse | 4, FAKE, ws, None) == -1
    assert step(ctx, C.byref(view), 1, C.byref(aset([0, 10, 5])), C.byref(io), fuse, FAKE, ws, None) == -4
    assert step(ctx, C.byref(view), 1, C.byref(aset([0, 2000, 2001])), C.byref(io), fuse, FAKE, ws, None) == -4
    assert step(ctx, C.byref(view), 1, C.byref(a), C.byref(io), fuse | abi.RC_VALIDATE, FAKE, 8, None) == -1
    f32, keep2 = make_ctx(abi.RC_F32)
    assert build(f32, C.byref(view), 0, C.byref(io), FAKE, ws, None) == -8
    assert step(f32, C.byref(view), 1, C.byref(a), C.byref(io), fuse, FAKE, ws, None) == -8
    if NO_GPU:
        assert build(ctx, C.byref(view), 0, C.byref(io), FAKE, ws, None) == -6
        assert step(ctx, C.byref(view), 1, C.byref(a), C.byref(io), fuse, FAKE, ws, None) == -6
    abi.rc_destroy(ctx)
    abi.rc_destroy(f32)


def test_quant_weight_refusals():
    ctx, keep = make_ctx()

    def layers(**over):
        q = (abi.rc_quant_layer * 2)()
        for i in range(2):
            q[i].qkv_w = qmat(rows=3456, cols=1152, ld=1152, scale_ld=32, block_rows=128)
            q[i].fc1_w = qmat(rows=4608, cols=1152, ld=1152, scale_ld=48, block_rows=128)
            q[i].fc2_w = qmat(rows=1152, cols=4608, ld=4608, scale_ld=16, block_rows=128)
        for k, v in over.items():
            setattr(q[1], k, v)
        return q

    put = abi.LIB.rc_set_quant_weights
    assert put(ctx, layers()) == 0 and put(ctx, None) == 0
    assert put(None, layers()) == -1
    assert put(ctx, layers(fc1_w=qmat(rows=4608, cols=1152, ld=1152, scale_ld=4608))) == -2             # a scale per row
    assert put(ctx, layers(fc2_w=qmat(rows=4608, cols=1152, ld=1152, scale_ld=48, block_rows=128))) == -2
    assert put(ctx, layers(qkv_w=qmat(rows=3456, cols=1152, ld=1152, scale_ld=32, block_rows=128, data=None))) == -1
    f32, keep2 = make_ctx(abi.RC_F32)
    assert put(f32, layers()) == -8
    abi.rc_destroy(ctx)
    abi.rc_destroy(f32)


def test_python_refusals():
    f8 = torch.float8_e4m3fn
    with pytest.raises(ValueError, match="GPU"):
        quant.QuantMatrix(torch.zeros((4, 32)).to(f8), torch.zeros((1, 16), dtype=torch.uint8), 1)
    with pytest.raises(ValueError, match="float8"):
        quant.QuantMatrix(torch.zeros((4, 32)), torch.zeros((1, 16), dtype=torch.uint8), 1)
    with pytest.raises(ValueError, match="cover"):
        quant.QuantMatrix(torch.zeros((4, 160)).to(f8), torch.zeros((1, 16), dtype=torch.uint8), 1)
    with pytest.raises(ValueError, match="cover"):
        quant.QuantMatrix(torch.zeros((20, 32)).to(f8), torch.zeros((1, 16), dtype=torch.uint8), 1)
    with pytest.raises(ValueError, match="block_rows"):
        quant.QuantMatrix(torch.zeros((4, 32)).to(f8), torch.zeros((1, 16), dtype=torch.uint8), 32)
    with pytest.raises(ValueError, match="multiple"):
        quant.QuantCache.alloc(1, 2, 100, device="cpu")
    with pytest.raises(ValueError, match="GPU"):
        quant.QuantCache.alloc(1, 2, 128, device="cpu")
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        quant.quantize(torch.zeros((2, 32), dtype=torch.float16))
    with pytest.raises(ValueError):
        quant.quantize(torch.zeros((2, 32)))


def test_plain_quantisation_is_the_definition():
    """The plain form's codes are the nearest of all 8-bit numbers, its scale the least that fits."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((40, 200)) * 10.0 ** rng.uniform(-8, 8, (40, 1))
    for tile in (1, 128):
        q, e = R.quantize(x, tile)
        y = R.dequantize(q, e, tile)
        step = R.dequantize(np.maximum(np.abs(q), 2.0 ** -6), e, tile)
        assert (np.abs(x - y) <= 2.0 ** -4 * step).all()
        assert (np.abs(q) <= 448).all() and (R.amax_finite(q, None) > 216)
    t = torch.from_numpy(np.linspace(-448, 448, 9973))
    np.testing.assert_array_equal(R.round_e4m3(t.numpy()), t.to(torch.float8_e4m3fn).double().numpy())


def test_plain_attention_against_softmax():
    rng = np.random.default_rng(1)
    v = R.round_e4m3(rng.standard_normal((1, 1, 2, 2, 64, 72)) * 100)
    e = rng.integers(118, 123, (1, 1, 2, 2))
    q = rng.standard_normal((3, 72))
    o, _ = R.attention(v, e, [0, 3], [100], q, 0.1)
    f = torch.from_numpy(v * 2.0 ** (e[..., None, None] - 127.0))
    k, w = f[0, 0, :, 0].reshape(-1, 72)[:100], f[0, 0, :, 1].reshape(-1, 72)[:100]
    ref = torch.softmax(torch.from_numpy(q) @ k.T * 0.1, -1) @ w
    np.testing.assert_allclose(o, ref.numpy(), rtol=1e-12)


def test_attention_grid_limits():
    """One long chain among very many: the grid holds the longest one's tiles for each."""
    n = 32767
    rows = aset([0, 1 << 20] + [(1 << 20) + i for i in range(1, n)], idx=None)
    c = qcache(batch=n, heads=16, tokens=64, chain_stride=16 * 64 * 144, scale_stride=32)
    f = abi.LIB.rc_qcache_attention
    assert f(C.byref(c), C.byref(rows), None, FAKE, 1152, 0.1, FAKE, 1152, FAKE, 1 << 40, None) == -2
    assert "too many" in abi.rc_last_error()
    ctx, keep = make_ctx(grid=(128, 128))
    nb, ws = abi.rc_quant_cache_bytes(ctx, n, 1), abi.rc_quant_workspace_bytes(ctx, 1 << 17, n)
    rows = aset([0, 16384] + [16384 + i for i in range(1, n)])
    assert abi.LIB.rc_reuse_step_quant(ctx, C.byref(abi.rc_cache_view(FAKE, nb, n, 1)), 0, C.byref(rows), C.byref(step_io()),
                                       abi.RC_FUSE_UPDATE, FAKE, ws, None) == -2
    assert "too many" in abi.rc_last_error()
    abi.rc_destroy(ctx)


@pytest.mark.parametrize("scale", [3.0e38, -2.4e38])
def test_attention_scale_limit(scale):
    """The scale times log2(e) has to be finite too."""
    rows = aset([0, 5, 9], idx=None)
    assert abi.LIB.rc_qcache_attention(C.byref(qcache()), C.byref(rows), None, FAKE, 288, scale, FAKE, 288, FAKE, 1 << 40,
                                       None) == -1


class _Range(C.Structure):
    _fields_ = [("p", C.c_void_p), ("lines", C.c_longlong)]


@pytest.mark.parametrize("rows,cols,ld", [(4608, 1152, 1152), (1152, 4608, 4608), (1152, 4608, 4624), (1, 16, 16), (3, 48, 4096)])
def test_what_is_warmed_is_what_is_read(rows, cols, ld):
    """A step's kernels warm the weights that its later products read: whole lines inside the 8-bit matrix where there
    is one, else the bfloat16 one's."""
    f = abi.LIB._ZN2rc10warm_rangeEPKvxPK7rc_qmat
    f.restype, f.argtypes = _Range, [C.c_void_p, C.c_longlong, C.POINTER(abi.rc_qmat)]
    r = f(2 * FAKE, 1000, C.byref(qmat(rows=rows, cols=cols, ld=ld, block_rows=128)))
    assert r.p == FAKE and 0 <= ((rows - 1) * ld + cols) - r.lines * 128 < 128
    r = f(2 * FAKE, 1000, None)
    assert r.p == 2 * FAKE and r.lines == 1000
