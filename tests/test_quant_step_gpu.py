"""Steps on an 8-bit pool against the oracle, block by block: each block of the
oracle takes the GPU's own input rows (the block output before it) and the keys
and values that the GPU left in the slot.

Keys and values: stored values are off by the rounding to e4m3, half a step or
2^-4 of the largest, and what the bfloat16 step's own gate allows.  Block
outputs with bfloat16 weights: that gate.  With 8-bit weights the oracle
quantises as the step does, but a value that the two sides see 2^-8 apart is
rounded to another neighbour in about 4 % of the cases (2^-8 over a spacing of
2^-3.5), a difference of 9 %, so of 1.8 % rms per operand and 3 % through both
MLP products, which is 3 % of the largest element too (both 4.5 sigma); twice
that is allowed."""
import numpy as np
import pytest
import torch

import _quant_ref as R
import oracle as O
import synth
from _cases import BF16_U, relerr, to_np, tol, weights

pytestmark = pytest.mark.gpu


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def linear(lw, name, x, w8):
    w = np.asarray(lw[name + "_w"], np.float64)
    if w8:
        x, w = R.dequantize(*R.quantize(x, 1), 1), R.dequantize(*R.quantize(bf16(w), 128), 128)
    return x @ w.T


def block(lw, X, mod, tk, tv, K, V, heads, w8):
    """Block output, and the fresh keys and values [rows][C], of active rows X over a slot's K, V [H][N][72]."""
    sh1, sc1, g1, sh2, sc2, g2 = mod
    C = X.shape[1]
    qkv = linear(lw, "qkv", O.modulate(O.layer_norm(X), sh1, sc1), w8) + lw["qkv_b"]
    o = O.attention(qkv[:, :C].reshape(-1, heads, 72), K.transpose(1, 0, 2), V.transpose(1, 0, 2))
    X = X + g1 * (o.reshape(-1, C) @ np.asarray(lw["proj_w"], np.float64).T + lw["proj_b"])
    X, _ = O.cross_and_mlp(lw, X, (sh1, sc1, g1, sh2, sc2, np.zeros_like(g2)), tk, tv, heads, None, np.float64)
    f = O.gelu_tanh(linear(lw, "fc1", O.modulate(O.layer_norm(X), sh2, sc2), w8) + lw["fc1_b"])
    return X + g2 * (linear(lw, "fc2", f, w8) + lw["fc2_b"]), qkv[:, C:2 * C], qkv[:, 2 * C:]


def slot_values(cache, t, l):
    """Stored keys and values [B][2][H][N][72], and scale factors [B][2][H][N / 64]."""
    q = cache.quant(t, l)
    v = q.data.cpu().float().double().numpy() * 2.0 ** (q.scales.cpu().numpy().astype(np.float64) - 127.0)[..., None, None]
    B, H, nb = v.shape[:3]
    f = 2.0 ** (q.scales.cpu().numpy().astype(np.float64) - 127.0)
    return v.transpose(0, 3, 1, 2, 4, 5).reshape(B, 2, H, nb * 64, 72), f.transpose(0, 3, 1, 2)


class Case:
    def __init__(self, B=2, layers=2, grid=(16, 16)):
        self.s = s = synth.ModelShape(layers=layers, grid_h=grid[0], grid_w=grid[1], dtype="bf16")
        self.W = weights(s, 3, True)
        self.B = B
        self.txt, self.lat = synth.make_text(s, B, 3), synth.make_latent(s, B, 3)
        from paper_2608_29809_amd.runtime import RegionCacheModel
        self.model = RegionCacheModel(s, self.W)
        self.tkv = self.model.prepare_text(self.model.to_storage(self.txt))
        self.tkv_o = [[O.text_kv(lw, O.caption_projection(self.W, self.txt[b]), s.heads) for lw in self.W["layers"]]
                      for b in range(B)]
        self.latent = torch.from_numpy(self.lat).cuda()

    def check(self, cache, t, timestep, per_chain, w8, before=None):
        """Every block of step t over the active tokens; before: slot values per block of a region step."""
        s, tl = self.s, tol(self.s)
        t0 = O.adaln_single(self.W, O.timestep_embedding(self.W, timestep))
        for b, idx in enumerate(per_chain):
            X = O.patch_embed(self.W, self.lat[b], s.grid_h, s.grid_w, s.patch)[idx]
            for l, lw in enumerate(self.W["layers"]):
                vals, unit = slot_values(cache, t, l)
                out, k, v = block(lw, X, O.layer_modulation(lw, t0), *self.tkv_o[b][l], vals[b, 0], vals[b, 1], s.heads, w8)
                for which, rows in ((0, k), (1, v)):
                    got = vals[b, which][:, idx].transpose(1, 0, 2).reshape(len(idx), -1)
                    assert relerr(got, rows) < 2.0 ** -4 + (6e-2 if w8 else tl), (b, l, which)
                if before is not None:
                    rest = np.setdiff1d(np.arange(s.tokens), idx)
                    step = 2.0 ** -10 * np.repeat(unit[b], 64, 2)[..., None]  # half the subnormal step
                    assert (np.abs(vals[b] - before[l][b])[:, :, rest] <= step[:, :, rest]).all(), (b, l)
                H = to_np(cache.H(b, t, l))[idx].astype(np.float64)
                lim = 6e-2 if w8 else tl
                floor = BF16_U * (np.abs(H).max() + np.abs(X).max()) / np.abs(out - X).max()
                assert relerr(H, out) < lim, (b, l)
                assert relerr(H - X, out - X) < lim + floor, (b, l)
                X = H


@pytest.fixture(scope="module")
def case():
    return Case()


def fill(case, cache, t, seed):
    """Random keys, values, hidden states and next latent of step t."""
    from paper_2608_29809_amd import quant
    from paper_2608_29809_amd.runtime import ActiveSet
    s, m = case.s, case.model
    slot = synth.make_cache_slot(s, case.B, seed)
    every = ActiveSet.from_lists([np.arange(s.tokens)] * case.B)
    for l in range(s.layers):
        rows = [m.to_storage(slot[n][l].transpose(0, 2, 1, 3).reshape(case.B * s.tokens, -1)) for n in ("K", "V")]
        quant.qcache_store(cache.quant(t, l), every, *rows)
        for b in range(case.B):
            cache.H(b, t, l).copy_(m.to_storage(slot["H"][l, b]))
    for b in range(case.B):
        cache.latent(b, t + 1).copy_(torch.from_numpy(synth.make_latent(s, case.B, seed, stream=77)[b]))


@pytest.mark.parametrize("w8", [False, True])
def test_dense_step(case, w8):
    s, m = case.s, case.model
    m.quantize_weights(w8)
    cache = m.alloc_cache(case.B, 2, bits=8)
    out = torch.empty_like(case.latent)
    m.build_cache(cache, 1, case.latent, 500, 450, case.tkv, latent_out=out)
    torch.cuda.synchronize()
    case.check(cache, 1, 500, [np.arange(s.tokens)] * case.B, w8)
    assert (cache.quant(0, 0).data.view(torch.uint8) == 0).all()  # other slots as they were
    for b in range(case.B):
        assert torch.equal(cache.latent(b, 1), case.latent[b]) and torch.equal(cache.latent(b, 2), out[b])


@pytest.mark.parametrize("w8", [False, True])
@pytest.mark.parametrize("validate", [False, True])
def test_region_step(case, w8, validate):
    from paper_2608_29809_amd.runtime import ActiveSet
    s, m = case.s, case.model
    m.quantize_weights(w8)
    cache = m.alloc_cache(case.B, 2, bits=8)
    fill(case, cache, 0, 5)
    before = [slot_values(cache, 0, l)[0] for l in range(s.layers)]
    h_before = [to_np(cache.H(0, 0, l)) for l in range(s.layers)]
    per = [np.flatnonzero(synth.rect_mask(16, 16, 7, 5, 4, 6)), np.array([0, 63, 64, 200, 255])]
    act, out = ActiveSet.from_lists(per), torch.empty_like(case.latent)
    maps = torch.zeros((case.B, s.tokens, 2), device="cuda")
    m.reuse_step(cache, 0, act, case.latent, 500, 450, case.tkv, delta=[3, 9], maps=maps, latent_out=out, validate=validate)
    torch.cuda.synchronize()
    case.check(cache, 0, 500, per, w8, before)
    rest = np.setdiff1d(np.arange(s.tokens), per[0])
    assert all(np.array_equal(to_np(cache.H(0, 0, l))[rest], h_before[l][rest]) for l in range(s.layers))
    assert torch.isfinite(out).all() and maps[0, per[0]].gt(0).all() and maps[0, rest].eq(0).all()


def test_region_step_many_chains(case):
    """More chains than travel in the kernels' arguments, some without active tokens."""
    from paper_2608_29809_amd.runtime import ActiveSet
    c = Case(B=18, layers=1, grid=(8, 8))
    cache = c.model.alloc_cache(18, 1, bits=8)
    fill(c, cache, 0, 6)
    rng = np.random.default_rng(1)
    per = [np.sort(rng.choice(64, int(n), replace=False)) if n else np.zeros(0, np.int64) for n in rng.integers(0, 12, 18)]
    per[17] = np.arange(64)
    before = [slot_values(cache, 0, 0)[0]]
    c.model.reuse_step(cache, 0, ActiveSet.from_lists(per), c.latent, 700, 650, c.tkv, latent_out=torch.empty_like(c.latent))
    torch.cuda.synchronize()
    keep = [b for b in range(18) if len(per[b])]
    full = c.B
    for b in range(full):
        if b not in keep:
            assert np.array_equal(slot_values(cache, 0, 0)[0][b], before[0][b])
    vals = [per[b] for b in range(full)]
    t0 = O.adaln_single(c.W, O.timestep_embedding(c.W, 700))
    v, _ = slot_values(cache, 0, 0)
    lw = c.W["layers"][0]
    for b in keep:
        X = O.patch_embed(c.W, c.lat[b], 8, 8, 2)[vals[b]]
        out, _, _ = block(lw, X, O.layer_modulation(lw, t0), *c.tkv_o[b][0], v[b, 0], v[b, 1], c.s.heads, False)
        assert relerr(to_np(cache.H(b, 0, 0))[vals[b]], out) < tol(c.s), b


def test_steps_of_many_rows():
    """Products in 256 x 256 and 192 x 256 tiles, whose chains are alike: the first one against the oracle, the others equal to it."""
    from paper_2608_29809_amd.runtime import ActiveSet
    B = 10
    c = Case(B=B, layers=1, grid=(32, 32))
    c.txt[:], c.lat[:] = c.txt[0], c.lat[0]
    s, m = c.s, c.model
    c.tkv, c.latent = m.prepare_text(m.to_storage(c.txt)), torch.from_numpy(c.lat).cuda()
    m.quantize_weights()
    cache, out = m.alloc_cache(B, 1, bits=8), torch.empty_like(c.latent)
    m.build_cache(cache, 0, c.latent, 500, 450, c.tkv, latent_out=out)
    c.check(cache, 0, 500, [np.arange(s.tokens)], True)
    H = [cache.H(b, 0, 0).clone() for b in range(B)]
    assert all(torch.equal(H[b], H[0]) and torch.equal(out[b], out[0]) for b in range(B))
    # 8000 rows: chains that end inside a tile, a partial last tile
    idx = np.sort(np.random.default_rng(4).choice(s.tokens, 800, replace=False))
    before = [slot_values(cache, 0, 0)[0]]
    m.reuse_step(cache, 0, ActiveSet.from_lists([idx] * B), c.latent, 300, 250, c.tkv, latent_out=out)
    c.check(cache, 0, 300, [idx], True, before)
    rest = np.setdiff1d(np.arange(s.tokens), idx)
    for b in range(B):
        assert torch.equal(cache.H(b, 0, 0), cache.H(0, 0, 0)) and torch.equal(out[b], out[0])
        assert torch.equal(cache.H(b, 0, 0)[rest], H[0][rest])


def test_empty_region_copies_the_latent(case):
    from paper_2608_29809_amd.runtime import ActiveSet
    m = case.model
    cache = m.alloc_cache(case.B, 1, bits=8)
    fill(case, cache, 0, 7)
    state, out = cache.buf.clone(), torch.empty_like(case.latent)
    m.reuse_step(cache, 0, ActiveSet.from_lists([np.zeros(0, np.int32)] * case.B), case.latent, 500, 450, case.tkv, latent_out=out)
    torch.cuda.synchronize()
    assert torch.equal(state, cache.buf)
    assert all(torch.equal(out[b], cache.latent(b, 1)) for b in range(case.B))


def test_other_pools_keep_their_results(case):
    """8-bit weights change no step on a bfloat16 pool."""
    m, outs = case.model, []
    for w8 in (False, True):
        m.quantize_weights(w8)
        cache = m.alloc_cache(case.B, 1)
        cache.buf.zero_()
        out = torch.empty_like(case.latent)
        m.build_cache(cache, 0, case.latent, 500, 450, case.tkv, latent_out=out)
        torch.cuda.synchronize()
        outs.append((out, cache.buf))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


@pytest.mark.parametrize("w8", [False, True])
def test_step_captured_and_replayed(case, w8):
    from paper_2608_29809_amd.runtime import ActiveSet
    m = case.model
    m.quantize_weights(w8)
    cache = m.alloc_cache(case.B, 1, bits=8)
    fill(case, cache, 0, 8)
    first = cache.buf.clone()
    act = ActiveSet.from_lists([np.arange(30, 120), np.arange(3)])
    x, out = case.latent.clone(), torch.empty_like(case.latent)

    def step(inp):
        m.reuse_step(cache, 0, act, inp, 500, 450, case.tkv, latent_out=out)

    step(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(x)
    for k in range(3):
        new = torch.roll(case.latent, k, 2).contiguous()
        cache.buf.copy_(first)
        step(new)
        want = out.clone(), cache.buf.clone()
        cache.buf.copy_(first)
        x.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(cache.buf, want[1])


@pytest.mark.parametrize("w8", [False, True])
def test_session_on_an_8_bit_pool(case, w8):
    """A first turn and an edit: finite latents, unedited patches of every reuse step from the cached trajectory."""
    from paper_2608_29809_amd import schedule as S
    m, s = case.model, case.s
    m.quantize_weights(w8)
    sess = S.EditSession(m, case.B, T=4, rho=0.25, threshold=0.5, cache_bits=8)
    x_T = torch.from_numpy(synth.make_latent(s, case.B, 9)).cuda()
    first = sess.first_turn(m.to_storage(case.txt), x_T)
    txt, delta = synth.edit_text(s, case.txt, 3, 4)
    out = sess.edit_turn(m.to_storage(txt), x_T, [int(d) for d in delta])
    torch.cuda.synchronize()
    assert torch.isfinite(first).all() and torch.isfinite(out["latent"]).all()
    mask = out["mask"].view(case.B, 1, s.grid_h, s.grid_w).bool()
    mask = mask.repeat_interleave(2, 2).repeat_interleave(2, 3).expand_as(first)
    assert torch.equal(out["latent"][~mask], first[~mask]) and (out["latent"][mask] != first[mask]).any()


def test_python_refusals(case):
    m = case.model
    cache, plain = m.alloc_cache(1, 1, bits=8), m.alloc_cache(1, 1)
    for f in (lambda: cache.K(0, 0, 0), lambda: cache.V(0, 0, 0), lambda: plain.quant(0, 0),
              lambda: m.alloc_cache(1, 1, bits=4), lambda: m.alloc_cache(1, 1, host=True, bits=8),
              lambda: m.update_cache(cache, 0, None, None)):
        with pytest.raises(ValueError):
            f()
