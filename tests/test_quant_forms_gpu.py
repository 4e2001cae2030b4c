"""Steps on an 8-bit pool in the other forms that models and calls have: token inputs, narrow MLPs, guidance."""
import numpy as np
import pytest
import torch

import oracle as O
import synth
from _cases import oracle_text_kv, relerr, to_np, tol
from test_quant_step_gpu import block, slot_values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("w8", [False, True])
@pytest.mark.parametrize("mlp,counts", [(128, [40, 0, 3]), (4608, [1, 130]), (256, [(5 * b) % 60 for b in range(19)])])
def test_token_mode_blocks(mlp, counts, w8):
    """A block over given tokens: the dense step of every chain, then a region step."""
    from paper_2608_29809_amd.runtime import ActiveSet, RegionCacheModel
    s = synth.ModelShape(layers=1, mlp=mlp, text_dim=1152, grid_h=16, grid_w=16, dtype="bf16", token_mode=True)
    W = synth.make_weights(s, seed=mlp, stress=True)
    B, rng = len(counts), np.random.default_rng(mlp)
    x = [synth.bf16_round(rng.standard_normal((B, s.tokens, s.hidden)).astype(np.float32)) for _ in range(2)]
    t_vec, text = rng.standard_normal(s.hidden).astype(np.float32), synth.make_text(s, B, mlp)
    m = RegionCacheModel(s, W)
    m.quantize_weights(w8)
    tkv, tv = m.prepare_text(m.to_storage(text)), torch.from_numpy(t_vec).cuda()
    cache = m.alloc_cache(B, 1, bits=8)
    m.build_cache(cache, 0, m.to_storage(x[0]), 0, -1, tkv, t_vec=tv)
    mod = O.layer_modulation(W["layers"][0], O.adaln_single(W, t_vec))
    lim = 6e-2 if w8 else tol(s)

    def check(x, per):
        v, _ = slot_values(cache, 0, 0)
        for b, idx in enumerate(per):
            if not len(idx):
                continue
            out, k, fresh_v = block(W["layers"][0], np.asarray(x[b], np.float64)[idx], mod, *oracle_text_kv(s, W, text[b])[0],
                                    v[b, 0], v[b, 1], s.heads, w8)
            for which, rows in ((0, k), (1, fresh_v)):
                got = v[b, which][:, idx].transpose(1, 0, 2).reshape(len(idx), -1)
                assert relerr(got, rows) < 2.0 ** -4 + lim, (b, which)
            assert relerr(to_np(cache.H(b, 0, 0))[idx], out) < lim, b

    torch.cuda.synchronize()
    check(x[0], [np.arange(s.tokens)] * min(B, 2))
    per = [np.sort(rng.choice(s.tokens, n, replace=False)) for n in counts]
    m.reuse_step(cache, 0, ActiveSet.from_lists(per), m.to_storage(x[1]), 0, -1, tkv, t_vec=tv)
    torch.cuda.synchronize()
    check(x[1], per)


@pytest.mark.parametrize("w8", [False, True])
def test_guided_pair(w8):
    """The next latent of a guided pair is that of the unguided steps combined: it is linear in the predicted noise
    (float32: 2^-19 of the largest value for the few operations and the scale 4.5)."""
    from paper_2608_29809_amd.runtime import ActiveSet, RegionCacheModel
    s = synth.ModelShape(layers=2, grid_h=16, grid_w=16, dtype="bf16")
    m = RegionCacheModel(s, synth.make_weights(s, seed=5, stress=True))
    m.quantize_weights(w8)
    tkv = m.prepare_text(m.to_storage(synth.make_text(s, 2, 5)))
    x = torch.from_numpy(synth.make_latent(s, 1, 5)).cuda().expand(2, -1, -1, -1).contiguous()
    idx = np.flatnonzero(synth.rect_mask(16, 16, 5, 6, 3, 4))
    act, g = ActiveSet.from_lists([idx] * 2), 4.5
    cache = m.alloc_cache(2, 2, bits=8)
    m.build_cache(cache, 1, x, 700, 650, tkv, latent_out=torch.empty_like(x), guidance=g)
    first, slots = cache.buf.clone(), cache.latent(0, 0).data_ptr() - cache.buf.data_ptr()
    outs, pools = [], []
    for guidance in (None, g):
        cache.buf.copy_(first)
        out = torch.empty_like(x)
        m.reuse_step(cache, 1, act, x, 500, 450, tkv, latent_out=out, guidance=guidance)
        torch.cuda.synchronize()
        outs.append(out.double())
        pools.append(cache.buf.clone())
    assert torch.equal(pools[0][:slots], pools[1][:slots])  # keys, values and hidden states alike
    want = outs[0][1] + g * (outs[0][0] - outs[0][1])
    mask = torch.zeros(s.tokens, dtype=torch.bool, device="cuda")
    mask[torch.from_numpy(idx).cuda()] = True
    mask = mask.view(1, 16, 16).repeat_interleave(2, 1).repeat_interleave(2, 2).expand(4, -1, -1)
    for b in range(2):
        assert (outs[1][b] - want)[mask].abs().max() <= 2.0 ** -19 * (1 + 2 * g) * outs[0].abs().max()
        assert torch.equal(outs[1][b][~mask], outs[0][b][~mask])
    assert (outs[1][0] - outs[0][0])[mask].abs().max() > 1e-3
