"""Memory and gradients of the operators' tensors on the GPU: exchanged memory is refused or not seen, never read."""
import numpy as np
import pytest
import torch

from paper_2608_29809_amd import norm, quant
from paper_2608_29809_amd.runtime import ActiveSet

pytestmark = pytest.mark.gpu


def rnd(*shape, seed=0):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float32)).cuda()


@pytest.mark.parametrize("part", ["weight", "bias"])
def test_weights_of_tensors(part):
    """A norm keeps the memory that it was made of, of a plain tensor and of a view as of a parameter."""
    x = rnd(3, 1152, seed=1)
    for view in (False, True):
        w = torch.full((2304,), 2.0, device="cuda")[1152:] if view else torch.full((1152,), 2.0, device="cuda")
        n = norm.Norm("rms", **{part: w})
        y = norm.norm_modulate(x, n, dtype=torch.float32)
        plain = norm.norm_modulate(x, norm.Norm("rms"), dtype=torch.float32)
        assert torch.equal(y, plain * 2 if part == "weight" else plain + 2)
        w.data = torch.zeros(7, device="cuda")
        others = [torch.full((1152,), 5.0, device="cuda") for _ in range(64)]  # (the memory would be theirs)
        assert torch.equal(norm.norm_modulate(x, n, dtype=torch.float32), y) and len(others) == 64
        getattr(n, part).fill_(0.0)
        assert torch.equal(norm.norm_modulate(x, n, dtype=torch.float32), plain * 0 if part == "weight" else plain)
        getattr(n, part).untyped_storage().resize_(0)
        with pytest.raises(ValueError, match="resized"):
            norm.norm_modulate(x, n)


def test_exchanged_matrices():
    x, w, z = rnd(40, 256), quant.quantize_int8(rnd(48, 256, seed=1)), quant.quantize(rnd(48, 256, seed=1), 128)
    active, q = ActiveSet.from_lists([np.arange(3)]), rnd(3, 144)
    made = [(lambda: quant.quantize_int8(x), lambda m: quant.igemm(m, w)), (lambda: quant.quantize(x), lambda m: quant.qgemm(m, z)),
            (lambda: quant.QuantCache.alloc(1, 2, 64), lambda m: quant.qcache_store(m, active, q, q))]
    for make, use in made:
        for part in ("data", "scales"):
            for exchange in (lambda t: setattr(t, "data", t.clone()), lambda t: t.untyped_storage().resize_(0)):
                m = make()
                use(m)
                exchange(getattr(m, part))
                with pytest.raises(ValueError, match="exchanged or resized"):
                    use(m)


def test_gradients():
    """Refused while they are recorded; a graph that saved what a call updates fails instead of using the new values."""
    x, h, gate = rnd(5, 1152), rnd(5, 1152, seed=1), rnd(1152, seed=2)
    want = norm.norm_modulate(x, norm.Norm(), gate)
    with pytest.raises(ValueError, match="gradient"):
        norm.norm_modulate(x, norm.Norm(), gate.clone().requires_grad_())
    with torch.no_grad():
        assert torch.equal(norm.norm_modulate(x, norm.Norm(), gate.clone().requires_grad_()), want)
    a = quant.quantize_int8(rnd(40, 256))
    with pytest.raises(ValueError, match="gradient"):
        quant.igemm(a, a, torch.zeros(40, device="cuda", requires_grad=True))
    loss = (x * gate.requires_grad_()).sum()
    norm.residual_norm(x, h, gate.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_update_in_a_graph():
    """An update that is captured and replayed, with eager calls between, as the calls one after another."""
    h, gate, n = rnd(70, 1152, seed=1), rnd(1152, seed=2), norm.Norm("rms", weight=rnd(1152, seed=3))
    x, eager = rnd(70, 1152), rnd(70, 1152)
    out = torch.empty(70, 1152, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        norm.residual_norm(x.clone(), h, gate, pre=n, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        norm.residual_norm(x, h, gate, pre=n, out=out)
    for _ in range(4):
        graph.replay()
        want = norm.residual_norm(eager, h, gate, pre=n)
        torch.cuda.synchronize()
        assert torch.equal(x, eager) and torch.equal(out, want)


def test_weights_on_two_devices():
    with pytest.raises(ValueError, match="cpu"):
        norm.Norm(weight=torch.zeros(8, device="cuda"), bias=torch.zeros(8))
