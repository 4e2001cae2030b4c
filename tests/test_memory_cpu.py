"""Matrices and caches whose tensors are given other memory after they were made: refused before any launch (on
tensors in host memory, which nothing reads)."""
import pytest
import torch

from _host_calls import calls  # noqa: F401  (a fixture)
from paper_2608_29809_amd import norm, quant
from paper_2608_29809_amd.runtime import ActiveSet

F8 = torch.float8_e4m3fn


def rows(n, cols=16):
    return torch.zeros(n, cols)


MADE = {
    "int8": lambda: quant.IntMatrix(torch.zeros(40, 16, dtype=torch.int8), torch.ones(40)),
    "int8 view": lambda: quant.IntMatrix(torch.zeros(50, 32, dtype=torch.int8)[8:48, 16:], torch.ones(50)[5:45]),
    "int8 alloc": lambda: quant.IntMatrix.alloc(40, 16, "cpu"),
    "e4m3": lambda: quant.QuantMatrix(torch.zeros(40, 16, dtype=torch.uint8).view(F8), torch.ones(1, 48, dtype=torch.uint8), 1),
    "e4m3 alloc": lambda: quant.QuantMatrix.alloc(40, 16, 1, "cpu"),
    "cache": lambda: quant.QuantCache.alloc(1, 2, 64, "cpu"),
}
# of a tensor: where it or its storage is given other memory
EXCHANGED = {
    "data": lambda t: setattr(t, "data", torch.zeros(4).to(t.dtype)),
    "same shape": lambda t: setattr(t, "data", t.clone()),
    "set_": lambda t: t.set_(torch.zeros(4).to(t.dtype)),
    "resize_": lambda t: t.resize_(1 << 20),
    "storage": lambda t: t.untyped_storage().resize_(0),
    "cut": lambda t: t.untyped_storage().resize_(16),
}


def uses(m):
    """The calls that take m, by what they call."""
    x, w = rows(40), MADE["int8" if isinstance(m, quant.IntMatrix) else "e4m3"]()
    if isinstance(m, quant.IntMatrix):
        return {"rc_igemm": [lambda: quant.igemm(m, w, out=rows(40, 40)), lambda: quant.igemm(w, m, out=rows(40, 40))],
                "rc_quantize_int8": [lambda: quant.quantize_int8(x, out=m)],
                "rc_residual_norm": [lambda: norm.norm_modulate(x, norm.Norm(), out=m), lambda: norm.residual_norm(x, x, pre=norm.Norm(), out=m)]}
    if isinstance(m, quant.QuantMatrix):
        return {"rc_qgemm": [lambda: quant.qgemm(m, w, out=rows(40, 40)), lambda: quant.qgemm(w, m, out=rows(40, 40))],
                "rc_quantize": [lambda: quant.quantize(x, out=m)], "rc_residual_norm": [lambda: norm.norm_modulate(x, norm.Norm(), out=m)]}
    active, k = ActiveSet.from_lists([range(3)], device="cpu"), rows(3, 144)
    return {"rc_qcache_store": [lambda: quant.qcache_store(m, active, k, k)],
            "rc_qcache_attention": [lambda: quant.qcache_attention(m, active, k.bfloat16())]}


@pytest.mark.parametrize("made", MADE)
@pytest.mark.parametrize("how", EXCHANGED)
@pytest.mark.parametrize("part", ["data", "scales"])
def test_exchanged_memory_is_refused(calls, made, how, part):
    m = MADE[made]()
    for name, fs in uses(m).items():
        for f in fs:
            f()
        assert calls == [name] * len(fs), name
        calls.clear()
    with torch.no_grad():
        getattr(m, part).view(torch.uint8).fill_(1)  # (in place: the same memory)
    m.struct()
    EXCHANGED[how](getattr(m, part))
    for fs in uses(m).values():
        for f in fs:
            with pytest.raises(ValueError, match="exchanged or resized"):
                f()
    assert not calls


@pytest.mark.parametrize("made", ["int8", "int8 alloc", "e4m3", "e4m3 alloc"])
def test_sizes_are_those_it_was_made_with(calls, made):
    """A tensor that was made smaller where it lies does not change how many rows a call writes."""
    m = MADE[made]()
    m.data.resize_(10, 16)
    quantised = quant.quantize_int8 if isinstance(m, quant.IntMatrix) else quant.quantize
    with pytest.raises(ValueError, match="another shape"):
        quantised(rows(10), out=m)
    quantised(rows(40), out=m)
    assert len(calls) == 1
