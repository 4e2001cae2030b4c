"""What the operators do to a graph that autograd keeps: nothing in silence (on tensors in host memory, up to the launch)."""
import pytest
import torch

from _host_calls import calls  # noqa: F401  (a fixture)
from paper_2608_29809_amd import norm, quant
from paper_2608_29809_amd.runtime import ActiveSet

F8 = torch.float8_e4m3fn
N = norm.Norm


def rows(n=40, cols=16, **more):
    return torch.zeros(n, cols, **more)


def imat(scales=None):
    return quant.IntMatrix(torch.zeros(40, 16, dtype=torch.int8), torch.ones(40) if scales is None else scales)


def qmat(block_rows=1):
    return quant.QuantMatrix(torch.zeros(40, 16, dtype=torch.uint8).view(F8), torch.ones(1, 48, dtype=torch.uint8), block_rows)


def parts(m):
    return [m.data, m.scales]


def writes():
    """A call, what it writes and what it only reads."""
    x, h, y, m, e, c = rows(), rows(), rows(), imat(), qmat(), quant.QuantCache.alloc(1, 2, 64, "cpu")
    z, q, active = rows(40, 40), rows(3, 144), ActiveSet.from_lists([range(3)], device="cpu")
    o, k = rows(3, 144).bfloat16(), rows(3, 144).bfloat16()
    return {
        "update": (lambda: norm.residual_norm(x, h), [x], [h]),
        "update and result": (lambda: norm.residual_norm(x, h, pre=N(), out=y), [x, y], [h]),
        "update and int8": (lambda: norm.residual_norm(x, h, pre=N(), out=m), [x] + parts(m), [h]),
        "norm": (lambda: norm.norm_modulate(x, N(), out=y), [y], [x]),
        "norm in place": (lambda: norm.norm_modulate(x, N(), out=x), [x], []),
        "norm to int8": (lambda: norm.norm_modulate(x, N(), out=m), parts(m), [x]),
        "norm to e4m3": (lambda: norm.norm_modulate(x, N(), out=e), parts(e), [x]),
        "int8": (lambda: quant.quantize_int8(x, out=m), parts(m), [x]),
        "e4m3": (lambda: quant.quantize(x, out=e), parts(e), [x]),
        "int8 product": (lambda: quant.igemm(m, imat(), out=z), [z], parts(m)),
        "e4m3 product": (lambda: quant.qgemm(e, qmat(), out=z), [z], parts(e)),
        "store": (lambda: quant.qcache_store(c, active, q, q), parts(c), [q]),
        "attention": (lambda: quant.qcache_attention(c, active, k, out=o), [o], [k] + parts(c)),
    }


@pytest.mark.parametrize("name", ["update", "update and result", "update and int8", "norm", "norm in place", "norm to int8", "norm to e4m3", "int8",
                                  "e4m3", "int8 product", "e4m3 product", "store", "attention"])
def test_writes_are_told(calls, name):
    """What a call writes in place has another version behind it, what it reads has not."""
    call, written, read = writes()[name]
    before = [t._version for t in written], [t._version for t in read]
    call()
    assert len(calls) == 1
    assert all(t._version > v for t, v in zip(written, before[0])) and [t._version for t in read] == before[1]


def test_graph_that_saved_an_updated_tensor(calls):
    """Its backward pass fails; it would use the values of after the update."""
    for call in (lambda x: norm.residual_norm(x, rows()), lambda x: norm.norm_modulate(rows(), N(), out=x[:]), lambda x: norm.norm_modulate(x, N(), out=x)):
        x, w = rows(), rows().requires_grad_()
        y = (w * x).sum()
        with torch.no_grad():
            call(x)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()


def test_inference_tensors(calls):
    """They have no version."""
    with torch.inference_mode():
        x = rows()
        norm.residual_norm(x, rows(), pre=N(), out=rows())
    norm.residual_norm(x, rows())
    assert len(calls) == 2


def takes():
    """A call of tensors, and those tensors, each of which autograd would expect a gradient through."""
    v = [torch.zeros(16) for _ in range(3)]
    return {
        "norm_modulate": (lambda x, scale, shift, out: norm.norm_modulate(x, N(), scale, shift, out=out), [rows(), v[0], v[1], rows()]),
        "residual_norm": (lambda x, h, gate, scale, shift, out: norm.residual_norm(x, h, gate, pre=N(), scale=scale, shift=shift, out=out),
                          [rows(), rows(), *v, rows()]),
        "norm_modulate to int8": (lambda x, scales: norm.norm_modulate(x, N(), out=imat(scales)), [rows(), torch.ones(40)]),
        "igemm": (lambda a, w, bias, out: quant.igemm(imat(a), imat(w), bias, out=out), [torch.ones(40), torch.ones(40), torch.zeros(40), rows(40, 40)]),
    }


@pytest.mark.parametrize("name", takes())
def test_gradients_are_refused(calls, name):
    """A tensor that requires a gradient, a leaf or a result, is refused while gradients are recorded, and only then."""
    call, tensors = takes()[name]
    for i in range(len(tensors)):
        leaf = [t.clone().requires_grad_(k == i) for k, t in enumerate(tensors)]
        result = [t.clone() for t in tensors]
        result[i] = tensors[i].clone().requires_grad_() * 2
        for given in (leaf, result):
            with pytest.raises(ValueError, match=f"{name.split()[0]} has no gradient"):
                call(*given)
            assert not calls
            for off in (torch.no_grad, torch.inference_mode):
                with off():
                    call(*given)
            call(*[t.detach() for t in given])
            assert len(calls) == 3
            calls.clear()
    norm.norm_modulate(rows(), N(weight=torch.nn.Parameter(torch.zeros(16))), out=rows())  # (a norm's weights are constants)
    with torch.no_grad():
        quant.quantize_int8(rows().requires_grad_(), out=imat())
    quant.quantize_int8(rows().requires_grad_(), out=imat())  # (integers, of which none is expected)
