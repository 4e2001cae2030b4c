"""Host-side checks of the norms around a block: refusals before any launch (a
call that would pass is made only where there is no GPU)."""
import ctypes as C

import numpy as np
import pytest
import torch

import _norm_ref as R
from paper_2608_29809_amd import abi, norm

NO_GPU = torch.cuda.device_count() == 0
FAKE = 1 << 20  # aligned, never dereferenced
LAYER = dict(kind=1, eps=1e-6, weight=None, bias=None)


def spec(**over):
    return abi.rc_norm(*[{**LAYER, **over}[f] for f in ("kind", "eps", "weight", "bias")])


NONE = None


def aset(offs, offsets=FAKE, batch=None):
    h = (C.c_int32 * len(offs))(*offs)
    a = abi.rc_active_set(None, offsets, C.cast(h, C.POINTER(C.c_int32)), len(offs) - 1 if batch is None else batch)
    a.keep = h
    return a


def call(**over):
    """An update with a bfloat16 result, but for what is given; e4m3, int8: keyword arguments of a matrix."""
    d = dict(rows=40, cols=256, x=FAKE, ldx=256, h=FAKE, ldh=256, x_dtype=0, h_dtype=1, post=NONE, pre=spec(), residual_scale=1.0,
             gate_stride=0, scale_stride=0, shift_stride=0, gate=FAKE, scale=FAKE, shift=FAKE, out=FAKE, ldo=256, out_dtype=1)
    e4m3, int8, chains = over.pop("e4m3", None), over.pop("int8", None), over.pop("chains", None)
    d.update(over)
    keep = [d["post"], d["pre"]]
    d.update(post=C.addressof(d["post"]) if d["post"] else None, pre=C.addressof(d["pre"]) if d["pre"] else None)
    a = abi.rc_norm_args(**d)
    if e4m3 is not None:
        keep.append(abi.rc_qmat(**{**dict(data=FAKE, scales=FAKE, ld=256, rows=40, cols=256, scale_ld=48, block_rows=1), **e4m3}))
        a.out_e4m3 = C.addressof(keep[-1])
    if int8 is not None:
        keep.append(abi.rc_imat(**{**dict(data=FAKE, scales=FAKE, ld=256, rows=40, cols=256), **int8}))
        a.out_int8 = C.addressof(keep[-1])
    if chains is not None:
        a.chains = C.addressof(chains)
    return abi.LIB.rc_residual_norm(C.byref(a), None)


@pytest.mark.parametrize("over,status", [
    (dict(rows=-1), -2), (dict(cols=0), -2), (dict(cols=16385, ldx=1 << 15, ldh=1 << 15, ldo=1 << 15), -8),
    (dict(x=None), -1), (dict(x=FAKE + 2), -3), (dict(h=FAKE + 1), -3), (dict(out=FAKE + 1), -3),
    (dict(out=FAKE + 2, out_dtype=0), -3), (dict(x_dtype=2), -1), (dict(h_dtype=-1), -1), (dict(out_dtype=3), -1),
    (dict(ldx=255), -2), (dict(ldh=0), -2), (dict(ldo=-256), -2), (dict(ldx=(1 << 31) + 8), -2),
    (dict(residual_scale=float("nan")), -1), (dict(residual_scale=float("inf")), -1),
    (dict(pre=spec(kind=3)), -1), (dict(pre=spec(kind=-1)), -1), (dict(post=spec(kind=5)), -1),
    (dict(pre=spec(eps=0.0)), -1), (dict(pre=spec(eps=-1e-6)), -1), (dict(post=spec(eps=float("inf"))), -1),
    (dict(pre=spec(eps=float("nan"))), -1), (dict(post=spec(kind=0)), -1), (dict(pre=spec(kind=0)), -1), (dict(pre=NONE), -1),
    (dict(pre=spec(weight=FAKE + 2)), -3), (dict(pre=spec(bias=FAKE + 1)), -3), (dict(post=spec(weight=FAKE + 2)), -3),
    (dict(gate=FAKE + 2), -3), (dict(scale=FAKE + 2), -3), (dict(shift=FAKE + 3), -3),
    (dict(gate_stride=255), -2), (dict(scale_stride=-1), -2), (dict(shift_stride=1), -2),
    (dict(out=None), -1),                                          # a norm, but no result
    (dict(out=None, pre=NONE), -1),                                # scale and shift, but no result
    (dict(h=None), -1), (dict(h=None, gate=None, post=spec()), -1), (dict(h=None, gate=None, out=None, pre=NONE, scale=None, shift=None), -1),
    (dict(e4m3={}), -1), (dict(int8={}), -1), (dict(out=None, e4m3={}, int8={}), -1),  # two results
    (dict(out=None, e4m3=dict(rows=39)), -2), (dict(out=None, e4m3=dict(block_rows=128)), -8), (dict(out=None, e4m3=dict(data=FAKE + 8)), -3),
    (dict(out=None, int8=dict(cols=240)), -2), (dict(out=None, int8=dict(scales=None)), -1), (dict(out=None, int8=dict(ld=264)), -3),
    (dict(cols=250, out=None, int8=dict(cols=250)), -8),
])
def test_refusals(over, status):
    assert call(**over) == status
    assert abi.rc_last_error()


def test_refusals_of_chains():
    assert call(chains=aset([0, 40], batch=0)) == -2
    assert call(chains=aset([0] * 40000)) == -2
    assert call(chains=aset([0, 10, 39])) == -4
    assert call(chains=aset([0, 10, 41])) == -4
    assert call(chains=aset([0, 20, 10, 40])) == -4
    assert call(chains=aset([1, 20, 40])) == -4
    assert call(chains=aset([0, 20, 40], offsets=None)) == -1
    assert abi.LIB.rc_residual_norm(None, None) == -1


def test_calls_that_pass():
    assert call(rows=0, x=None, h=FAKE) == 0  # nothing to do
    assert call(rows=0, chains=aset([0, 0, 0], offsets=None)) == 0
    if NO_GPU:
        for over in (dict(), dict(chains=aset([0, 0, 40])), dict(out=None, pre=NONE, scale=None, shift=None), dict(h=None, gate=None),
                     dict(out=None, e4m3={}), dict(out=None, int8={}), dict(x=FAKE + 4, h=FAKE + 2, out=FAKE + 6, ldx=257, ldh=259, ldo=256),
                     dict(post=spec(kind=2, weight=FAKE + 4, bias=FAKE)), dict(gate_stride=256, scale_stride=6 * 256)):
            assert call(**over) == -6, over


@pytest.mark.skipif(not NO_GPU, reason="needs tensors that are not on a GPU")
def test_python_refusals():
    x, v = torch.zeros(4, 32), torch.zeros(32)
    N = norm.Norm()
    for f in (lambda: norm.Norm("batch"), lambda: norm.Norm(weight=v.double()), lambda: norm.Norm(weight=x), lambda: norm.Norm(bias=torch.zeros(64)[::2]),
              lambda: norm.Norm(weight=v, bias=v[:31]), lambda: norm.norm_modulate(x, N), lambda: norm.norm_modulate(x[0], N),
              lambda: norm.norm_modulate(x, None), lambda: norm.norm_modulate(x.half(), N), lambda: norm.norm_modulate(x, norm.Norm(weight=v[:31])),
              lambda: norm.norm_modulate(x, N, v[:31]), lambda: norm.norm_modulate(x, N, v.double()), lambda: norm.norm_modulate(x, N, x),
              lambda: norm.norm_modulate(x, N, x[None]), lambda: norm.norm_modulate(x, N, dtype=torch.float16),
              lambda: norm.norm_modulate(x.t(), N), lambda: norm.residual_norm(x, None), lambda: norm.residual_norm(x, x[:3]),
              lambda: norm.residual_norm(x, x, scale=v), lambda: norm.residual_norm(x, x, out=x), lambda: norm.residual_norm(x, x.double())):
        with pytest.raises(ValueError):
            f()


def test_arguments_as_bytes():
    """Those of the C structure, field by field."""
    fields = [f for f, _ in abi.rc_norm_args._fields_]
    values = [1.0 + i if f == "residual_scale" else (0x1234567890 if t is not C.c_int32 else 0x12345600) + i
              for i, (f, t) in enumerate(abi.rc_norm_args._fields_)]
    assert abi.norm_args(*values) == bytes(abi.rc_norm_args(*values))
    nulls = [1.0 if f == "residual_scale" else 0 for f in fields]
    assert abi.norm_args(*nulls) == bytes(abi.rc_norm_args(*[None if t is C.c_void_p else v for v, (_, t) in zip(nulls, abi.rc_norm_args._fields_)]))


def test_plain_form_in_float32():
    """The bounds hold for float32 arithmetic that adds in another order."""
    rng = np.random.default_rng(0)
    for cols, off in ((1, 0.0), (7, 3.0), (1152, 0.3), (1152, 1e3), (16384, 5.0)):
        x = (rng.standard_normal((9, cols)) + off).astype(np.float32)
        x[3] = x[3, 0]
        for kind in ("layer", "rms"):
            m = x.mean(1, keepdims=True, dtype=np.float32) if kind == "layer" else np.float32(0)
            d = x - m
            y = d / np.sqrt((d * d).mean(1, keepdims=True, dtype=np.float32) + np.float32(1e-6))
            ref, tol = R.norm(x.astype(np.float64), np.zeros(x.shape), kind, 1e-6)
            assert (np.abs(y - ref) <= tol).all(), (cols, off, kind)


GIVEN = {"tensor": lambda t: t, "parameter": torch.nn.Parameter, "view": lambda t: torch.cat([t, t])[t.numel():]}


@pytest.mark.parametrize("part", ["weight", "bias"])
@pytest.mark.parametrize("given", GIVEN)
def test_memory_of_weights(given, part):
    """A norm holds the memory that it was made of; where that is resized it is refused instead of read."""
    def made(**more):
        t = GIVEN[given](torch.full((1152,), 2.0))
        return t, norm.Norm("rms", **{part: t, **more})

    def held(n):  # (as the C structure has it)
        assert norm._norm(n, 1152, -1, "the norm") == C.addressof(n._struct)
        assert getattr(n, part).data_ptr() == getattr(n._struct, part) and not getattr(n, part).requires_grad
        return getattr(n, part)

    t, n = made()
    with torch.no_grad():
        t.fill_(3.0)
    assert held(n).data_ptr() == t.data_ptr() and torch.equal(held(n), torch.full((1152,), 3.0))
    t.data = torch.zeros(4)
    others = [torch.full((1152,), 5.0) for _ in range(64)]  # (the memory would be theirs)
    assert torch.equal(held(n), torch.full((1152,), 3.0)) and len(others) == 64
    t, n = made()
    with torch.no_grad():
        t.set_(torch.zeros(4))
    assert torch.equal(held(n), torch.full((1152,), 2.0))
    t, n = made()
    getattr(n, part).set_(torch.zeros(4))  # (a tensor of that memory, not what the norm holds)
    assert torch.equal(held(n), torch.full((1152,), 2.0))
    for resize in (lambda t: t.detach().resize_(1 << 20), lambda t: t.untyped_storage().resize_(0), lambda t: t.untyped_storage().resize_(64)):
        for more in ({}, {"weight" if part == "bias" else "bias": torch.zeros(1152)}):
            t, n = made(**more)
            resize(t)
            with pytest.raises(ValueError, match="resized"):
                norm._norm(n, 1152, -1, "the norm")
            with pytest.raises(ValueError, match="resized"):
                getattr(n, part)


def test_weights_without_values():
    for w in (torch.zeros(0), torch.zeros(64)[32:32], torch.zeros(64)[:0]):
        assert norm.Norm(weight=w).weight.shape == (0,)


def test_weights_elsewhere():
    n = norm.Norm(weight=torch.zeros(8))
    assert norm._norm(n, 8, -1, "post")
    with pytest.raises(ValueError, match="the CPU"):
        norm._norm(n, 8, 0, "post")
