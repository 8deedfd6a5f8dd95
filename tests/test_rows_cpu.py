"""What the row operators (element dropout, layer norm: arxiv 2411.01238, Sections 2.1 and 4.2) refuse, on the host."""
import ctypes

import pytest
import torch

from paper_2411_01238_amd import sdrop


@pytest.fixture
def mem():
    buf = ctypes.create_string_buffer(1 << 16)      # host memory: never dereferenced by these calls
    addr = (ctypes.addressof(buf) + 15) // 16 * 16
    yield addr
    del buf


def _with(f, ok, **kw):
    a = list(ok)
    for k, v in kw.items():
        a[int(k[1:])] = v
    return f(*a)


def test_dropout_arguments(mem):
    f, p = sdrop.lib().sdrop_dropout, mem
    ok = (p, None, p, 64, 64, 0.5, 1, 2, sdrop.BF16, 0, 0, 0, None)
    for bad in (dict(a0=None), dict(a2=None), dict(a5=1.5), dict(a5=-0.1), dict(a5=float("nan"))):
        assert _with(f, ok, **bad) == sdrop.EINVAL
    for bad in (dict(a3=0), dict(a4=0), dict(a4=(1 << 24) + 1), dict(a3=(1 << 30) + 1), dict(a9=63), dict(a10=1), dict(a11=(1 << 24) + 1), dict(a9=-64)):
        assert _with(f, ok, **bad) == sdrop.ESHAPE
    assert _with(f, ok, a8=3) == sdrop.EDTYPE
    assert _with(f, ok, a0=p + 1) == sdrop.EALIGN and _with(f, ok, a8=sdrop.F32, a2=p + 2) == sdrop.EALIGN


def test_layer_norm_arguments(mem):
    L, p = sdrop.lib(), mem
    f = L.sdrop_layer_norm
    ok = (p, p, p, p, p, p, p, p, 64, 64, 1e-5, 0.5, 1, 2, sdrop.BF16, sdrop.F32, 0, 0, 0, 0, None)
    for bad in (dict(a0=None), dict(a2=None), dict(a5=None), dict(a10=-1.0), dict(a10=float("inf")), dict(a10=float("nan")), dict(a11=2.0),
                dict(a4=None), dict(a1=None, a4=None), dict(a4=None, a11=0.0)):
        assert _with(f, ok, **bad) == sdrop.EINVAL
    for bad in (dict(a8=0), dict(a9=-1), dict(a16=63), dict(a17=63), dict(a18=63), dict(a19=63)):
        assert _with(f, ok, **bad) == sdrop.ESHAPE
    for bad in (dict(a14=5), dict(a15=sdrop.F16), dict(a14=sdrop.F32, a15=sdrop.BF16)):
        assert _with(f, ok, **bad) == sdrop.EDTYPE
    for bad in (dict(a0=p + 1), dict(a2=p + 2), dict(a6=p + 2), dict(a7=p + 1)):
        assert _with(f, ok, **bad) == sdrop.EALIGN
    g = L.sdrop_layer_norm_bwd
    need = L.sdrop_layer_norm_bwd_workspace_bytes(64, 64)
    assert need > 0 and need % (2 * 64 * 4) == 0
    assert L.sdrop_layer_norm_bwd_workspace_bytes(0, 64) == 0 and L.sdrop_layer_norm_bwd_workspace_bytes(64, 1 << 25) == 0
    okb = (p, None, p, p, p, p, p, p, p, p, 64, 64, 0.5, 1, 2, sdrop.BF16, sdrop.BF16, 0, 0, 0, 0, 0, None, 0, None)
    assert _with(g, okb) == sdrop.EWORKSPACE
    assert _with(g, okb, a22=p + 4, a23=need) == sdrop.EWORKSPACE and _with(g, okb, a22=p, a23=need - 1) == sdrop.EWORKSPACE
    for bad in (dict(a0=None), dict(a2=None), dict(a3=None), dict(a4=None), dict(a5=None), dict(a6=None, a7=None, a8=None, a9=None), dict(a12=-1.0)):
        assert _with(g, okb, **bad) == sdrop.EINVAL
    for bad in (dict(a10=0), dict(a17=3), dict(a18=3), dict(a19=3), dict(a20=3), dict(a21=3)):
        assert _with(g, okb, **bad) == sdrop.ESHAPE
    assert _with(g, okb, a16=sdrop.F16) == sdrop.EDTYPE
    assert _with(g, okb, a9=p + 1) == sdrop.EALIGN


def test_the_binding_refuses_what_is_no_gpu_matrix():
    x = torch.zeros(4, 4)
    for call in (lambda: sdrop.sdrop_dropout(x, 0.5, 1), lambda: sdrop.sdrop_layer_norm(x, x[0]), lambda: sdrop.sdrop_layer_norm_bwd(x, x, x[0], x[0], x[0])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(sdrop.SdropError):
        sdrop.sdrop_dropout(x.double(), 0.5, 1)
    with pytest.raises(ValueError):
        sdrop.sdrop_dropout(x, 0.5, 1, residual=x.half())


def test_models_refuse_unknown_operators():
    from paper_2411_01238_amd import model_step as ms
    for name in ("mlp", "gpt", "vit"):
        with pytest.raises(ValueError):
            ms.MODELS[name]("dense", 0.0, device="cpu", ops="other")
