"""What attention (arxiv 2411.01238, Section 4.2's models) refuses, on the host."""
import ctypes

import pytest
import torch

from paper_2411_01238_amd import sdrop


@pytest.fixture
def mem():
    buf = ctypes.create_string_buffer(1 << 16)      # host memory: never dereferenced by these calls
    yield (ctypes.addressof(buf) + 15) // 16 * 16
    del buf


def _desc(**kw):
    a = dict(B=2, max_q=64, max_k=64, Hq=4, Hkv=2, D=64, scale=0.125, causal=1, dtype=sdrop.BF16)
    for n in ("q", "o", "do", "dq"):
        a.update({n + "_b": 64 * 256, n + "_t": 256, n + "_h": 64})
    for n in ("k", "v", "dk", "dv"):
        a.update({n + "_b": 64 * 128, n + "_t": 128, n + "_h": 64})
    a.update(kw)
    return ctypes.byref(sdrop.Attn(**a))


BAD = [
    (dict(scale=0.0), sdrop.EINVAL), (dict(scale=-1.0), sdrop.EINVAL), (dict(scale=float("inf")), sdrop.EINVAL), (dict(scale=float("nan")), sdrop.EINVAL),
    (dict(scale=1e-60), sdrop.EINVAL), (dict(scale=1e300), sdrop.EINVAL), (dict(scale=3e38), sdrop.EINVAL),      # not in fp32 (the last: times log2 e)
    (dict(causal=2), sdrop.EINVAL), (dict(dtype=sdrop.F32), sdrop.EDTYPE), (dict(dtype=9), sdrop.EDTYPE),
    (dict(B=0), sdrop.ESHAPE), (dict(max_q=0), sdrop.ESHAPE), (dict(max_k=0), sdrop.ESHAPE), (dict(Hq=3), sdrop.ESHAPE), (dict(Hkv=0), sdrop.ESHAPE),
    (dict(D=0), sdrop.ESHAPE), (dict(D=60), sdrop.ESHAPE), (dict(D=136), sdrop.ESHAPE), (dict(max_q=1 << 31), sdrop.ESHAPE), (dict(max_q=1 << 29), sdrop.ESHAPE),
    (dict(q_t=4), sdrop.ESHAPE), (dict(k_h=-8), sdrop.ESHAPE), (dict(v_t=(1 << 24) + 8), sdrop.ESHAPE), (dict(o_b=3), sdrop.ESHAPE),
]


def test_descriptions(mem):
    L, p = sdrop.lib(), mem
    assert L.sdrop_attn_workspace_bytes(None) == 0 and L.sdrop_attn_bwd_workspace_bytes(None) == 0
    for kw, code in BAD:
        assert L.sdrop_attn(p, p, p, p, None, None, _desc(**kw), p, 1 << 40, None) == code, kw
        assert L.sdrop_attn_bwd(p, p, p, p, p, None, p, p, p, p, _desc(**kw), p, 1 << 40, None) == code, kw
        assert L.sdrop_attn_workspace_bytes(_desc(**kw)) == 0
    for kw in (dict(do_t=4), dict(dq_h=-8), dict(dk_t=1 << 25), dict(dv_b=1), dict(dq_t=0), dict(dk_h=0), dict(dv_b=0)):
        assert L.sdrop_attn_bwd(p, p, p, p, p, None, p, p, p, p, _desc(**kw), p, 1 << 40, None) == sdrop.ESHAPE, kw
    assert L.sdrop_attn(p, p, p, p, None, None, _desc(o_t=0), p, 1 << 40, None) == sdrop.ESHAPE
    # packed arrays have a size; lengths go with dense keys
    assert L.sdrop_attn(p, p, p, p, None, None, _desc(cu_q=p), p, 1 << 40, None) == sdrop.ESHAPE
    assert L.sdrop_attn(p, p, p, p, None, None, _desc(cu_k=p, total_k=64, k_len=p), p, 1 << 40, None) == sdrop.EINVAL
    assert L.sdrop_attn(p, p, p, p, None, None, None, p, 1 << 40, None) == sdrop.EINVAL


def test_pointers_and_workspaces(mem):
    L, p = sdrop.lib(), mem
    ok = [p, p, p, p, None, None]
    for i in range(4):
        a = list(ok)
        a[i] = None
        assert L.sdrop_attn(*a, _desc(), None, 0, None) == sdrop.EINVAL
        a[i] = p + 8
        assert L.sdrop_attn(*a, _desc(), None, 0, None) == sdrop.EALIGN
    assert L.sdrop_attn(p, p, p, p, p + 8, None, _desc(), None, 0, None) == sdrop.EALIGN
    assert L.sdrop_attn(p, p, p, p, None, p + 2, _desc(), None, 0, None) == sdrop.EALIGN
    # one query, many keys: parts of the keys need room for their results
    few = dict(max_q=1, max_k=1 << 16)
    need = L.sdrop_attn_workspace_bytes(_desc(**few))
    assert need > 0
    assert L.sdrop_attn(*ok, _desc(**few), None, 0, None) == sdrop.EWORKSPACE
    assert L.sdrop_attn(*ok, _desc(**few), p, need - 1, None) == sdrop.EWORKSPACE
    assert L.sdrop_attn(*ok, _desc(**few), p + 4, need, None) == sdrop.EWORKSPACE
    okb = [p, p, p, p, p, None, p, p, p, p]
    need = L.sdrop_attn_bwd_workspace_bytes(_desc())
    # two floats for each row of each head, and a little more
    assert 2 * 4 * 64 * 8 <= need <= 2 * 4 * 64 * 8 + 1024
    assert 4 * 100 * 8 <= L.sdrop_attn_bwd_workspace_bytes(_desc(cu_q=p, total_q=100)) <= 4 * 100 * 8 + 1024
    for i in (0, 1, 2, 3, 4, 6, 7, 8, 9):
        a = list(okb)
        a[i] = None
        assert L.sdrop_attn_bwd(*a, _desc(), p, need, None) == sdrop.EINVAL
        a[i] = p + (8 if i != 6 else 2)
        assert L.sdrop_attn_bwd(*a, _desc(), p, need, None) == sdrop.EALIGN
    assert L.sdrop_attn_bwd(*okb, _desc(), p, need - 1, None) == sdrop.EWORKSPACE
    assert L.sdrop_attn_bwd(*okb, _desc(), None, need, None) == sdrop.EWORKSPACE


def test_the_binding_refuses_what_does_not_fit():
    q = torch.zeros(2, 8, 4, 64, dtype=torch.float16)
    cu = torch.zeros(3, dtype=torch.int32)
    for call in (lambda: sdrop.sdrop_attn(q, q, q), lambda: sdrop.sdrop_attn(q[0], q, q), lambda: sdrop.sdrop_attn(q[0], q[0], q[0], cu_q=cu, cu_k=cu)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(sdrop.SdropError):
        sdrop.sdrop_attn(q.float(), q.float(), q.float())
