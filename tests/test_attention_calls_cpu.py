"""Descriptions of attention calls (arxiv 2411.01238, Section 4.2's models) that programs come to make, on the host."""
import ctypes

import pytest

from paper_2411_01238_amd import sdrop


@pytest.mark.parametrize("total,ok", [(1, True), (2, False)])
def test_packed_arrays_of_one_token_have_no_step(total, ok):
    # the bound of the lengths is not the number of tokens: one token's step is of no consequence, two tokens' must not be 0
    buf = ctypes.create_string_buffer(64)
    p = ctypes.addressof(buf)
    a = dict(B=2, max_q=150, max_k=150, Hq=2, Hkv=2, D=64, scale=0.125, causal=1, dtype=sdrop.BF16, cu_q=p, cu_k=p, total_q=total, total_k=total)
    a.update({n + "_h": 64 for n in ("q", "k", "v", "o", "do", "dq", "dk", "dv")})
    need = sdrop.lib().sdrop_attn_bwd_workspace_bytes(ctypes.byref(sdrop.Attn(**a)))
    assert (need > 0) == ok
