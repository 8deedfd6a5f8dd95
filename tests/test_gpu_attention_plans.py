"""Which launches attention's backward pass (arxiv 2411.01238, Section 4.2's models) makes of sequences of up to 256 keys, and that its gradients
are right on either side of the rule."""
import pytest
import torch

from paper_2411_01238_amd import sdrop
from _util import kernel_names
from test_gpu_attention_precision import check_heads, gradients, randn

pytestmark = pytest.mark.gpu

# B, Tq, Tk, heads, D, causal: one launch? (a quarter of the CUs' heads up to 256 rows, half of them, or three quarters for small heads, beyond)
PLANS = [
    (8, 256, 256, 8, 128, False, True), (8, 257, 256, 8, 128, False, False), (8, 700, 77, 8, 128, True, False), (16, 300, 200, 8, 128, True, True),
    (16, 300, 200, 8, 64, True, False), (24, 290, 77, 8, 64, False, True), (7, 200, 200, 8, 64, False, False), (64, 1500, 40, 1, 64, False, False),
    (64, 20, 257, 1, 64, False, False),
]


@pytest.mark.parametrize("B,Tq,Tk,H,D,causal,one", PLANS)
def test_rows_decide_too(B, Tq, Tk, H, D, causal, one):
    if torch.cuda.get_device_properties(0).multi_processor_count != 256:
        pytest.skip("the rule counts CUs: these are calls on 256")
    print("plan", B, Tq, Tk, H, D, causal, flush=True)
    td = torch.bfloat16
    q, k, v, do = (randn((B, T, H, D), td, i) for i, T in enumerate((Tq, Tk, Tk, Tq)))
    o, lse, rest = sdrop.sdrop_attn(q, k, v, causal, need_rest=True)
    names = " ".join(kernel_names(lambda: sdrop.sdrop_attn_bwd(do, q, k, v, o, lse, causal, rest=rest)))
    assert ("attn_bwd_short_kernel" in names) == one and ("attn_dq_kernel" in names) == (not one)
    check_heads(q, k, v, do, gradients(q, k, v, do, causal), causal, td, "plan", some=[(0, 0), (B - 1, H - 1)])


def test_query_heads_of_a_key_head_are_rows():
    # 32 query heads to a key head: 64 workgroups would walk 2048 rows each
    td = torch.float16
    q, k, v, do = randn((64, 64, 32, 64), td, 1), randn((64, 100, 1, 64), td, 2), randn((64, 100, 1, 64), td, 3), randn((64, 64, 32, 64), td, 4)
    o, lse, rest = sdrop.sdrop_attn(q, k, v, True, need_rest=True)
    assert "attn_dq_kernel" in " ".join(kernel_names(lambda: sdrop.sdrop_attn_bwd(do, q, k, v, o, lse, True, rest=rest)))
    dq, dk, dv = sdrop.sdrop_attn_bwd(do, q, k, v, o, lse, True, rest=rest)
    # the same with the key head given 32 times, dk and dv summed
    many = [t.expand(64, 100, 32, 64) for t in (k, v)]
    o2, lse2, rest2 = sdrop.sdrop_attn(q, *many, True, need_rest=True)
    outs = [torch.empty((64, 100, 32, 64), dtype=td, device="cuda") for _ in range(2)]
    dq2, dk2, dv2 = sdrop.sdrop_attn_bwd(do, q, *many, o2, lse2, True, rest=rest2, out_dk=outs[0], out_dv=outs[1])
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    # dq: two orders of the same fp32 sums of values that each were rounded, and the result's own rounding
    e = torch.finfo(td).eps / 2
    for a, b in ((dq, dq2), (dk, dk2.float().sum(2, keepdim=True)), (dv, dv2.float().sum(2, keepdim=True))):
        assert float((a.float() - b.float()).norm()) <= 2 * e * float(b.float().norm())
