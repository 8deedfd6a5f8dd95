"""Attention (arxiv 2411.01238, Section 4.2's models) against its float64 definition.

Tolerances, with e = eps / 2 of the type, a rounding's most (2^-8 for bf16, 2^-11 for fp16), and a = 2^-18 for the fp32 arithmetic: a
score is a sum of at most 128 products in fp32 (|error| <= 128 * 2^-24 of the magnitudes), and the exponential passes on an
absolute error of the score as a relative one of P; scores here stay below 2^4, so P and its sum are off by at most 2^4 * 2^-17 = 2^-13
for large scores and far less for usual ones.
    O      P is rounded once (e), O once: |error| <= e |O| + (e + 2^-13) sum_j P |v|
    dV     the same with P^T |dO|;  dQ, dK: dS = P (dP - delta) is rounded once, and delta = dO O carries what is left of O's
           rounding after its second part (e^2, below 2^-13 |dO| |O|)
lse is fp32: 2^-13 absolute.
"""
import numpy as np
import pytest
import torch

from oracle import transformer_oracle as orc
from paper_2411_01238_amd import sdrop
from paper_2411_01238_amd import transformer as tr
from _util import f64

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
A = 2.0 ** -13


def _randn(shape, dtype, seed, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * std).to(dtype).cuda()


def _bounds(q, k, v, do, scale, causal, e):
    """Bounds of (o, dq, dk, dv), element by element, without the final rounding."""
    group = q.shape[1] // k.shape[1]
    o, dq, dk, dv = (np.zeros(t.shape) for t in (q, q, k, v))
    for h in range(q.shape[1]):
        j = h // group
        p, _ = orc._scores(q[:, h], k[:, j], scale, causal)
        o[:, h] = (e + A) * (p @ np.abs(v[:, j]))
        if do is None:
            continue
        dp = do[:, h] @ v[:, j].T
        delta = (p * dp).sum(axis=1, keepdims=True)
        mag = np.abs(do[:, h]) @ np.abs(v[:, j]).T + (np.abs(do[:, h]) * np.abs(p @ v[:, j])).sum(axis=1, keepdims=True)
        err = p * ((e + A) * np.abs(dp - delta) + A * mag)
        dq[:, h] = scale * (err @ np.abs(k[:, j]))
        dk[:, j] += scale * (err.T @ np.abs(q[:, h]))
        dv[:, j] += (e + A) * (p.T @ np.abs(do[:, h]))
    return o, dq, dk, dv


def _near(got, want, bound, dtype, what):
    got = f64(got)
    e = torch.finfo(dtype).eps / 2
    bound = np.abs(want) * e + bound * (1 + e) + (2.0 ** -24 if dtype == torch.float16 else 1e-30)
    assert np.all(np.isfinite(got)), what
    bad = np.abs(got - want) > bound
    assert not bad.any(), "%s: %d of %d off, worst %.3g of its bound" % (what, bad.sum(), bad.size, (np.abs(got - want) / bound).max())
    # (and on the whole no more than three roundings' worth: a wrong scale or a lost tile of small values shows here)
    n = np.linalg.norm(want)
    assert np.linalg.norm(got - want) <= 3 * e * n + A * np.sqrt(want.size), what


def _check(q, k, v, do, causal, dtype, got, lse, what, scale=None):
    """One sequence [T, H, D]; got: (o,) or (o, dq, dk, dv)."""
    qd, kd, vd = f64(q), f64(k), f64(v)
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    o, l64 = orc.attention(qd, kd, vd, scale, causal)
    bound = _bounds(qd, kd, vd, None if do is None else f64(do), scale, causal, torch.finfo(dtype).eps / 2)
    _near(got[0], o, bound[0], dtype, what + " o")
    if lse is not None:
        l = f64(lse)
        assert np.array_equal(np.isneginf(l), np.isneginf(l64)), what
        fin = np.isfinite(l64)
        assert np.all(np.abs(l[fin] - l64[fin]) <= A), what + " lse"
    if do is not None:
        for n, g, w, b in zip(("dq", "dk", "dv"), got[1:], orc.attention_bwd(f64(do), qd, kd, vd, scale, causal), bound[1:]):
            _near(g, w, b, dtype, what + " " + n)


DENSE = [
    # B, Tq, Tk, Hq, Hkv, D, causal
    (1, 1, 1, 1, 1, 8, True), (2, 1, 1, 2, 1, 64, False), (1, 2, 3, 1, 1, 16, True), (3, 31, 33, 2, 2, 128, True),
    (1, 64, 64, 3, 1, 72, True), (2, 65, 129, 4, 2, 64, False), (1, 128, 128, 1, 1, 128, True), (1, 257, 300, 2, 1, 120, True),
    (2, 100, 40, 2, 1, 80, True),       # 60 tokens that see no key
    (1, 130, 7, 1, 1, 128, False), (1, 33, 1025, 7, 1, 128, True), (2, 40, 700, 5, 5, 40, False), (1, 500, 500, 6, 2, 32, True),
]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("B,Tq,Tk,Hq,Hkv,D,causal", DENSE)
def test_dense_forward_and_backward(B, Tq, Tk, Hq, Hkv, D, causal, dtype):
    print("attention", B, Tq, Tk, Hq, Hkv, D, causal, dtype, flush=True)
    td = DT[dtype]
    q, k, v, do = (_randn(s, td, i) for i, s in enumerate(((B, Tq, Hq, D), (B, Tk, Hkv, D), (B, Tk, Hkv, D), (B, Tq, Hq, D))))
    o, lse, rest = sdrop.sdrop_attn(q, k, v, causal, need_rest=True)
    grads = sdrop.sdrop_attn_bwd(do, q, k, v, o, lse, causal, rest=rest)
    for b in range(B):
        _check(q[b], k[b], v[b], do[b], causal, td, [t[b] for t in (o,) + grads], lse[b], "b=%d" % b)
    assert sdrop.status() == 0


# heads enough that a workgroup takes a sequence's gradients whole: up to 256 keys, group sizes that divide 16 and others
SHORT = [
    (16, 197, 197, 4, 4, 64, False), (64, 33, 33, 2, 1, 128, True), (22, 100, 256, 9, 3, 72, True), (64, 1, 9, 1, 1, 8, True), (13, 40, 31, 25, 5, 40, False),
    (16, 70, 130, 16, 4, 128, True), (8, 90, 60, 32, 8, 96, True), (64, 64, 128, 1, 1, 64, False), (64, 129, 256, 1, 1, 128, False), (2, 3, 2, 64, 32, 16, True),
]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("B,Tq,Tk,Hq,Hkv,D,causal", SHORT)
def test_many_short_sequences(B, Tq, Tk, Hq, Hkv, D, causal, dtype):
    test_dense_forward_and_backward(B, Tq, Tk, Hq, Hkv, D, causal, dtype)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 2, 64), (6, 2, 128)])
def test_many_short_packed_sequences(Hq, Hkv, D, dtype):
    print("short packed", Hq, Hkv, D, dtype, flush=True)
    td = DT[dtype]
    g = np.random.default_rng(5)
    lq = [0, 1, 32, 33, 150, 0] + [int(n) for n in g.integers(0, 90, 34)]
    lk = [9, 0, 32, 1, 250, 0] + [int(n) for n in g.integers(0, 90, 34)]
    cq, ck = (torch.tensor(np.concatenate([[0], np.cumsum(l)]), dtype=torch.int32, device="cuda") for l in (lq, lk))
    nq, nk = sum(lq) + 5, sum(lk) + 5
    q, do, k, v = _randn((nq, Hq, D), td, 1), _randn((nq, Hq, D), td, 4), _randn((nk, Hkv, D), td, 2), _randn((nk, Hkv, D), td, 3)
    for t in (q, do, k, v):
        t[-5:] = float("nan")
    out = [torch.full_like(t, 7.0) for t in (q, k, v)]
    kw = dict(cu_q=cq, cu_k=ck, max_q=150, max_k=256)
    o, lse, rest = sdrop.sdrop_attn(q, k, v, True, need_rest=True, **kw)
    sdrop.sdrop_attn_bwd(do, q, k, v, o, lse, True, rest=rest, out_dq=out[0], out_dk=out[1], out_dv=out[2], **kw)
    assert all(bool((t[-5:] == 7.0).all()) for t in out)
    for b in range(len(lq)):
        a, z = slice(int(cq[b]), int(cq[b + 1])), slice(int(ck[b]), int(ck[b + 1]))
        if lk[b] == 0:
            assert not out[0][a].any()
        if lq[b] == 0:
            assert not out[1][z].any() and not out[2][z].any()
        if lq[b] and lk[b]:
            _check(q[a], k[z], v[z], do[a], True, td, [o[a], out[0][a], out[1][z], out[2][z]], lse[:, a], "seq %d" % b)
    assert sdrop.status() == 0


def test_short_sequences_padded_and_as_slices_of_one_tensor():
    td = torch.bfloat16
    B, T, H, D = 16, 120, 4, 64
    q, k, v, do = (_randn((B, T, H, D), td, i) for i in range(4))
    lens = [T, 0, 1, 33, 64, 119] + [7 * b for b in range(6, B)]
    for b, n in enumerate(lens):
        k[b, n:], v[b, n:] = float("nan"), float("inf")
    kl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse, rest = sdrop.sdrop_attn(q, k, v, True, k_len=kl, need_rest=True)
    dq, dk, dv = sdrop.sdrop_attn_bwd(do, q, k, v, o, lse, True, k_len=kl, rest=rest)
    for b, n in enumerate(lens):
        if n:
            _check(q[b], k[b, :n], v[b, :n], do[b], True, td, (o[b], dq[b], dk[b, :n], dv[b, :n]), lse[b], "b=%d n=%d" % (b, n))
        assert not dk[b, n:].any() and not dv[b, n:].any() and (n or not dq[b].any())
    # a fused projection's slices, and heads before tokens: the same bits
    x = _randn((B, T, 3 * H, D), td, 9).requires_grad_()
    parts = [t.detach().contiguous().requires_grad_() for t in (x[:, :, :H], x[:, :, H:2 * H], x[:, :, 2 * H:])]
    turned = [t.detach().transpose(1, 2).contiguous().transpose(1, 2).requires_grad_() for t in parts]
    gx, = torch.autograd.grad(tr.qkv_attention(x, H), x, do)
    gp = torch.autograd.grad(tr.attention(*parts), parts, do)
    gt = torch.autograd.grad(tr.attention(*turned), turned, do)
    assert torch.equal(gx, torch.cat(gp, dim=2)) and all(torch.equal(a, b) for a, b in zip(gp, gt))
    assert sdrop.status() == 0


FEW = [(1, 1, 5000, 1, 1, 128, True), (3, 1, 777, 8, 2, 128, True), (2, 4, 3000, 8, 1, 64, True), (1, 8, 9000, 3, 1, 96, False), (64, 1, 130, 4, 4, 64, True)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("B,Tq,Tk,Hq,Hkv,D,causal", FEW)
def test_few_queries_over_many_keys(B, Tq, Tk, Hq, Hkv, D, causal, dtype):
    print("few", B, Tq, Tk, Hq, Hkv, D, causal, dtype, flush=True)
    td = DT[dtype]
    q, k, v = _randn((B, Tq, Hq, D), td, 1), _randn((B, Tk, Hkv, D), td, 2), _randn((B, Tk, Hkv, D), td, 3)
    # a cache filled to different lengths, 0 and 1 among them; what lies behind is anything
    lens = [Tk if b == 0 else max(0, Tk - 97 * b) if b % 3 else b // 3 % 2 for b in range(B)]
    for b, n in enumerate(lens):
        k[b, n:], v[b, n:] = float("nan"), float("inf")
    o, lse = sdrop.sdrop_attn(q, k, v, causal, k_len=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    for b, n in enumerate(lens):
        _check(q[b], k[b, :n], v[b, :n], None, causal, td, (o[b],), lse[b], "b=%d n=%d" % (b, n))
    o2, _, rest = sdrop.sdrop_attn(q, k, v, causal, k_len=torch.tensor(lens, dtype=torch.int32, device="cuda"), need_rest=True)
    assert torch.equal(o2, o)
    for b, n in enumerate(lens):
        if n + (Tq - 1 if not causal else 0) <= 128:        # what is kept of O's rounding: at most half a step
            assert bool((rest[b].abs().float() <= torch.finfo(td).eps / 2 * o[b].abs().float() * 1.01 + 1e-6).all())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 2, 64), (3, 3, 128), (5, 1, 48)])
def test_packed_sequences(Hq, Hkv, D, causal, dtype):
    print("packed", Hq, Hkv, D, causal, dtype, flush=True)
    td = DT[dtype]
    lq, lk = [1, 0, 200, 63, 64, 0, 129, 5], [1, 3, 200, 100, 30, 0, 129, 0]
    cq, ck = (torch.tensor(np.concatenate([[0], np.cumsum(l)]), dtype=torch.int32, device="cuda") for l in (lq, lk))
    tail = 37                                   # rows behind the last sequence
    nq, nk = sum(lq) + tail, sum(lk) + tail
    q, do, k, v = _randn((nq, Hq, D), td, 1), _randn((nq, Hq, D), td, 4), _randn((nk, Hkv, D), td, 2), _randn((nk, Hkv, D), td, 3)
    for t in (q, do, k, v):
        t[-tail:] = float("nan")
    out = [torch.full_like(t, 7.0) for t in (q, q, k, v)]
    kw = dict(cu_q=cq, cu_k=ck, max_q=200, max_k=333)
    o, lse, rest = sdrop.sdrop_attn(q, k, v, causal, out=out[0], need_rest=True, **kw)
    sdrop.sdrop_attn_bwd(do, q, k, v, o, lse, causal, rest=rest, out_dq=out[1], out_dk=out[2], out_dv=out[3], **kw)
    for t, n in zip(out, (nq, nq, nk, nk)):
        assert bool((t[n - tail:] == 7.0).all())
    for b in range(len(lq)):
        a, z = slice(int(cq[b]), int(cq[b + 1])), slice(int(ck[b]), int(ck[b + 1]))
        if lk[b] == 0:
            assert not out[0][a].any() and not out[1][a].any()
        if lq[b] == 0:
            assert not out[2][z].any() and not out[3][z].any()
        if lq[b] and lk[b]:
            _check(q[a], k[z], v[z], do[a], causal, td, [out[0][a], out[1][a], out[2][z], out[3][z]], lse[:, a], "seq %d" % b)
    # the same through autograd, which clears what no sequence owns
    leaves = [t.detach().requires_grad_() for t in (q, k, v)]
    y = tr.attention(*leaves, causal=causal, **kw)
    grads = torch.autograd.grad(y, leaves, do)
    for x, w, n in zip((y,) + grads, out, (nq, nq, nk, nk)):
        assert torch.equal(x[:n - tail], w[:n - tail]) and not x[n - tail:].any()
    assert sdrop.status() == 0


def test_padded_keys_in_training():
    td = torch.bfloat16
    B, T, H, D = 3, 150, 2, 64
    q, k, v, do = (_randn((B, T, H, D), td, i) for i in range(4))
    lens = [150, 61, 0]
    for b, n in enumerate(lens):
        k[b, n:], v[b, n:] = float("inf"), float("nan")
    kl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    leaves = [t.requires_grad_() for t in (q, k, v)]
    o = tr.attention(*leaves, k_len=kl)
    dq, dk, dv = torch.autograd.grad(o, leaves, do)
    for b, n in enumerate(lens):
        if n:
            _check(q[b], k[b, :n], v[b, :n], do[b], False, td, (o[b], dq[b], dk[b, :n], dv[b, :n]), None, "b=%d" % b)
        else:
            assert not o[b].any() and not dq[b].any()
        assert not dk[b, n:].any() and not dv[b, n:].any()


def test_strides_slices_and_other_orders():
    # a fused projection's slices; [B, H, T, D] tensors; a key head repeated by stride 0; a wider cache
    td = torch.float16
    B, T, Hq, Hkv, D = 2, 90, 4, 2, 64
    qkv = _randn((B, T, Hq + 2 * Hkv, D + 8), td, 1)
    q, k, v = qkv[:, :, :Hq, :D], qkv[:, :, Hq:Hq + Hkv, 8:], qkv[:, :, Hq + Hkv:, :D]
    do = _randn((B, Hq, T, D), td, 2).transpose(1, 2)
    want = sdrop.sdrop_attn(q.contiguous(), k.contiguous(), v.contiguous(), True, 0.3, need_rest=True)
    out = torch.full((B, Hq, T, D), 7.0, dtype=td, device="cuda").transpose(1, 2)
    o, lse, rest = sdrop.sdrop_attn(q, k, v, True, 0.3, out=out, need_rest=True)
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1]) and torch.equal(rest, want[2])     # (90 tokens: all of them are kept)
    g = sdrop.sdrop_attn_bwd(do.contiguous(), q.contiguous(), k.contiguous(), v.contiguous(), want[0], want[1], True, 0.3, rest=want[2])
    grad = torch.full((B, T, Hq + 2 * Hkv, D + 8), 7.0, dtype=td, device="cuda")
    outs = dict(out_dq=grad[:, :, :Hq, :D], out_dk=grad[:, :, Hq:Hq + Hkv, :D], out_dv=grad[:, :, Hq + Hkv:, :D])
    sdrop.sdrop_attn_bwd(do, q, k, v, o, lse, True, 0.3, rest=rest, **outs)
    for x, y in zip(g, outs.values()):
        assert torch.equal(x, y)
    assert bool((grad[..., D:] == 7.0).all())
    _check(q[1], k[1], v[1], do[1], True, td, (o[1],) + tuple(t[1] for t in g), lse[1], "scale 0.3", scale=0.3)
    one = _randn((B, T, 1, D), td, 3)
    a = sdrop.sdrop_attn(q, one.expand(B, T, 2, D), one.expand(B, T, 2, D))[0]
    assert torch.equal(a, sdrop.sdrop_attn(q, one, one)[0])
    # autograd copies what the kernels cannot take in place
    odd = torch.randn((B, T, Hq, D + 1), device="cuda", dtype=td)[..., 1:]
    leaf = odd.detach().requires_grad_()
    y = tr.attention(leaf, k, v)
    assert torch.equal(y, sdrop.sdrop_attn(odd.contiguous(), k, v)[0])
    assert torch.autograd.grad(y.sum(), leaf)[0].shape == odd.shape


def test_infinite_scores_and_values_stay_where_they_are_seen():
    # causal: what a later key or value holds reaches no earlier token through the keys' tiles it does not see
    td = torch.bfloat16
    T, D = 200, 64
    q, k, v = (_randn((1, T, 1, D), td, i) for i in range(3))
    want = sdrop.sdrop_attn(q, k, v, True)[0]
    k2 = k.clone()
    k2[0, 192:] = float("nan")
    o = sdrop.sdrop_attn(q, k2, v, True)[0]
    assert torch.equal(o[0, :192], want[0, :192]) and bool(torch.isnan(o[0, 192:]).all())
    # large scores: no overflow, the largest key takes all
    big = q * 200
    o, lse = sdrop.sdrop_attn(big, k, v, False)
    s = (f64(big)[0, :, 0] @ f64(k)[0, :, 0].T) * D ** -0.5
    assert bool(torch.isfinite(o).all()) and np.allclose(f64(lse)[0, 0], s.max(axis=1), rtol=1e-2)


def test_bad_offsets_and_lengths_leave_a_sequence_out():
    # what the device finds in offsets: the sequence is skipped, others are computed, the status word says so
    td = torch.bfloat16
    q = _randn((300, 2, 64), td, 1)
    good = torch.tensor([0, 100, 200, 300], dtype=torch.int32, device="cuda")
    want, _ = sdrop.sdrop_attn(q, q, q, cu_q=good, cu_k=good, max_q=100, max_k=100)
    for cu in ([0, 100, 50, 300], [0, 100, 200, 301], [-5, 100, 200, 300]):
        bad = torch.tensor(cu, dtype=torch.int32, device="cuda")
        out = torch.full_like(q, 7.0)
        sdrop.sdrop_attn(q, q, q, cu_q=bad, cu_k=bad, max_q=100, max_k=100, out=out)
        assert sdrop.status() == sdrop.STATUS_BAD_LENGTHS and sdrop.status() == 0
        for b in range(3):
            a, e = cu[b], cu[b + 1]
            if (a, e) == (100 * b, 100 * b + 100):
                assert torch.equal(out[a:e], want[a:e])
        assert bool((out[200:] == 7.0).all()) if cu[3] == 301 else True
    kl = torch.tensor([5, -1, 51], dtype=torch.int32, device="cuda")
    x = _randn((3, 50, 2, 64), td, 2)
    out = torch.full_like(x, 7.0)
    sdrop.sdrop_attn(x, x, x, k_len=kl, out=out)
    assert sdrop.status() == sdrop.STATUS_BAD_LENGTHS
    assert bool((out[1:] == 7.0).all()) and torch.equal(out[0], sdrop.sdrop_attn(x[:1], x[:1, :5], x[:1, :5])[0][0])


def test_offsets_beyond_32_bits():
    # a cache of 9.7 GB: the last sequences lie behind 2^32 elements
    td = torch.bfloat16
    B, T, H, D = 9, 33000, 128, 128
    kv = torch.empty((B, T, H, D), dtype=td, device="cuda").normal_()
    q = _randn((B, 1, H, D), td, 1)
    n = torch.full((B,), 700, dtype=torch.int32, device="cuda")
    n[-1] = T
    o, lse = sdrop.sdrop_attn(q, kv, kv, k_len=n)
    for b, L in ((0, 700), (B - 2, 700), (B - 1, T)):
        _check(q[b, :, 124:], kv[b, :L, 124:], kv[b, :L, 124:], None, False, td, (o[b, :, 124:],), lse[b, 124:], "b=%d" % b)
    # heads far apart: [H, T, D] order
    x = kv[B - 1:].transpose(1, 2)
    o2, _ = sdrop.sdrop_attn(q[B - 1:, :, :1], kv[B - 1:, :, 127:], kv[B - 1:, :, 127:])
    _check(q[B - 1, :, :1], kv[B - 1, :, 127:], kv[B - 1, :, 127:], None, False, td, (o2[0],), None, "last head")


@pytest.mark.parametrize("B,T", [(1, 300), (64, 100)])
def test_gradients_of_heads_far_apart(B, T):
    # the two query heads of a key head 2 GiB apart: the same bits as side by side
    td = torch.bfloat16
    D, far = 64, 1 << 30
    q, do = _randn((B, T, 2, D), td, 1), _randn((B, T, 2, D), td, 2)
    k, v = _randn((B, T, 1, D), td, 3), _randn((B, T, 1, D), td, 4)
    apart = []
    for t in (q, do, q):
        x = torch.empty(far + B * T * D, dtype=td, device="cuda").as_strided(t.shape, (T * D, D, far, 1))
        x.copy_(t)
        apart.append(x)
    o, lse, rest = sdrop.sdrop_attn(q, k, v, True, need_rest=True)
    want = sdrop.sdrop_attn_bwd(do, q, k, v, o, lse, True, rest=rest)
    o2, lse2, rest2 = sdrop.sdrop_attn(apart[0], k, v, True, need_rest=True)
    got = sdrop.sdrop_attn_bwd(apart[1], apart[0], k, v, o2, lse2, True, rest=rest2, out_dq=apart[2])
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    for b in {0, B - 1}:
        _check(q[b], k[b], v[b], do[b], True, td, [t[b] for t in (o,) + want], lse[b], "b=%d" % b)


def test_results_repeat_on_another_stream_and_in_a_graph():
    td = torch.bfloat16
    q, do, k, v = _randn((2, 300, 4, 128), td, 1), _randn((2, 300, 4, 128), td, 2), _randn((2, 300, 2, 128), td, 3), _randn((2, 300, 2, 128), td, 4)
    cache_k, cache_v = _randn((2, 4000, 2, 128), td, 5), _randn((2, 4000, 2, 128), td, 6)

    def step():
        o, lse, rest = sdrop.sdrop_attn(q, k, v, True, need_rest=True)
        return (o, lse, rest[:, :128].clone()) + sdrop.sdrop_attn_bwd(do, q, k, v, o, lse, True, rest=rest) + (sdrop.sdrop_attn(q[:, :1], cache_k, cache_v)[0],)

    ref = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(ref, other):
        assert torch.equal(a, b)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = step()
    for _ in range(3):
        for o in outs:
            o.fill_(7.0)
        step()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for o, r in zip(outs, ref):
            assert torch.equal(o, r)


def test_block_of_operators_trains():
    # a pre-norm block's operators in a row, with torch's linear layers between them: gradients against the same graph in float64
    td = torch.float16
    B, T, d, H = 2, 65, 128, 2
    ws = [_randn((3 * d, d), td, 1, 0.08), _randn((d, d), td, 2, 0.08), _randn((d,), td, 3, 0.1) + 1, _randn((d,), td, 4, 0.1)]
    x = _randn((B, T, d), td, 5)
    do = _randn((B, T, d), td, 6)
    keep = torch.from_numpy(orc.element_keep(B * T, d, 0.25, 3, 1)).view(B, T, d)

    def native(x, wq, wp, g, b):
        n = tr.layer_norm(x, g, b)
        qkv = (n @ wq.t()).view(B, T, 3 * H, d // H)
        a = tr.attention(qkv[:, :, :H], qkv[:, :, H:2 * H], qkv[:, :, 2 * H:], causal=True).reshape(B, T, d)
        y, h = tr.dropout_add_norm(a @ wp.t(), x, g, b, 0.25, 1e-5, 3, 1)
        return y + h

    def plain(x, wq, wp, g, b):
        n = torch.nn.functional.layer_norm(x, (d,), g, b)
        q, k, v = (n @ wq.t()).view(B, T, 3, H, d // H).permute(2, 0, 3, 1, 4)
        s = (q @ k.transpose(2, 3)) * (d // H) ** -0.5
        s = s.masked_fill(torch.ones(T, T, dtype=torch.bool).triu(1), float("-inf"))
        a = (torch.softmax(s, -1) @ v).transpose(1, 2).reshape(B, T, d)
        h = x + (a @ wp.t()) * keep / 0.75
        return torch.nn.functional.layer_norm(h, (d,), g, b) + h

    leaves = [t.detach().requires_grad_() for t in [x] + ws]
    ref = [t.detach().cpu().double().requires_grad_() for t in leaves]
    y, yr = native(*leaves), plain(*ref)
    got, want = torch.autograd.grad(y, leaves, do), torch.autograd.grad(yr, ref, do.cpu().double())
    # the longest chain rounds about 12 times to fp16
    tol = 12 * torch.finfo(td).eps
    for a, b in [(y, yr)] + list(zip(got, want)):
        assert (a.detach().cpu().double() - b.detach()).norm() <= tol * b.detach().norm()


def test_block_captured_with_its_backward_pass():
    # all operators and their gradients through autograd, captured; no eager graph of the leaves lives meanwhile
    td = torch.bfloat16
    B, T, H, D = 2, 150, 4, 64
    x, r = _randn((B, T, 3 * H * D), td, 1).requires_grad_(), _randn((B, T, H * D), td, 2).requires_grad_()
    w3, w1 = _randn((3 * H * D,), td, 3).requires_grad_(), _randn((H * D,), td, 4).requires_grad_()
    gy, gz = _randn((B, T, H * D), td, 5), _randn((B, T, H * D), td, 6)
    leaves = (x, r, w3, w1)

    def step():
        a = tr.qkv_attention(tr.layer_norm(x, w3).view(B, T, 3 * H, D), H, causal=True).view(B, T, H * D)
        y, h = tr.dropout_add_norm(a, r, w1, None, 0.2, 1e-5, 7, 8)
        z = tr.dropout(y, 0.3, 7, 9, residual=h)
        return [y.detach(), z.detach()] + list(torch.autograd.grad((y, z), leaves, (gy, gz)))

    ref = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, c in zip(ref, other):
        assert torch.equal(a, c)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = step()
    for _ in range(3):
        for o in outs:
            o.fill_(7.0)
        step()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for o, c in zip(outs, ref):
            assert torch.equal(o, c)


def test_gradients_refuse_to_be_differentiated_again():
    x = _randn((2, 20, 6, 64), torch.bfloat16, 1).requires_grad_()
    w = _randn((64,), torch.bfloat16, 2).requires_grad_()
    forms = [lambda: tr.dropout(x, 0.5, 1), lambda: tr.layer_norm(x, w), lambda: tr.dropout_add_norm(x, x, w, None, 0.5)[0],
             lambda: tr.attention(x, x, x), lambda: tr.qkv_attention(x, 2)]
    for f in forms:
        y = f()
        g, = torch.autograd.grad((y * y).sum(), x, create_graph=True)
        plain, = torch.autograd.grad((f().detach() * 2 * f()).sum(), x)
        assert g.requires_grad and torch.equal(g, plain)
        with pytest.raises(RuntimeError, match="differentiated once"):
            torch.autograd.grad(g.sum(), x)
        with pytest.raises(RuntimeError, match="differentiated once"):
            g.sum().backward()


def test_two_streams_at_once():
    # two calls that overlap, each with partial results of its own
    td = torch.float16
    q, k, v = _randn((1, 1, 8, 128), td, 1), _randn((1, 30000, 8, 128), td, 2), _randn((1, 30000, 8, 128), td, 3)
    want = [sdrop.sdrop_attn(q, k, v)[0], sdrop.sdrop_attn(q, v, k)[0]]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(8):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(sdrop.sdrop_attn(q, *((k, v) if i == 0 else (v, k)))[0])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(t, want[i]) for t in got[i])
