"""Rounding errors of attention's gradients (arxiv 2411.01238, Section 4.2's models) where the usual inputs do not show them: scores so
far apart that a few keys carry a row, and gradients whose products with P are far smaller than fp16's usual numbers.

Tolerances are on norms of the errors.  A rounding is off by at most e = eps / 2 of the value and evenly spread over half a step, so the mean
of its square is at most e^2 / 3, and roundings have signs of their own: in sums the squares add.  What a gradient may have:
    dS                one rounding per value: e^2 / 3 of dS^2
    delta             row sums of dO O.  P is rounded for O, but for keys that have more than half of their row: squared, e^2 / 3 of the sum
                      of the others' (P dP)^2, which reaches every key of the row by P.  O's second part is rounded: e^2 of O
    fp32              sums of 128 products: 128 roundings of 2^-24, below 2^-20 of the magnitudes; P by the error of its score, below 2^-13
                      for scores below 2^7, which reaches dS and delta as a rounding does
    the result        e^2 / 3 of its square, or half a step of fp16's smallest numbers (2^-25), squared, / 3
The square of an even error has a mean of 1 / 3 of the largest and a variance of 1 / 5 - 1 / 9: over n values the mean of the squares is off by a
share of sqrt(0.8 / n), and four of these are allowed.
The mantissas of usual values are larger than 1: the mean square of a rounding is 0.18 e^2 for them, so that 0.74 of these tolerances is what
an implementation with exactly these errors shows.
"""
import numpy as np
import pytest
import torch

from paper_2411_01238_amd import sdrop
from _util import f64

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}


def head_bounds(q, k, v, do, scale, causal, e):
    """One head in float64: ((dq, dk, dv), and the mean square of the error allowed in each row of dq, in each of dk, without the result's
    own rounding)."""
    s = scale * (q @ k.T)
    if causal:
        i, j = np.arange(q.shape[0])[:, None], np.arange(k.shape[0])[None, :]
        s = np.where(j <= i + k.shape[0] - q.shape[0], s, -np.inf)
    top = s.max(axis=1, keepdims=True)
    p = np.exp(s - np.where(np.isfinite(top), top, 0.0))
    p /= np.maximum(p.sum(axis=1, keepdims=True), 1e-300)           # (a row that sees no key has P = 0)
    o, dp = p @ v, do @ v.T
    delta = (do * o).sum(axis=1, keepdims=True)
    ds = p * (dp - delta)
    grads = scale * (ds @ k), scale * (ds.T @ q), p.T @ do
    small = 2.0 ** -13
    arith = 2.0 ** -20 * p * (np.abs(do) @ np.abs(v).T + (np.abs(do) * np.abs(o)).sum(axis=1, keepdims=True))
    rounded = e ** 2 / 3 + small ** 2
    row = rounded * (np.where(p > 0.5, ds, p * dp) ** 2).sum(axis=1) + e ** 4 * ((do * o) ** 2).sum(axis=1)         # delta's error, squared
    own = rounded * ds ** 2 + arith ** 2
    k2, q2 = (k ** 2).sum(axis=1), (q ** 2).sum(axis=1)
    return grads, (scale ** 2 * (own @ k2 + row * ((p @ k) ** 2).sum(axis=1)), scale ** 2 * (own.T @ q2 + (p ** 2).T @ (row * q2)))


def check_heads(q, k, v, do, got, causal, dtype, what, scale=None, some=None, rows=slice(None), keys=slice(None)):
    """got: (dq, dk, dv), [B, T, H, D] each; one key head per query head.  rows, keys: those of dq and of dk that are looked at."""
    e, tiny = torch.finfo(dtype).eps / 2, 2.0 ** -25 if dtype == torch.float16 else 0.0
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    for b, h in (some or [(b, h) for b in range(q.shape[0]) for h in range(q.shape[2])]):
        qd, kd, vd, gd = (f64(t[b, :, h]) for t in (q, k, v, do))
        want, allow = head_bounds(qd, kd, vd, gd, scale, causal, e)
        for name, at, g, w, a in zip(("dq", "dk"), (rows, keys), got, want, allow):
            w = w[at]
            err = np.linalg.norm(f64(g[b, :, h])[at] - w)
            bound = np.sqrt((a[at].sum() + e ** 2 / 3 * (w ** 2).sum() + tiny ** 2 / 3 * w.size) * (1 + 4 * np.sqrt(0.8 / w.size)))
            assert err <= bound, "%s, b=%d h=%d, %s: error %.3g of its bound (%.3g of the gradient)" % (what, b, h, name, err / bound, err / np.linalg.norm(w))


def randn(shape, dtype, seed, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * std).to(dtype).cuda()


def gradients(q, k, v, do, causal, scale=None, **kw):
    o, lse, rest = sdrop.sdrop_attn(q, k, v, causal, scale, need_rest=True, **kw)
    return sdrop.sdrop_attn_bwd(do, q, k, v, o, lse, causal, scale, rest=rest, **kw)


# two launches on tiles of 64 and of 128, sequences that one workgroup takes whole, few rows over parts of the keys
SHAPES = [(1, 1024, 1024, 2, 128, True), (2, 700, 700, 3, 64, False), (4, 1000, 1000, 16, 64, False), (32, 250, 250, 4, 128, True), (64, 200, 256, 2, 64, False), (1, 16, 4096, 2, 128, True)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("std", [1, 3, 10])
@pytest.mark.parametrize("B,Tq,Tk,H,D,causal", SHAPES)
def test_gradients_where_few_keys_carry_a_row(B, Tq, Tk, H, D, causal, std, dtype):
    print("scores of deviation", std, B, Tq, Tk, H, D, causal, dtype, flush=True)
    td = DT[dtype]
    q, k = randn((B, Tq, H, D), td, 1, std ** 0.5), randn((B, Tk, H, D), td, 2, std ** 0.5)
    v, do = randn((B, Tk, H, D), td, 3), randn((B, Tq, H, D), td, 4)
    check_heads(q, k, v, do, gradients(q, k, v, do, causal), causal, td, "deviation %d" % std, some=[(0, 0), (B - 1, H - 1), (B // 2, H // 2)])
    assert sdrop.status() == 0


# two launches on tiles of 64 and of 128, sequences that one workgroup takes whole
SMALL = [(1, 2048, 2048, 2, 64, False), (4, 3000, 3000, 16, 64, True), (1, 3000, 3000, 2, 128, False), (4, 1000, 1000, 16, 128, False), (64, 256, 256, 2, 128, False),
         (64, 256, 256, 2, 64, True), (64, 128, 128, 2, 64, False)]


@pytest.mark.parametrize("size", [1e-2, 1e-3, 1e-5, 200.0])
@pytest.mark.parametrize("B,Tq,Tk,H,D,causal", SMALL)
def test_fp16_gradients_of_any_size(B, Tq, Tk, H, D, causal, size):
    # dS is far below fp16's smallest usual number (2^-14), or above its largest; the results are not
    print("gradients of deviation", size, B, Tq, Tk, H, D, causal, flush=True)
    td = torch.float16
    q, k, v = randn((B, Tq, H, D), td, 1), randn((B, Tk, H, D), td, 2), randn((B, Tk, H, D), td, 3, 20.0 if size > 1 else 1.0)
    do = randn((B, Tq, H, D), td, 4, size)
    check_heads(q, k, v, do, gradients(q, k, v, do, causal), causal, td, "dO of %g" % size, some=[(0, 0), (B - 1, H - 1)])


@pytest.mark.parametrize("B,Tq,Tk,H,D,causal", SMALL)
def test_fp16_gradients_of_different_sizes_in_one_call(B, Tq, Tk, H, D, causal):
    # rows of dO from 1 down to 2^-10 and up again, in runs of 37: each size's rows by themselves
    print("mixed", B, Tq, Tk, H, D, causal, flush=True)
    td = torch.float16
    q, k, v = randn((B, Tq, H, D), td, 1), randn((B, Tk, H, D), td, 2), randn((B, Tk, H, D), td, 3)
    power = np.array([0, -10, -3, -6])[np.arange(Tq) // 37 % 4]
    do = (randn((B, Tq, H, D), torch.float32, 4) * torch.tensor(2.0 ** power, dtype=torch.float32, device="cuda")[None, :, None, None]).to(td)
    got = gradients(q, k, v, do, causal)
    for n in (0, -3, -6, -10):
        check_heads(q, k, v, do, got, causal, td, "rows of 2^%d" % n, some=[(0, 0), (B - 1, H - 1)], rows=power == n)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("B,Tq,Tk,H,D,causal", [s for s in SMALL if s[5]] + [(1, 2048, 2048, 2, 128, True), (64, 200, 200, 2, 128, True)])
def test_fp16_rows_that_are_not_finite_reach_no_other(B, Tq, Tk, H, D, causal, bad):
    print("not finite", bad, B, Tq, Tk, H, D, flush=True)
    td = torch.float16
    q, k, v, do = randn((B, Tq, H, D), td, 1), randn((B, Tk, H, D), td, 2), randn((B, Tk, H, D), td, 3), randn((B, Tq, H, D), td, 4, 0.01)
    at = Tq // 3
    whole = do.clone()
    do[:, at, :, 5] = bad
    got = gradients(q, k, v, do, causal)
    assert not bool(torch.isfinite(got[0][:, at]).all())
    # the rows that are on no tile with it, and the keys behind it
    check_heads(q, k, v, whole, got, causal, td, "beside it", some=[(0, 0), (B - 1, H - 1)], rows=np.arange(Tq) != at, keys=np.arange(Tk) >= (at // 128 + 1) * 128)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Tq", [1, 200])
def test_many_keys_of_a_small_share_each(Tq, D):
    # fp16: one key takes half, 16000 others, each of them among fp16's smallest numbers as a share of it, the rest.  A rounding there is
    # at most 2^-25 of the largest P
    td = torch.float16
    T = 16000
    q = torch.zeros((1, Tq, 1, D), dtype=td, device="cuda")
    q[..., 0] = 1.0
    k, v = randn((1, T, 1, D), td, 1), randn((1, T, 1, D), td, 2)
    k[..., 0] = torch.linspace(-10.0, -9.5, T, device="cuda").to(td)[None, :, None]
    k[0, 777, 0, 0] = 0.0
    o, lse = sdrop.sdrop_attn(q, k, v, False, 1.0)
    sc, vd = f64(k)[0, :, 0, 0], f64(v)[0, :, 0]
    p = np.exp(sc)
    want = p @ vd / p.sum()
    e = torch.finfo(td).eps / 2
    bound = e * np.abs(want) + ((np.maximum(e * p, 2.0 ** -25) + 2.0 ** -18 * p) / p.sum()) @ np.abs(vd)
    assert (np.abs(f64(o)[0, :, 0] - want) <= bound).all()
    assert (np.abs(f64(lse)[0, 0] - np.log(p.sum())) <= 2.0 ** -13).all()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("B,Tq,Tk,Hq,Hkv,D", [(2, 1, 9000, 4, 1, 128), (1, 3, 5000, 8, 2, 64), (3, 1, 300, 2, 2, 96)])
def test_few_queries_are_as_exact_as_their_type(B, Tq, Tk, Hq, Hkv, D, dtype):
    # the error is that of rounding the exact result, and of values next to a tie: P's own rounding does not show
    td = DT[dtype]
    q, k, v = randn((B, Tq, Hq, D), td, 1), randn((B, Tk, Hkv, D), td, 2), randn((B, Tk, Hkv, D), td, 3)
    o = f64(sdrop.sdrop_attn(q, k, v, True)[0])
    got = want = 0.0
    for b in range(B):
        for h in range(Hq):
            s = f64(q[b, :, h]) @ f64(k[b, :, h * Hkv // Hq]).T * D ** -0.5
            s[np.arange(Tk)[None, :] > np.arange(Tq)[:, None] + Tk - Tq] = -np.inf
            p = np.exp(s - s.max(axis=1, keepdims=True))
            w = p / p.sum(axis=1, keepdims=True) @ f64(v[b, :, h * Hkv // Hq])
            got += ((o[b, :, h] - w) ** 2).sum()
            want += ((f64(torch.from_numpy(w).to(td)) - w) ** 2).sum()
    assert got <= 1.05 ** 2 * want, np.sqrt(got / want)
