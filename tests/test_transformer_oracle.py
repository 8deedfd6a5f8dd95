"""The float64 definitions of the operators around the substituted layers (arxiv 2411.01238, Sections 2.1 and 4.2): the generator
against published vectors, the rest against differences."""
import os

import numpy as np
import pytest

from oracle import transformer_oracle as orc

HERE = os.path.dirname(os.path.abspath(__file__))


def test_generator_matches_the_published_vectors():
    n = 0
    for line in open(os.path.join(HERE, "golden", "philox4x32_10_kat.txt")):
        v = [int(x, 16) for x in line.split("#")[0].replace("philox4x32", "").split() if len(x) == 8]
        if len(v) != 10:
            continue
        got = orc.philox4x32([np.array([x]) for x in v[:4]], v[4:6])
        assert [int(g[0]) for g in got] == v[6:]
        n += 1
    assert n >= 3


def test_mask_rate_chunks_and_independence():
    keep = orc.element_keep(400, 1000, 0.3, 7, 2)
    assert abs(keep.mean() - 0.7) < 4 * np.sqrt(0.21 / keep.size)
    # a row's mask does not depend on the rows before it, and other seeds, streams and columns give other masks
    assert np.array_equal(orc.element_keep(400, 1000, 0.3, 7, 2, rows=[399]), keep[399:])
    for other in (orc.element_keep(400, 1000, 0.3, 8, 2), orc.element_keep(400, 1000, 0.3, 7, 3), orc.element_keep(400, 1000, 0.3, 7 + (1 << 32), 2)):
        assert abs((other != keep).mean() - 0.42) < 0.01
    assert orc.element_keep(3, 9, 0.0, 1).all() and not orc.element_keep(3, 9, 1.0, 1).any()
    assert orc.element_scale(0.5) == 2.0 and orc.element_scale(1.0) == 0.0 and orc.element_scale(0.0) == 1.0


def _difference(f, x, i, e):
    a, b = x.copy(), x.copy()
    a.flat[i] += e
    b.flat[i] -= e
    return (f(a) - f(b)) / (2 * e)


def test_layer_norm_gradients_against_differences():
    r = np.random.RandomState(0)
    h, g, b, dy, dh = r.randn(5, 13), 1 + 0.1 * r.randn(13), r.randn(13), r.randn(5, 13), r.randn(5, 13)
    dr, dg, db = orc.layer_norm_bwd(dy, h, g, 1e-5, dh)
    for i in range(h.size):
        want = _difference(lambda t: (orc.layer_norm(t, g, b, 1e-5)[0] * dy).sum() + (t * dh).sum(), h, i, 1e-5)
        assert dr.flat[i] == pytest.approx(want, abs=1e-7)
    for i in range(13):
        assert dg[i] == pytest.approx(_difference(lambda t: (orc.layer_norm(h, t, b, 1e-5)[0] * dy).sum(), g, i, 1e-5), abs=1e-7)
        assert db[i] == pytest.approx(_difference(lambda t: (orc.layer_norm(h, g, t, 1e-5)[0] * dy).sum(), b, i, 1e-5), abs=1e-7)


@pytest.mark.parametrize("Tq,Tk,causal", [(5, 5, True), (4, 7, True), (6, 3, True), (3, 4, False), (1, 6, True)])
def test_attention_and_its_gradients_against_differences(Tq, Tk, causal):
    r = np.random.RandomState(1)
    q, k, v, do = r.randn(Tq, 4, 3), r.randn(Tk, 2, 3), r.randn(Tk, 2, 3), r.randn(Tq, 4, 3)
    o, lse = orc.attention(q, k, v, 0.7, causal)
    for i in range(Tq):
        n = min(Tk, i + Tk - Tq + 1) if causal else Tk
        if n <= 0:
            assert not o[i].any() and np.all(np.isneginf(lse[:, i]))
            continue
        s = 0.7 * np.einsum("hd,jd->hj", q[i, :2], k[:n, 0])            # the first two query heads read the first key head
        assert np.allclose(lse[:2, i], np.log(np.exp(s).sum(axis=1)))
        assert np.allclose(o[i, :2], np.exp(s) / np.exp(s).sum(axis=1, keepdims=True) @ v[:n, 0])
    grads = orc.attention_bwd(do, q, k, v, 0.7, causal)
    for which, (x, g) in enumerate(zip((q, k, v), grads)):
        def f(t, which=which):
            a = [q, k, v]
            a[which] = t
            return (orc.attention(*a, 0.7, causal)[0] * do).sum()
        for i in range(x.size):
            assert g.flat[i] == pytest.approx(_difference(f, x, i, 1e-6), abs=1e-7)
