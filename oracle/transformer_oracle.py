"""Float64 definitions of the operators around the substituted layers (arxiv 2411.01238: element dropout of Section 2.1, layer norm
and attention of Section 4.2's models), in numpy, independent of the library's code.  Test infrastructure only."""
import numpy as np

_LOW = np.uint64(0xFFFFFFFF)


def philox4x32(counter, key, rounds=10):
    """Philox4x32 (Salmon et al., SC'11): counter, a sequence of four uint64 arrays of 32-bit words; key, two Python integers."""
    c = [np.asarray(w, dtype=np.uint64) for w in counter]
    k0, k1 = int(key[0]), int(key[1])
    for _ in range(rounds):
        p0, p1 = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & _LOW, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & _LOW]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def element_threshold(p):
    return 65536 if p >= 1.0 else min(65535, int(np.floor(p * 65536 + 0.5)))


def element_keep(M, N, p, seed, rng_stream=0, rows=None):
    """Keep flags of the element dropout, [M, N] (or of the given rows): 16 bits per element, one generator call for 8 elements."""
    rows = np.arange(M) if rows is None else np.asarray(rows)
    per_row = (N + 7) // 8
    c = (rows.astype(np.uint64)[:, None] * np.uint64(per_row) + np.arange(per_row, dtype=np.uint64)[None, :])
    full = lambda v: np.full(c.shape, v, dtype=np.uint64)     # noqa: E731
    w = philox4x32((c & _LOW, (c >> np.uint64(32)) | np.uint64(1 << 31), full(rng_stream & 0xFFFFFFFF), full(rng_stream >> 32)),
                   (seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF))
    halves = np.stack([h for x in w for h in (x & np.uint64(0xFFFF), x >> np.uint64(16))], axis=-1).reshape(len(rows), per_row * 8)
    return halves[:, :N] >= np.uint64(element_threshold(p))


def element_scale(p):
    t = element_threshold(p)
    return 65536.0 / (65536 - t) if t < 65536 else 0.0


def dropout(x, keep, p, residual=None):
    y = np.where(keep, x * element_scale(p), 0.0)
    return y if residual is None else y + residual


def layer_norm(h, gamma, beta, eps):
    """(y, mean, rstd) of the rows of h."""
    mean = h.mean(axis=1)
    rstd = 1.0 / np.sqrt(((h - mean[:, None]) ** 2).mean(axis=1) + eps)
    return (h - mean[:, None]) * rstd[:, None] * gamma + (0.0 if beta is None else beta), mean, rstd


def layer_norm_bwd(dy, h, gamma, eps, dh=None):
    """(dr, dgamma, dbeta): the gradient at h (with dh, what reaches it from elsewhere) and at the weights."""
    _, mean, rstd = layer_norm(h, gamma, None, eps)
    z, w = (h - mean[:, None]) * rstd[:, None], dy * gamma
    dr = rstd[:, None] * (w - w.mean(axis=1, keepdims=True) - z * (w * z).mean(axis=1, keepdims=True))
    return dr if dh is None else dr + dh, (dy * z).sum(axis=0), dy.sum(axis=0)


def _scores(q, k, scale, causal):
    s = scale * (q @ k.T)
    if causal:
        i, j = np.arange(q.shape[0])[:, None], np.arange(k.shape[0])[None, :]
        s = np.where(j <= i + k.shape[0] - q.shape[0], s, -np.inf)
    top = s.max(axis=1, initial=-np.inf)
    ref = np.where(np.isfinite(top), top, 0.0)[:, None]
    e = np.exp(s - ref)
    total = e.sum(axis=1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = np.log(total[:, 0]) + ref[:, 0]
    return e / np.where(total > 0, total, 1.0), lse


def attention(q, k, v, scale, causal):
    """One sequence: q [Tq, Hq, D], k and v [Tk, Hkv, D] -> (o, lse [Hq, Tq]).  A token that sees no key has o = 0, lse = -inf."""
    group = q.shape[1] // k.shape[1]
    o, lse = np.zeros(q.shape), np.zeros((q.shape[1], q.shape[0]))
    for h in range(q.shape[1]):
        p, lse[h] = _scores(q[:, h], k[:, h // group], scale, causal)
        o[:, h] = p @ v[:, h // group]
    return o, lse


def attention_bwd(do, q, k, v, scale, causal):
    """(dq, dk, dv) of that sequence."""
    group = q.shape[1] // k.shape[1]
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for h in range(q.shape[1]):
        j = h // group
        p, _ = _scores(q[:, h], k[:, j], scale, causal)
        dp = do[:, h] @ v[:, j].T
        ds = p * (dp - (p * dp).sum(axis=1, keepdims=True))
        dq[:, h] = scale * (ds @ k[:, j])
        dk[:, j] += scale * (ds.T @ q[:, h])
        dv[:, j] += p.T @ do[:, h]
    return dq, dk, dv
