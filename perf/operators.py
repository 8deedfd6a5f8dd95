"""The operators around the substituted layers of a transformer block, as a list of timed cases: element dropout, layer norm
(alone, and with the dropout and the residual add in front of it) and attention.

A case is one pass of one of the library's public paths:

    dropout    y = r + m x / (1 - p) through autograd: forward and backward.  m is drawn from a counter-based generator and
               never stored; r (the residual) may be missing
    norm       layer norm through autograd: forward, and backward with the gradients of weight and bias
    add_norm   h = r + m x / (1 - p), y = norm(h): the two outputs, and the backward from the gradients of both
    attn       attention through autograd: forward and backward, causal or not, grouped heads, dense or packed sequences
    prompt     the same, forward only (inference)
    decode     one new token per sequence against a padded key / value cache, through the binding

Rows x features, types and head sizes are those of the models in model_step.py (width 1024, feed-forward 4096, 8 heads of 128,
batches of 32 x 128 and 64 x 256 tokens) and of the tests, and generic ones around them.

The plain forms below are the definitions in elementary operations.  The dropout's mask is part of the definition: Philox4x32-10
with one call per 8 consecutive elements of a row, 16 random bits each, an element kept where they are >= round(65536 p).
"""
import math
import random

import torch

own = False

_DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"f16": 2, "bf16": 2, "f32": 4}
_EPS = 1e-5


def _rows(name, path, M, N, dtype, p=0.0, residual=False):
    c = {"path": path, "M": M, "N": N, "dtype": dtype}
    if path != "norm":
        c["p"] = p
    if path == "dropout":
        c["residual"] = residual
    return dict(c, name=name) if name else c


def _attn(name, path, B, T, Hq, Hkv, D, dtype, causal=True, packed=False, lens=0):
    """B sequences of T tokens; packed: B sequences of 1 .. T tokens one behind the other; decode: T is the cache's length, of
    which every sequence has filled its own part.  lens: seed of the ragged lengths."""
    c = {"path": path, "B": B, "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "dtype": dtype}
    if path != "decode":
        c["causal"], c["packed"] = causal, packed
    if path == "decode" or packed:
        c["lens"] = lens
    return dict(c, name=name) if name else c


def listed():
    return [
        # the input of a classifier's hidden layer in the smallest batch of the tests: launches are all of it
        _rows("dropout_small", "dropout", 256, 1024, "bf16", 0.5),
        # what the dropout_dense variant of the ViT puts in front of its second feed-forward layer
        _rows("dropout_ffn_hidden", "dropout", 16384, 4096, "bf16", 0.1),
        # a norm of a small GPT batch in fp32
        _rows("norm_small_f32", "norm", 512, 384, "f32"),
        # the final norm of the character GPT
        _rows("norm_gpt", "norm", 4096, 1024, "f16"),
        # residual dropout, add and norm of the ViT's blocks
        _rows("add_norm_vit", "add_norm", 16384, 1024, "bf16", 0.1),
        # a wider model, rows and features that are no multiple of anything, fp32 (no 16-byte rows)
        _rows("add_norm_odd_f32", "add_norm", 8191, 2501, "f32", 0.3),
        # attention of the character GPT at its own batch: many short causal sequences
        _attn("attn_gpt", "attn", 32, 128, 8, 8, 128, "bf16"),
        # the ViT's: 256 tokens, no mask
        _attn("attn_vit", "attn", 64, 256, 8, 8, 128, "bf16", causal=False),
        # documents of different lengths packed into one row of tokens, grouped heads
        _attn("attn_packed_grouped", "attn", 12, 2048, 16, 4, 64, "f16", packed=True, lens=1),
        # one long document, training
        _attn("attn_long", "attn", 1, 8192, 16, 8, 128, "bf16"),
        # a batch of prompts before generation, forward only
        _attn("prompt_batch", "prompt", 4, 4000, 16, 4, 128, "bf16"),
        # generation: one token a sequence, caches of up to 16384 tokens
        _attn("decode_cache", "decode", 16, 16384, 32, 8, 128, "bf16", lens=2),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / 1e15)


def draw(rng):
    """One more case: the paths, types and shapes of the listed ones over the ranges between and around them."""
    largest = max(_cost(c) for c in listed())
    while True:
        path = rng.choice(("dropout", "norm", "add_norm", "attn", "attn", "prompt", "decode"))
        dtype = rng.choice(("bf16", "bf16", "f16"))
        if path in ("dropout", "norm", "add_norm"):
            M = max(1, round(_log_uniform(rng, 64, 32768)))
            # widths are mostly whole multiples of 64; some are odd
            N = _log_uniform(rng, 64, 8192)
            N = max(1, round(N / 64)) * 64 if rng.random() < 0.7 else max(3, round(N))
            c = _rows("", path, M, N, rng.choice((dtype, dtype, "f32")), rng.choice((0.1, 0.1, 0.2, 0.5)), rng.random() < 0.5)
        else:
            Hkv = rng.choice((1, 2, 4, 8))
            Hq = Hkv * rng.choice((1, 1, 2, 4, 5, 8))
            D = rng.choice((64, 64, 128, 128, 128, 32, 80, 96))
            T = max(16, round(_log_uniform(rng, 32, 8192)))
            if path == "decode":
                T = max(16, round(_log_uniform(rng, 256, 32768)))
            B = max(1, round(_log_uniform(rng, 1, 64)))
            c = _attn("", path, B, T, Hq, Hkv, D, dtype, causal=rng.random() < 0.7, packed=rng.random() < 0.4, lens=rng.randrange(1000))
            if path != "decode" and 4.0 * Hq * (B * T * T if not c["packed"] else sum(_lengths(c)) ** 2) > 5e9:
                continue        # (the plain form keeps the scores of all heads)
        if _cost(c) <= largest:
            return c


def _lengths(c):
    r = random.Random(c["lens"])
    return [r.randint(max(1, c["T"] // 4) if c["path"] == "decode" else 1, c["T"]) for _ in range(c["B"])]


def _normal(shape, g, std, dtype):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g).to(dtype)


def prepare(case, seed):
    dt = _DT[case["dtype"]]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case, "seed": seed}
    if case["path"] in ("dropout", "norm", "add_norm"):
        M, N = case["M"], case["N"]
        s["x"] = _normal((M, N), g, 1.0, dt).requires_grad_(True)
        s["dy"] = _normal((M, N), g, 1.0, dt)
        if case.get("residual") or case["path"] == "add_norm":
            s["r"] = _normal((M, N), g, 1.0, dt).requires_grad_(True)
        if case["path"] != "dropout":
            s["gamma"] = (1.0 + _normal((N,), g, 0.1, torch.float32)).to(dt).requires_grad_(True)
            s["beta"] = _normal((N,), g, 0.1, dt).requires_grad_(True)
        if case["path"] == "add_norm":
            s["dh"] = _normal((M, N), g, 1.0, dt)       # what the rest of the residual stream sends back
        return s
    B, T, Hq, Hkv, D = (case[k] for k in ("B", "T", "Hq", "Hkv", "D"))
    if case["path"] == "decode":
        s["q"] = _normal((B, 1, Hq, D), g, 1.0, dt)
        s["k"], s["v"] = _normal((B, T, Hkv, D), g, 1.0, dt), _normal((B, T, Hkv, D), g, 1.0, dt)
        s["k_len"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
        return s
    lead = (B, T)
    if case["packed"]:
        lens = _lengths(case)
        ends = [0]
        for n in lens:
            ends.append(ends[-1] + n)
        s["cu"], s["max"] = torch.tensor(ends, dtype=torch.int32, device="cuda"), max(lens)
        lead = (ends[-1],)
    # query, key and value heads of a token lie side by side, as one projection writes them
    qkv = _normal(lead + (Hq + 2 * Hkv, D), g, 1.0, dt)
    s["q"], s["k"], s["v"] = qkv[..., :Hq, :], qkv[..., Hq:Hq + Hkv, :], qkv[..., Hq + Hkv:, :]
    if case["path"] == "attn":
        s["q"], s["k"], s["v"] = (t.detach().requires_grad_(True) for t in (s["q"], s["k"], s["v"]))
        s["do"] = _normal(lead + (Hq, D), g, 1.0, dt)
    return s


# ---- the plain forms ----

def _mulhi(a, b):
    """High word of the product of two 32-bit numbers held in 64-bit integers (a full product would pass 63 bits)."""
    return (a * (b >> 16) + ((a * (b & 0xFFFF)) >> 16)) >> 16


def _keep_scale(M, N, p, seed, rng_stream, device):
    """The dropout's mask [M, N] and its scale.  Counter of 8-element chunk c of a row: (its number over all rows, with the top
    bit of the 64 set; rng_stream), key: seed."""
    chunks = (N + 7) // 8
    c = torch.arange(M * chunks, dtype=torch.int64, device=device)
    low = 0xFFFFFFFF
    x = [c & low, (c >> 32) | 0x80000000, torch.full_like(c, rng_stream & low), torch.full_like(c, rng_stream >> 32)]
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):
        h0, l0 = _mulhi(0xD2511F53, x[0]), (0xD2511F53 * x[0]) & low
        h1, l1 = _mulhi(0xCD9E8D57, x[2]), (0xCD9E8D57 * x[2]) & low
        x = [h1 ^ x[1] ^ k0, l1, h0 ^ x[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    bits = torch.stack([h for w in x for h in (w & 0xFFFF, w >> 16)], dim=-1).reshape(M, chunks * 8)[:, :N]
    t = 65536 if p >= 1.0 else min(65535, int(p * 65536.0 + 0.5))
    return bits >= t, (65536.0 / (65536 - t) if t < 65536 else 0.0)


def _norm_forward(h, gamma, beta):
    mu = h.mean(dim=1, keepdim=True)
    d = h - mu
    rstd = torch.rsqrt((d * d).mean(dim=1, keepdim=True) + _EPS)
    return d * rstd, rstd, d * rstd * gamma + beta


def _norm_backward(dy, xh, rstd, gamma):
    w = dy * gamma
    dh = rstd * (w - w.mean(dim=1, keepdim=True) - xh * (w * xh).mean(dim=1, keepdim=True))
    return dh, (dy * xh).sum(dim=0), dy.sum(dim=0)


def _plain_rows(s):
    c, dt = s["case"], s["x"].dtype
    x, dy = s["x"].float(), s["dy"].float()
    if c["path"] == "norm":
        gamma, beta = s["gamma"].float(), s["beta"].float()
        xh, rstd, y = _norm_forward(x, gamma, beta)
        return [t.to(dt) for t in (y,) + _norm_backward(dy, xh, rstd, gamma)]
    keep, scale = _keep_scale(c["M"], c["N"], c["p"], s["seed"], 1, x.device)
    m = keep * scale
    if c["path"] == "dropout":
        return [(s["r"].float() + x * m if "r" in s else x * m).to(dt), (dy * m).to(dt)]
    gamma, beta = s["gamma"].float(), s["beta"].float()
    h = (s["r"].float() + x * m).to(dt)          # the residual stream is a tensor of its own, of this type
    xh, rstd, y = _norm_forward(h.float(), gamma, beta)
    dh, dg, db = _norm_backward(dy, xh, rstd, gamma)
    dr = dh + s["dh"].float()
    return [y.to(dt), h] + [t.to(dt) for t in (dr * m, dr, dg, db)]


def _allowed(s, device):
    """[.., Tq, Tk]: may this query see this key?  None: every one."""
    c = s["case"]
    if c["path"] == "decode":
        return (torch.arange(c["T"], device=device)[None, :] < s["k_len"][:, None])[:, None, None, :]
    if c["packed"]:
        n = s["q"].shape[0]
        at = torch.arange(n, device=device)
        seq = torch.bucketize(at, s["cu"][1:].to(torch.int64), right=True)
        ok = seq[:, None] == seq[None, :]
        return ok & (at[:, None] >= at[None, :]) if c["causal"] else ok
    if c["causal"]:
        at = torch.arange(c["T"], device=device)
        return at[:, None] >= at[None, :]
    return None


def _plain_attn(s):
    c, dt = s["case"], s["q"].dtype
    group = c["Hq"] // c["Hkv"]
    heads = lambda t: (t if t.dim() == 4 else t[None]).float().transpose(1, 2).contiguous()     # noqa: E731  [B, H, T, D]
    q, k, v = heads(s["q"]), heads(s["k"]), heads(s["v"])
    B, Hq, Tq, D = q.shape
    # grouped heads: the queries of a group one below the other, against the same keys
    q = q.reshape(B, c["Hkv"], group * Tq, D)
    ok = _allowed(s, q.device)
    scores = (torch.matmul(q, k.transpose(2, 3).contiguous()) * D ** -0.5).view(B, c["Hkv"], group, Tq, -1)
    if ok is not None:
        scores = scores.masked_fill(~(ok[:, :, None] if ok.dim() == 4 else ok), -math.inf)
    e = torch.exp(scores - scores.amax(dim=-1, keepdim=True))
    del scores
    p = (e / e.sum(dim=-1, keepdim=True)).view(B, c["Hkv"], group * Tq, -1)
    del e
    o = torch.matmul(p, v)
    back = lambda t, H: t.reshape(B, H, -1, D).transpose(1, 2).reshape((B, -1, H, D) if s["q"].dim() == 4 else (-1, H, D)).to(dt)   # noqa: E731
    if c["path"] != "attn":
        return [back(o, Hq)]
    do = heads(s["do"]).reshape(B, c["Hkv"], group * Tq, D)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = p * (ds - (do * o).sum(dim=-1, keepdim=True))
    del p
    dq = torch.matmul(ds, k) * D ** -0.5
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q) * D ** -0.5
    return [back(o, Hq), back(dq, Hq), back(dk, c["Hkv"]), back(dv, c["Hkv"])]


# ---- the framework's calls ----

def _own(s):
    from paper_2411_01238_amd import sdrop, transformer
    c = s["case"]
    path = c["path"]
    if path == "dropout":
        y = transformer.dropout(s["x"], c["p"], s["seed"], 1, residual=s.get("r"))
        return [y.detach(), torch.autograd.grad(y, s["x"], s["dy"])[0]]
    if path == "norm":
        y = transformer.layer_norm(s["x"], s["gamma"], s["beta"], _EPS)
        return [y.detach()] + list(torch.autograd.grad(y, (s["x"], s["gamma"], s["beta"]), s["dy"]))
    if path == "add_norm":
        y, h = transformer.dropout_add_norm(s["x"], s["r"], s["gamma"], s["beta"], c["p"], _EPS, s["seed"], 1)
        return [y.detach(), h.detach()] + list(torch.autograd.grad((y, h), (s["x"], s["r"], s["gamma"], s["beta"]), (s["dy"], s["dh"])))
    if path == "decode":
        return [sdrop.sdrop_attn(s["q"], s["k"], s["v"], k_len=s["k_len"])[0]]
    packed = dict(cu_q=s["cu"], cu_k=s["cu"], max_q=s["max"], max_k=s["max"]) if c["packed"] else {}
    if path == "prompt":
        return [sdrop.sdrop_attn(s["q"], s["k"], s["v"], causal=c["causal"], **packed)[0]]
    o = transformer.attention(s["q"], s["k"], s["v"], causal=c["causal"], **packed)
    return [o.detach()] + list(torch.autograd.grad(o, (s["q"], s["k"], s["v"]), s["do"]))


def run(s):
    if own:
        return _own(s)
    with torch.no_grad():
        return _plain_rows(s) if "x" in s else _plain_attn(s)


def _pairs(c):
    """Query-key pairs that the mask leaves, over all sequences, for one head."""
    if c["path"] == "decode":
        return sum(_lengths(c))
    lens = _lengths(c) if c["packed"] else [c["T"]] * c["B"]
    return sum(n * (n + 1) // 2 if c["causal"] else n * n for n in lens)


def work(case):
    """Each input read once, each output written once.  Attention: two products of the pairs forward, five backward."""
    sz = _SIZE[case["dtype"]]
    if "M" in case:
        n, w = case["M"] * case["N"], case["N"]
        arrays = {"dropout": 4 + (1 if case.get("residual") else 0), "norm": 4, "add_norm": 8}[case["path"]]
        return {"bytes": float(sz * (arrays * n + (0 if case["path"] == "dropout" else 4 * w))), "flops": 0.0}
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    if case["path"] == "decode":
        rows = sum(_lengths(case))
        return {"bytes": float(sz * D * (2 * Hkv * rows + 2 * Hq * case["B"])), "flops": 4.0 * D * Hq * rows}
    tokens = sum(_lengths(case)) if case["packed"] else case["B"] * case["T"]
    train = case["path"] == "attn"
    return {"bytes": float(sz * D * tokens * ((4 * Hq + 4 * Hkv) if train else 2 * (Hq + Hkv))),
            "flops": (14.0 if train else 4.0) * D * Hq * _pairs(case)}


# ---- the definitions once more, in 64 bits ----

def _philox_bits(counter, seed, rng_stream):
    """Four words per counter.  Products of 32-bit numbers in two halves of 16 bits."""
    def product(a, b):
        lo, hi = a * (b & 0xFFFF), a * (b >> 16)
        t = (lo >> 16) + (hi & 0xFFFF)
        return (hi >> 16) + (t >> 16), ((t & 0xFFFF) << 16) | (lo & 0xFFFF)

    full = lambda v: torch.full_like(counter, v)        # noqa: E731
    w = 2 ** 32
    a, b, c, d = counter % w, counter // w + 2 ** 31, full(rng_stream % w), full(rng_stream // w)
    key = [seed % w, (seed // w) % w]
    for r in range(10):
        (ah, al), (ch, cl) = product(0xD2511F53, a), product(0xCD9E8D57, c)
        u, v = (key[0] + r * 0x9E3779B9) % w, (key[1] + r * 0xBB67AE85) % w
        a, b, c, d = ch ^ b ^ u, cl, ah ^ d ^ v, al
    return a, b, c, d


def _exact_rows(case, s):
    M, N, path = case["M"], case["N"], case["path"]
    dt = _DT[case["dtype"]]
    x, dy = s["x"].detach().double(), s["dy"].double()
    mult, h = 1.0, x
    if path != "norm":
        per_row = -(-N // 8)
        mult = torch.empty((M, N), dtype=torch.float64, device=x.device)
        t = math.floor(case["p"] * 65536 + 0.5)
        counter = torch.arange(per_row, device=x.device)[None, :] + per_row * torch.arange(M, device=x.device)[:, None]
        for i, word in enumerate(_philox_bits(counter, s["seed"], 1)):
            for half in (0, 1):
                n = mult[:, 2 * i + half::8].shape[1]
                u = (word // 65536 if half else word % 65536)[:, :n]
                mult[:, 2 * i + half::8] = torch.where(u >= t, 65536.0 / (65536 - t), 0.0)
        h = x * mult + (s["r"].detach().double() if "r" in s else 0.0)
        if path == "dropout":
            return [h, dy * mult]
        h = h.to(dt).double()
    var, mu = torch.var_mean(h, dim=1, correction=0, keepdim=True)
    s1 = 1.0 / torch.sqrt(var + _EPS)
    z = (h - mu) * s1
    gamma = s["gamma"].detach().double()
    y = z * gamma + s["beta"].detach().double()
    u = dy * gamma
    grad = s1 * (u - (u.sum(1, keepdim=True) + z * (u * z).sum(1, keepdim=True)) / N)
    dg, db = (dy * z).sum(0), dy.sum(0)
    if path == "norm":
        return [y, grad, dg, db]
    grad = grad + s["dh"].double()
    return [y, h, grad * mult, grad, dg, db]


def _exact_attn(case, s):
    """Sequence by sequence and head by head."""
    Hq, Hkv, D, train = case["Hq"], case["Hkv"], case["D"], case["path"] == "attn"
    if case["path"] != "decode" and _pairs(dict(case, causal=False)) * Hq * D * (14 if train else 4) > 2e13:
        return None
    outs = {n: torch.zeros(s[n[-1]].shape, dtype=torch.float64, device="cuda") for n in (("q", "dq", "dk", "dv") if train else ("q",))}
    for b in range(case["B"]):
        if case["path"] == "decode":
            rows, cols = (b, slice(0, 1)), (b, slice(0, int(s["k_len"][b])))
        elif case["packed"]:
            rows = cols = (slice(int(s["cu"][b]), int(s["cu"][b + 1])),)
        else:
            rows = cols = (b, slice(0, case["T"]))
        for h in range(Hq):
            j = h // (Hq // Hkv)
            q, k, v = (s[n].detach()[i + (m,)].double() for n, i, m in (("q", rows, h), ("k", cols, j), ("v", cols, j)))
            a = q @ k.t().contiguous() / math.sqrt(D)
            if case.get("causal"):
                a = a + torch.full_like(a, -math.inf).triu(1)
            p = torch.softmax(a, dim=1)
            o = p @ v
            outs["q"][rows + (h,)] = o
            if train:
                g = s["do"][rows + (h,)].double()
                d = g @ v.t().contiguous()
                d = p * (d - (p * d).sum(1, keepdim=True)) / math.sqrt(D)
                outs["dq"][rows + (h,)] = d @ k
                outs["dk"][cols + (j,)] += d.t().contiguous() @ q
                outs["dv"][cols + (j,)] += p.t().contiguous() @ g
    return list(outs.values())


def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        return _exact_rows(case, s) if "M" in case else _exact_attn(case, s)
