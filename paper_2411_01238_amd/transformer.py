"""torch.autograd wrappers over the binding for what a transformer block (arxiv 2411.01238, Section 4.2) is made of besides its
linear layers: element dropout, layer norm, and dropout + residual add + layer norm in one pass.  Everything runs in libsdrop's
kernels; this file only wires them into autograd.

The dropout's mask is a function of a seed and a stream number (`rng_stream`: one per call, e.g. a step counter) and is never
stored: the backward pass draws it again.  A captured graph replays the mask of the numbers it was captured with.
"""
import torch

from . import sdrop


def _rows(t):
    """t [.., N] as a matrix whose rows are contiguous (a view where that is possible)."""
    m = t if t.dim() == 2 else t.reshape(-1, t.shape[-1])
    return m if m.stride(1) == 1 or m.shape[1] == 1 else m.contiguous()


def _grad_rows(g):
    # (a gradient that autograd has expanded from fewer values has rows of stride 0)
    g = _rows(g)
    return g if g.shape[0] == 1 or g.stride(0) >= g.shape[1] else g.contiguous()


def _once(backward):
    """once_differentiable, whose own work (a third of a small backward's host time) is left out where no graph is asked for."""
    with_graph = torch.autograd.function.once_differentiable(backward)

    def call(ctx, *grads):
        return (with_graph if torch.is_grad_enabled() else backward)(ctx, *grads)
    return call


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed, rng_stream):
        ctx.args = (p, seed, rng_stream)
        y = sdrop.sdrop_dropout(_grad_rows(x), p, seed, rng_stream, residual=None if residual is None else _grad_rows(residual))
        return y.view(x.shape)

    @staticmethod
    @_once
    def backward(ctx, dy):
        dx = sdrop.sdrop_dropout(_grad_rows(dy), *ctx.args).view(dy.shape) if ctx.needs_input_grad[0] else None
        return dx, dy if ctx.needs_input_grad[1] else None, None, None, None


def dropout(x, p, seed=0, rng_stream=0, residual=None):
    """residual + m . x / (1 - p) with a fresh element mask m (Bernoulli(1 - p), in steps of 2^-16), drawn from (seed,
    rng_stream) and not stored.  x [.., N]: a GPU tensor in fp16, bf16 or fp32; residual: of its shape and type, or None."""
    if residual is not None and residual.shape != x.shape:
        raise ValueError("residual must have x's shape")
    return _Dropout.apply(x, residual, float(p), int(seed), int(rng_stream))


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        m = _grad_rows(x)
        y, h, mean, rstd = sdrop.sdrop_layer_norm(m, weight, bias, eps)
        ctx.save_for_backward(h, weight, mean, rstd)
        return y.view(x.shape)

    @staticmethod
    @_once
    def backward(ctx, dy):
        h, weight, mean, rstd = ctx.saved_tensors
        nx, nw, nb = ctx.needs_input_grad[:3]
        dx, _, dg, db = sdrop.sdrop_layer_norm_bwd(_grad_rows(dy), h, weight, mean, rstd, need_dr=False, need_dx=nx, need_dgamma=nw, need_dbeta=nb)
        return None if dx is None else dx.view(dy.shape), dg, db, None


def layer_norm(x, weight, bias=None, eps=1e-5):
    """(x - mean) / sqrt(var + eps) * weight + bias over the last dimension.  x [.., N] in fp16, bf16 or fp32; weight and bias
    (or None) [N] of x's type or fp32."""
    return _LayerNorm.apply(x, weight, bias, float(eps))


class _DropoutAddNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, bias, p, eps, seed, rng_stream):
        ctx.set_materialize_grads(False)
        y, h, mean, rstd = sdrop.sdrop_layer_norm(_grad_rows(x), weight, bias, eps, _grad_rows(residual), p, seed, rng_stream)
        ctx.save_for_backward(h, weight, mean, rstd)
        ctx.args = (p, seed, rng_stream)
        return y.view(x.shape), h.view(x.shape)

    @staticmethod
    @_once
    def backward(ctx, dy, dh):
        h, weight, mean, rstd = ctx.saved_tensors
        p, seed, rng_stream = ctx.args
        nx, nr, nw, nb = ctx.needs_input_grad[:4]
        if dy is None:          # only the residual stream is used further on
            if dh is None:
                return (None,) * 8
            dx = None if not nx else dh if p == 0.0 else sdrop.sdrop_dropout(_grad_rows(dh), p, seed, rng_stream).view(dh.shape)
            return dx, dh if nr else None, None, None, None, None, None, None
        dx, dr, dg, db = sdrop.sdrop_layer_norm_bwd(_grad_rows(dy), h, weight, mean, rstd, None if dh is None else _grad_rows(dh), p, seed,
                                                    rng_stream, need_dr=nr, need_dx=nx, need_dgamma=nw, need_dbeta=nb)
        return (None if dx is None else dx.view(dy.shape), None if dr is None else dr.view(dy.shape), dg, db, None, None, None, None)


def dropout_add_norm(x, residual, weight, bias=None, p=0.0, eps=1e-5, seed=0, rng_stream=0):
    """h = residual + dropout(x, p), y = layer_norm(h): returns (y, h), each pass over the rows in one launch.  h is the
    residual stream in x's type; its gradient and y's are joined in the backward pass."""
    if residual.shape != x.shape:
        raise ValueError("residual must have x's shape")
    return _DropoutAddNorm.apply(x, residual, weight, bias, float(p), float(eps), int(seed), int(rng_stream))


def _last_contiguous(t):
    # (what the kernels take in place: contiguous heads, 16-byte steps; anything else is copied once)
    ok = t.stride(-1) == 1 and all(n == 1 or (s > 0 and s % 8 == 0) for n, s in zip(t.shape[:-1], t.stride()[:-1])) and t.data_ptr() % 16 == 0
    return t if ok else t.contiguous()


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, causal, scale, cu_q, cu_k, max_q, max_k, k_len):
        q, k, v = _last_contiguous(q), _last_contiguous(k), _last_contiguous(v)
        if not any(ctx.needs_input_grad[:3]):
            return sdrop.sdrop_attn(q, k, v, causal, scale, cu_q, cu_k, max_q, max_k, k_len, need_lse=False)[0]
        o, lse, rest = sdrop.sdrop_attn(q, k, v, causal, scale, cu_q, cu_k, max_q, max_k, k_len, need_rest=True)
        ctx.save_for_backward(q, k, v, o, lse, rest, cu_q, cu_k, k_len)
        ctx.args = (causal, scale, max_q, max_k)
        return o

    @staticmethod
    @_once
    def backward(ctx, do):
        q, k, v, o, lse, rest, cu_q, cu_k, k_len = ctx.saved_tensors
        causal, scale, max_q, max_k = ctx.args
        dq, dk, dv = sdrop.sdrop_attn_bwd(_last_contiguous(do), q, k, v, o, lse, causal, scale, cu_q, cu_k, max_q, max_k, k_len, rest)
        return dq, dk, dv, None, None, None, None, None, None, None


def attention(q, k, v, causal=False, scale=None, cu_q=None, cu_k=None, max_q=None, max_k=None, k_len=None):
    """softmax(scale q k^T) v per head; see sdrop.sdrop_attn for shapes, packed sequences, grouped heads and k_len."""
    return _Attention.apply(q, k, v, bool(causal), scale, cu_q, cu_k, max_q, max_k, k_len)


class ElementDropout(torch.nn.Module):
    """Element-wise dropout (optionally + a residual) whose mask is never stored; a new mask every forward call in training mode."""

    def __init__(self, p=0.5, seed=0):
        super().__init__()
        if not 0.0 <= p <= 1.0:
            raise ValueError("p must lie in [0, 1]")
        self.p, self.seed, self.calls = float(p), int(seed), 0

    def forward(self, x, residual=None):
        if not self.training or self.p == 0.0:
            return x if residual is None else x + residual
        y = dropout(x, self.p, self.seed, self.calls, residual)
        self.calls += 1
        return y


class LayerNorm(torch.nn.Module):
    """torch.nn.LayerNorm over the last dimension, in libsdrop's kernels (its state dict loads as it is)."""

    def __init__(self, normalized_shape, eps=1e-5, bias=True, dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        self.eps = float(eps)
        self.weight = torch.nn.Parameter(torch.ones(normalized_shape, dtype=dtype, device=device))
        self.bias = torch.nn.Parameter(torch.zeros(normalized_shape, dtype=dtype, device=device)) if bias else None

    def forward(self, x):
        return layer_norm(x, self.weight, self.bias, self.eps)


class DropoutAddNorm(LayerNorm):
    """(y, h): h = residual + dropout(x), y = norm(h).  In eval mode nothing is dropped."""

    def __init__(self, normalized_shape, p=0.1, eps=1e-5, bias=True, seed=0, dtype=torch.bfloat16, device="cuda"):
        super().__init__(normalized_shape, eps, bias, dtype, device)
        if not 0.0 <= p <= 1.0:
            raise ValueError("p must lie in [0, 1]")
        self.p, self.seed, self.calls = float(p), int(seed), 0

    def forward(self, x, residual):
        p = self.p if self.training else 0.0
        out = dropout_add_norm(x, residual, self.weight, self.bias, p, self.eps, self.seed, self.calls)
        if self.training:
            self.calls += 1
        return out
