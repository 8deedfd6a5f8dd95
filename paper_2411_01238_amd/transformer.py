"""What a transformer block (arxiv 2411.01238, Section 4.2) is made of besides its linear layers, as differentiable functions and
modules: element dropout, layer norm, dropout + residual add + layer norm in one pass, attention.  Everything runs in libsdrop's
kernels; the autograd nodes around them are in csrc/autograd_native.cpp.  Each can be differentiated once.  Tensors with nothing in them give
results with nothing in them (attention over no keys: 0).

The dropout's mask is a function of a seed and a stream number (`rng_stream`: one per call, e.g. a step counter) and is never
stored: the backward pass draws it again.  A captured graph replays the mask of the numbers it was captured with.  A module numbers its calls,
so that one that is run again by a backward pass, to save memory, would draw another mask and is refused: use the functions there, with a
stream number of the step's own.  Capture a backward pass only
after the eager graphs of the same leaves are gone (torch would add their gradients on those graphs' stream, outside the capture).
"""
import torch

try:
    from . import _native
except ImportError as e:
    raise RuntimeError("_native.so is not built or does not fit this torch: run `python -m paper_2411_01238_amd.build` "
                       "(there is no fallback path)") from e

_U64 = (1 << 64) - 1


def dropout(x, p, seed=0, rng_stream=0, residual=None):
    """residual + m . x / (1 - p) with a fresh element mask m (Bernoulli(1 - p), in steps of 2^-16), drawn from (seed,
    rng_stream) and not stored.  x [.., N]: a GPU tensor in fp16, bf16 or fp32; residual: of its shape and type, or None."""
    return _native.dropout(x, residual, p, int(seed) & _U64, int(rng_stream) & _U64)


def layer_norm(x, weight, bias=None, eps=1e-5):
    """(x - mean) / sqrt(var + eps) * weight + bias over the last dimension.  x [.., N] in fp16, bf16 or fp32; weight and bias
    (or None) [N] of x's type or fp32."""
    return _native.layer_norm(x, weight, bias, eps)


def dropout_add_norm(x, residual, weight, bias=None, p=0.0, eps=1e-5, seed=0, rng_stream=0):
    """h = residual + dropout(x, p), y = layer_norm(h): returns (y, h), each pass over the rows in one launch.  h is the
    residual stream in x's type; its gradient and y's are joined in the backward pass."""
    return _native.dropout_add_norm(x, residual, weight, bias, p, eps, int(seed) & _U64, int(rng_stream) & _U64)


def attention(q, k, v, causal=False, scale=None, cu_q=None, cu_k=None, max_q=None, max_k=None, k_len=None):
    """softmax(scale q k^T) v per head; see sdrop.sdrop_attn for shapes, packed sequences, grouped heads and k_len.  Tensors that the
    kernels cannot take in place (heads that are not contiguous, steps of other than 16 bytes) are copied once."""
    return _native.attention(q, k, v, causal, _scale(scale), cu_q, cu_k, _bound(cu_q, max_q), _bound(cu_k, max_k), k_len)


def qkv_attention(qkv, n_kv_head, causal=False, scale=None, cu=None, max_len=None, k_len=None):
    """attention() of the slices of one tensor [.., Hq + 2 Hkv, D] (query, key and value heads of a token side by side, as one
    projection writes them): its gradient is one tensor too.  cu, max_len: packed sequences [tokens, Hq + 2 Hkv, D]."""
    return _native.qkv_attention(qkv, n_kv_head, causal, _scale(scale), cu, _bound(cu, max_len), k_len)


def _scale(scale):
    if scale is None:
        return 0.0                      # the nodes' own default, D ** -0.5
    if not scale > 0.0:
        raise ValueError("scale must be positive")
    return scale


def _bound(cu, n):
    if cu is not None and n is None:
        raise ValueError("packed sequences need an upper bound of their lengths")
    return 0 if n is None else n


def _seed(seed):
    """A module's seed.  None: one of its own from torch's CPU generator, so that two modules, and ranks with seeds of their own, draw different
    masks."""
    return int(torch.randint(1 << 62, (), dtype=torch.int64, device="cpu")) if seed is None else int(seed)


def refuse_recomputation():
    """Raises where a backward pass is running: a call number of its own would draw another mask than the forward pass did."""
    if torch._C._current_graph_task_id() != -1:
        raise RuntimeError("a module that numbers its dropout masks cannot be run again in the backward pass (recomputation): it would draw another "
                           "mask; use the functions with a seed and rng_stream of the step's own")


class ElementDropout(torch.nn.Module):
    """Element-wise dropout (optionally + a residual) whose mask is never stored; a new mask every forward call in training mode.
    seed: None for one of the module's own (a repeated number repeats the masks).  The call's number (`calls`) is no part of the state
    dict."""

    def __init__(self, p=0.5, seed=None):
        super().__init__()
        if not 0.0 <= p <= 1.0:
            raise ValueError("p must lie in [0, 1]")
        self.p, self.seed, self.calls = float(p), _seed(seed), 0

    def forward(self, x, residual=None):
        if not self.training or self.p == 0.0:
            return x if residual is None else x + residual
        refuse_recomputation()
        y = dropout(x, self.p, self.seed, self.calls, residual)
        self.calls += 1
        return y


class LayerNorm(torch.nn.Module):
    """torch.nn.LayerNorm over the last dimension, in libsdrop's kernels (its state dict loads as it is).  Called with a residual, it is
    dropout_add_norm: (y, h), the dropout's numbers being the caller's."""

    def __init__(self, normalized_shape, eps=1e-5, bias=True, dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        self.eps = float(eps)
        self.weight = torch.nn.Parameter(torch.ones(normalized_shape, dtype=dtype, device=device))
        self.bias = torch.nn.Parameter(torch.zeros(normalized_shape, dtype=dtype, device=device)) if bias else None

    def forward(self, x, residual=None, p=0.0, seed=0, rng_stream=0):
        if residual is None:
            return layer_norm(x, self.weight, self.bias, self.eps)
        return dropout_add_norm(x, residual, self.weight, self.bias, p, self.eps, seed, rng_stream)


class DropoutAddNorm(LayerNorm):
    """(y, h): h = residual + dropout(x), y = norm(h).  In eval mode nothing is dropped.  seed: as for ElementDropout."""

    def __init__(self, normalized_shape, p=0.1, eps=1e-5, bias=True, seed=None, dtype=torch.bfloat16, device="cuda"):
        super().__init__(normalized_shape, eps, bias, dtype, device)
        if not 0.0 <= p <= 1.0:
            raise ValueError("p must lie in [0, 1]")
        self.p, self.seed, self.calls = float(p), _seed(seed), 0

    def forward(self, x, residual):
        p = self.p if self.training else 0.0
        if p > 0.0:
            refuse_recomputation()
        out = super().forward(x, residual, p, self.seed, self.calls)
        if self.training:
            self.calls += 1
        return out
