"""PyTorch layers over libtopk: top-k attention as a drop-in multi-head attention
layer (Section 2.1 with Eq. 4 per head) and the top-k feed-forward layer (Eq. 3),
each with a backward pass by input checkpointing (Section 2.2): the forward keeps
only its inputs and the selected keys with their raw scores, the backward calls
``topk_attn_backward`` / ``topk_ffn_backward``.

The projections around the attention are plain GEMMs left to PyTorch (rocBLAS);
every top-k step runs in libtopk's kernels, and so do head norms and rotary positions
(``rotary``, ``norm_rotary_heads``), which the attention layer takes as options.
"""
from __future__ import annotations

import math

import torch
from torch.autograd.function import once_differentiable

from . import (attn, attn_backward, attn_dense, attn_prefix, ffn, ffn_backward, qk_norm_rope, qk_norm_rope_append,
               qk_norm_rope_backward, rope, rope_axes, rope_frequencies)


class TopkAttentionFunction(torch.autograd.Function):
    """out = top-k attention(q, k, v) over [B, H, L, d] tensors, differentiable in
    q, k and v. The selection itself carries no gradient (the index set is piecewise
    constant in the inputs)."""

    @staticmethod
    def forward(ctx, q, k, v, topk: int, chunk: int, causal: bool, scale: float):
        out, idx, dots = attn(q, k, v, topk, chunk, causal, scale, cache=True)
        ctx.save_for_backward(q, k, v, idx, dots)
        ctx.scale = scale
        return out

    @staticmethod
    def backward(ctx, d_out):
        q, k, v, idx, dots = ctx.saved_tensors
        dq, dk, dv = attn_backward(q, k, v, idx, dots, d_out.contiguous(), ctx.scale)
        return dq, dk, dv, None, None, None, None


class TopkFFNFunction(torch.autograd.Function):
    """out = top-k feed-forward layer(x) with keys w1 and values w2 (Eq. 3, ReLU after
    the selection), differentiable in x, w1 and w2."""

    @staticmethod
    def forward(ctx, x, w1, w2, topk: int, chunk: int):
        out, idx, dots = ffn(x, w1, w2, topk, chunk, cache=True)
        ctx.save_for_backward(x, w1, w2, idx, dots)
        return out

    @staticmethod
    def backward(ctx, d_out):
        x, w1, w2, idx, dots = ctx.saved_tensors
        dx, dw1, dw2 = ffn_backward(x, w1, w2, idx, dots, d_out.contiguous())
        return dx, dw1, dw2, None, None


class RotaryFunction(torch.autograd.Function):
    """out = rope(x, ...), differentiable in x: the gradient turns back."""

    @staticmethod
    def forward(ctx, x, positions, freqs, axes, adjacent: bool):
        ctx.save_for_backward(positions, freqs)
        ctx.axes, ctx.adjacent = axes, adjacent
        return rope(x, positions, freqs, axes, adjacent)

    @staticmethod
    @once_differentiable
    def backward(ctx, d_out):
        positions, freqs = ctx.saved_tensors
        if d_out.stride(-1) != 1:
            d_out = d_out.contiguous()
        return rope(d_out, positions, freqs, ctx.axes, ctx.adjacent, inverse=True), None, None, None, None


class NormRotaryHeadsFunction(torch.autograd.Function):
    """q, k, v = qk_norm_rope(qkv, ...), differentiable in qkv and the weights; the backward
    recomputes from qkv, which it needs, and keeps, for the norm alone."""

    @staticmethod
    def forward(ctx, qkv, q_weight, k_weight, positions, freqs, heads, kv_heads, axes, adjacent, eps, norm):
        ctx.save_for_backward(qkv if norm else None, q_weight, k_weight, positions, freqs)
        ctx.how = heads, kv_heads, axes, adjacent, eps, norm
        return qk_norm_rope(qkv, heads, kv_heads, q_weight, k_weight, positions, freqs, axes, adjacent, eps, norm)

    @staticmethod
    @once_differentiable
    def backward(ctx, d_q, d_k, d_v):
        qkv, q_weight, k_weight, positions, freqs = ctx.saved_tensors
        heads, kv_heads, axes, adjacent, eps, norm = ctx.how
        if qkv is None:  # (not read: one row stands for all)
            B, _, L, d = d_q.shape
            qkv = d_q.new_empty((heads + 2 * kv_heads) * d).expand(B, L, -1)
        d_qkv, d_wq, d_wk = qk_norm_rope_backward(
            qkv, heads, kv_heads, d_q.contiguous(), d_k.contiguous(), d_v.contiguous(), q_weight, k_weight, positions, freqs,
            axes, adjacent, eps, norm, weights=any(ctx.needs_input_grad[1:3]))
        return (d_qkv, d_wq, d_wk) + (None,) * 8


def rotary(x, positions, freqs, axes=None, adjacent: bool = False):
    """Differentiable rotary positions on [B, H, L, d] heads; arguments as ``rope``."""
    return RotaryFunction.apply(x, positions, freqs, None if axes is None else tuple(axes), bool(adjacent))


def norm_rotary_heads(qkv, heads: int, kv_heads: int, q_weight=None, k_weight=None, positions=None, freqs=None, axes=None,
                      adjacent: bool = False, eps: float = 1e-6, norm: bool = True):
    """Differentiable q, k, v heads of the packed projection; arguments as ``qk_norm_rope``."""
    return NormRotaryHeadsFunction.apply(qkv, q_weight, k_weight, positions, freqs, int(heads), int(kv_heads),
                                         None if axes is None else tuple(axes), bool(adjacent), float(eps), bool(norm))


def topk_attention(q, k, v, topk: int, chunk: int = 0, causal: bool = False, scale: float | None = None):
    """Differentiable top-k attention over contiguous [B, H, L, d] tensors."""
    if scale is None:
        scale = 1.0 / math.sqrt(q.shape[-1])
    return TopkAttentionFunction.apply(q, k, v, int(topk), int(chunk), bool(causal), float(scale))


def dense_attention(q, k, v, chunk: int = 0, causal: bool = False, scale: float | None = None):
    """Query chunking with the top-k disabled (every valid key, Eq. 1): the paper's
    comparison baseline. Forward only (no backward is provided for it)."""
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad):
        raise RuntimeError("dense_attention has no backward pass; call it under torch.no_grad()")
    if scale is None:
        scale = 1.0 / math.sqrt(q.shape[-1])
    return attn_dense(q, k, v, int(chunk), bool(causal), float(scale))


def topk_feed_forward(x, w1, w2, topk: int, chunk: int = 0):
    """Differentiable top-k feed-forward layer: x [N, d_model], w1 / w2 [d_ff, d_model]."""
    return TopkFFNFunction.apply(x, w1, w2, int(topk), int(chunk))


class TopkMultiheadAttention(torch.nn.Module):
    """Multi-head self-attention whose heads use top-k attention: a drop-in for a
    BERT-style attention block on batch-first input x [B, L, d_model].

    [q | k | v] = x W_qkv^T + b_qkv, head h takes columns h*d_h .. (h+1)*d_h - 1 of
    each; every head runs top-k attention (temperature 1/sqrt(d_h) unless given);
    y = concat(heads) W_o^T + b_o. With topk=None the heads keep every key (query
    chunking without top-k, the paper's baseline; forward only).

    With ``qk_norm`` every query and key head is divided by its root mean square and scaled
    by weights of its own (q_norm, k_norm, [d_h]); with ``rope_theta`` heads are rotated by
    their positions, by one axis, or by several with ``rope_sections``, the pairs of each
    (see ``rope_frequencies``, ``rope_axes``, and there ``rope_adjacent``). ``decode`` is the
    serving form for a batch of requests behind a shared prefix (topk=None, causal)."""

    def __init__(self, d_model: int, n_heads: int, topk: int, chunk: int = 1024, causal: bool = False,
                 bias: bool = True, scale: float | None = None, device=None, dtype=torch.bfloat16, qk_norm: bool = False,
                 rope_theta: float | None = None, rope_sections=None, rope_adjacent: bool = False):
        super().__init__()
        if d_model % n_heads:
            raise ValueError(f"d_model {d_model} is not a multiple of n_heads {n_heads}")
        self.d_model, self.n_heads, self.topk, self.chunk, self.causal = d_model, n_heads, topk, chunk, causal
        self.d_head = d_model // n_heads
        self.scale = 1.0 / math.sqrt(self.d_head) if scale is None else float(scale)
        kw = dict(device=device, dtype=dtype)
        self.qkv = torch.nn.Linear(d_model, 3 * d_model, bias=bias, **kw)
        self.out = torch.nn.Linear(d_model, d_model, bias=bias, **kw)
        self.qk_norm, self.rope_axes, self.rope_adjacent = bool(qk_norm), None, bool(rope_adjacent)
        if qk_norm:
            self.q_norm = torch.nn.Parameter(torch.ones(self.d_head, **kw))
            self.k_norm = torch.nn.Parameter(torch.ones(self.d_head, **kw))
        if rope_theta is None and rope_sections is not None:
            raise ValueError("rope_sections need rope_theta")
        # the frequencies' bits as integers: a change of the module's type leaves them whole
        self.register_buffer("rope_bits", None, persistent=False)
        if rope_theta is not None:
            pairs = self.d_head // 2 if rope_sections is None else tuple(rope_sections)
            if rope_sections is not None:
                self.rope_axes = rope_axes(pairs)
            self.rope_of = pairs, float(rope_theta)
            bits = self._rope_bits()
            if 2 * bits.numel() > self.d_head:
                raise ValueError(f"{bits.numel()} pairs do not fit into {self.d_head} features")
            self.rope_bits = bits.to(self.qkv.weight.device)

    def _rope_bits(self):
        return rope_frequencies(*self.rope_of, device="cpu").view(torch.int64)

    def _axes(self):
        return max(self.rope_axes, default=0) + 1

    def _apply(self, fn, recurse=True):
        # (a layer built without memory gets it here; the frequencies are in no state_dict)
        bare = self.rope_bits is not None and self.rope_bits.is_meta
        super()._apply(fn, recurse)
        if bare and not self.rope_bits.is_meta:
            self.rope_bits.copy_(self._rope_bits())
        return self

    def _rotation(self, positions, L: int, device):
        if self.rope_bits is None:
            if positions is not None:
                raise ValueError("positions need rope_theta")
            return dict(norm=self.qk_norm)
        if self.rope_bits.is_meta:  # (weights that were assigned to a layer without memory)
            self.rope_bits = self._rope_bits().to(device)
        if positions is None:
            positions = torch.arange(L, device=device)
            if self.rope_axes is not None:
                positions = positions.expand(self._axes(), 1, L)
        return dict(positions=positions, freqs=self.rope_bits.view(torch.float64), axes=self.rope_axes,
                    adjacent=self.rope_adjacent, norm=self.qk_norm)

    def heads(self, x, positions=None):
        """q, k, v [B, n_heads, L, d_h] as the attention sees them (the keys and values of a
        shared prefix are k[0], v[0] of its own call)."""
        if not self.qk_norm and self.rope_bits is None and positions is None:
            B, L, D = x.shape
            p = self.qkv(x).view(B, L, 3, self.n_heads, self.d_head).permute(2, 0, 3, 1, 4)
            return tuple(p[t].contiguous() for t in range(3))
        w = (self.q_norm, self.k_norm) if self.qk_norm else (None, None)
        return norm_rotary_heads(self.qkv(x), self.n_heads, self.n_heads, *w, **self._rotation(positions, x.shape[1], x.device))

    def forward(self, x, positions=None):
        """x [B, L, d_model]; positions as ``rope`` takes them (default: 0 .. L - 1 on every axis)."""
        B, L, D = x.shape
        q, k, v = self.heads(x, positions)
        if self.topk is None:
            o = dense_attention(q, k, v, self.chunk, self.causal, self.scale)
        else:
            o = topk_attention(q, k, v, self.topk, self.chunk, self.causal, self.scale)
        return self.out(o.permute(0, 2, 1, 3).reshape(B, L, D))

    @torch.no_grad()
    def decode(self, x, prefix_k, prefix_v, k_cache, v_cache, lengths, positions=None):
        """The next L tokens x [B, L, d_model] of B requests that share the prefix [n_heads, P,
        d_h] and hold ``lengths[b]`` tokens in their caches [B, n_heads, S, d_h]: their keys and
        values are appended (the caller advances lengths by L, and leaves room for them), and
        each attends to the prefix, its own cache and the new tokens up to itself. positions
        default to P + lengths[b] + 0 .. L - 1 on every axis. Caches may be cut from longer ones
        (see ``attn_prefix``)."""
        if self.topk is not None or not self.causal:
            raise ValueError("decode attends to every earlier key: it needs topk=None and causal=True")
        B, L, D = x.shape
        if positions is None and self.rope_bits is not None:
            positions = prefix_k.shape[1] + lengths[:, None] + torch.arange(L, device=x.device, dtype=torch.int32)
            if self.rope_axes is not None:
                positions = positions.expand(self._axes(), B, L)
        w = (self.q_norm, self.k_norm) if self.qk_norm else (None, None)
        q = qk_norm_rope_append(self.qkv(x), self.n_heads, self.n_heads, k_cache, v_cache, lengths, *w,
                                **self._rotation(positions, L, x.device))
        o = attn_prefix(q, prefix_k, prefix_v, k_cache, v_cache, lengths + L, True, self.scale)
        return self.out(o.permute(0, 2, 1, 3).reshape(B, L, D))


class TopkFeedForward(torch.nn.Module):
    """The feed-forward sub-layer cast as attention (Eq. 3): keys are the rows of w1,
    values the rows of w2 (both [d_ff, d_model]); each token keeps its top-k hidden
    units, ReLU after the selection. Input [..., d_model]."""

    def __init__(self, d_model: int, d_ff: int, topk: int, chunk: int = 1024, device=None,
                 dtype=torch.bfloat16):
        super().__init__()
        self.topk, self.chunk = topk, chunk
        kw = dict(device=device, dtype=dtype)
        self.w1 = torch.nn.Parameter(torch.empty(d_ff, d_model, **kw))
        self.w2 = torch.nn.Parameter(torch.empty(d_ff, d_model, **kw))
        torch.nn.init.normal_(self.w1, std=d_model ** -0.5)
        torch.nn.init.normal_(self.w2, std=d_ff ** -0.5)

    def forward(self, x):
        shape = x.shape
        y = topk_feed_forward(x.reshape(-1, shape[-1]).contiguous(), self.w1, self.w2, self.topk, self.chunk)
        return y.reshape(shape)
