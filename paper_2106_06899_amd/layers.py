"""PyTorch layers over libtopk: top-k attention as a drop-in multi-head attention
layer (Section 2.1 with Eq. 4 per head) and the top-k feed-forward layer (Eq. 3),
each with a backward pass by input checkpointing (Section 2.2): the forward keeps
only its inputs and the selected keys with their raw scores, the backward calls
``topk_attn_backward`` / ``topk_ffn_backward``.

The projections around the attention are plain GEMMs left to PyTorch (rocBLAS);
every top-k step runs in libtopk's kernels, and so do head norms and rotary positions
(``rotary``, ``norm_rotary_heads``), which the attention layer takes as options, and attention over packed
sequences (``packed_attention``) and over caches in pages, which it offers beside the padded form.
"""
from __future__ import annotations

import math

import torch
from torch.autograd.function import once_differentiable

from . import (attn, attn_backward, attn_dense, attn_packed, attn_packed_backward, attn_prefix, attn_tree, ffn, ffn_backward,
               pages_append, qk_norm_rope, qk_norm_rope_append, qk_norm_rope_backward, rope, rope_axes, rope_frequencies)


def _whole(t):
    """A gradient in one piece at an address that the kernels take. (Autograd may hand over a part of another
    gradient, in one piece but at any address: that of ``cat``, of a view of one flat tensor.)"""
    t = t.contiguous()
    return t.clone() if t.data_ptr() % 16 else t


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
        dq, dk, dv = attn_backward(q, k, v, idx, dots, _whole(d_out), ctx.scale)
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
        dx, dw1, dw2 = ffn_backward(x, w1, w2, idx, dots, _whole(d_out))
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


class PackedAttentionFunction(torch.autograd.Function):
    """out = attn_packed(q, k, v, offsets), differentiable in q, k and v; the backward recomputes the
    weights from the inputs and each row's logarithm of their sum."""

    @staticmethod
    def forward(ctx, q, k, v, offsets, causal: bool, scale: float):
        if not any(ctx.needs_input_grad):
            return attn_packed(q, k, v, offsets, causal, scale)
        out, lse, rest = attn_packed(q, k, v, offsets, causal, scale, lse=True, rest=True)
        ctx.save_for_backward(q, k, v, offsets, out, lse, rest)
        ctx.how = causal, scale
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, d_out):
        q, k, v, offsets, out, lse, rest = ctx.saved_tensors
        head, token, one = d_out.stride()
        if one != 1 or head % 8 or token % 8 or d_out.data_ptr() % 16:
            d_out = _whole(d_out)
        return (*attn_packed_backward(q, k, v, offsets, out, lse, d_out, *ctx.how, rest), None, None, None)


def packed_attention(q, k, v, offsets, causal: bool = True, scale: float | None = None):
    """Differentiable attention over packed sequences; arguments as ``attn_packed``. (As with any function of PyTorch's:
    a backward pass that is captured into a graph must not find an earlier eager graph of the same leaves alive, whose
    stream the captured work would wait for.)"""
    if scale is None:
        scale = 1.0 / math.sqrt(q.shape[-1])
    return PackedAttentionFunction.apply(q, k, v, offsets, bool(causal), float(scale))


def packed_positions(offsets, N: int):
    """Each of N packed tokens' place in its own sequence, int64 [N] (for tokens of no sequence any)."""
    t = torch.arange(N, device=offsets.device)
    return t - offsets[torch.searchsorted(offsets[1:], t, right=True, out_int32=True).clamp(max=offsets.shape[0] - 2)]


def tree_depths(parents):
    """How many drafts each draft follows, int64 [T] or [B, T]: what it adds to its request's position
    (parents as ``attn_tree`` takes them)."""
    i = torch.arange(parents.shape[-1], device=parents.device)
    up = torch.where((parents >= 0) & (parents < i), parents.long(), i)  # (the text: itself)
    depth = (up != i).long()
    for _ in range((parents.shape[-1] - 1).bit_length()):  # twice as far up each time
        depth = depth + torch.gather(depth, -1, up)
        up = torch.gather(up, -1, up)
    return depth


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
    (see ``rope_frequencies``, ``rope_axes``, and there ``rope_adjacent``).

    With topk=None there are forms for more than a padded batch: ``packed`` for sequences that lie
    one behind the other (with a backward pass), ``draft`` for the next tokens of requests whose
    caches lie in pages, alone or as a tree of guesses, and ``decode`` for a batch of requests behind
    a shared prefix (the last two causal)."""

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

    def packed(self, x, offsets, positions=None, kv: bool = False):
        """x [N, d_model], sequences one behind the other (``attn_packed``'s offsets); positions
        [N] or [axes, 1, N] (default: each token's place in its own sequence, on every axis). With
        ``kv`` also the keys and values [n_heads, N, d_h], as ``pages_append`` takes them."""
        if self.topk is not None:
            raise ValueError("packed attends to every key: it needs topk=None")
        N, D = x.shape
        if self.qk_norm or self.rope_bits is not None or positions is not None:
            if positions is None and self.rope_bits is not None:
                positions = packed_positions(offsets, N)
                if self.rope_axes is not None:
                    positions = positions.expand(self._axes(), 1, N)
            q, k, v = (t[0] for t in self.heads(x[None], positions))
        else:
            q, k, v = self.qkv(x).view(N, 3, self.n_heads, self.d_head).permute(1, 2, 0, 3)
        o = packed_attention(q, k, v, offsets, self.causal, self.scale)
        y = self.out(o.transpose(0, 1).reshape(N, D))
        return (y, k, v) if kv else y

    @torch.no_grad()
    def draft(self, x, k_pages, v_pages, table, lengths, parents=None, positions=None):
        """The next T tokens x [B, T, d_model] of B requests whose caches lie in pages k_pages, v_pages
        [pages, n_heads, page_rows, d_h], or T guesses that form a tree (``parents`` as ``attn_tree``
        takes them): their keys and values go to the rows behind the ``lengths[b]`` that a request
        has (``pages_reserve`` makes room for them; the caller advances lengths, with
        ``pages_keep`` by those that are accepted), and each attends to its request's rows, itself
        and the guesses that it follows. positions default to lengths[b] and how many guesses each
        follows, on every axis. (A request of negative length writes nothing, and its output means nothing.)"""
        if self.topk is not None or not self.causal:
            raise ValueError("draft attends to every earlier key: it needs topk=None and causal=True")
        B, T, D = x.shape
        if positions is None and self.rope_bits is not None:
            steps = torch.arange(T, device=x.device) if parents is None else tree_depths(parents)
            positions = lengths[:, None] + steps
            if self.rope_axes is not None:
                positions = positions.expand(self._axes(), B, T)
        w = (self.q_norm, self.k_norm) if self.qk_norm else (None, None)
        q, k, v = qk_norm_rope(self.qkv(x), self.n_heads, self.n_heads, *w, **self._rotation(positions, T, x.device))
        pages_append(k, v, k_pages, v_pages, table, lengths)
        o = attn_tree(q, k_pages, v_pages, lengths + T, table, parents, self.scale)
        return self.out(o.permute(0, 2, 1, 3).reshape(B, T, D))

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
