"""GPU parity of head norms and rotary positions against the formulas in 64 bits.

Tolerances, element by element, with e = 2^-24 (half a step of fp32):
* the result's own rounding, half a step of its type relative to the value;
* rotation: the fraction of a turn is rounded to fp32 (angle off by pi e / 2), sine and cosine by
  up to 2 steps of 2e, products and sum by e each: below 10 e (|a| + |b|) for a pair (a, b);
* norm: a sum of d squares in a tree of at most 16 + 4 + 6 levels, mean, root and two products:
  below 20 e relative, and as much again for the second sum of the backward pass;
* weight gradients: N terms of the above in fp32, below (N + 40) e times the sum of their sizes.
"""
import math

import pytest
import torch

import paper_2106_06899_amd as tk
from paper_2106_06899_amd import layers

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    tk.lib()
    yield


def _randn(seed, *shape, dtype=F32, std=1.0, mean=0.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=gen, device="cuda") * std + mean).to(dtype)


def _pairs(d_rot, adjacent):
    p = torch.arange(d_rot // 2, device="cuda")
    return (2 * p, 2 * p + 1) if adjacent else (p, p + d_rot // 2)


def _turn(x, pos, freqs, axes, adjacent, back=False):
    """(rotated, |a| + |b| of each element's pair, 0 where it passes); x float64 [B, h, L, d], pos [A, B, L]."""
    n = len(freqs)
    ang = torch.stack([pos[a].double() * f for a, f in zip(axes, freqs.tolist())], -1)[:, None]  # [B, 1, L, n]
    c, s = torch.cos(ang), torch.sin(ang) * (-1 if back else 1)
    i, j = _pairs(2 * n, adjacent)
    a, b = x[..., i], x[..., j]
    y, size = x.clone(), torch.zeros_like(x)
    y[..., i], y[..., j] = a * c - b * s, a * s + b * c
    size[..., i] = size[..., j] = a.abs() + b.abs()
    return y, size


def _close(got, ref, tol, what):
    err = (got.double() - ref).abs()
    half = torch.finfo(got.dtype).eps / 2
    bad = err > ref.abs() * half * (1 + 1e-6) + tol + 1e-37
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float(err.max()):.3e}"
    assert got.isfinite().all()


ROPE = {
    # name: dtype, B, H, L, d, pairs of each axis, adjacent, far
    "one_token": (BF16, 1, 1, 1, 64, (32,), False, 0),
    "widest_lanes": (BF16, 2, 3, 37, 128, (64,), False, 0),
    "adjacent": (BF16, 2, 3, 37, 128, (64,), True, 5),
    "far": (F32, 1, 2, 33, 64, (32,), False, 10 ** 9),
    "half_rotated": (F32, 2, 2, 21, 80, (20,), False, 1000),
    "half_rotated_adjacent": (F32, 2, 2, 21, 80, (20,), True, 1000),
    "eight_byte_lanes": (BF16, 2, 2, 40, 72, (36,), False, 7),
    "three_axes": (BF16, 2, 2, 50, 128, (16, 24, 24), False, 3),
    "four_axes_f32": (F32, 1, 3, 19, 96, (12, 12, 12, 12), True, 3),
    "single_features": (BF16, 2, 2, 9, 70, (7, 3), False, 3),
    "single_features_adjacent": (F32, 1, 1, 70, 6, (1, 1, 1), True, 3),
    "two_features": (F32, 3, 1, 5, 2, (1,), False, 3),
    "widest_head": (BF16, 1, 2, 17, 512, (256,), False, 3),
    "widest_head_f32": (F32, 1, 2, 17, 512, (256,), True, 3),
    "widest_odd_pairs": (F32, 1, 2, 17, 510, (255,), False, 3),
    "many_tokens": (BF16, 3, 1, 4097, 64, (16, 16), False, 0),
    "many_heads": (BF16, 1, 300, 3, 64, (32,), False, 0),
}


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("name", sorted(ROPE))
def test_rope(name, inverse):
    dt, B, H, L, d, sections, adjacent, far = ROPE[name]
    x = _randn(1, B, H, L, d, dtype=dt, std=2.0)
    gen = torch.Generator(device="cuda").manual_seed(2)
    pos = torch.randint(-50, 5000, (len(sections), B, L), generator=gen, device="cuda") + far
    freqs, axes = tk.rope_frequencies(sections), tk.rope_axes(sections, interleaved=True)
    y = tk.rope(x, pos, freqs, axes, adjacent, inverse)
    ref, size = _turn(x.double(), pos, freqs, axes, adjacent, inverse)
    _close(y, ref, 10 * E * size, name)
    if 2 * len(freqs) < d:
        assert torch.equal(y[..., 2 * len(freqs):], x[..., 2 * len(freqs):])


def test_rope_shapes_of_positions():
    x = _randn(3, 3, 2, 11, 64)
    f = tk.rope_frequencies(32)
    one = torch.arange(11, device="cuda", dtype=torch.int32) * 7
    want = tk.rope(x, one.long().expand(1, 3, 11).contiguous(), f)
    for p in (one, one[None], one.expand(3, 11), one.expand(1, 3, 11), one.long(), torch.stack((one, one), -1)[:, 0]):
        assert torch.equal(tk.rope(x, p, f), want)
    each = torch.randint(0, 99, (3, 1), device="cuda")
    assert torch.equal(tk.rope(x, each, f), tk.rope(x, each.expand(3, 11).contiguous(), f))
    axes = (0, 1) * 16
    assert torch.equal(tk.rope(x, one.expand(2, 3, 11), f, axes), want)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_rope_strided_and_unaligned_inputs(dt):
    f, pos = tk.rope_frequencies(32), torch.arange(19, device="cuda")
    packed = _randn(4, 2, 19, 5 * 64, dtype=dt)
    views = [packed.view(2, 19, 5, 64).transpose(1, 2)[:, 1:4], packed.view(2, 19, 5, 64).transpose(1, 2)[1:].expand(2, 5, 19, 64),
             packed.flatten()[3:3 + 2 * 2 * 19 * 64].view(2, 2, 19, 64), packed.view(2, 19, 320)[..., 5:5 + 64][:, None]]
    for x in views:
        assert torch.equal(tk.rope(x, pos, f), tk.rope(x.contiguous().clone(), pos, f))


def test_rope_turns_back_and_passes_through():
    x = _randn(5, 2, 3, 21, 64)
    pos, f = torch.arange(21, device="cuda") + 10 ** 7, tk.rope_frequencies(32)
    back = tk.rope(tk.rope(x, pos, f), pos, f, inverse=True)
    s = x.double().abs() + x.double().abs().roll(32, -1)
    assert bool(((back.double() - x.double()).abs() <= 24 * E * s).all())
    assert torch.equal(tk.rope(x, pos, f[:0]), x)
    assert torch.equal(tk.rope(x, torch.zeros_like(pos), f), x)


HEADS = {
    # name: dtype, B, L, H, Hkv, d, pairs of each axis, adjacent, norm, weights
    "one_token": (BF16, 1, 1, 1, 1, 64, (32,), False, True, True),
    "encoder": (BF16, 2, 65, 12, 12, 64, (32,), False, True, True),
    "shared_heads": (BF16, 3, 33, 8, 2, 128, (64,), False, True, True),
    "odd_groups_f32": (F32, 2, 41, 5, 1, 96, (20, 14, 14), True, True, True),
    "no_rotation": (BF16, 2, 9, 3, 3, 64, (), False, True, True),
    "no_norm": (BF16, 2, 9, 4, 2, 64, (16,), False, False, False),
    "no_weights": (F32, 2, 9, 4, 2, 80, (20,), False, True, False),
    "split_only": (F32, 1, 7, 2, 1, 10, (), False, False, False),
    "eight_byte_lanes": (BF16, 2, 40, 2, 1, 72, (36,), False, True, True),
    "single_features": (BF16, 2, 11, 3, 1, 70, (7, 3), True, True, True),
    "widest_head": (BF16, 1, 5, 2, 2, 512, (256,), False, True, True),
    "widest_odd_pairs": (F32, 1, 5, 2, 2, 510, (255,), True, True, True),
    "several_tiles": (BF16, 1, 3000, 2, 1, 64, (32,), False, True, True),
    "many_tokens_f32": (F32, 2, 1100, 3, 3, 128, (64,), False, True, True),
}


def _case(name, seed=0):
    dt, B, L, H, Hkv, d, sections, adjacent, norm, weights = HEADS[name]
    qkv = _randn(10 + seed, B, L, (H + 2 * Hkv) * d, dtype=dt, std=1.5)
    wq, wk = (_randn(s, d, dtype=dt, std=0.2, mean=1.0) if weights else None for s in (11, 12))
    kw = dict(norm=norm)
    gen = torch.Generator(device="cuda").manual_seed(13)
    pos = torch.randint(0, 100000, (max(1, len(sections)), B, L), generator=gen, device="cuda")
    if sections:
        kw.update(positions=pos, freqs=tk.rope_frequencies(sections), axes=tk.rope_axes(sections), adjacent=adjacent)
    return qkv, H, Hkv, wq, wk, kw


def _reference(qkv, H, Hkv, wq, wk, kw):
    """64-bit q, k, v with the tolerance of q and k."""
    B, L, W = qkv.shape
    d = W // (H + 2 * Hkv)
    x = qkv.double().view(B, L, H + 2 * Hkv, d).transpose(1, 2)
    out = []
    for t, w in ((x[:, :H], wq), (x[:, H:H + Hkv], wk)):
        n = t
        if kw["norm"]:
            n = t / torch.sqrt(t.pow(2).mean(-1, keepdim=True) + 1e-6)
            n = n * w.double() if w is not None else n
        y, size = _turn(n, kw["positions"], kw["freqs"], kw["axes"], kw["adjacent"]) if "freqs" in kw else (n, torch.zeros_like(n))
        out += [(y, 10 * E * size + (20 * E * torch.maximum(size, n.abs()) if kw["norm"] else 0))]
    return out[0], out[1], x[:, H + Hkv:]


@pytest.mark.parametrize("name", sorted(HEADS))
def test_qk_norm_rope(name):
    qkv, H, Hkv, wq, wk, kw = _case(name)
    q, k, v = tk.qk_norm_rope(qkv, H, Hkv, wq, wk, **kw)
    (rq, tq), (rk, tk_), rv = _reference(qkv, H, Hkv, wq, wk, kw)
    _close(q, rq, tq, "q")
    _close(k, rk, tk_, "k")
    assert torch.equal(v.double(), rv)


def _grad_reference(qkv, H, Hkv, wq, wk, kw, grads):
    B, L, W = qkv.shape
    d = W // (H + 2 * Hkv)
    x = qkv.double().view(B, L, H + 2 * Hkv, d).transpose(1, 2)
    dx, tol, dw = torch.empty_like(x), torch.zeros_like(x), []
    for at, h, w, g in ((0, H, wq, grads[0]), (H, Hkv, wk, grads[1])):
        t, m = x[:, at:at + h], g.double()
        size = torch.zeros_like(m)
        if "freqs" in kw:
            m, size = _turn(m, kw["positions"], kw["freqs"], kw["axes"], kw["adjacent"], back=True)
        size = torch.maximum(size, m.abs())
        if not kw["norm"]:
            dx[:, at:at + h], tol[:, at:at + h] = m, 10 * E * size
            dw.append(None)
            continue
        ww = w.double() if w is not None else torch.ones(d, dtype=torch.float64, device="cuda")
        r = 1 / torch.sqrt(t.pow(2).mean(-1, keepdim=True) + 1e-6)
        u = t * r
        dx[:, at:at + h] = r * (m * ww - u * (m * ww * u).mean(-1, keepdim=True))
        # the rotation's error, the norm's and the second sum's (each at most 20 e, three factors r)
        tol[:, at:at + h] = 90 * E * r * (size * ww.abs() + u.abs() * (size * ww.abs() * u.abs()).mean(-1, keepdim=True))
        terms = (size * u.abs()).sum((0, 1, 2))
        dw.append(((m * u).sum((0, 1, 2)), (B * L * h + 40) * E * terms) if w is not None else None)
    dx[:, H + Hkv:] = grads[2].double()
    flat = lambda z: z.transpose(1, 2).reshape(B, L, W)  # noqa: E731
    return flat(dx), flat(tol), dw


@pytest.mark.parametrize("name", sorted(HEADS))
def test_qk_norm_rope_backward(name):
    qkv, H, Hkv, wq, wk, kw = _case(name)
    B, L, W = qkv.shape
    d = W // (H + 2 * Hkv)
    grads = [_randn(20 + i, B, h, L, d, dtype=qkv.dtype) for i, h in enumerate((H, Hkv, Hkv))]
    got = tk.qk_norm_rope_backward(qkv, H, Hkv, *grads, wq, wk, **kw)
    dx, tol, dw = _grad_reference(qkv, H, Hkv, wq, wk, kw, grads)
    _close(got[0], dx, tol, "d_qkv")
    for g, r, n in zip(got[1:], dw, ("d_q_weight", "d_k_weight")):
        assert (g is None) == (r is None)
        if g is not None:
            _close(g, r[0], r[1], n)
    again = tk.qk_norm_rope_backward(qkv, H, Hkv, *grads, wq, wk, **kw)
    for a, b in zip(got, again):
        assert a is None or torch.equal(a, b)
    alone = tk.qk_norm_rope_backward(qkv, H, Hkv, *grads, wq, wk, weights=False, **kw)
    assert torch.equal(alone[0], got[0]) and alone[1] is None and alone[2] is None


@pytest.mark.parametrize("adjacent", [False, True])
def test_gradients_against_differences(adjacent):
    """Central differences of the call itself in 32 bits, with steps of 2^-6: off by the third
    derivative (below 40 h^2 of the gradient's size here) and by rounding over the step."""
    H, Hkv, d = 2, 1, 16
    qkv = _randn(30, 1, 3, (H + 2 * Hkv) * d).requires_grad_()
    wq, wk = (_randn(s, d, std=0.2, mean=1.0).requires_grad_() for s in (31, 32))
    rot = dict(positions=torch.arange(3, device="cuda") + 5, freqs=tk.rope_frequencies(6), adjacent=adjacent)
    g = [_randn(33 + i, 1, h, 3, d) for i, h in enumerate((H, Hkv, Hkv))]

    def loss(a, b, c):
        return sum((y.double() * z.double()).sum() for y, z in zip(layers.norm_rotary_heads(a, H, Hkv, b, c, **rot), g))
    loss(qkv, wq, wk).backward()
    h = 2.0 ** -6
    for i, t in enumerate((qkv, wq, wk)):
        args = [z.detach().clone() for z in (qkv, wq, wk)]
        flat = args[i].flatten()
        pick = torch.arange(0, flat.numel(), 5)
        for j in pick.tolist():
            v = flat[j].item()
            ends = []
            for s in (h, -h):
                args[i].view(-1)[j] = v + s
                ends.append(loss(*args).item())
            args[i].view(-1)[j] = v
            diff = (ends[0] - ends[1]) / (2 * h)
            size = float(t.grad.abs().max())
            assert abs(diff - t.grad.flatten()[j].item()) <= (40 * h * h + 1e-3) * size, (i, j)


def test_layers_equal_direct_calls_and_refuse_second_order():
    qkv, H, Hkv, wq, wk, kw = _case("shared_heads")
    grads = [_randn(40 + i, 3, h, 33, 128, dtype=BF16) for i, h in enumerate((H, Hkv, Hkv))]
    leaves = [t.clone().requires_grad_() for t in (qkv, wq, wk)]
    outs = layers.norm_rotary_heads(leaves[0], H, Hkv, leaves[1], leaves[2], **kw)
    got = torch.autograd.grad(outs, leaves, grads, retain_graph=True)
    want = tk.qk_norm_rope_backward(qkv, H, Hkv, *grads, wq, wk, **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # an unused output and an expanded gradient
    one = torch.autograd.grad(outs[0].sum(), leaves[0], retain_graph=True)[0]
    ones = [torch.ones_like(grads[0]), torch.zeros_like(grads[1]), torch.zeros_like(grads[2])]
    assert torch.equal(one, tk.qk_norm_rope_backward(qkv, H, Hkv, *ones, wq, wk, **kw)[0])
    first = torch.autograd.grad(outs[0].float().square().sum(), leaves[0], create_graph=True)[0]
    with pytest.raises(RuntimeError):
        torch.autograd.grad(first.float().sum(), leaves[0])
    x = _randn(43, 2, 3, 33, 128, dtype=BF16).requires_grad_()
    pos, f = torch.arange(33, device="cuda"), tk.rope_frequencies(64)
    y = layers.rotary(x, pos, f)
    assert torch.equal(torch.autograd.grad(y, x, y.detach(), retain_graph=True)[0], tk.rope(y.detach(), pos, f, inverse=True))
    assert torch.equal(torch.autograd.grad(y.sum(), x)[0], tk.rope(torch.ones_like(y), pos, f, inverse=True))


def test_padded_projection_rows():
    """A projection cut from a wider one (strides of its own, not a multiple of 16 bytes)."""
    for pad in (64, 3):
        wide = _randn(50, 2, 13, 4 * 64 + pad, dtype=BF16)
        qkv = wide[..., pad:]
        rot = dict(positions=torch.arange(13, device="cuda"), freqs=tk.rope_frequencies(32))
        grads = [_randn(51 + i, 2, h, 13, 64, dtype=BF16) for i, h in enumerate((2, 1, 1))]
        w = _randn(55, 64 + 1, dtype=BF16, mean=1.0)[1:].contiguous()
        for f in (lambda t: tk.qk_norm_rope(t, 2, 1, w, w, **rot), lambda t: tk.qk_norm_rope_backward(t, 2, 1, *grads, w, w, **rot)):
            assert all(torch.equal(a, b) or torch.allclose(a.float(), b.float(), rtol=2 ** -7) for a, b in zip(f(qkv), f(qkv.contiguous())))


@pytest.mark.parametrize("dt", [F32, BF16])
def test_append(dt):
    """Rows lengths[b] .. + L of the caches, and nothing else; rows without a place are dropped."""
    B, L, H, Hkv, S, d = 6, 3, 4, 2, 20, 64
    lengths = torch.tensor([0, 5, 17, 18, 20, -2], dtype=torch.int32, device="cuda")
    qkv = _randn(60, B, L, (H + 2 * Hkv) * d, dtype=dt)
    w = _randn(61, d, dtype=dt, mean=1.0)
    rot = dict(positions=lengths[:, None] + torch.arange(L, device="cuda", dtype=torch.int32), freqs=tk.rope_frequencies(32))
    q, k, v = tk.qk_norm_rope(qkv, H, Hkv, w, w, **rot)
    base = _randn(62, 2, B, S + 4, Hkv, d, dtype=dt)
    for layout in ("heads first", "tokens first"):
        if layout == "heads first":
            kc, vc = base[:, :, :S].transpose(2, 3).contiguous().unbind(0)
        else:
            kc, vc = (t.clone()[:, :S].transpose(1, 2) for t in base)  # cut from a longer cache, heads behind tokens
        wants = [kc.clone(), vc.clone()]
        for b, n in enumerate(lengths.tolist()):
            for i in range(L):
                if 0 <= n + i < S:
                    wants[0][b, :, n + i], wants[1][b, :, n + i] = k[b, :, i], v[b, :, i]
        got = tk.qk_norm_rope_append(qkv, H, Hkv, kc, vc, lengths, w, w, **rot)
        assert torch.equal(got, q) and torch.equal(kc, wants[0]) and torch.equal(vc, wants[1]), layout
    none = torch.empty(B, Hkv, 0, d, dtype=dt, device="cuda")
    assert torch.equal(tk.qk_norm_rope_append(qkv, H, Hkv, none, none, lengths, w, w, **rot), q)


def test_refusals_of_the_binding():
    x, f, p = _randn(70, 2, 2, 5, 64), tk.rope_frequencies(32), torch.arange(5, device="cuda")
    bad = [
        lambda: tk.rope(x[0], p, f), lambda: tk.rope(x.transpose(2, 3), p, f), lambda: tk.rope(x.half(), p, f),
        lambda: tk.rope(x, p.float(), f), lambda: tk.rope(x, p.cpu(), f), lambda: tk.rope(x, p, f.float()), lambda: tk.rope(x, p, f[::2]),
        lambda: tk.rope(x, p[:4], f), lambda: tk.rope(x, None, f), lambda: tk.rope(x, p, None), lambda: tk.rope(x, p, tk.rope_frequencies(33)),
        lambda: tk.rope(x, p.expand(2, 2, 5), f), lambda: tk.rope(x, p, f, axes=(0,) * 31), lambda: tk.rope(x, p, f, axes=(1,) * 32),
        lambda: tk.rope(x, p.expand(5, 2, 5), f, axes=(0,) * 32), lambda: tk.rope(x[..., :63], p, f[:4]),
    ]
    qkv = _randn(71, 2, 5, 4 * 64)
    kc, vc, n = torch.zeros(2, 1, 8, 64, device="cuda"), torch.zeros(2, 1, 8, 64, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    w = torch.ones(64, device="cuda")
    bad += [
        lambda: tk.qk_norm_rope(qkv, 3, 1), lambda: tk.qk_norm_rope(qkv, 2, 0), lambda: tk.qk_norm_rope(qkv[0], 2, 1),
        lambda: tk.qk_norm_rope(qkv, 2, 1, w[:32]), lambda: tk.qk_norm_rope(qkv, 2, 1, w.bfloat16()), lambda: tk.qk_norm_rope(qkv, 2, 1, w, norm=False),
        lambda: tk.qk_norm_rope(qkv, 2, 1, eps=-1.0), lambda: tk.qk_norm_rope(qkv, 2, 1, positions=p),
        lambda: tk.qk_norm_rope_append(qkv, 2, 1, kc, kc, n), lambda: tk.qk_norm_rope_append(qkv, 2, 1, kc, vc, n.long()),
        lambda: tk.qk_norm_rope_append(qkv, 2, 1, kc, vc, n[:1]), lambda: tk.qk_norm_rope_append(qkv, 2, 1, kc, vc[:, :, :7], n),
        lambda: tk.qk_norm_rope_append(qkv, 2, 1, kc[:1].expand(2, 1, 8, 64), vc, n), lambda: tk.qk_norm_rope_append(qkv, 2, 1, kc.bfloat16(), vc, n),
        lambda: tk.qk_norm_rope_backward(qkv, 2, 1, *[torch.zeros(2, h, 5, 64, device="cuda") for h in (2, 1, 2)]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, TypeError, tk.TopkError)):
            call()
            print("accepted:", i)


def test_other_streams_and_a_replayed_graph():
    """Forward, backward and append on a side stream, and captured and replayed with new inputs."""
    qkv, H, Hkv, wq, wk, kw = _case("shared_heads")
    B, L, d = 3, 33, 128
    grads = [_randn(80 + i, B, h, L, d, dtype=BF16) for i, h in enumerate((H, Hkv, Hkv))]
    kc, vc = (torch.zeros(B, Hkv, 64, d, dtype=BF16, device="cuda") for _ in range(2))
    n = torch.tensor([0, 9, 31], dtype=torch.int32, device="cuda")

    def everything():
        a = tk.qk_norm_rope(qkv, H, Hkv, wq, wk, **kw)
        b = tk.qk_norm_rope_backward(qkv, H, Hkv, *grads, wq, wk, **kw)
        c = tk.qk_norm_rope_append(qkv, H, Hkv, kc, vc, n, wq, wk, **kw)
        return (*a, *b, c, tk.rope(a[0], kw["positions"], kw["freqs"], kw["axes"], inverse=True))
    want = [t.clone() for t in (*everything(), kc, vc)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = (*everything(), kc, vc)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = everything()
    first = qkv.clone()
    for rep in range(4):
        qkv.copy_(first if rep % 2 == 0 else _randn(90 + rep, *qkv.shape, dtype=BF16))
        kc.zero_(), vc.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*held, kc, vc)]
        kc.zero_(), vc.zero_()
        eager = (*everything(), kc, vc)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager)), f"replay {rep}"


def test_gradient_of_empty_tokens_with_a_tiny_eps():
    """Tokens of zeros (padding): r = eps^(-1/2) = 1e15, whose third power is beyond fp32, and
    dx = r w times the gradient. r, its products and w: a few e relative each, below 20 e."""
    H, Hkv, d, L = 2, 1, 64, 5
    qkv = _randn(21, 1, L, (H + 2 * Hkv) * d)
    qkv[0, 2:4] = 0
    w = _randn(22, d, mean=1.0, std=0.1)
    grads = [_randn(23 + i, 1, h, L, d) for i, h in enumerate((H, Hkv, Hkv))]
    dx, dwq, dwk = tk.qk_norm_rope_backward(qkv, H, Hkv, *grads, w, w, eps=1e-30)
    eps = float(torch.tensor(1e-30, dtype=F32).double())
    for h in range(H + Hkv):
        ref = (grads[0][0, h] if h < H else grads[1][0, h - H])[2:4].double() * w.double() * eps ** -0.5
        _close(dx[0, 2:4, h * d:(h + 1) * d], ref, 20 * E * ref.abs(), f"head {h}")
    assert dx.isfinite().all() and dwq.isfinite().all() and dwk.isfinite().all()


def test_more_tiles_than_a_grid_and_offsets_past_31_bits():
    """2^22 + 5 tokens of 512 features: a workgroup takes a second tile of tokens, elements lie past 2^31."""
    L, d = 2 ** 22 + 5, 512
    x = torch.empty(1, 1, L, d, dtype=BF16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(31))
    pos, f = torch.arange(L, device="cuda"), tk.rope_frequencies(d // 2)
    y = tk.rope(x, pos, f)
    for a, b in ((0, 9), (L // 2 - 3, L // 2 + 4), (2 ** 22 - 6, L)):
        assert torch.equal(y[:, :, a:b], tk.rope(x[:, :, a:b], pos[a:b], f))
    ref, size = _turn(x[:, :, -7:].double(), pos[None, None, -7:], f, (0,) * (d // 2), False)
    _close(y[:, :, -7:], ref, 10 * E * size, "last rows")


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("d,pairs", [(128, 64), (70, 11)])
@pytest.mark.parametrize("adjacent", [False, True])
def test_rope_over_its_input(dt, d, pairs, adjacent):
    """The C call with out = x, by whole accesses and by single elements."""
    x = _randn(41, 2, 3, 301, d, dtype=dt)
    pos, f = torch.arange(301, device="cuda") * 3, tk.rope_frequencies(pairs)
    want = tk.rope(x, pos, f, adjacent=adjacent)
    rot = tk._Rotation(pos.data_ptr(), f.data_ptr(), None, 2 * pairs, 0, 0, 1, 1, 8, int(adjacent), 0)
    rc = tk.lib().topk_rope(x.data_ptr(), x.data_ptr(), 2, 3, 301, d, *x.stride()[:3], rot, int(dt is BF16), torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and torch.equal(x, want)


def _same(a, b):
    """Equal, with the sign of zeros; NaN equals NaN."""
    return bool((((a == b) & (a.signbit() == b.signbit())) | (a.isnan() & b.isnan())).all())


PASSING = [(80, 20, False), (80, 20, True), (70, 11, False), (70, 11, True), (64, 0, False), (70, 0, False), (512, 128, False)]
# features behind the rotated ones: places in (B, H, L) and what stands there
ODD = {(0, 0, 0): math.inf, (1, 1, 4): -math.inf, (0, 1, 2): math.nan, (1, 0, 3): -0.0}


def _spoil(t, first):
    """t [B, h, L, d] with ODD in its features from `first` on (one each)."""
    t = t.clone()
    for i, (at, x) in enumerate(ODD.items()):
        t[at[0], at[1] % t.shape[1], at[2], first + (5 * i) % (t.shape[-1] - first)] = x
    return t


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("d,pairs,adjacent", PASSING)
def test_features_that_are_not_rotated_stay_alone(dt, d, pairs, adjacent):
    """What is infinite, NaN or minus zero behind the rotated features comes out as it went in, and meets
    no other feature."""
    x = _randn(100, 2, 2, 5, d, dtype=dt)
    odd = _spoil(x, 2 * pairs)
    pos, f = torch.arange(5, device="cuda") + 3, tk.rope_frequencies(pairs) if pairs else torch.zeros(0, dtype=torch.float64, device="cuda")
    for inverse in (False, True):
        y, plain = (tk.rope(t, pos, f, adjacent=adjacent, inverse=inverse) for t in (odd, x))
        assert _same(y[..., 2 * pairs:], odd[..., 2 * pairs:])
        assert torch.equal(y[..., :2 * pairs], plain[..., :2 * pairs])
    # the packed form without a norm: the same numbers
    rot = dict(positions=pos, freqs=f, adjacent=adjacent) if pairs else {}
    packed = torch.cat((odd, x[:, :1].roll(1, 2), odd[:, 1:]), 1)
    q, k, v = tk.qk_norm_rope(packed.transpose(1, 2).reshape(2, 5, 4 * d), 2, 1, norm=False, **rot)
    assert _same(q, tk.rope(odd, pos, f, adjacent=adjacent)) and _same(v, odd[:, 1:])


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("d,pairs,adjacent", [p for p in PASSING if p[1]])
def test_infinite_features_beside_a_norm(dt, d, pairs, adjacent):
    """An infinite feature makes its head's root mean square infinite: it becomes NaN, the others 0. An
    infinite gradient of a feature that is not rotated reaches the gradient of that feature's weight alone."""
    rot = dict(positions=torch.arange(5, device="cuda") + 3, freqs=tk.rope_frequencies(pairs), adjacent=adjacent)
    x = _randn(102, 2, 5, 4, d, dtype=dt)
    w = _randn(103, d, dtype=dt, mean=1.0)
    odd, at = x.clone(), 2 * pairs + 3
    odd[1, 2, 0, at] = math.inf
    q, k, v = tk.qk_norm_rope(odd.view(2, 5, 4 * d), 2, 1, w, w, **rot)
    want = tk.qk_norm_rope(x.view(2, 5, 4 * d), 2, 1, w, w, **rot)
    assert bool(q[1, 0, 2, at].isnan())
    rest = torch.arange(d, device="cuda") != at
    assert not q[1, 0, 2, rest].any()
    q[1, 0, 2] = want[0][1, 0, 2]
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, want[2])
    g = [_randn(104 + i, 2, h, 5, d, dtype=dt) for i, h in enumerate((2, 1, 1))]
    dwq = tk.qk_norm_rope_backward(x.view(2, 5, 4 * d), 2, 1, *g, w, w, **rot)[1]
    g[0][1, 0, 2, at] = math.inf
    got = tk.qk_norm_rope_backward(x.view(2, 5, 4 * d), 2, 1, *g, w, w, **rot)[1]
    assert not bool(got[at].isfinite()) and torch.equal(got[rest], dwq[rest])


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("d,pairs,adjacent", PASSING)
def test_gradient_of_a_rotation_does_not_depend_on_its_input(dt, d, pairs, adjacent):
    """Without a norm the gradient is the turned one, to the sign of its zeros, whatever the projection holds."""
    rot = dict(positions=torch.arange(5, device="cuda") + 3, freqs=tk.rope_frequencies(pairs), adjacent=adjacent) if pairs else {}
    g = [_randn(110 + i, 2, h, 5, d, dtype=dt) for i, h in enumerate((2, 1, 1))]
    qkv = _randn(113, 2, 5, 4 * d, dtype=dt)
    want = tk.qk_norm_rope_backward(qkv, 2, 1, *g, norm=False, **rot)[0]
    for x in (math.inf, -math.inf, math.nan):
        assert _same(tk.qk_norm_rope_backward(torch.full_like(qkv, x), 2, 1, *g, norm=False, **rot)[0], want)
    pos, f = torch.arange(5, device="cuda") + 3, tk.rope_frequencies(pairs) if pairs else torch.zeros(0, dtype=torch.float64, device="cuda")
    g = [_spoil(t, 2 * pairs) for t in g]
    back = tk.qk_norm_rope_backward(qkv, 2, 1, *g, norm=False, **rot)[0].view(2, 5, 4, d).transpose(1, 2)
    for t, at in zip(g[:2], (0, 2)):
        assert _same(back[:, at:at + t.shape[1]], tk.rope(t, pos, f, adjacent=adjacent, inverse=True))
    assert _same(back[:, 3:], g[2])


def test_rotation_alone_keeps_no_input():
    """Nothing of the projection is held for the gradient where there is no norm: it may be overwritten."""
    pos, f = torch.arange(9, device="cuda"), tk.rope_frequencies(32)
    leaf = _randn(120, 2, 9, 4 * 64, dtype=BF16).requires_grad_()
    g = [_randn(121 + i, 2, h, 9, 64, dtype=BF16) for i, h in enumerate((2, 1, 1))]
    for kw in (dict(positions=pos, freqs=f), dict()):
        qkv = leaf * 2
        outs = layers.norm_rotary_heads(qkv, 2, 1, norm=False, **kw)
        want = tk.qk_norm_rope_backward(qkv.detach().clone(), 2, 1, *g, norm=False, **kw)[0] * 2
        with torch.no_grad():
            qkv.fill_(math.nan)
        assert torch.equal(torch.autograd.grad(outs, leaf, g)[0], want)


LOOPS = {
    # name: dtype, L, H, Hkv, d, pairs of each axis, adjacent (each with two tiles of tokens a workgroup in the
    # backward pass, the last workgroup's second tile missing, the last tile ragged)
    "rotated": (BF16, 11003, 3, 3, 128, (64,), False),
    "single_features": (F32, 11003, 3, 3, 70, (7, 3), True),
    "not_rotated": (BF16, 24004, 3, 3, 64, (), False),
    "half_rotated": (BF16, 21861, 2, 1, 128, (32,), True),
}


@pytest.mark.parametrize("name", sorted(LOOPS))
def test_backward_over_several_tiles_a_workgroup(name):
    dt, L, H, Hkv, d, sections, adjacent = LOOPS[name]
    qkv = _randn(130, 1, L, (H + 2 * Hkv) * d, dtype=dt, std=1.5)
    wq, wk = (_randn(s, d, dtype=dt, std=0.2, mean=1.0) for s in (131, 132))
    kw = dict(norm=True)
    if sections:
        pos = torch.randint(0, 100000, (len(sections), 1, L), generator=torch.Generator(device="cuda").manual_seed(133), device="cuda")
        kw.update(positions=pos, freqs=tk.rope_frequencies(sections), axes=tk.rope_axes(sections), adjacent=adjacent)
    grads = [_randn(134 + i, 1, h, L, d, dtype=dt) for i, h in enumerate((H, Hkv, Hkv))]
    dx, tol, dw = _grad_reference(qkv, H, Hkv, wq, wk, kw, grads)
    got = tk.qk_norm_rope_backward(qkv, H, Hkv, *grads, wq, wk, **kw)
    _close(got[0], dx, tol, "d_qkv")
    for g, r, n in zip(got[1:], dw, ("d_q_weight", "d_k_weight")):
        _close(g, r[0], r[1], n)
    if sections:
        got = tk.qk_norm_rope_backward(qkv, H, Hkv, *grads, **dict(kw, norm=False))
        dx, tol, _ = _grad_reference(qkv, H, Hkv, None, None, dict(kw, norm=False), grads)
        _close(got[0], dx, tol, "d_qkv without a norm")
