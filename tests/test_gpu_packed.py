"""GPU parity of attention over packed sequences against Eq. 1 in 64 bits.

Tolerance of an output element: half a step of bf16 relative to it, and twice the relative error
of a weight times sum_j w_j |v_j|. A weight is off by its score's rounding (d products summed in fp32:
at most (d + 8) 2^-24 sum |q k| scale), by the rounding of the exponent (2^-22 of the largest) and by
its own to bf16 (2^-9 at most; the sum that it is divided by is of the rounded ones, off by no more: that is the
doubling).

Tolerances of the gradients. With u = 2^-9 (half a step of bf16 relative to the number), w the weights,
a = d_out v^T and D = d_out . out: a recomputed weight is off by delta' = delta and the rounding of lse
(2^-21 (1 + |lse|), as tested), D by u |d_out| . |out| (out is stored in bf16; 2^-17 where what rounding took is
passed on too) and sums' rounding, and
ds = w (a - D) by its own rounding u besides; so with e = delta' and A = (d + 8) 2^-24 |d_out| |v|^T
    dv: half a step of the result, and (u + e) w^T |d_out|
    dq: half a step, and scale (u + e) |ds| |k| + scale (w (A + u |d_out| . |out| + its sums)) |k|, dk likewise with |q|.
Every bound is doubled for terms of second order.
"""
import math

import pytest
import torch

import paper_2106_06899_amd as tk
from paper_2106_06899_amd import layers

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    tk.lib()
    yield


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _inputs(offsets, N, H, Hkv, d, seed=0, std=2.0, tokens=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(heads, std):
        x = (torch.randn(N, heads, d, generator=gen, device="cuda") * std).to(BF16).transpose(0, 1)
        return x if tokens else x.contiguous()

    return normal(H, std), normal(Hkv, 1.0), normal(Hkv, 1.0), _int(offsets)


def _sequence(q, k, causal, scale):
    """Scores of one sequence and head in 64 bits, what is hidden, and the size of the scores' terms."""
    s = q.double() @ k.double().t() * scale
    n = len(q)
    hidden = torch.ones(n, n, dtype=torch.bool, device="cuda").triu_(1) if causal else torch.zeros(n, n, dtype=torch.bool, device="cuda")
    size = (q.double().abs() @ k.double().abs().t()).masked_fill(hidden, 0).amax(-1, keepdim=True) * scale
    return s.masked_fill(hidden, -math.inf), hidden, size


def _check(q, k, v, offsets, causal, scale, out, lse=None):
    H, N, d = q.shape
    G = H // k.shape[0]
    off, worst = offsets.tolist(), 0.0
    outside = torch.ones(N, dtype=torch.bool, device="cuda")
    for a, z in zip(off, off[1:]):
        outside[a:z] = False
        for h in range(H if z > a else 0):
            vv = v[h // G, a:z].double()
            s, hidden, size = _sequence(q[h, a:z], k[h // G, a:z], causal, scale)
            w = torch.softmax(s, -1)
            ref = w @ vv
            delta = ((d + 8) * 2.0 ** -24 + 2.0 ** -22) * size
            tol = 2.0 ** -8 * ref.abs() + 2 * (delta + 2.0 ** -9) * (w @ vv.abs()) + 1e-37
            err = (out[h, a:z].double() - ref).abs()
            assert bool((err <= tol).all()), f"sequence {a}:{z} head {h}: error {float((err / tol).max()):.2f} of its bound"
            worst = max(worst, float((err / tol).max()))
            if lse is not None:
                want = torch.logsumexp(s, -1)
                assert bool(((lse[h, a:z].double() - want).abs() <= 2 * delta[:, 0] + 2.0 ** -21 * (1 + want.abs())).all())
    assert not out[:, outside].any()
    assert lse is None or bool((lse[:, outside] == -math.inf).all())
    print(f"[case] worst error {worst:.3f} of its bound", flush=True)


CASES = {
    # name: offsets, N, H, Hkv, d, causal
    "one_token": ([0, 1], 1, 1, 1, 64, True),
    "one_token_each": ([0, 1, 2, 3], 3, 2, 1, 128, False),
    "two_tokens": ([0, 2], 2, 8, 8, 128, True),
    "empty_ones": ([0, 0, 5, 5, 5, 12, 12], 12, 4, 2, 64, True),
    "only_empty": ([3, 3, 3], 7, 2, 2, 128, True),
    "outside": ([5, 40, 90], 133, 3, 1, 64, True),
    "outside_all_keys": ([1, 300], 301, 2, 2, 128, False),
    "tile_edges": ([0, 63, 127, 255, 256, 320, 449, 705], 705, 2, 1, 64, True),
    "tile_edges_d128": ([0, 64, 192, 320, 449, 641], 641, 2, 1, 128, True),
    "tile_edges_all_keys": ([0, 64, 129, 256, 449, 641], 641, 2, 1, 128, False),
    "odd_groups": ([0, 77, 300], 300, 15, 3, 64, True),
    "eight_heads": ([0, 130, 201, 700], 700, 16, 4, 128, True),
    "many": ([i * (i + 1) // 2 for i in range(64)], 2016, 2, 1, 64, True),
    "more_than_a_wave_of_them": ([i * 7 for i in range(150)], 1043, 2, 2, 64, True),
    "more_all_keys": ([i * 13 for i in range(70)], 897, 1, 1, 128, False),
    "hundreds_of_them": ([(i * 5) // 2 for i in range(700)], 1748, 1, 1, 64, True),
    "thousands": ([min(i, 2500) for i in range(2600)], 2510, 1, 1, 128, False),
    "mostly_padding": ([100, 200, 330], 9000, 4, 2, 64, True),
    "mostly_padding_d128": ([1000, 1200, 1201], 9001, 4, 1, 128, False),
    "padding_behind_many": ([7 * i + 500 for i in range(100)], 7000, 2, 2, 64, True),
    # more than 256 workgroups of 128 rows: a workgroup's waves have rows of their own
    "many_workgroups": ([0, 1000, 1003, 3200], 3210, 12, 3, 64, True),
    "many_workgroups_d128": ([0, 1000, 1064, 3200], 3200, 12, 12, 128, True),
    "many_workgroups_all_keys": ([5, 1000, 1003, 3200], 3210, 12, 3, 64, False),
    "many_workgroups_all_keys_d128": ([0, 1000, 1003, 3200], 3210, 12, 4, 128, False),
    "more_than_two_a_cu": ([0, 130, 3300, 3301, 5600], 5600, 14, 2, 64, True),
    "long": ([0, 2000, 5003], 5003, 2, 1, 128, True),
    "long_d64": ([0, 3001, 3002, 5000], 5000, 2, 2, 64, True),
    "shared_out": ([0, 1100, 1133, 2300], 2310, 4, 1, 128, True),
    "shared_out_d64": ([3, 1500], 1500, 6, 2, 64, True),
    "shared_out_all_keys": ([0, 900, 900], 905, 5, 1, 128, False),
    "long_all_keys": ([0, 1500, 3333], 3333, 2, 1, 64, False),
}


@pytest.mark.parametrize("name", sorted(CASES))
@pytest.mark.parametrize("tokens", [False, True])
def test_packed(name, tokens):
    offsets, N, H, Hkv, d, causal = CASES[name]
    q, k, v, off = _inputs(offsets, N, H, Hkv, d, tokens=tokens)
    out, lse = tk.attn_packed(q, k, v, off, causal, lse=True)
    assert out.stride() == q.stride()
    _check(q, k, v, off, causal, d ** -0.5, out, lse)
    same = torch.equal(tk.attn_packed(q, k, v, off, causal), out)
    assert same


def test_what_rounding_took():
    """out and rest together are the result to 16 bits, 0 for tokens of no sequence."""
    q, k, v, off = _inputs([3, 100, 300], 310, 4, 2, 128, tokens=True)
    out, rest = tk.attn_packed(q, k, v, off, rest=True)
    same = torch.equal(out, tk.attn_packed(q, k, v, off)) and rest.stride() == out.stride()
    assert same and not rest[:, :3].any() and not rest[:, 300:].any()
    assert bool((rest.float().abs() <= 2.0 ** -8 * out.float().abs()).all()) and bool(rest.any())
    # What rounding took is at most half a step, which bf16 holds: rounded itself, it leads midway to the next number
    # at most (the low half of the exact sum's bits is then 0x8000), where the sum may round the other way.
    both = out.float() + rest.float()
    other = both.bfloat16() != out
    assert bool(((both.contiguous().view(torch.int32) & 0xFFFF)[other] == 0x8000).all())


@pytest.mark.parametrize("name", [n for n, (off, N, _, _, d, _) in sorted(CASES.items()) if d == 64 or N <= 1024 or N <= 64 * (len(off) - 1)])
def test_weights_of_two_numbers(name):
    """In a training pass over heads of 64, or a short one, out and rest together have the weights to 16 bits: off by at
    most 2^-16 from the weights' second rounding, as much from rest's, and from sums of n terms in 32 bits."""
    offsets, N, H, Hkv, d, causal = CASES[name]
    q, k, v, off = _inputs(offsets, N, H, Hkv, d)
    out, lse, rest = tk.attn_packed(q, k, v, off, causal, lse=True, rest=True)
    _check(q, k, v, off, causal, d ** -0.5, out, lse)
    both = out.double() + rest.double()
    for a, z in zip(offsets, offsets[1:]):
        for h in range(H if z > a else 0):
            vv = v[h // (H // Hkv), a:z].double()
            s, _, size = _sequence(q[h, a:z], k[h // (H // Hkv), a:z], causal, d ** -0.5)
            w = torch.softmax(s, -1)
            ref = w @ vv
            delta = ((d + 8) * 2.0 ** -24 + 2.0 ** -22) * size
            tol = 2.0 ** -16 * ref.abs() + 2 * (delta + 2.0 ** -17 + (z - a + 8) * 2.0 ** -24) * (w @ vv.abs()) + 1e-37
            assert bool(((both[h, a:z] - ref).abs() <= tol).all()), (a, z, h)


@pytest.mark.parametrize("far", ["tokens", "heads"])
def test_tokens_and_heads_far_apart(far):
    """Offsets past 32 bits: the same numbers as of tensors that lie in one piece."""
    N, d = 290, 128
    H, Hkv = (4, 2) if far == "tokens" else (2, 2)
    q, k, v, off = _inputs([0, 130, 290], N, H, Hkv, d)
    g, want = _gradient(q, k, v, off)
    ref, lse = tk.attn_packed(q, k, v, off, lse=True)
    head, token = (d, (1 << 24) - 8) if far == "tokens" else ((1 << 31) + 8, 2 * d)
    buf = torch.zeros((N - 1) * token + (H - 1) * head + 8 * d, dtype=BF16, device="cuda")  # 5 to 10 GB

    def there(x, at):
        return buf[at:].as_strided(x.shape, (head, token, 1)).copy_(x)

    second = 4 * d if far == "tokens" else d  # beside the first
    for first, other in ((0, 1), (3, 2)):  # queries and keys; gradients and values
        x = [q, k, v, g]
        x[first], x[other] = there(x[first], 0), there(x[other], second)
        out, sums = tk.attn_packed(*x[:3], off, lse=True)
        got = tk.attn_packed_backward(*x[:3], off, out.contiguous(), sums, x[3])
        same = torch.equal(out, ref) and torch.equal(sums, lse) and all(torch.equal(a, b) for a, b in zip(got, want))
        assert same, first


def test_scale_and_large_scores():
    q, k, v, off = _inputs([0, 200, 333], 333, 2, 1, 64, std=8.0)
    for scale in (1e-3, 0.7):
        _check(q, k, v, off, True, scale, *tk.attn_packed(q, k, v, off, scale=scale, lse=True))


def test_cut_from_a_projection():
    """q, k and v as columns of one packed projection; the result as contiguous heads would give it."""
    H, Hkv, d, N = 4, 2, 64, 300
    x = torch.randn(N, (H + 2 * Hkv) * d, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(BF16)
    q, k, v = x.view(N, H + 2 * Hkv, d).transpose(0, 1).split((H, Hkv, Hkv))
    off = _int([0, 111, 300])
    out = tk.attn_packed(q, k, v, off)
    same = torch.equal(out, tk.attn_packed(q.contiguous(), k.contiguous(), v.contiguous(), off))
    assert same


# (few heads: two waves share rows; a hundred: rows of their own)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("d,H", [(64, 2), (128, 2), (64, 100), (128, 100)])
@pytest.mark.parametrize("rest", [False, True])
def test_hidden_rows_may_hold_anything(bad, d, H, rest):
    """Later tokens, other sequences and tokens of none hold numbers that are not finite: rows that
    do not see them are as if they were not there."""
    off, N = [0, 150, 200, 420], 430
    q, k, v, o = _inputs(off, N, H, H // 2, d, seed=3)
    want, wl = tk.attn_packed(q, k, v, o, lse=True, rest=rest)[:2]
    k2, v2 = k.clone(), v.clone()
    for t in (149, 100, 330, 425):
        v2[:, t, t % d] = bad
    k2[:, 427] = v2[:, 428] = bad
    got, gl = tk.attn_packed(q, k2, v2, o, lse=True, rest=rest)[:2]
    same = torch.equal(gl, wl)
    assert same
    for a, z, ts in ((0, 150, (100, 149)), (150, 200, ()), (200, 420, (330,))):
        for i in range(a, z):
            cols = {t % d for t in ts if t <= i}
            clean = [f for f in range(d) if f not in cols]
            assert torch.equal(got[:, i, clean], want[:, i, clean]), i
            assert all(not got[:, i, f].isfinite().any() for f in cols), i
    assert not got[:, 420:].any()
    k3 = k.clone()
    k3[:, 300] = bad  # a key: rows before it are untouched
    same = torch.equal(tk.attn_packed(q, k3, v, o, lse=True, rest=rest)[0][:, :300], want[:, :300])
    assert same


def test_tiny_weights_and_a_late_maximum():
    """Weights below 2^-126 still count against large values, before and behind a maximum that leads
    them by far."""
    for H in (1, 300):
        _tiny(64, 200, H), _tiny(128, 100, H)


def _tiny(d, n, H):
    q = torch.zeros(H, n, d, device="cuda", dtype=BF16)
    k, v = torch.zeros_like(q), torch.zeros_like(q)
    q[..., 0] = 1
    for at in (10, n - 10):
        k[:] = 0
        k[:, at, 0] = 88.5
        v[:] = 2.0 ** 100
        v[:, at] = 1.0
        off = _int([0, n])
        out = tk.attn_packed(q, k, v, off, causal=False, scale=1.0)
        s = q[0].double() @ k[0].double().t()
        ref = torch.softmax(s, -1) @ v[0].double()
        assert bool(((out.double() - ref).abs() <= 2.0 ** -7 * ref.abs()).all()), at
        out = tk.attn_packed(q, k, v, off, causal=False, scale=1.0, lse=True, rest=True)[0]
        assert bool(((out.double() - ref).abs() <= 2.0 ** -7 * ref.abs()).all()), at


def test_streams_and_graphs():
    q, k, v, off = _inputs([0, 90, 400], 400, 4, 2, 128, seed=5)
    want = tk.attn_packed(q, k, v, off)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = tk.attn_packed(q, k, v, off)
    torch.cuda.current_stream().wait_stream(s)
    same = torch.equal(got, want)
    assert same
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = tk.attn_packed(q, k, v, off)
    for o in ([0, 90, 400], [0, 5, 300], [7, 333, 400]):
        off.copy_(_int(o))
        g.replay()
        torch.cuda.synchronize()
        same = torch.equal(out, tk.attn_packed(q, k, v, off))
        assert same


@pytest.mark.parametrize("more", [0, 100])  # (so many sequences more)
def test_offsets_that_decrease_stay_inside(more):
    """No meaningful result, but nothing outside the tensors is read or written."""
    q, k, v, off = _inputs([0, 200, 100, 300] + more * [300], 300, 2, 1, 64)
    for o in ([0, 200, 100, 300], [-50, 100, 1000, 3], [2 ** 31 - 1, -2 ** 31, 300, 300]):
        off.copy_(_int((o * (1 + more // 4))[:4 + more]))
        out, lse = tk.attn_packed(q, k, v, off, lse=True)
        grads = tk.attn_packed_backward(q, k, v, off, out, lse, q)
        torch.cuda.synchronize()
        assert [t.shape for t in (out, *grads)] == [q.shape, q.shape, k.shape, v.shape]


def test_refused_on_the_gpu():
    q, k, v, off = _inputs([0, 50], 50, 4, 2, 64)
    for args in ((q[0], k, v, off), (q, k[:, :40], v, off), (q, k, v, off[:1]), (q, k, v[..., ::2], off), (q.cpu(), k, v, off)):
        with pytest.raises(ValueError):
            tk.attn_packed(*args)
    with pytest.raises(TypeError):
        tk.attn_packed(q, k, v, off.long())
    with pytest.raises(TypeError):
        tk.attn_packed(q, k.float(), v, off)
    for args in ((q.float(), k.float(), v.float(), off), (q[:3], k, v, off), (q[..., :32], k[..., :32], v[..., :32], off)):
        with pytest.raises(tk.TopkError):
            tk.attn_packed(*args)
    assert tk.attn_packed(q[:, :0], k[:, :0], v[:, :0], off).shape == (4, 0, 64)


def _grad_check(q, k, v, offsets, g, causal, scale, grads, rest=False):
    H, N, d = q.shape
    Hkv = k.shape[0]
    G = H // Hkv
    dq, dk, dv = grads
    u = 2.0 ** -9
    outside = torch.ones(N, dtype=torch.bool, device="cuda")
    off, worst = offsets.tolist(), 0.0
    for a, z in zip(off, off[1:]):
        outside[a:z] = False
        if z <= a:
            continue
        for hk in range(Hkv):
            kk, vv = k[hk, a:z].double(), v[hk, a:z].double()
            want = [torch.zeros(z - a, d, dtype=torch.float64, device="cuda") for _ in range(2)]
            tol = [torch.zeros_like(want[0]) for _ in range(2)]
            for h in range(hk * G, hk * G + G):
                qq, gg = q[h, a:z].double(), g[h, a:z].double()
                s, hidden, size = _sequence(q[h, a:z], k[hk, a:z], causal, scale)
                w = torch.softmax(s, -1)
                lse = torch.logsumexp(s, -1, keepdim=True)
                out = w @ vv
                x = gg @ vv.t()
                D = (gg * out).sum(-1, keepdim=True)
                ds = w * (x - D)
                # (out is off by its weights too: their bound is part of D's)
                e = 2 * ((d + 8) * 2.0 ** -24 + 2.0 ** -22) * size + 2.0 ** -21 * (1 + lse.abs())
                out_off = 2.0 ** (-17 if rest else -9) * out.abs() + 2 * (e + u) * (w @ vv.abs())
                D_off = (gg.abs() * out_off).sum(-1, keepdim=True) + d * 2.0 ** -24 * (gg.abs() * out.abs()).sum(-1, keepdim=True)
                A = (d + 8) * 2.0 ** -24 * (gg.abs() @ vv.abs().t())
                ds_off = ((u + e) * ds.abs() + w * (A + D_off)).masked_fill(hidden, 0)
                for name, got, ref, t in (("dq", dq[h, a:z], scale * ds @ kk, 2 * scale * ds_off @ kk.abs()),):
                    t = t + 2.0 ** -8 * ref.abs() + 1e-37
                    err = (got.double() - ref).abs()
                    assert bool((err <= t).all()), f"{name} of sequence {a}:{z} head {h}: error {float((err / t).max()):.2f} of its bound"
                    worst = max(worst, float((err / t).max()))
                want[0] += scale * ds.t() @ qq
                tol[0] += 2 * scale * ds_off.t() @ qq.abs()
                want[1] += w.t() @ gg
                tol[1] += 2 * ((u + e) * w).t() @ gg.abs()
            for name, got, ref, t in (("dk", dk[hk, a:z], want[0], tol[0]), ("dv", dv[hk, a:z], want[1], tol[1])):
                t = t + 2.0 ** -8 * ref.abs() + 1e-37
                err = (got.double() - ref).abs()
                assert bool((err <= t).all()), f"{name} of sequence {a}:{z} head {hk}: error {float((err / t).max()):.2f} of its bound"
                worst = max(worst, float((err / t).max()))
    for t in grads:
        assert not t[:, outside].any()
    print(f"[case] worst gradient error {worst:.3f} of its bound", flush=True)


def _gradient(q, k, v, off, causal=True, scale=None, seed=9, tokens=False):
    g = torch.randn(q.shape[1], q.shape[0], q.shape[2], generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(BF16).transpose(0, 1)
    if not tokens:
        g = g.contiguous()
    if tokens:  # with what rounding took from out
        out, lse, rest = tk.attn_packed(q, k, v, off, causal, scale, lse=True, rest=True)
        return g, tk.attn_packed_backward(q, k, v, off, out, lse, g, causal, scale, rest)
    out, lse = tk.attn_packed(q, k, v, off, causal, scale, lse=True)
    return g, tk.attn_packed_backward(q, k, v, off, out, lse, g, causal, scale)


@pytest.mark.parametrize("name", sorted(CASES))
@pytest.mark.parametrize("tokens", [False, True])
def test_packed_backward(name, tokens):
    offsets, N, H, Hkv, d, causal = CASES[name]
    q, k, v, off = _inputs(offsets, N, H, Hkv, d, tokens=tokens)
    g, grads = _gradient(q, k, v, off, causal, tokens=tokens)
    assert [t.stride() for t in grads] == [t.stride() for t in (q, k, v)]
    _grad_check(q, k, v, off, g, causal, d ** -0.5, grads, rest=tokens)
    same = all(torch.equal(a, b) for a, b in zip(grads, _gradient(q, k, v, off, causal, tokens=tokens)[1]))
    assert same


def test_keys_shared_by_expansion():
    """Keys and values that are one head expanded: the gradient is whole, and autograd's sum over the heads is that of
    one shared head but for its roundings."""
    off = _int([0, 60, 200])
    q, k, v, _ = _inputs([0, 200], 200, 4, 1, 64)
    g = _gradient(q, k, v, off)[0]
    k1, v1 = k.clone().requires_grad_(), v.clone().requires_grad_()
    out = layers.packed_attention(q, k1.expand(4, -1, -1), v1.expand(4, -1, -1), off)
    same = torch.equal(out, tk.attn_packed(q, k, v, off, lse=True, rest=True)[0])
    assert same
    got = torch.autograd.grad(out, (k1, v1), g)
    k2, v2 = k.clone().requires_grad_(), v.clone().requires_grad_()
    want = torch.autograd.grad(layers.packed_attention(q, k2, v2, off), (k2, v2), g)
    for a, b in zip(got, want):  # four roundings of parts and their sum's
        parts = 4 * b.float().abs().amax()
        assert bool(((a.float() - b.float()).abs() <= 5 * 2.0 ** -9 * parts).all())


def test_gradients_against_differences():
    """Central differences of the 64-bit definition in a few directions: what the tests above take for the
    gradient is the gradient."""
    d, off = 64, [0, 9, 30]
    q, k, v, o = _inputs(off, 30, 2, 1, d, std=1.0)
    g, grads = _gradient(q, k, v, o)

    def loss(q, k, v):
        total = 0.0
        for a, z in zip(off, off[1:]):
            for h in range(2):
                s = q[h, a:z] @ k[0, a:z].t() / 8
                s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu_(1), -math.inf)
                total += float((torch.softmax(s, -1) @ v[0, a:z] * g[h, a:z].double()).sum())
        return total

    gen = torch.Generator(device="cuda").manual_seed(2)
    x = [t.double() for t in (q, k, v)]
    for i in range(3):
        for _ in range(3):
            u = torch.randn(x[i].shape, generator=gen, device="cuda", dtype=torch.float64)
            step = 1e-5
            up, down = ([t + s * step * u if j == i else t for j, t in enumerate(x)] for s in (1, -1))
            slope = (loss(*up) - loss(*down)) / (2 * step)
            got = float((grads[i].double() * u).sum())
            # each element is within 2^-6 of its size at most, and independent: their sum stays within 2^-6 of the whole
            assert abs(got - slope) <= 2.0 ** -6 * float((grads[i].double() * u).norm()) + 1e-6, (i, got, slope)


def test_autograd_on_layouts_and_broadcast_gradients():
    """Leaves as tokens, a gradient that is one number expanded, and values that need no gradient."""
    N, H, Hkv, d = 200, 4, 2, 64
    off = _int([0, 70, 200])
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(N, H + 2 * Hkv, d, generator=gen, device="cuda").to(BF16).requires_grad_()
    q, k, v = x.transpose(0, 1).split((H, Hkv, Hkv))
    out = layers.packed_attention(q, k, v, off)
    out.sum().backward()
    ones = torch.ones(H, N, d, dtype=BF16, device="cuda")
    o, lse, rest = tk.attn_packed(q.detach(), k.detach(), v.detach(), off, lse=True, rest=True)
    want = torch.cat(tk.attn_packed_backward(q.detach(), k.detach(), v.detach(), off, o, lse, ones, rest=rest)).transpose(0, 1)
    same = torch.equal(x.grad, want)
    assert same
    y = x.detach().transpose(0, 1)[:H].requires_grad_()
    (dq,) = torch.autograd.grad(layers.packed_attention(y, k.detach(), v.detach(), off).float().sum(), y)
    same = torch.equal(dq, want.transpose(0, 1)[:H])
    assert same


@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("d,H", [(64, 2), (128, 2), (64, 100), (128, 100)])
@pytest.mark.parametrize("N", [300, 1300])  # (a short pass, and not)
def test_gradients_of_hidden_rows(bad, d, H, N):
    """Numbers that are not finite reach the gradients of what meets them, no other."""
    off = [0, 150, 290]
    q, k, v, o = _inputs(off, N, H, H // 2, d, seed=3)
    g, want = _gradient(q, k, v, o)
    out, lse = tk.attn_packed(q, k, v, o, lse=True)
    # d_out of token 100: dq of that token, dk and dv of the keys that it sees
    g2 = g.clone()
    g2[:, 100, 5] = bad
    g2[:, 295] = bad
    got = tk.attn_packed_backward(q, k, v, o, out, lse, g2)
    rows = [t for t in range(N) if t != 100]
    assert torch.equal(got[0][:, rows], want[0][:, rows]) and not got[0][:, 100].isfinite().any()
    for i in (1, 2):
        assert torch.equal(got[i][:, 101:], want[i][:, 101:])
    assert not got[2][:, :101, 5].isfinite().any()
    cols = [f for f in range(d) if f != 5]
    assert torch.equal(got[2][:, :, cols], want[2][:, :, cols])
    # a query of token 100: its output and logarithm with it
    q2 = q.clone()
    q2[:, 100, 3] = bad
    out2, lse2 = tk.attn_packed(q2, k, v, o, lse=True)
    got = tk.attn_packed_backward(q2, k, v, o, out2, lse2, g)
    for i in (1, 2):
        assert torch.equal(got[i][:, 101:], want[i][:, 101:])
    assert torch.equal(got[0][:, rows], want[0][:, rows])
    # a key and a value of token 100: rows that do not see them
    for which in (0, 1):
        kv = [k.clone(), v.clone()]
        kv[which][:, 100, 7] = bad
        out2, lse2 = tk.attn_packed(q, *kv, o, lse=True)
        got = tk.attn_packed_backward(q, *kv, o, out2, lse2, g)
        seen = list(range(100)) + list(range(150, N))
        assert torch.equal(got[0][:, seen], want[0][:, seen])
        assert torch.equal(got[1][:, 150:], want[1][:, 150:]) and torch.equal(got[2][:, 150:], want[2][:, 150:])


@pytest.mark.parametrize("N", [400, 1500])
def test_backward_in_graphs_and_streams(N):
    q, k, v, off = _inputs([0, 90, 400], N, 4, 2, 128, seed=5)
    g = _gradient(q, k, v, off)[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _gradient(q, k, v, off)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = tk.attn_packed(q, k, v, off, lse=True)
        grads = tk.attn_packed_backward(q, k, v, off, out, lse, g)
    for o in ([0, 90, 400], [0, 5, 300], [7, 333, 400]):
        off.copy_(_int(o))
        graph.replay()
        torch.cuda.synchronize()
        same = all(torch.equal(a, b) for a, b in zip(grads, _gradient(q, k, v, off)[1]))
        assert same


@pytest.mark.parametrize("behind", [1, 3, 8])  # (8 numbers are 16 bytes: an address that is taken as it is)
def test_gradients_at_any_address(behind):
    """A gradient that is in one piece, but at an address that the kernels do not take: the same numbers as at one that
    they do. Handed over, and as the backward of a flat vector of several results makes it."""
    off = _int([0, 60, 200])
    q, k, v, _ = _inputs([0, 200], 200, 4, 2, 64)
    x = [t.clone().requires_grad_() for t in (q, k, v)]
    g = _gradient(q, k, v, off)[0]
    want = torch.autograd.grad(layers.packed_attention(*x, off), x, g)
    odd = torch.cat((g.new_zeros(behind), g.flatten()))[behind:].view(g.shape)
    assert odd.is_contiguous() and bool(odd.data_ptr() % 16) == (behind < 8)
    got = torch.autograd.grad(layers.packed_attention(*x, off), x, odd)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    first = torch.ones(behind, device="cuda", dtype=BF16, requires_grad=True)
    both = torch.cat((first, layers.packed_attention(*x, off).flatten()))
    got = torch.autograd.grad(both, x, torch.cat((torch.ones_like(first), g.flatten())))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,H", [(64, 2), (128, 2), (64, 100), (128, 100)])
@pytest.mark.parametrize("rest", [False, True])
def test_infinite_values_that_are_seen(d, H, rest, causal):
    """By the definition a weight above 0 makes an infinite value an infinite output, of the same sign, two of different
    signs NaN, wherever the key lies: in a tile that all rows see, on the diagonal, last of its sequence."""
    off, N = [0, 150, 200, 420], 430
    q, k, v, o = _inputs(off, N, H, H // 2, d, seed=3)
    want, wl = tk.attn_packed(q, k, v, o, causal, lse=True, rest=rest)[:2]
    inf, nan = math.inf, math.nan
    v2 = v.clone()
    at = [(149, 0, inf), (100, 1, -inf), (20, 2, inf), (101, 2, -inf), (199, 3, -inf), (200, 4, inf), (330, 5, nan), (300, 6, -inf), (419, 7, inf), (419, d - 1, -inf),
          (400, d - 1, -inf), (201, 8, inf), (390, 8, -inf), (3, d - 2, nan)]
    for t, f, x in at:
        v2[:, t, f] = x
    for a, z in zip(off, off[1:]):
        here = torch.zeros(z - a, d, dtype=torch.float64)
        for t, f, x in at:
            if a <= t < z:
                here[t - a if causal else 0:, f] += x
        here = here.to(BF16).cuda()[None]
        want[:, a:z] = torch.where(here == 0, want[:, a:z], here)
    got = tk.attn_packed(q, k, v2, o, causal, lse=True, rest=rest)
    assert torch.equal(got[1], wl)
    assert bool(((got[0] == want) | (got[0].isnan() & want.isnan())).all())
    if rest:  # nothing was taken from what is not finite
        assert not got[2][~want.isfinite()].any()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,H", [(64, 2), (128, 2), (64, 100), (128, 100)])
@pytest.mark.parametrize("rest", [False, True])
def test_infinite_values_of_weights_that_32_bits_hold_as_0(d, H, rest, causal):
    """e^-200 is above 0 all the same."""
    n = 500
    q, k, v = (torch.zeros(H, n, d, device="cuda", dtype=BF16) for _ in range(3))
    q[..., 0] = 1
    for top in (3, 250, 499):
        k[:] = 0
        k[:, top, 0] = 200
        v[:] = 1
        for t, f, x in ((0, 1, math.inf), (100, 2, -math.inf), (300, 3, math.inf), (480, 4, -math.inf), (10, 5, math.inf), (470, 5, -math.inf)):
            v[:, t, f] = x
        want = v.float().cumsum(1) if causal else v.float().sum(1, keepdim=True).expand(-1, n, -1)
        want = torch.where(want.isfinite(), 1.0, want)
        out = tk.attn_packed(q, k, v, _int([0, n]), causal, 1.0, lse=True, rest=rest)[0].float()
        assert bool(((out == want) | (out.isnan() & want.isnan())).all()), top


TINY = 2.0 ** -127.68  # e^-88.5: as a bf16 number a multiple of 2^-133, off by 2^-134 at most, that is 2^-6.32 of it


@pytest.mark.parametrize("lse,rest", [(False, False), (True, False), (True, True)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d,n,H", [(64, 200, 1), (64, 200, 300), (128, 100, 1), (128, 100, 300), (64, 1100, 2), (64, 1100, 40), (128, 1100, 2), (128, 1100, 40)])
def test_tiny_weights_are_the_result(d, n, H, causal, lse, rest):
    """Values of 2^116 whose weights are e^-88.5 beside a value of 0 that has all the rest: the output is theirs alone, before
    and behind the key that leads them. (Rounding of the weight 2^-6.32, of the output 2^-8, of the rest less than 2^-10.)"""
    q, k, v = (torch.zeros(H, n, d, device="cuda", dtype=BF16) for _ in range(3))
    q[..., 0] = 1
    for at in (0, 10, 70, n - 10, n - 1):
        k[:], v[:] = 0, 2.0 ** 116
        k[:, at, 0], v[:, at] = 88.5, 0
        got = tk.attn_packed(q, k, v, _int([0, n]), causal, 1.0, lse=lse, rest=rest)
        out = (got[0] if lse else got).double()
        want = torch.full((n,), (n - 1) * math.exp(-88.5) * 2.0 ** 116, dtype=torch.float64, device="cuda")
        if causal:
            i = torch.arange(n, device="cuda").double()
            want = torch.where(i >= at, i * math.exp(-88.5) * 2.0 ** 116, 2.0 ** 116)
        assert bool(((out - want[None, :, None]).abs() <= (2.0 ** -6.32 + 2.0 ** -8 + 2.0 ** -10) * want[None, :, None]).all()), at


def _gradients_in_64_bits(q, k, v, offsets, g, causal, scale, rounded=lambda x: x):
    """dq, dk, dv; rounded: what is done to weights and score gradients on their way into the products."""
    H, N, d = q.shape
    G = H // k.shape[0]
    out = [torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (q, k, v)]
    for a, z in zip(offsets, offsets[1:]):
        for h in range(H if z > a else 0):
            qq, kk, vv, gg = (t[i, a:z].double() for t, i in ((q, h), (k, h // G), (v, h // G), (g, h)))
            w = torch.softmax(_sequence(q[h, a:z], k[h // G, a:z], causal, scale)[0], -1)
            ds = w * (gg @ vv.t() - (gg * (w @ vv)).sum(-1, keepdim=True))
            w, ds = rounded(w), rounded(ds)
            out[0][h, a:z] += scale * ds @ kk
            out[1][h // G, a:z] += scale * ds.t() @ qq
            out[2][h // G, a:z] += w.t() @ gg
    return out


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("offsets", [[0, 200, 201, 700], [0, 1000], [25 * i for i in range(81)]])
def test_gradients_of_two_numbers(offsets, d, causal):
    """A short pass has its weights and score gradients to 16 bits and D to as many: its gradients are off by what their own
    rounding to bf16 is. In the 2-norm that is 2^-16 of the sums' terms and the scores' roundings beside it, less than a
    tenth of it, and errors add in squares: a hundredth. With weights and score gradients of one bf16 number it would be 1.2 times
    as much at least."""
    N = offsets[-1] + 20
    q, k, v, off = _inputs(offsets, N, 4, 2, d, seed=6, std=1.0)
    g = torch.randn(q.shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(BF16)
    out, lse, rest = tk.attn_packed(q, k, v, off, causal, lse=True, rest=True)
    got = tk.attn_packed_backward(q, k, v, off, out, lse, g, causal, rest=rest)
    want = _gradients_in_64_bits(q, k, v, offsets, g, causal, d ** -0.5)
    one = _gradients_in_64_bits(q, k, v, offsets, g, causal, d ** -0.5, lambda x: x.to(BF16).double())
    for name, x, y, z in zip(("dq", "dk", "dv"), got, want, one):
        own = float((y.to(BF16).double() - y).norm())
        assert float((z.to(BF16).double() - y).norm()) >= 1.2 * own, name  # (the test can tell them apart)
        print(f"[case] {name}: {float((x.double() - y).norm()) / own:.3f} of its rounding", flush=True)
        assert float((x.double() - y).norm()) <= 1.05 * own, name


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d,H,Hkv", [(64, 2, 1), (128, 6, 2)])
@pytest.mark.parametrize("n", [3, 64, 65, 300])
@pytest.mark.parametrize("N", [300, 1500])  # (a short pass, and not)
def test_offsets_of_any_kind_stay_inside(N, n, d, H, Hkv, causal):
    """Whatever the offsets are, nothing outside the tensors is written, and nothing that is read there (NaN) reaches a
    result."""
    pad = 1 << 16
    rng = torch.Generator().manual_seed(n + d)
    shapes = dict(q=(H, N, d), k=(Hkv, N, d), v=(Hkv, N, d), g=(H, N, d), out=(H, N, d), rest=(H, N, d), dq=(H, N, d), dk=(Hkv, N, d), dv=(Hkv, N, d), lse=(H, N))
    whole, x = {}, {}
    for name, s in shapes.items():
        read = name in "qkvg"
        whole[name] = torch.full((math.prod(s) + 2 * pad,), math.nan if read else 3.0, dtype=torch.float32 if name == "lse" else BF16, device="cuda")
        x[name] = whole[name][pad:-pad].view(s)
        if read:
            x[name].copy_(torch.randn(s, generator=rng))
    off = _int([0] * (n + 1))
    st = tk._PackedStrides(*(N * d, d) * 8)
    p = {name: t.data_ptr() for name, t in x.items()}
    L, stream = tk.lib(), torch.cuda.current_stream().cuda_stream
    ws = tk.lib().topk_attn_packed_backward_workspace_bytes(n, N, H, Hkv, d, 1)
    far = torch.randint(-2 ** 31, 2 ** 31 - 1, (n + 1,), generator=rng)
    near = torch.randint(-50, N + 50, (n + 1,), generator=rng)
    inside = torch.randint(0, N + 1, (n + 1,), generator=rng)
    for o in (far, near, inside, inside.sort(descending=True)[0], torch.tensor([0, N] * n)[:n + 1]):
        off.copy_(o.int())
        for name in shapes:
            if name not in "qkvg":
                x[name].fill_(3.0)
        tk._launch(off.device, L.topk_attn_packed, (p["q"], p["k"], p["v"], off.data_ptr(), p["out"], p["lse"], p["rest"], n, N, H, Hkv, d, st, int(causal), d ** -0.5, 1, stream))
        tk._launch(off.device, L.topk_attn_packed_backward, (p["q"], p["k"], p["v"], off.data_ptr(), p["out"], p["lse"], p["rest"], p["g"], p["dq"], p["dk"], p["dv"], n, N, H, Hkv, d, st,
                                                             int(causal), d ** -0.5, 1, stream), ws)
        torch.cuda.synchronize()
        for name in shapes:
            if name not in "qkvg":
                assert bool((whole[name][:pad] == 3).all()) and bool((whole[name][-pad:] == 3).all()), name
                if N == 300 or name in ("out", "rest", "lse"):  # (shares of tokens that no tile covers are added up as they are)
                    assert not x[name].isnan().any(), name


@pytest.mark.parametrize("d", [64, 128])
def test_many_infinite_values(d):
    """Half of all values are infinite or NaN."""
    q, k, v, o = _inputs([0, 333, 600], 600, 4, 2, d, seed=5)
    gen = torch.Generator(device="cuda").manual_seed(0)
    kind = torch.randint(0, 40, v.shape, generator=gen, device="cuda")
    v = torch.where(kind == 0, math.inf, torch.where((kind == 1) & (torch.arange(d, device="cuda") % 2 == 0), -math.inf, v))
    v[:, 200, 7] = math.nan
    v[:, 300:] = torch.where(kind[:, 300:] >= 20, math.inf, v[:, 300:])
    for causal in (True, False):
        for rest in (True, False):
            out = tk.attn_packed(q, k, v, o, causal, lse=True, rest=rest)[0]
            for a, z in ((0, 333), (333, 600)):
                here = torch.where(v[:, a:z].isfinite(), 0.0, v[:, a:z].float())
                here = here.cumsum(1) if causal else here.sum(1, keepdim=True).expand(-1, z - a, -1)
                here = here.repeat_interleave(2, 0)
                got = out[:, a:z].float()
                assert bool(((got == here) | (got.isnan() & here.isnan()) | (here == 0) & got.isfinite()).all())
