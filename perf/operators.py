"""Rotary positions, head norms and shared-prefix attention: the calls whose speed is measured.

* ``rope`` (``layers.rotary`` in training): rotates the feature pairs of ``[B, H, L, d]`` heads by
  positions on one or several axes (a token's place, or time, height and width of a video).
* ``qk_norm_rope`` (``layers.norm_rotary_heads`` in training, ``qk_norm_rope_append`` for serving):
  takes the packed ``[q | k | v]`` projection apart into heads, divides every query and key head by
  its root mean square, scales and rotates it; the serving form writes keys and values to a cache.
* ``attn_prefix``: attention of a batch whose requests share a long prefix of keys and values and
  have a cache of their own behind it.

With ``own`` false ``run`` computes the same from elementary torch operations in 32 bits (angles in
64, which far positions need), rounded once at the end.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _rope(name, **kw):
    c = dict(op="rope", dtype="bf16", B=1, H=1, L=1, d=64, d_rot=64, axes=1, interleaved=False, adjacent=False,
             far=0, train=False)
    c.update(kw)
    return dict(c, name=name) if name else c


def _heads(name, **kw):
    c = dict(op="heads", form="forward", dtype="bf16", B=1, L=1, H=1, Hkv=1, d=64, d_rot=64, axes=1, interleaved=False,
             adjacent=False, far=0, S=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def _prefix(name, **kw):
    c = dict(op="prefix", B=1, H=1, Hkv=1, Lq=1, P=0, S=0, shortest=1, d=64, causal=True, lse=False)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one short 32-bit sequence far into a text, half of each head rotated: a call bound by its launch
        _rope("rope_f32_short", dtype="f32", H=3, L=77, d=80, d_rot=40, far=1000000),
        # two clips of 8 frames of 32 x 32 patches, three axes, forward and backward
        _rope("rope_video_train", B=2, H=16, L=8192, d=128, d_rot=128, axes=3, train=True),
        # a batch of images of 1025 patches, two axes, neighbouring features paired, 32 bits
        _rope("rope_images_f32", dtype="f32", B=8, H=12, L=1025, axes=2, interleaved=True, adjacent=True),
        # one new token of each of 32 requests, its keys and values written to their caches
        _heads("heads_decode", form="append", B=32, L=1, H=32, Hkv=8, d=128, d_rot=128, S=1024),
        # training step of an encoder layer's heads on a batch of 512-token sequences
        _heads("heads_encoder_train", form="train", B=8, L=512, H=12, Hkv=12),
        # a causal decoder's prefill over a batch of 8192-token sequences
        _heads("heads_prefill", B=4, L=8192, H=16, Hkv=16, d=128, d_rot=128),
        # 32-bit training at odd sizes with shared key heads
        _heads("heads_f32_ragged_train", form="train", dtype="f32", B=2, L=1511, H=4, Hkv=2, d=96, d_rot=96),
        # a handful of requests behind a short prompt, where launches and latency count
        _prefix("prefix_decode_few", B=4, H=12, Hkv=12, P=500, S=130),
        # serving: 64 requests at various lengths behind one system prompt
        _prefix("prefix_decode_batch", B=64, H=32, Hkv=8, d=128, P=8192, S=512, shortest=100),
        # a few requests about one long document
        _prefix("prefix_decode_long", B=8, H=16, Hkv=16, d=128, P=65536, S=1024, shortest=1, lse=True),
        # five tokens of each request at once (drafts to be verified)
        _prefix("prefix_verify", B=16, H=16, Hkv=4, Lq=5, P=20001, S=300, shortest=5),
        # the requests' own prompts of 512 tokens behind the shared one
        _prefix("prefix_prefill", B=4, H=16, Hkv=4, Lq=512, d=128, P=16384, S=512, shortest=512),
    ]


# ----------------------------------------------------------------------------- drawn cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """One more case of the same ranges: sizes spread over their logarithm, odd ones among them;
    bytes and operations are bounded by the largest listed case's."""
    op = rng.choice(["rope", "heads", "heads", "prefix", "prefix"])
    if op in ("rope", "heads"):
        d = rng.choice([32, 64, 64, 80, 96, 128, 128, 256, 72])
        d_rot = d if rng.random() < 0.7 else max(2, d // 4 * 2)
        if op == "heads" and rng.random() < 0.1:
            d_rot = 0
        axes = rng.choice([1, 1, 2, 3]) if d_rot >= 6 else 1
        kw = dict(dtype=rng.choice(["f32", "bf16", "bf16"]), d=d, d_rot=d_rot, axes=axes, interleaved=axes > 1 and rng.random() < 0.5,
                  adjacent=rng.random() < 0.3, far=rng.choice([0, 0, 70001, 1000000]))
        B, Hkv = _log(rng, 1, 32), rng.choice([1, 2, 3, 4, 8, 12, 16])
        H = Hkv * rng.choice([1, 1, 2, 4, 5])
        if op == "rope":
            L = _log(rng, 1, min(20000, int(6e7 / (B * H * d))))
            return _rope(None, B=B, H=H, L=L, train=rng.random() < 0.5, **kw)
        form = rng.choice(["forward", "train", "append"])
        L = _log(rng, 1, min(200 if form == "append" else 20000, int(6e7 / (B * (H + 2 * Hkv) * d))))
        S = L + _log(rng, 1, 1000) if form == "append" else 0
        return _heads(None, form=form, B=B, L=L, H=H, Hkv=Hkv, S=S, **kw)
    d, Hkv = rng.choice([64, 128]), rng.choice([1, 2, 4, 8, 12, 16])
    H = Hkv * rng.choice([1, 1, 2, 4, 5, 8])
    Lq = rng.choice([1, 1, 1, rng.randint(2, 8), _log(rng, 9, 600)])
    B = _log(rng, 1, 128 if Lq <= 8 else 8)
    P = _log(rng, 1, min(70000, 2.5e8 / (Hkv * d), 2.5e11 / (4.0 * d * H * B * Lq)))
    S = _log(rng, Lq, max(Lq, min(3000, int(1.2e8 / (B * Hkv * d)))))
    return _prefix(None, B=B, H=H, Hkv=Hkv, Lq=Lq, P=P, S=S, shortest=rng.randint(Lq, S), d=d,
                   causal=rng.random() < 0.8, lse=rng.random() < 0.3)


# ----------------------------------------------------------------------------- inputs
def _sections(case):
    """Pairs of each axis: the first axes take what does not divide evenly."""
    n, A = case["d_rot"] // 2, case["axes"]
    return [n // A + (a < n % A) for a in range(A)]


def _pair_axes(case):
    """The axis that each pair turns by."""
    left, out = _sections(case), []
    if not case["interleaved"]:
        return [a for a, n in enumerate(left) for _ in range(n)]
    while any(left):
        for a in range(len(left)):
            if left[a]:
                out.append(a)
                left[a] -= 1
    return out


def _positions(case, gen):
    """int64 [axes, B, L]: places in a text, or the axes of a grid that is scanned in rows."""
    B, L, A = case["B"], case["L"], case["axes"]
    start = torch.randint(0, 64, (1, B, 1), generator=gen, device="cuda") + case["far"]
    t = torch.arange(L, device="cuda")
    if A == 1:
        return (start + t).expand(1, B, L).contiguous()
    side = max(1, round((L / 8 if A > 2 else L) ** 0.5))
    grid = [t // side, t % side] if A == 2 else [t // (side * side), t // side % side, t % side]
    return (start + torch.stack(grid)[:, None]).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": case}

    def normal(dt, *shape, std=1.0, mean=0.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * std + mean).to(DTYPES[dt])

    if case["op"] == "prefix":
        B, H, Hkv, Lq, P, S, d = (case[n] for n in ("B", "H", "Hkv", "Lq", "P", "S", "d"))
        # heads that look for something: scores of a few units
        s["q"] = normal("bf16", B, H, Lq, d, std=2.0)
        s["pk"], s["pv"] = normal("bf16", Hkv, P, d), normal("bf16", Hkv, P, d)
        s["k"], s["v"] = normal("bf16", B, Hkv, S, d), normal("bf16", B, Hkv, S, d)
        s["lengths"] = _lengths(case)[torch.randperm(B, generator=gen, device="cuda")].contiguous()
        return s
    dt, d, n = case["dtype"], case["d"], case["d_rot"] // 2
    s["positions"] = _positions(case, gen)
    s["freqs"] = 10000.0 ** (-torch.arange(n, dtype=torch.float64, device="cuda") / max(n, 1))
    s["axes"] = tuple(_pair_axes(case))
    s["axis_of"] = torch.tensor(s["axes"], dtype=torch.int64, device="cuda")
    B, L = case["B"], case["L"]
    if case["op"] == "rope":
        s["x"] = normal(dt, B, case["H"], L, d).requires_grad_(case["train"])
        s["g"] = normal(dt, B, case["H"], L, d) if case["train"] else None
        return s
    H, Hkv, train = case["H"], case["Hkv"], case["form"] == "train"
    s["qkv"] = normal(dt, B, L, (H + 2 * Hkv) * d).requires_grad_(train)
    s["wq"] = normal(dt, d, std=0.1, mean=1.0).requires_grad_(train)
    s["wk"] = normal(dt, d, std=0.1, mean=1.0).requires_grad_(train)
    if train:
        s["gq"], s["gk"], s["gv"] = normal(dt, B, H, L, d), normal(dt, B, Hkv, L, d), normal(dt, B, Hkv, L, d)
    if case["form"] == "append":
        S = case["S"]
        s["k_cache"], s["v_cache"] = normal(dt, B, Hkv, S, d), normal(dt, B, Hkv, S, d)
        s["lengths"] = torch.randint(0, S - L + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    return s


def _lengths(case):
    """int32 [B] on the GPU: lengths from the shortest to the whole cache, evenly spread."""
    B, lo, hi = case["B"], case["shortest"], case["S"]
    return torch.tensor([hi - (hi - lo) * b // max(1, B - 1) for b in range(B)], dtype=torch.int32, device="cuda")


# ----------------------------------------------------------------------------- the plain forms
def _plain_angles(s):
    """cos and sin of every token's pairs, [B, 1, L, pairs], from angles in 64 bits."""
    a = s["positions"].double()[s["axis_of"]].permute(1, 2, 0)[:, None] * s["freqs"]
    return torch.cos(a).float(), torch.sin(a).float()


def _plain_rotate(x, s):
    """x: 32-bit heads [B, H, L, d]."""
    d_rot = s["case"]["d_rot"]
    if not d_rot:
        return x
    c, n = _plain_angles(s)
    if s["case"]["adjacent"]:
        a, b = x[..., 0:d_rot:2], x[..., 1:d_rot:2]
        y = torch.stack((a * c - b * n, a * n + b * c), -1).flatten(-2)
    else:
        a, b = x[..., :d_rot // 2], x[..., d_rot // 2:d_rot]
        y = torch.cat((a * c - b * n, a * n + b * c), -1)
    return torch.cat((y, x[..., d_rot:]), -1)


def _plain_heads(s, qkv, wq, wk):
    """32-bit q, k, v heads from the 32-bit packed projection."""
    c = s["case"]
    B, L, H, Hkv, d = c["B"], c["L"], c["H"], c["Hkv"], c["d"]
    q, k, v = qkv.view(B, L, H + 2 * Hkv, d).transpose(1, 2).split((H, Hkv, Hkv), 1)
    q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + 1e-6) * wq
    k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + 1e-6) * wk
    return _plain_rotate(q, s), _plain_rotate(k, s), v


def _plain_prefix(s):
    c = s["case"]
    B, H, Hkv, Lq, P, S, d = (c[n] for n in ("B", "H", "Hkv", "Lq", "P", "S", "d"))
    G = H // Hkv
    q = s["q"].float().view(B, Hkv, G * Lq, d) * d ** -0.5
    sp = torch.matmul(q.transpose(0, 1).reshape(Hkv, B * G * Lq, d), s["pk"].float().transpose(1, 2))
    sp = sp.view(Hkv, B, G * Lq, P).transpose(0, 1)
    ss = torch.matmul(q, s["k"].float().transpose(2, 3))
    first = s["lengths"].long().view(B, 1, 1, 1) - (Lq - 1 if c["causal"] else 0)
    seen = first + (torch.arange(Lq, device="cuda").repeat(G).view(-1, 1) if c["causal"] else 0)
    ss = ss.masked_fill(torch.arange(S, device="cuda") >= seen, -math.inf)
    top = torch.maximum(sp.amax(-1, keepdim=True), ss.amax(-1, keepdim=True))
    sp, ss = torch.exp(sp - top), torch.exp(ss - top)
    total = sp.sum(-1, keepdim=True) + ss.sum(-1, keepdim=True)
    o = torch.matmul(sp.transpose(0, 1).reshape(Hkv, B * G * Lq, P), s["pv"].float()).view(Hkv, B, G * Lq, d)
    o = (o.transpose(0, 1) + torch.matmul(ss, s["v"].float())) / total
    out = o.reshape(B, H, Lq, d).bfloat16()
    return (out, (top + torch.log(total)).view(B, H, Lq)) if c["lse"] else out


def _plain(s):
    c = s["case"]
    if c["op"] == "prefix":
        return _plain_prefix(s)
    dt = DTYPES[c["dtype"]]
    if c["op"] == "rope":
        y = _plain_rotate(s["x"].float(), s).to(dt)
        return (y.detach(), *torch.autograd.grad(y, s["x"], s["g"])) if c["train"] else y
    q, k, v = (t.to(dt).contiguous() for t in _plain_heads(s, s["qkv"].float(), s["wq"].float(), s["wk"].float()))
    if c["form"] == "forward":
        return q, k, v
    if c["form"] == "train":
        grads = torch.autograd.grad((q, k, v), (s["qkv"], s["wq"], s["wk"]), (s["gq"], s["gk"], s["gv"]))
        return (q.detach(), k.detach(), v.detach(), *grads)
    b = torch.arange(c["B"], device="cuda")[:, None]
    at = s["lengths"].long()[:, None] + torch.arange(c["L"], device="cuda")
    s["k_cache"][b, :, at] = k.transpose(1, 2)
    s["v_cache"][b, :, at] = v.transpose(1, 2)
    return q, s["k_cache"], s["v_cache"]


# ----------------------------------------------------------------------------- one pass
def run(state):
    if not own:
        return _plain(state)
    import paper_2106_06899_amd as tk
    from paper_2106_06899_amd import layers
    s, c = state, state["case"]
    if c["op"] == "prefix":
        return tk.attn_prefix(s["q"], s["pk"], s["pv"], s["k"], s["v"], s["lengths"], causal=c["causal"], lse=c["lse"])
    rot = dict(axes=s["axes"], adjacent=c["adjacent"])
    if c["op"] == "rope":
        if not c["train"]:
            return tk.rope(s["x"], s["positions"], s["freqs"], **rot)
        y = layers.rotary(s["x"], s["positions"], s["freqs"], **rot)
        return (y.detach(), *torch.autograd.grad(y, s["x"], s["g"]))
    if c["d_rot"]:
        rot.update(positions=s["positions"], freqs=s["freqs"])
    else:
        rot = {}
    if c["form"] == "forward":
        return tk.qk_norm_rope(s["qkv"], c["H"], c["Hkv"], s["wq"], s["wk"], **rot)
    if c["form"] == "append":
        q = tk.qk_norm_rope_append(s["qkv"], c["H"], c["Hkv"], s["k_cache"], s["v_cache"], s["lengths"], s["wq"], s["wk"], **rot)
        return q, s["k_cache"], s["v_cache"]
    q, k, v = layers.norm_rotary_heads(s["qkv"], c["H"], c["Hkv"], s["wq"], s["wk"], **rot)
    grads = torch.autograd.grad((q, k, v), (s["qkv"], s["wq"], s["wk"]), (s["gq"], s["gk"], s["gv"]))
    return (q.detach(), k.detach(), v.detach(), *grads)


def work(case):
    """Bytes and operations of one pass: inputs read once, outputs written once."""
    if case["op"] == "prefix":
        B, H, Hkv, Lq, P, S, d = (case[n] for n in ("B", "H", "Hkv", "Lq", "P", "S", "d"))
        lo = case["shortest"]
        lengths = [S - (S - lo) * b // max(1, B - 1) for b in range(B)]
        pairs = sum(Lq * (P + n) - (Lq * (Lq - 1) // 2 if case["causal"] else 0) for n in lengths) * H
        rows = B * H * Lq
        return {"bytes": 2 * d * (2 * rows + 2 * Hkv * P + 2 * Hkv * sum(lengths)) + 4 * B + (4 * rows if case["lse"] else 0),
                "flops": 4 * d * pairs}
    es, B, L, d = (4 if case["dtype"] == "f32" else 2), case["B"], case["L"], case["d"]
    place = 8 * case["axes"] * B * L + 4 * case["d_rot"]
    if case["op"] == "rope":
        n = B * case["H"] * L * d
        return {"bytes": (4 if case["train"] else 2) * n * es + place, "flops": (6 if case["train"] else 3) * n}
    n = B * L * (case["H"] + 2 * case["Hkv"]) * d
    return {"bytes": (4 if case["form"] == "train" else 2) * n * es + place, "flops": (20 if case["form"] == "train" else 8) * n}


# ----------------------------------------------------------------------------- 64 bits
def _turns(s):
    """complex128 [B, L, pairs]: e^(i angle) of each token's pairs."""
    ang = torch.stack([s["positions"][a].double() * f for a, f in zip(s["axes"], s["freqs"].tolist())], -1)
    return torch.polar(torch.ones_like(ang), ang)


def _exact_turn(x, s, back=False):
    """x: 64-bit [B, L, H, d]; rotated as complex numbers, by the opposite angles if back."""
    n = s["case"]["d_rot"] // 2
    if n == 0:
        return x
    e = _turns(s)[:, :, None]
    e = e.conj() if back else e
    i = torch.arange(n, device=x.device)
    i, j = (2 * i, 2 * i + 1) if s["case"]["adjacent"] else (i, i + n)
    z = torch.complex(x[..., i], x[..., j]) * e
    y = x.clone()
    y[..., i], y[..., j] = z.real, z.imag
    return y


def _exact_rope(s):
    y = _exact_turn(s["x"].detach().double().transpose(1, 2), s).transpose(1, 2)
    if not s["case"]["train"]:
        return y
    return y, _exact_turn(s["g"].double().transpose(1, 2), s, back=True).transpose(1, 2)


def _exact_heads(s):
    c = s["case"]
    B, L, H, Hkv, d = c["B"], c["L"], c["H"], c["Hkv"], c["d"]
    x = s["qkv"].detach().double().view(B, L, H + 2 * Hkv, d)
    parts = [(x[:, :, :H], s["wq"].detach().double()), (x[:, :, H:H + Hkv], s["wk"].detach().double())]
    r = [1.0 / torch.sqrt(t.pow(2).sum(-1, keepdim=True) / d + 1e-6) for t, _ in parts]
    q, k = (_exact_turn(t * i * w, s).transpose(1, 2) for (t, w), i in zip(parts, r))
    v = x[:, :, H + Hkv:].transpose(1, 2)
    if c["form"] == "forward":
        return q, k, v
    if c["form"] == "append":
        kc, vc = s["k_cache"].double(), s["v_cache"].double()
        for b, n in enumerate(s["lengths"].tolist()):
            kc[b, :, n:n + L], vc[b, :, n:n + L] = k[b], v[b]
        return q, kc, vc
    dx, dw = torch.empty_like(x), []
    for (t, w), i, g, at in zip(parts, r, (s["gq"], s["gk"]), (0, H)):
        g = _exact_turn(g.double().transpose(1, 2), s, back=True)
        u = t * i
        dw.append((g * u).sum((0, 1, 2)))
        g = g * w
        dx[:, :, at:at + t.shape[2]] = i * (g - u * (g * u).sum(-1, keepdim=True) / d)
    dx[:, :, H + Hkv:] = s["gv"].double().transpose(1, 2)
    return q, k, v, dx.view(B, L, -1), dw[0], dw[1]


def _exact_prefix(s):
    c = s["case"]
    B, H, Hkv, Lq, P, d = (c[n] for n in ("B", "H", "Hkv", "Lq", "P", "d"))
    G = H // Hkv
    out = torch.empty(B, H, Lq, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(B, H, Lq, dtype=torch.float64, device="cuda")
    for h in range(Hkv):
        pk, pv = s["pk"][h].double(), s["pv"][h].double()
        for b, n in enumerate(s["lengths"].tolist()):
            keys = torch.cat((pk, s["k"][b, h, :n].double()))
            values = torch.cat((pv, s["v"][b, h, :n].double()))
            q = s["q"][b, h * G:(h + 1) * G].double().reshape(G * Lq, d)
            w = q @ keys.t() / math.sqrt(d)
            if c["causal"]:
                last = P + n - Lq + torch.arange(Lq, device="cuda").repeat(G)
                w.masked_fill_(torch.arange(P + n, device="cuda") > last[:, None], -math.inf)
            lse[b, h * G:(h + 1) * G] = torch.logsumexp(w, -1).view(G, Lq)
            out[b, h * G:(h + 1) * G] = (torch.softmax(w, -1) @ values).view(G, Lq, d)
    return (out, lse) if c["lse"] else out


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "heads": _exact_heads, "prefix": _exact_prefix}[case["op"]](s)
