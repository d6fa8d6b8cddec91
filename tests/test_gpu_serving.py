"""Packed prompts, pages and trees of drafted tokens together, as a serving loop and a training step use
them through the attention layer."""
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


def _layer(causal=True, **kw):
    torch.manual_seed(0)
    layer = layers.TopkMultiheadAttention(256, 4, None, causal=causal, device="cuda", **kw)
    with torch.no_grad():
        layer.qkv.weight.mul_(3)  # heads that look for something
        if layer.qk_norm:
            layer.q_norm.mul_(2)
    return layer


def _plain(layer, x, positions):
    """The layer on one sequence x [n, d_model] in 32 bits (the frequencies' angles in 64)."""
    n, D = x.shape
    H, d = layer.n_heads, layer.d_head
    p = (x.float() @ layer.qkv.weight.float().t() + layer.qkv.bias.float()).to(BF16).float().view(n, 3, H, d)
    q, k, v = (p[:, i].transpose(0, 1) for i in range(3))
    if layer.qk_norm:
        q, k = (t * torch.rsqrt((t * t).mean(-1, keepdim=True) + 1e-6) * w.float() for t, w in ((q, layer.q_norm), (k, layer.k_norm)))
    if layer.rope_bits is not None:
        a = positions.double()[:, None] * layer.rope_bits.view(torch.float64)
        c, s = torch.cos(a).float(), torch.sin(a).float()
        q, k = (torch.cat((t[..., :d // 2] * c - t[..., d // 2:] * s, t[..., :d // 2] * s + t[..., d // 2:] * c), -1) for t in (q, k))
    q, k = q.to(BF16).float(), k.to(BF16).float()
    x = q @ k.transpose(1, 2) * layer.scale
    if layer.causal:
        x = x.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu_(1), -float("inf"))
    o = (torch.softmax(x, -1) @ v).to(BF16).float()
    return o.transpose(0, 1).reshape(n, D) @ layer.out.weight.float().t() + layer.out.bias.float()


def _near(got, want):
    """Within 2^-5 of the row's largest: five bf16 roundings on the way (projection, heads, weights, heads' outputs,
    result) of 2^-9 each, which the projections' sums of 256 terms of mixed signs may bring to three times that
    relative to a result smaller than its terms."""
    return bool(((got.float() - want).abs().amax(-1) <= 2.0 ** -5 * want.abs().amax(-1)).all())


@pytest.mark.parametrize("kw", [dict(), dict(qk_norm=True, rope_theta=10000.0), dict(rope_theta=500.0, bias=True)])
@pytest.mark.parametrize("causal", [False, True])
def test_packed_layer(kw, causal):
    layer = _layer(causal, **kw)
    lens = [1, 70, 0, 133, 20]
    off = [sum(lens[:i]) for i in range(len(lens) + 1)]
    x = torch.randn(off[-1], 256, device="cuda", dtype=BF16)
    y = layer.packed(x, _int(off))
    for a, z in zip(off, off[1:]):
        if z > a:
            assert _near(y[a:z], _plain(layer, x[a:z], torch.arange(z - a, device="cuda")))
    at = torch.cat([torch.arange(n, device="cuda") for n in lens])
    same = torch.equal(layers.packed_positions(_int(off), off[-1]), at)
    assert same


def test_packed_layer_learns():
    """A training step on packed sequences: gradients of every weight, as autograd has them of the same
    layer sequence by sequence in 32 bits."""
    layer = _layer(True, qk_norm=True, rope_theta=10000.0)
    off = [0, 50, 51, 180]
    x = torch.randn(180, 256, device="cuda", dtype=BF16)
    g = torch.randn(180, 256, device="cuda", dtype=BF16)
    layer.packed(x, _int(off)).backward(g)
    got = {n: p.grad.clone() for n, p in layer.named_parameters()}
    layer.zero_grad()
    sum((_plain(layer, x[a:z], torch.arange(z - a, device="cuda")) * g[a:z].float()).sum() for a, z in zip(off, off[1:])).backward()
    for n, p in layer.named_parameters():
        # sums over 180 tokens of terms that a handful of bf16 roundings (2^-9 each) have moved: 2^-6 of the whole, in the 2-norm
        assert float((got[n].float() - p.grad.float()).norm()) <= 2.0 ** -6 * float(p.grad.float().norm()), n


def test_captured_training_step():
    """Forward and backward of packed sequences in a graph: every replay has the gradients of the eager step, with
    other offsets and inputs and with eager steps in between."""
    layer = _layer(True, qk_norm=True, rope_theta=10000.0)
    weights = list(layer.parameters())
    x, g = (torch.randn(180, 256, device="cuda", dtype=BF16) for _ in range(2))
    off = _int([0, 50, 51, 180])
    step = lambda: torch.autograd.grad(layer.packed(x, off), weights, g)  # noqa: E731
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for o in ([0, 50, 51, 180], [0, 0, 180, 180], [0, 100, 130, 180], [0, 50, 51, 180]):
        off.copy_(_int(o))
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            same = torch.equal(a, b)
            assert same


def test_tree_depths():
    par = [[-1, 0, 1, 1, 3, -1, 5, 9], [3, 0, 1, 2, 3, 4, 5, 6]]
    want = [[0, 1, 2, 2, 3, 0, 1, 0], [0, 1, 2, 3, 4, 5, 6, 7]]
    assert layers.tree_depths(_int(par)).tolist() == want
    assert layers.tree_depths(_int(par[0])).tolist() == want[0]
    assert layers.tree_depths(_int(list(range(-1, 63)))).tolist() == list(range(64))


@pytest.mark.parametrize("page", [7, 16])
def test_serving_loop(page):
    """Prompts in one packed call, their rows into pages, two answers forked from each, drafts in trees, the
    accepted ones kept, requests ended, the pool moved to a smaller one and used on: every step's output is
    what the layer gives for the accepted text so far in one piece."""
    layer = _layer(True, qk_norm=True, rope_theta=10000.0)
    H, d, T = layer.n_heads, layer.d_head, 6
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(BF16)  # noqa: E731
    lens = [40, 9, 77]
    off = [0, 40, 49, 126]
    x = rand(126, 256)
    texts = [x[a:z] for a, z in zip(off, off[1:])] * 2  # requests 3 .. 5 will go on from 0 .. 2
    n_pages, M, B = 80, 40, 6
    kp, vp = (torch.full((1, n_pages, H, page, d), float("nan"), device="cuda", dtype=BF16) for _ in range(2))
    table, refs = torch.full((B, M), -1, dtype=torch.int32, device="cuda"), torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
    with torch.no_grad():
        y, k, v = layer.packed(x, _int(off), kv=True)
    for a, z, t in zip(off, off[1:], texts):
        assert _near(y[a:z], _plain(layer, t, torch.arange(z - a, device="cuda")))
    rows = _int(lens + [0, 0, 0])
    assert int(tk.pages_reserve(kp, vp, table, refs, lengths, rows)) == 0
    tk.pages_append(k, v, kp[0], vp[0], table, lengths, _int(off + [126] * 3))
    lengths += rows
    tk.pages_fork(table, refs, lengths, _int([0, 1, 2, 0, 1, 2]), page)
    assert lengths.tolist() == lens * 2
    parents = [[-1, 0, 0, 1, 3, 2], [-1, 0, 1, 2, 3, 4], [-1, -1, 1, 0, 2, 2]] * 2
    kept = [[0, 1, 3, 4], [0, 1, 2, 3], [1, 2, 5, -1], [0, 2, 5, -1], [-1, -1, -1, -1], [0, 3, -1, -1]]
    for step in range(4):
        drafts = rand(B, T, 256)
        assert int(tk.pages_reserve(kp, vp, table, refs, lengths, T)) == 0
        y = layer.draft(drafts, kp[0], vp[0], table, lengths, _int(parents))
        for b in range(B):
            n = len(texts[b])
            for i in range(T):
                path, j = [], i
                while j >= 0:
                    path.insert(0, j)
                    j = parents[b][j]
                t = torch.cat((texts[b], drafts[b, path]))
                assert _near(y[b, i:i + 1], _plain(layer, t, torch.arange(len(t), device="cuda"))[-1:]), (step, b, i)
        lengths = tk.pages_keep(kp, vp, table, lengths, _int(kept))
        tk.pages_release(table, refs, lengths, page)
        texts = [torch.cat((t, drafts[b, [i for i in kept[b] if i >= 0]])) for b, t in enumerate(texts)]
        assert lengths.tolist() == [len(t) for t in texts]
        held = [-(-len(t) // page) for t in texts]
        assert (table >= 0).sum(1).tolist() == held and int(refs.sum()) == sum(held)
        if step == 1:  # request 1 ends, 4 goes on in its place too
            tk.pages_fork(table, refs, lengths, _int([0, 4, 2, 3, 4, 5]), page)
            texts[1] = texts[4]
        if step == 2:  # the used pages to a pool that has just enough, and a few
            used = int((refs > 0).sum())
            k2, v2 = (torch.full((1, used + 14, H, page, d), float("nan"), device="cuda", dtype=BF16) for _ in range(2))
            table, refs, missing = tk.pages_compact(kp, vp, table, refs, k2, v2)
            assert int(missing) == 0
            kp, vp = k2, v2
    # single tokens, one after the other
    for _ in range(2):
        tokens = rand(B, 1, 256)
        assert int(tk.pages_reserve(kp, vp, table, refs, lengths, 1)) == 0
        y = layer.draft(tokens, kp[0], vp[0], table, lengths)
        lengths += 1
        texts = [torch.cat((t, tokens[b])) for b, t in enumerate(texts)]
        for b in range(B):
            assert _near(y[b], _plain(layer, texts[b], torch.arange(len(texts[b]), device="cuda"))[-1:])
    lengths.zero_()
    tk.pages_release(table, refs, lengths, page)
    assert not refs.any() and bool((table == -1).all())


def test_refusals_of_the_layer():
    layer = layers.TopkMultiheadAttention(256, 4, 16, device="cuda")
    x = torch.zeros(10, 256, device="cuda", dtype=BF16)
    with pytest.raises(ValueError):
        layer.packed(x, _int([0, 10]))
    layer = _layer(False)
    with pytest.raises(ValueError):
        layer.draft(x[None], None, None, None, None)
    with pytest.raises(ValueError):
        layer.packed(x, _int([0, 10]), positions=torch.arange(10, device="cuda"))
