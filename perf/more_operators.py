"""Packed prompts, paged caches and trees of drafted tokens: the calls whose speed is measured.

* ``attn_packed`` (``layers.packed_attention`` in training): attention over prompts of different
  lengths that lie one behind the other, with shared key heads.
* ``attn_tree``: drafted tokens of each request (a tree of guesses, or the one next token) against
  the request's cache, which lies in pages.
* ``pages_*``: the work on such a cache between the attention calls: room for new rows
  (``pages_reserve``, which copies a shared page before it is written), writing them
  (``pages_append``), forking and ending requests (``pages_fork``), keeping the accepted drafts
  (``pages_keep``), giving pages back (``pages_release``) and moving the used pages to another pool
  (``pages_compact``).

With ``own`` false ``run`` computes the same from elementary torch operations in 32 bits, rounded
once at the end.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BF16 = torch.bfloat16


def _packed(name, **kw):
    c = dict(op="packed", n=1, shortest=1, longest=1, H=1, Hkv=1, d=64, causal=True, tokens=False, train=False, lse=False)
    c.update(kw)
    return dict(c, name=name) if name else c


def _tree(name, **kw):
    c = dict(op="tree", B=1, H=1, Hkv=1, T=1, page=16, shortest=1, longest=1, d=64, chain=False, lse=False)
    c.update(kw)
    return dict(c, name=name) if name else c


def _pages(name, **kw):
    c = dict(op="pages", form="drafts", B=1, T=1, beams=1, layers=1, Hkv=1, d=64, page=16, shortest=1, longest=1, spare=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # three short prompts: a call bound by its launch and by one tile's latency
        _packed("packed_few", n=3, shortest=5, longest=77, H=12, Hkv=12, lse=True),
        # a serving step's new prompts, from an empty one to 3000 tokens, heads as the projection left them
        _packed("packed_batch", n=12, shortest=0, longest=3000, H=16, Hkv=4, d=128, tokens=True),
        # one long document, causal
        _packed("packed_long", n=1, shortest=16384, longest=16384, H=16, Hkv=4, d=128),
        # training of an encoder on texts of 1 to 512 tokens without padding
        _packed("packed_encoder_train", n=24, shortest=1, longest=512, H=12, Hkv=12, causal=False, train=True, tokens=True),
        # training of a decoder with shared key heads on long texts of different lengths
        _packed("packed_decoder_train", n=3, shortest=1000, longest=8192, H=16, Hkv=4, d=128, train=True),
        # the next token of each of 32 requests
        _tree("tree_decode", B=32, H=32, Hkv=8, d=128, shortest=100, longest=4096),
        # a small tree for each of a few short requests, where launches and latency count; odd pages
        _tree("tree_few", B=4, H=12, Hkv=12, T=13, page=24, shortest=50, longest=600, lse=True),
        # trees of 24 drafts for a batch of requests
        _tree("tree_batch", B=48, H=32, Hkv=8, T=24, page=64, shortest=500, longest=8192, d=128),
        # the largest tree behind two long documents
        _tree("tree_long", B=2, H=16, Hkv=16, T=64, page=128, shortest=30000, longest=100000, d=128),
        # a beam search step: eight requests of eight beams go on from the best beam
        _pages("pages_beams", form="beams", B=64, beams=8, layers=2, Hkv=8, d=128, shortest=200, longest=2000, spare=500),
        # a step with drafts: room, their rows, the accepted ones, what is left over
        _pages("pages_drafts", form="drafts", B=32, T=16, layers=4, Hkv=8, d=128, shortest=30, longest=3000, spare=3000),
        # the used pages of a scattered pool into a smaller one
        _pages("pages_compact", form="compact", B=24, layers=2, Hkv=8, d=128, shortest=100, longest=4000, spare=2500),
    ]


# ----------------------------------------------------------------------------- drawn cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """One more case of the same ranges: sizes spread over their logarithm, odd ones among them;
    bytes, operations and the plain form's scores are bounded by the largest listed case's."""
    op = rng.choice(["packed", "packed", "tree", "tree", "pages"])
    d, Hkv = rng.choice([64, 128]), rng.choice([1, 2, 4, 8, 12, 16])
    if op == "packed":
        H, n, train = Hkv * rng.choice([1, 1, 2, 4, 5]), _log(rng, 1, 40), rng.random() < 0.5
        longest = _log(rng, 8 if train else 1, min(16384, math.sqrt((2.5e9 if train else 4e9) / (H * n))))
        return _packed(None, n=n, shortest=rng.choice([0, 1, rng.randint(0, longest)]), longest=longest, H=H, Hkv=Hkv, d=d,
                       causal=rng.random() < 0.7, tokens=rng.random() < 0.5, train=train, lse=not train and rng.random() < 0.3)
    if op == "tree":
        H, B = Hkv * rng.choice([1, 1, 2, 4, 5, 8]), _log(rng, 1, 96)
        T = rng.choice([1, rng.randint(2, 16), _log(rng, 1, 64)])
        longest = _log(rng, T, max(T, min(100000, 2e8 / (B * Hkv * d), 2e9 / (B * H * T))))
        return _tree(None, B=B, H=H, Hkv=Hkv, T=T, page=rng.choice([1, 8, 16, 16, 24, 32, 64, 128, 100, 256]),
                     shortest=rng.randint(T, longest), longest=longest, d=d, chain=rng.random() < 0.2, lse=rng.random() < 0.3)
    form = rng.choice(["beams", "drafts", "compact"])
    beams = rng.randint(1, 12) if form == "beams" else 1
    B, layers, page = _log(rng, 1, 10) * beams if form == "beams" else _log(rng, 1, 100), rng.randint(1, 4), rng.choice([1, 8, 16, 16, 24, 64, 100])
    longest = _log(rng, 1, min(4000, 1e8 / (B / beams * layers * Hkv * d)))
    return _pages(None, form=form, B=B, T=_log(rng, 1, 64) if form == "drafts" else 1, beams=beams, layers=layers, Hkv=Hkv, d=d, page=page,
                  shortest=rng.randint(1, longest), longest=longest, spare=rng.randint(0, 200))


# ----------------------------------------------------------------------------- inputs
def _lens(case, n):
    """n lengths from the shortest to the longest, evenly spread."""
    lo, hi = case["shortest"], case["longest"]
    return [hi - (hi - lo) * b // max(1, n - 1) for b in range(n)]


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    rng = random.Random(int(seed))

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).to(BF16)

    s = {"case": case}
    return {"packed": _prepare_packed, "tree": _prepare_tree, "pages": _prepare_pages}[case["op"]](s, case, normal, rng)


def _prepare_packed(s, c, normal, rng):
    lens = _lens(c, c["n"])
    rng.shuffle(lens)
    s["offsets"] = _int([sum(lens[:i]) for i in range(c["n"] + 1)])
    N = sum(lens)
    # heads that look for something: scores of a few units
    for name, heads, std in (("q", c["H"], 2.0), ("k", c["Hkv"], 1.0), ("v", c["Hkv"], 1.0), ("g", c["H"], 1.0)):
        if name != "g" or c["train"]:
            s[name] = normal(*((N, heads) if c["tokens"] else (heads, N)), c["d"], std=std).requires_grad_(c["train"] and name != "g")
    return s


def _prepare_tree(s, c, normal, rng):
    B, T, page = c["B"], c["T"], c["page"]
    lens = _lens(c, B)
    rng.shuffle(lens)
    need = [-(-n // page) for n in lens]
    ids = list(range(sum(need)))
    rng.shuffle(ids)
    table = [[ids.pop() for _ in range(n)] + [-1] * (max(need) - n) for n in need]
    s["table"], s["lengths"] = _int(table), _int(lens)
    s["q"] = normal(B, c["H"], T, c["d"], std=2.0)
    s["k"], s["v"] = normal(sum(need), c["Hkv"], page, c["d"]), normal(sum(need), c["Hkv"], page, c["d"])
    # each draft follows a draft before it or the text itself (-1)
    s["parents"] = None if c["chain"] else _int([[rng.randint(max(-1, i - 6), i - 1) for i in range(T)] for _ in range(B)])
    return s


def _prepare_pages(s, c, normal, rng):
    B, T, page, W = c["B"], c["T"], c["page"], c["beams"]
    lens = [n for n in _lens(c, B // W) for _ in range(W)]
    M = -(-(c["longest"] + T) // page)
    used = sum(-(-n // page) for n in lens)
    total = used + B * (T // page + 2) + c["spare"]
    ids = list(range(total))
    rng.shuffle(ids)
    refs, table = [0] * total, []
    for b, n in enumerate(lens):
        whole = n // page
        row = list(table[b - b % W][:whole]) if b % W else [ids.pop() for _ in range(whole)]  # beams share what they have in common
        if n % page:
            row.append(ids.pop())
        for p in row:
            refs[p] += 1
        if c["form"] == "drafts" and b % 2 and n % page:
            refs[row[-1]] += 1  # kept for another request too: copied before it is written
        table.append(row + [-1] * (M - len(row)))
    s["table"], s["refs"], s["lengths"] = _int(table), _int(refs), _int(lens)
    shape = (c["layers"], total, c["Hkv"], page, c["d"])
    s["k_pages"], s["v_pages"] = normal(*shape), normal(*shape)
    if c["form"] == "compact":
        live = sum(r > 0 for r in refs)
        s["k_to"], s["v_to"] = (torch.zeros(c["layers"], live + 3, *shape[2:], dtype=BF16, device="cuda") for _ in range(2))
        return s
    s["k"], s["v"] = (normal(c["layers"], B, c["Hkv"], T, c["d"]) for _ in range(2))
    if c["form"] == "beams":
        s["parents"] = _int([b - b % W for b in range(B)])
    else:  # the accepted drafts of each request, in order
        kept = [sorted(rng.sample(range(T), rng.randint(0, min(T, 8)))) for _ in range(B)]
        s["kept"] = _int([a + [-1] * (min(T, 8) - len(a)) for a in kept])
    return s


# ----------------------------------------------------------------------------- the plain forms
def _attend(q, k, v, seen, scale):
    """Output and logarithm of the sum of rows q [..., R, d] on keys k, v [..., S, d], 32 bits; a
    row that sees nothing is 0."""
    x = (torch.matmul(q, k.transpose(-1, -2)) * scale).masked_fill(~seen, -math.inf)
    top = x.detach().amax(-1, keepdim=True).clamp(min=-1e30)
    w = torch.exp(x - top)
    total = w.sum(-1, keepdim=True)
    out = torch.matmul(w, v) / torch.where(total > 0, total, 1.0)
    return out, (top + torch.log(total)).squeeze(-1)


def _plain_packed(s):
    c = s["case"]
    H, Hkv, d, longest = c["H"], c["Hkv"], c["d"], c["longest"]
    q, k, v = ((s[n].transpose(0, 1) if c["tokens"] else s[n]).float() for n in ("q", "k", "v"))
    N, off = q.shape[1], s["offsets"].long()
    # every sequence at its own row of a padded batch
    i = torch.arange(longest, device="cuda")
    at = (off[:-1, None] + i).clamp(max=N - 1)
    seen = (i < (off[1:] - off[:-1])[:, None])[:, None, :].expand(-1, longest, -1)
    if c["causal"]:
        seen = seen & (i <= i[:, None])
    qp = q[:, at].view(Hkv, H // Hkv, c["n"], longest, d)
    out, lse = _attend(qp, k[:, at][:, None], v[:, at][:, None], seen, d ** -0.5)
    t = torch.arange(N, device="cuda")
    seq = torch.searchsorted(off[1:].contiguous(), t, right=True)
    out = out.reshape(H, -1, d)[:, seq * longest + t - off[seq]].to(BF16)
    if c["train"]:
        g = s["g"].transpose(0, 1) if c["tokens"] else s["g"]
        return (out.detach(), *torch.autograd.grad(out, (s["q"], s["k"], s["v"]), g))
    return (out, lse.reshape(H, -1)[:, seq * longest + t - off[seq]]) if c["lse"] else out


def _plain_tree(s):
    c = s["case"]
    B, H, Hkv, T, d = (c[n] for n in ("B", "H", "Hkv", "T", "d"))
    table, lengths = s["table"].long().clamp(min=0), s["lengths"].long()
    k, v = (s[n][table].float().transpose(1, 2).reshape(B, Hkv, -1, d) for n in ("k", "v"))
    i = torch.arange(T, device="cuda")
    if s["parents"] is None:
        sees = (i <= i[:, None]).expand(B, T, T)
    else:  # each draft sees itself and whatever it follows, over any number of steps
        step = (s["parents"][..., None] == i).float() + (i == i[:, None])
        sees = torch.linalg.matrix_power(step, T) > 0
    j = torch.arange(k.shape[2], device="cuda") - (lengths[:, None] - T)  # draft number of each cache row; before the drafts: negative
    seen = (j < 0)[:, None, :] | (torch.gather(sees, 2, j.clamp(0, T - 1)[:, None].expand(B, T, -1)) & (j < T)[:, None, :])
    seen = seen.repeat(1, H // Hkv, 1)[:, None]
    out, lse = _attend(s["q"].float().view(B, Hkv, -1, d), k, v, seen, d ** -0.5)
    out = out.view(B, H, T, d).to(BF16)
    return (out, lse.view(B, H, T)) if c["lse"] else out


def _plain_fork(s):
    """Every request goes on from its parent's pages."""
    table, refs, lengths, par = s["table"], s["refs"], s["lengths"], s["parents"].long()
    page, M = s["case"]["page"], table.shape[1]
    new = table[par].masked_fill(torch.arange(M, device="cuda") * page >= lengths[par][:, None], -1)
    new = torch.where((par == torch.arange(len(par), device="cuda"))[:, None], table, new)
    for t, by in ((table, -1), (new, 1)):
        refs.index_add_(0, t.long().clamp(min=0).flatten(), (t >= 0).int().flatten() * by)
    lengths.copy_(lengths[par])
    table.copy_(new)


def _plain_reserve(s):
    """Pages for T more rows of every request; those that others hold too are copied."""
    table, refs, n, page, T = s["table"].long(), s["refs"], s["lengths"].long()[:, None], s["case"]["page"], s["case"]["T"]
    total = refs.numel()
    e = torch.arange(table.shape[1], device="cuda")
    writes, held, p = (e >= n // page) & (e * page < n + T), table >= 0, table.clamp(min=0)
    shared = writes & held & (refs[p] > 1)
    number = torch.arange(table.numel(), device="cuda").view_as(table)
    writers = torch.zeros(total, dtype=torch.int32, device="cuda").index_add_(0, p.flatten(), shared.int().flatten())
    first = torch.full((total,), table.numel(), device="cuda")
    first.scatter_reduce_(0, p.flatten(), torch.where(shared, number, table.numel()).flatten(), "amin")
    # where all that hold a page write to it, the first keeps it
    leaves = shared & ~((writers[p] == refs[p]) & (first[p] == number))
    fresh = writes & (~held | leaves)
    free = torch.nonzero(refs == 0).flatten()
    missing = (fresh.sum() - len(free)).clamp(min=0).int()
    if int(missing):
        return missing
    new = torch.where(fresh, free[(fresh.flatten().cumsum(0) - 1).clamp(0, max(0, len(free) - 1))].view_as(table), table) if len(free) else table
    b, at = torch.nonzero(leaves & (e == n // page) & (n % page > 0), as_tuple=True)
    rows = (torch.arange(page, device="cuda") < (n % page)[b])[None, :, None, :, None]
    for t in (s["k_pages"], s["v_pages"]):
        t[:, new[b, at]] = torch.where(rows, t[:, table[b, at]], t[:, new[b, at]])
    refs.index_add_(0, p.flatten(), -leaves.int().flatten())
    refs.index_add_(0, new.clamp(min=0).flatten(), fresh.int().flatten())
    s["table"].copy_(new)
    return missing


def _plain_append(s):
    """T rows of each request behind those that it has."""
    page = s["case"]["page"]
    r = s["lengths"].long()[:, None] + torch.arange(s["case"]["T"], device="cuda")
    p = torch.gather(s["table"].long(), 1, r // page)
    for t, x in ((s["k_pages"], s["k"]), (s["v_pages"], s["v"])):
        t[:, p, :, r % page] = x.permute(1, 3, 0, 2, 4)


def _plain_keep(s):
    """The accepted drafts' rows, moved up behind the text; the lengths with them."""
    page, table, n, kept = s["case"]["page"], s["table"].long(), s["lengths"].long()[:, None], s["kept"].long()
    b, a = torch.nonzero(kept >= 0, as_tuple=True)
    src, dst = n[b, 0] + kept[b, a], n[b, 0] + a
    for t in (s["k_pages"], s["v_pages"]):
        t[:, table[b, dst // page], :, dst % page] = t[:, table[b, src // page], :, src % page]
    return (n[:, 0] + (kept >= 0).sum(1)).int()


def _plain_release(s, lengths):
    """Pages behind those that the lengths need are given back."""
    table = s["table"]
    gone = (torch.arange(table.shape[1], device="cuda") * s["case"]["page"] >= lengths[:, None]) & (table >= 0)
    s["refs"].index_add_(0, table.long().clamp(min=0).flatten(), -gone.int().flatten())
    table.masked_fill_(gone, -1)


def _plain_compact(s):
    table, refs = s["table"], s["refs"]
    live = torch.nonzero(refs > 0).flatten()
    number = ((refs > 0).cumsum(0) - 1).int()
    new_refs = torch.zeros(s["k_to"].shape[1], dtype=torch.int32, device="cuda")
    new_refs[:len(live)] = refs[live]
    s["k_to"][:, :len(live)] = s["k_pages"][:, live]
    s["v_to"][:, :len(live)] = s["v_pages"][:, live]
    return torch.where(table >= 0, number[table.long().clamp(min=0)], -1), new_refs, s["k_to"], s["v_to"]


def _plain_pages(s):
    form = s["case"]["form"]
    if form == "compact":
        return _plain_compact(s)
    if form == "beams":
        _plain_fork(s)
    missing = _plain_reserve(s)
    _plain_append(s)
    lengths = s["lengths"]
    if form == "drafts":
        lengths = _plain_keep(s)
        _plain_release(s, lengths)
    return missing, lengths, s["table"], s["refs"], s["k_pages"], s["v_pages"]


# ----------------------------------------------------------------------------- one pass
def run(state):
    if not own:
        return {"packed": _plain_packed, "tree": _plain_tree, "pages": _plain_pages}[state["case"]["op"]](state)
    import paper_2106_06899_amd as tk
    from paper_2106_06899_amd import layers
    s, c = state, state["case"]
    if c["op"] == "packed":
        q, k, v = (s[n].transpose(0, 1) if c["tokens"] else s[n] for n in ("q", "k", "v"))
        if not c["train"]:
            return tk.attn_packed(q, k, v, s["offsets"], causal=c["causal"], lse=c["lse"])
        out = layers.packed_attention(q, k, v, s["offsets"], causal=c["causal"])
        g = s["g"].transpose(0, 1) if c["tokens"] else s["g"]
        return (out.detach(), *torch.autograd.grad(out, (s["q"], s["k"], s["v"]), g))
    if c["op"] == "tree":
        return tk.attn_tree(s["q"], s["k"], s["v"], s["lengths"], s["table"], s["parents"], lse=c["lse"])
    pools, page, lengths = (s["k_pages"], s["v_pages"]), c["page"], s["lengths"]
    if c["form"] == "compact":
        table, refs, _ = tk.pages_compact(*pools, s["table"], s["refs"], s["k_to"], s["v_to"])
        return table, refs, s["k_to"], s["v_to"]
    if c["form"] == "beams":
        tk.pages_fork(s["table"], s["refs"], lengths, s["parents"], page)
    missing = tk.pages_reserve(*pools, s["table"], s["refs"], lengths, c["T"])
    tk.pages_append(s["k"], s["v"], *pools, s["table"], lengths)
    if c["form"] == "drafts":
        lengths = tk.pages_keep(*pools, s["table"], lengths, s["kept"])
        tk.pages_release(s["table"], s["refs"], lengths, page)
    return missing, lengths, s["table"], s["refs"], *pools


def work(case):
    """Bytes and operations of one pass: inputs read once, outputs written once."""
    c, d, Hkv = case, case["d"], case["Hkv"]
    if c["op"] == "packed":
        lens, H = _lens(c, c["n"]), c["H"]
        pairs = sum(n * (n + 1) // 2 if c["causal"] else n * n for n in lens) * H
        N = sum(lens)
        # forward: q, k, v in, out; backward: these and the gradient in, three gradients out
        moved = (2 * H + 2 * Hkv) * N * d * 2 + (4 * H * N if c["lse"] else 0)
        return {"bytes": moved + ((4 * H + 4 * Hkv) * N * d * 2 - H * N * d * 2 if c["train"] else 0) + 4 * (c["n"] + 1),
                "flops": (14 if c["train"] else 4) * d * pairs}
    if c["op"] == "tree":
        B, H, T = c["B"], c["H"], c["T"]
        lens = _lens(c, B)
        return {"bytes": 4 * d * (B * H * T + Hkv * sum(lens)) + 4 * (B * (T + 1) + sum(-(-n // c["page"]) for n in lens)) + (4 * B * H * T if c["lse"] else 0),
                "flops": 4 * d * H * T * sum(lens)}
    B, T, page, row = c["B"], c["T"], c["page"], c["layers"] * Hkv * d * 4  # a row: keys and values of all layers
    lens = _lens(c, B // c["beams"])
    held = sum(-(-n // page) for n in lens)
    books = 4 * B * (-(-(c["longest"] + T) // page) + 2)
    if c["form"] == "compact":
        return {"bytes": 2 * held * page * row + 2 * books, "flops": 0}
    if c["form"] == "beams":  # the shared last pages copied for all beams but one, one row each
        return {"bytes": 2 * row * ((c["beams"] - 1) * sum(n % page for n in lens) + B) + 2 * books, "flops": 0}
    # last pages that others hold copied (for every other request), the drafts written, half of eight moved
    return {"bytes": 2 * row * (sum(n % page for n in lens[1::2]) + B * T + B * min(T, 8) // 2) + 2 * books, "flops": 0}


# ----------------------------------------------------------------------------- 64 bits
def _exact_packed(s):
    c = s["case"]
    H, Hkv, d = c["H"], c["Hkv"], c["d"]
    G = H // Hkv
    by_head = lambda n: s[n].detach().transpose(0, 1) if c["tokens"] else s[n].detach()  # noqa: E731
    q, k, v = by_head("q"), by_head("k"), by_head("v")
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    dq, dk, dv = (torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (q, k, v))
    off = s["offsets"].tolist()
    for a, z in zip(off, off[1:]):
        for h in range(H if z > a else 0):
            qq, kk, vv = q[h, a:z].double(), k[h // G, a:z].double(), v[h // G, a:z].double()
            x = qq @ kk.t() / math.sqrt(d)
            if c["causal"]:
                x.masked_fill_(torch.ones(z - a, z - a, dtype=torch.bool, device="cuda").triu_(1), -math.inf)
            lse[h, a:z] = torch.logsumexp(x, -1)
            w = torch.softmax(x, -1)
            del x
            out[h, a:z] = w @ vv
            if c["train"]:
                g = by_head("g")[h, a:z].double()
                dv[h // G, a:z] += w.t() @ g
                dx = g @ vv.t()
                dx = w * (dx - (dx * w).sum(-1, keepdim=True)) / math.sqrt(d)
                dq[h, a:z] = dx @ kk
                dk[h // G, a:z] += dx.t() @ qq
    if c["train"]:
        back = lambda t: t.transpose(0, 1) if c["tokens"] else t  # noqa: E731
        return out, back(dq), back(dk), back(dv)
    return (out, lse) if c["lse"] else out


def _exact_tree(s):
    c = s["case"]
    B, H, Hkv, T, d, page = (c[n] for n in ("B", "H", "Hkv", "T", "d", "page"))
    G = H // Hkv
    out = torch.empty(B, H, T, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(B, H, T, dtype=torch.float64, device="cuda")
    parents = [list(range(-1, T - 1))] * B if s["parents"] is None else s["parents"].tolist()
    for b, n in enumerate(s["lengths"].tolist()):
        pages = s["table"][b, :-(-n // page)].long()
        hidden = torch.ones(T, T, dtype=torch.bool)
        for i in range(T):
            j = i
            while j >= 0:
                hidden[i, j] = False
                j = parents[b][j]
        hidden = torch.cat((torch.zeros(T, n - T, dtype=torch.bool), hidden), 1).cuda().repeat(G, 1)
        for h in range(Hkv):
            kk, vv = (s[t][pages, h].reshape(-1, d)[:n].double() for t in ("k", "v"))
            x = (s["q"][b, h * G:(h + 1) * G].double().reshape(G * T, d) @ kk.t() / math.sqrt(d)).masked_fill(hidden, -math.inf)
            lse[b, h * G:(h + 1) * G] = torch.logsumexp(x, -1).view(G, T)
            out[b, h * G:(h + 1) * G] = (torch.softmax(x, -1) @ vv).view(G, T, d)
    return (out, lse) if c["lse"] else out


def _exact_pages(s):
    """The books as lists, page by page; rows are copied one by one."""
    c = s["case"]
    page, T, B = c["page"], c["T"], c["B"]
    table, refs, lens = s["table"].tolist(), s["refs"].tolist(), s["lengths"].tolist()
    kp, vp = s["k_pages"].double(), s["v_pages"].double()
    if c["form"] == "compact":
        live = [p for p, r in enumerate(refs) if r > 0]
        new = {p: i for i, p in enumerate(live)}
        k_to, v_to = s["k_to"].double(), s["v_to"].double()
        at = torch.tensor(live, device="cuda")
        k_to[:, :len(live)], v_to[:, :len(live)] = kp[:, at], vp[:, at]
        return [_int([[new.get(p, -1) for p in row] for row in table]), _int([refs[p] for p in live] + [0] * (k_to.shape[1] - len(live))), k_to, v_to]
    if c["form"] == "beams":
        old = [list(row) for row in table]
        for b, p in enumerate(s["parents"].tolist()):
            if p != b:
                n = -(-lens[p] // page)
                table[b] = old[p][:n] + [-1] * (len(old[p]) - n)
                for x in old[b]:
                    refs[x] -= x >= 0
                for x in table[b]:
                    refs[x] += x >= 0
                lens[b] = lens[p]
    before, holders, left = [list(row) for row in table], list(refs), []
    for b in range(B):
        for e in range(lens[b] // page, -(-(lens[b] + T) // page)):
            if table[b][e] < 0 or holders[table[b][e]] > 1:
                left.append((b, e))
    for p in {before[b][e] for b, e in left if before[b][e] >= 0}:  # the last to hold a page keeps it
        mine = [x for x in left if before[x[0]][x[1]] == p]
        if len(mine) == holders[p]:
            left.remove(mine[0])
    free = iter([p for p, r in enumerate(refs) if r == 0])
    for b, e in left:
        p, q = table[b][e], next(free)
        table[b][e], refs[q] = q, 1
        if p >= 0:
            refs[p] -= 1
            if e == lens[b] // page and lens[b] % page:
                kp[:, q, :, :lens[b] % page], vp[:, q, :, :lens[b] % page] = kp[:, p, :, :lens[b] % page], vp[:, p, :, :lens[b] % page]
    for b in range(B):
        for t in range(T):
            p, r = table[b][(lens[b] + t) // page], (lens[b] + t) % page
            kp[:, p, :, r], vp[:, p, :, r] = s["k"][:, b, :, t].double(), s["v"][:, b, :, t].double()
    if c["form"] == "drafts":
        for b, kept in enumerate(s["kept"].tolist()):
            kept, n = [a for a in kept if a >= 0], lens[b]
            for i, a in enumerate(kept):
                p, q = table[b][(n + i) // page], table[b][(n + a) // page]
                kp[:, p, :, (n + i) % page], vp[:, p, :, (n + i) % page] = kp[:, q, :, (n + a) % page].clone(), vp[:, q, :, (n + a) % page].clone()
            lens[b] += len(kept)
            for e in range(-(-lens[b] // page), len(table[b])):
                if table[b][e] >= 0:
                    refs[table[b][e]] -= 1
                    table[b][e] = -1
    return [_int(0), _int(lens), _int(table), _int(refs), kp, vp]


def exact(case, seed):
    s = prepare(case, seed)
    return {"packed": _exact_packed, "tree": _exact_tree, "pages": _exact_pages}[case["op"]](s)
