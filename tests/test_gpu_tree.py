"""GPU parity of attention of drafted tokens over a cache in pages against Eq. 1 in 64 bits.

Tolerance of an output element: half a step of bf16 relative to it, and twice the relative error
of a weight times sum_j w_j |v_j|. A weight is off by its score's rounding (d products summed in fp32:
at most (d + 8) 2^-24 sum |q k| scale), by the rounding of the exponent (2^-22 of the largest) and by
its own on the way into the second product: 2^-16 as the sum of two bf16 numbers, 2^-9 as one, which
64 rows a request and key head and more take (the sum that it is divided by is not rounded).
"""
import math
import random

import pytest
import torch

import paper_2106_06899_amd as tk

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    tk.lib()
    yield


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _inputs(H, Hkv, T, d, page, lens, seed=0, spare=3, std=2.0, wide=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    need = [-(-max(n, 0) // page) for n in lens]
    ids = list(range(sum(need) + spare))
    rng.shuffle(ids)
    M = max(max(need), 1) + wide
    table = [[ids.pop() for _ in range(n)] + [-1] * (M - n) for n in need]
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    q = (normal(len(lens), H, T, d) * std).to(BF16)
    k, v = (normal(sum(need) + spare, Hkv, page, d).to(BF16) for _ in range(2))
    parents = [[rng.randint(max(-1, i - 5), i - 1) for i in range(T)] for _ in lens]
    return q, k, v, _int(lens), _int(table), parents


def _sees(parents):
    """Row i of the drafts sees those that it follows, and itself; any parent that is no earlier draft is the text."""
    out = []
    for i in range(len(parents)):
        p = parents[i]
        out.append((set(out[p]) if 0 <= p < i else set()) | {i})
    return out


def _check(q, k, v, lens, table, parents, out, lse=None, scale=None):
    B, H, T, d = q.shape
    n_pages, Hkv, page, _ = k.shape
    G = H // Hkv
    scale = d ** -0.5 if scale is None else scale
    wstep = 2.0 ** -16 if G * T < 64 else 2.0 ** -9
    worst = 0.0
    for b in range(B):
        row = table[b].tolist() if table is not None else [b]
        n = min(max(int(lens[b]), 0), len(row) * page)
        there = [0 <= row[j // page] < n_pages for j in range(n)] if any(not 0 <= p < n_pages for p in row[:-(-n // page)]) else [True] * n
        at = torch.tensor([min(max(p, 0), n_pages - 1) for p in row[:-(-n // page)]] or [0], device="cuda")
        sees = _sees(parents[b] if parents is not None else list(range(-1, T - 1)))
        hidden = torch.zeros(T, n, dtype=torch.bool)
        for i in range(T):
            for j in range(max(0, n - T), n):
                hidden[i, j] = (j - (n - T)) not in sees[i]
        hidden = (hidden | ~torch.tensor(there, dtype=torch.bool)[None, :n]).cuda()
        for h in range(H):
            kk, vv = (t[at, h // G].reshape(-1, d)[:n].double() for t in (k, v))
            s = (q[b, h].double() @ kk.t() * scale).masked_fill(hidden, -math.inf)
            w = torch.softmax(s, -1).nan_to_num(0.0) if n else s
            vv = torch.where(hidden.all(0)[:, None], 0.0, vv)
            ref = w @ vv
            size = (q[b, h].double().abs() @ kk.abs().t()).masked_fill(hidden, 0).amax(-1, keepdim=True) * scale if n else torch.zeros(T, 1, device="cuda")
            delta = ((d + 8) * 2.0 ** -24 + 2.0 ** -22) * size
            tol = 2.0 ** -8 * ref.abs() + 2 * (delta + wstep) * (w @ vv.abs()) + 1e-37
            err = (out[b, h].double() - ref).abs()
            assert bool((err <= tol).all()), f"request {b} head {h}: error {float((err / tol).max()):.2f} of its bound"
            worst = max(worst, float((err / tol).max()))
            if lse is not None:
                want = torch.logsumexp(s, -1) if n else torch.full((T,), -math.inf, device="cuda", dtype=torch.float64)
                none = want == -math.inf
                assert bool((lse[b, h][none] == -math.inf).all())
                assert bool(((lse[b, h].double() - want).abs() <= 2 * delta[:, 0] + 2.0 ** -21 * (1 + want.abs()))[~none].all())
    print(f"[case] worst error {worst:.3f} of its bound", flush=True)


CASES = {
    # name: H, Hkv, T, d, page, lengths
    "one": (1, 1, 1, 64, 1, [1]),
    "single_tokens": (8, 2, 1, 128, 16, [1, 16, 17, 33, 300]),
    "single_tokens_d64": (12, 12, 1, 64, 16, [130, 1, 0, 77]),
    "odd_pages": (6, 2, 3, 64, 7, [3, 50, 101]),
    "odd_pages_d128": (6, 2, 3, 128, 13, [3, 50, 101, 700]),
    "pages_of_one": (4, 4, 2, 128, 1, [40, 2, 129]),
    "small_tree": (3, 3, 13, 64, 24, [13, 14, 50, 200]),
    "two_blocks": (4, 2, 9, 64, 16, [300, 9]),
    "two_blocks_odd": (4, 2, 9, 64, 5, [300, 9]),
    "two_blocks_d128": (4, 2, 9, 128, 32, [300, 9]),
    "two_blocks_odd_d128": (4, 2, 9, 128, 6, [300, 9]),
    "forty_rows": (8, 1, 5, 128, 16, [64, 5, 333]),
    "forty_rows_d64": (8, 1, 5, 64, 10, [64, 5, 333]),
    "whole_tree": (2, 2, 64, 128, 64, [64, 65, 1000]),
    "whole_tree_d64": (2, 1, 64, 64, 16, [64, 200, 127]),
    "many_rows": (8, 2, 33, 64, 100, [33, 500]),
    "many_tiles": (16, 1, 64, 128, 128, [700, 64]),
    "shorter_than_its_drafts": (4, 2, 8, 64, 16, [0, 3, 8]),
    "shorter_than_its_drafts_d128": (8, 1, 40, 128, 16, [0, 3, 8, 100]),
    "long": (4, 2, 4, 128, 16, [9999, 3000]),
    "long_d64": (4, 4, 1, 64, 64, [20001]),
    "long_trees": (4, 2, 50, 128, 32, [5000, 60, 3333]),
    "uneven": (4, 1, 1, 128, 16, [6000] + [5] * 40),
    "more_than_a_wave": (2, 1, 2, 64, 8, [(37 * i) % 700 for i in range(150)]),
    "many_rows_in_one_range": (8, 4, 40, 64, 16, [(97 * i) % 400 + 40 for i in range(40)]),
    "many_rows_in_one_range_d128": (10, 5, 20, 128, 32, [(61 * i) % 450 for i in range(30)] + [0, 512]),
    "hundreds": (1, 1, 1, 64, 16, [(53 * i) % 301 for i in range(700)]),
    "hundreds_uneven": (2, 1, 3, 128, 16, [5000] + [(29 * i) % 97 + 3 for i in range(300)]),
    "out_of_range": (2, 1, 2, 64, 16, [-5, 40, 10]),
}


@pytest.mark.parametrize("name", sorted(CASES))
@pytest.mark.parametrize("chain", [False, True])
def test_tree(name, chain):
    H, Hkv, T, d, page, lens = CASES[name]
    q, k, v, lengths, table, parents = _inputs(H, Hkv, T, d, page, lens)
    if chain:
        parents = None
    par = None if chain else _int(parents)
    out, lse = tk.attn_tree(q, k, v, lengths, table, par, lse=True)
    _check(q, k, v, lens, table, parents, out, lse)
    same = torch.equal(tk.attn_tree(q, k, v, lengths, table, par), out)
    assert same


def test_lengths_beyond_the_table():
    q, k, v, lengths, table, parents = _inputs(2, 1, 3, 64, 16, [48, 20])
    lengths.copy_(_int([49, 2 ** 31 - 1]))
    out = tk.attn_tree(q, k, v, lengths, table, _int(parents))
    _check(q, k, v, [49, 2 ** 31 - 1], table, parents, out)


@pytest.mark.parametrize("T,H,d,page", [(1, 4, 128, 16), (13, 2, 64, 24), (13, 2, 64, 7), (20, 8, 128, 64), (64, 2, 64, 16)])
def test_wide_tables_and_one_tree_for_all(T, H, d, page):
    """A table far wider than the requests: the same numbers but for the ranges' rounding."""
    lens = [T, 400, 1500]
    q, k, v, lengths, table, parents = _inputs(H, 1, T, d, page, lens, wide=3000)
    out, lse = tk.attn_tree(q, k, v, lengths, table, _int(parents[0]), lse=True)
    _check(q, k, v, lens, table, [parents[0]] * 3, out, lse)
    same = torch.equal(out, tk.attn_tree(q, k, v, lengths, table, _int([parents[0]] * 3)))
    assert same


def test_parents_that_are_no_drafts_before():
    q, k, v, lengths, table, _ = _inputs(4, 2, 6, 64, 16, [40, 100])
    parents = [[0, -1, 2, 5, 3, 4], [1, 7, -9, 2 ** 31 - 1, 0, 4]]
    _check(q, k, v, [40, 100], table, parents, tk.attn_tree(q, k, v, lengths, table, _int(parents)))


@pytest.mark.parametrize("T,H,d,page", [(1, 4, 128, 16), (5, 2, 64, 24), (5, 2, 64, 7), (20, 8, 128, 64), (64, 2, 64, 16)])
def test_entries_that_name_no_page(T, H, d, page):
    """Rows without a page are not seen, and nothing is read for them."""
    lens = [300, 1500, T]
    q, k, v, lengths, table, parents = _inputs(H, 1, T, d, page, lens)
    bad = table.clone()
    bad[0, 1], bad[1, 0], bad[1, -1], bad[1, 2] = -1, len(k), 2 ** 31 - 1, -2 ** 31
    bad[2, 0] = -1
    out, lse = tk.attn_tree(q, k, v, lengths, bad, _int(parents), lse=True)
    _check(q, k, v, lens, bad, parents, out, lse)


def test_without_a_table():
    """A cache of one long page a request, cut from a larger one."""
    lens = [70, 1, 33]
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(4, 2, 90, 64, generator=gen, device="cuda").to(BF16)[:, :, 10:85] for _ in range(2))
    q = torch.randn(3, 4, 1, 64, generator=gen, device="cuda").to(BF16)
    out, lse = tk.attn_tree(q, k, v, _int(lens), lse=True)
    _check(q, k, v, lens, None, None, out, lse)
    want = tk.attn_prefix(q, None, None, k[:3], v[:3], _int(lens))
    assert bool(((out.float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + 2.0 ** -12).all())


@pytest.mark.parametrize("T,H,d,page", [(1, 4, 128, 16), (5, 2, 64, 7), (20, 8, 128, 64), (64, 2, 64, 16)])
def test_pages_far_apart(T, H, d, page):
    """A pool whose pages, heads or rows lie further apart than 32 bits reach."""
    q, k, v, lengths, table, parents = _inputs(H, 2, T, d, page, [3 * page, 77], spare=0)
    want = tk.attn_tree(q, k, v, lengths, table, _int(parents))
    P = len(k)
    buf = torch.zeros(5 << 30, dtype=BF16, device="cuda")  # 10 GB
    small = 2 * page * d
    for st in (((5 << 30) // P // 8 * 8, page * d, d), (small, (1 << 32) + 8, d), (small, page * d, d)):
        if st[0] * (P - 1) + st[1] + page * d > len(buf):
            continue
        far = buf.as_strided((P, 2, page, d), (*st, 1))
        far.copy_(k)
        same = torch.equal(tk.attn_tree(q, far, v, lengths, table, _int(parents)), want)
        far.copy_(v)
        same = same and torch.equal(tk.attn_tree(q, k, far, lengths, table, _int(parents)), want)
        assert same, st


def test_strided_pools():
    """The rows of all heads together, keys and values of a page side by side."""
    q, k, v, lengths, table, parents = _inputs(4, 2, 5, 128, 16, [200, 77])
    both = torch.stack((k, v)).permute(1, 3, 0, 2, 4).contiguous()  # [pages, rows, 2, heads, d]
    ks, vs = (both[:, :, i].transpose(1, 2) for i in range(2))
    same = torch.equal(tk.attn_tree(q, ks, vs, lengths, table, _int(parents)), tk.attn_tree(q, k, v, lengths, table, _int(parents)))
    assert same


@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("T,H,d,page", [(12, 2, 64, 8), (12, 2, 64, 7), (9, 4, 64, 16), (9, 2, 128, 16), (20, 8, 128, 16), (40, 4, 64, 64)])
def test_hidden_rows_may_hold_anything(bad, T, H, d, page):
    """Rows behind the request's, pages of others, and drafts that a row does not see."""
    lens = [300, 77]
    q, k, v, lengths, table, parents = _inputs(H, 1, T, d, page, lens, seed=2)
    par = _int(parents)
    want = tk.attn_tree(q, k, v, lengths, table, par)
    used = torch.zeros(k.shape[0], k.shape[2], dtype=torch.bool)
    for b, n in enumerate(lens):
        for j in range(n):
            used[table[b, j // page], j % page] = True
    k2, v2 = k.clone(), v.clone()
    free = (~used).cuda()
    k2.transpose(1, 2)[free] = bad
    v2.transpose(1, 2)[free] = bad
    same = torch.equal(tk.attn_tree(q, k2, v2, lengths, table, par), want)
    assert same
    for draft in (T // 2, T - 1):
        for which in (0, 1):
            kv = [k2.clone(), v2.clone()]
            for b, n in enumerate(lens):
                j = n - T + draft
                kv[which][table[b, j // page], 0, j % page, 3] = bad
            got = tk.attn_tree(q, *kv, lengths, table, par)
            for b in range(2):
                sees = _sees(parents[b])
                for i in range(T):
                    if draft not in sees[i]:
                        assert torch.equal(got[b, :, i], want[b, :, i]), (draft, which, b, i)
                    elif which:
                        assert not got[b, :, i, 3].isfinite().any()
                        assert torch.equal(got[b, :, i, 4:], want[b, :, i, 4:])


def test_tiny_weights_and_a_late_maximum():
    """Weights below 2^-126 still count against large values, before and behind a maximum that leads them."""
    for d, T in ((64, 1), (128, 1), (128, 64), (64, 40)):
        n = 1000
        q = torch.zeros(1, 2, T, d, device="cuda", dtype=BF16)
        q[..., 0] = 1
        for at in (10, n - T - 5):
            k, v = torch.zeros(1, 2, n, d, device="cuda", dtype=BF16), torch.full((1, 2, n, d), 2.0 ** 90, device="cuda", dtype=BF16)
            k[..., at, 0], v[..., at, :] = 88.5, 1.0
            out = tk.attn_tree(q, k, v, _int([n]), scale=1.0)
            s = k[0, 0, :, 0].double()
            ref = torch.softmax(s, 0) @ v[0, 0].double()
            near = n - T  # (drafts see fewer keys: their part is within T of n)
            assert bool(((out.double() - ref).abs() <= (2.0 ** -7 + T / near) * ref.abs()).all()), (d, T, at)


def test_streams_and_graphs():
    q, k, v, lengths, table, parents = _inputs(8, 2, 6, 128, 16, [3000, 200, 77], wide=20)
    par = _int(parents)
    want = tk.attn_tree(q, k, v, lengths, table, par)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = tk.attn_tree(q, k, v, lengths, table, par)
    torch.cuda.current_stream().wait_stream(s)
    same = torch.equal(got, want)
    assert same
    g, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = tk.attn_tree(q, k, v, lengths, table, par)
    with torch.cuda.graph(g2):
        out2 = tk.attn_tree(q[:, :2].contiguous(), k[:, :1], v[:, :1], lengths, table, par)
    for lens in ([3000, 200, 77], [6, 100, 70], [2500, 0, 9]):
        lengths.copy_(_int(lens))
        g.replay()
        g2.replay()
        torch.cuda.synchronize()
        same = torch.equal(out, tk.attn_tree(q, k, v, lengths, table, par))
        same &= torch.equal(out2, tk.attn_tree(q[:, :2].contiguous(), k[:, :1], v[:, :1], lengths, table, par))
        assert same


def test_refused_on_the_gpu():
    q, k, v, lengths, table, parents = _inputs(4, 2, 3, 64, 16, [40, 20])
    for args in ((q[0], k, v, lengths, table), (q, k, k, lengths, table), (q, k, v, lengths[:1], table), (q, k, v, lengths, table[:1]),
                 (q, k, v[:, :1], lengths, table), (q, k[..., :32], v[..., :32], lengths, table), (q, k[:1], v[:1], lengths), (q, k.cpu(), v, lengths, table),
                 (q, k, v, lengths, table, _int([0, 0])), (q.transpose(1, 2), k, v, lengths, table)):
        with pytest.raises(ValueError):
            tk.attn_tree(*args)
    with pytest.raises(TypeError):
        tk.attn_tree(q, k, v, lengths.long(), table)
    for args in ((q[:, :3].contiguous(), k, v, lengths, table), (q.float(), k.float(), v.float(), lengths, table),
                 (q.repeat(1, 1, 22, 1), k, v, lengths, table)):
        with pytest.raises(tk.TopkError):
            tk.attn_tree(*args)


@pytest.mark.parametrize("T,H,d,page", [(1, 2, 64, 8), (12, 2, 64, 8), (12, 2, 64, 7), (9, 4, 64, 16), (9, 4, 64, 5), (9, 2, 128, 16), (9, 2, 128, 7), (20, 8, 128, 16), (40, 4, 64, 64),
                                        (5, 8, 128, 16)])
def test_infinite_values_that_are_seen(T, H, d, page):
    """By the definition a weight above 0 makes an infinite value an infinite output, of the same sign, two of different
    signs NaN, whether the key is text, in a tile with drafts or not, or a draft."""
    lens = [300, 77, 2500, T]
    q, k, v, lengths, table, parents = _inputs(H, 1, T, d, page, lens, seed=2)
    par = _int(parents)
    want, wl = tk.attn_tree(q, k, v, lengths, table, par, lse=True)
    inf, nan = math.inf, math.nan
    v2 = v.clone()
    for b, n in enumerate(lens):
        text = n - T
        at = [(n - 1, 3, inf), (text + T // 2, 4, -inf), (n - 1, 5, inf), (text, 5, -inf), (text + T // 3, 6, nan), (text, d - 1, inf), (n - 1, d - 2, -inf)]
        if text:
            at += [(text - 1, 7, inf), (0, 8, -inf), (0, 9, inf), (n - 1, 9, -inf), (text - 1, 10, nan)]
        sees = _sees(parents[b])
        here = torch.zeros(T, d, dtype=torch.float64)
        put = {}
        for j, f, x in at:
            put[j, f] = x  # (with one draft some coincide: the last stands)
        for (j, f), x in put.items():
            v2[table[b, j // page], 0, j % page, f] = x
            for i in range(T):
                if j < text or j - text in sees[i]:
                    here[i, f] += x
        here = here.to(BF16).cuda()[None]
        want[b] = torch.where(here == 0, want[b], here)
    got, gl = tk.attn_tree(q, k, v2, lengths, table, par, lse=True)
    assert torch.equal(gl, wl)
    assert bool(((got == want) | (got.isnan() & want.isnan())).all())


@pytest.mark.parametrize("d,T,page", [(64, 1, 16), (64, 1, 7), (128, 1, 16), (64, 5, 16), (128, 5, 7), (128, 40, 16), (64, 40, 16)])
def test_infinite_values_of_weights_that_32_bits_hold_as_0(d, T, page):
    """e^-200 is above 0 all the same, in the leading key's range and in others."""
    n = 5000
    q, k, v, lengths, table, _ = _inputs(4, 1, T, d, page, [n, T, 300])
    q[:], k[:], v[:] = 0, 0, 1
    q[..., 0] = 1
    at = lambda j: (table[0, j // page], 0, j % page)  # noqa: E731
    for j, f, x in ((0, 1, math.inf), (1000, 2, -math.inf), (4000, 3, math.inf), (n - T, 4, -math.inf), (10, 5, math.inf), (4700, 5, -math.inf)):
        v[(*at(j), f)] = x
    want = torch.ones(d, device="cuda")
    want[1:6] = torch.tensor([math.inf, -math.inf, math.inf, -math.inf, math.nan])
    for top in (3, 2500, n - T - 1):
        k[:] = 0
        k[(*at(top), 0)] = 200
        out = tk.attn_tree(q, k, v, lengths, table, scale=1.0).float()
        assert bool(((out[0] == want) | (out[0].isnan() & want.isnan())).all()), top
        assert bool((out[1:] == 1).all())


@pytest.mark.parametrize("d,H,T", [(64, 2, 1), (64, 4, 13), (128, 2, 1), (128, 4, 9), (128, 8, 20), (64, 2, 64), (128, 2, 64)])
@pytest.mark.parametrize("n", [300, 1000, 16000])
def test_tiny_weights_are_the_result(d, H, T, n):
    """Values of 2^112 whose weights are e^-88.5 beside a value of 0 that has all the rest: the output is theirs alone, before
    and behind the key that leads them, in its range and in others. (As a bf16 number such a weight is a multiple of
    2^-133, off by 2^-6.32 of it at most; rounding of the output 2^-8, of the rest less than 2^-10.)"""
    q = torch.zeros(1, H, T, d, device="cuda", dtype=BF16)
    q[..., 0] = 1
    k, v = (torch.zeros(1, H // 2, n, d, device="cuda", dtype=BF16) for _ in range(2))
    for at in (0, 10, n // 2, n - T - 5):
        k[:], v[:] = 0, 2.0 ** 112
        k[..., at, 0], v[..., at, :] = 88.5, 0
        out = tk.attn_tree(q, k, v, _int([n]), scale=1.0, lse=True)[0].double()
        want = (n - T + torch.arange(T, device="cuda").double()) * math.exp(-88.5) * 2.0 ** 112  # (each follows the one before it)
        assert bool(((out - want[None, None, :, None]).abs() <= (2.0 ** -6.32 + 2.0 ** -8 + 2.0 ** -10) * want[None, None, :, None]).all()), at
