"""GPU tests of the page calls against books kept as Python lists, and rows copied one by one: every
result is exact, whole numbers and rows alike."""
import random

import pytest
import torch

import paper_2106_06899_amd as tk

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    tk.lib()
    yield


class Books:
    """A cache of pages on the CPU, one step at a time."""

    def __init__(self, k, v, table, refs, lengths):
        self.k, self.v, self.table, self.refs, self.lens = k.cpu().clone(), v.cpu().clone(), table.tolist(), refs.tolist(), lengths.tolist()
        self.page, self.n = k.shape[-2], k.shape[1]

    def held(self, p):
        return 0 <= p < self.n

    def reserve(self, rows):
        want, page = [], self.page
        for b, n in enumerate(self.lens):
            r = rows[b] if isinstance(rows, list) else rows
            if n >= 0 and r > 0:
                want += [(b, e) for e in range(n // page, min(len(self.table[b]), -(-(n + r) // page)))]
        leave = [x for x in want if self.held(self.table[x[0]][x[1]]) and self.refs[self.table[x[0]][x[1]]] > 1]
        holders = {}
        for x in leave:
            holders.setdefault(self.table[x[0]][x[1]], []).append(x)
        for p, xs in holders.items():
            if len(xs) == self.refs[p]:
                leave.remove(xs[0])
        need = [x for x in want if not self.held(self.table[x[0]][x[1]]) or x in leave]
        free = [p for p, r in enumerate(self.refs) if r == 0]
        if len(free) < len(need):
            return len(need) - len(free)
        for (b, e), q in zip(need, free):
            p, used = self.table[b][e], self.lens[b] - e * page
            if (b, e) in leave:
                self.refs[p] -= 1
                if used > 0:
                    for t in (self.k, self.v):
                        t[:, q, :, :used] = t[:, p, :, :used]
            self.table[b][e], self.refs[q] = q, 1
        return 0

    def at(self, b, r):
        e = r // self.page
        p = self.table[b][e] if e < len(self.table[b]) else -1
        return (p, r % self.page) if self.held(p) else None

    def write(self, b, r, k, v):
        x = self.at(b, r)
        if self.lens[b] >= 0 and x:
            self.k[:, x[0], :, x[1]], self.v[:, x[0], :, x[1]] = k, v

    def append(self, k, v):
        for b in range(len(self.lens)):
            for t in range(k.shape[3]):
                self.write(b, self.lens[b] + t, k[:, b, :, t], v[:, b, :, t])

    def keep(self, kept):
        new = []
        for b, row in enumerate(kept):
            n = next((i for i, x in enumerate(row) if x < 0), len(row)) if self.lens[b] >= 0 else 0
            old = (self.k.clone(), self.v.clone()) if n else None
            for i in range(n):
                f, t = self.at(b, self.lens[b] + row[i]), self.at(b, self.lens[b] + i)
                if f and t:
                    self.k[:, t[0], :, t[1]], self.v[:, t[0], :, t[1]] = old[0][:, f[0], :, f[1]], old[1][:, f[0], :, f[1]]
            new.append(self.lens[b] + n)
        return new

    def need(self, n):
        return -(-max(n, 0) // self.page)

    def fork(self, parents):
        old, lens = [list(r) for r in self.table], list(self.lens)
        for b, p in enumerate(parents):
            if p == b or p >= len(parents):
                continue
            n = self.need(lens[p]) if p >= 0 else 0
            self.table[b] = [x if i < n and self.held(x) else -1 for i, x in enumerate(old[p] if p >= 0 else old[b])]
            for x in old[b]:
                if self.held(x):
                    self.refs[x] -= 1
            for x in self.table[b]:
                if self.held(x):
                    self.refs[x] += 1
            self.lens[b] = lens[p] if p >= 0 else 0

    def release(self):
        for b, row in enumerate(self.table):
            for e in range(self.need(self.lens[b]), len(row)):
                if self.held(row[e]):
                    self.refs[row[e]] -= 1
                row[e] = -1


class Cache:
    """Books on the GPU and the CPU together."""

    def __init__(self, B, M, page, n_pages, layers=1, heads=2, d=64, dtype=torch.bfloat16, seed=0, longest=None):
        rng = self.rng = random.Random(seed)
        gen = self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.page, self.B, self.M = page, B, M
        self.k, self.v = (torch.randn(layers, n_pages, heads, page, d, generator=gen, device="cuda").to(dtype) for _ in range(2))
        ids = list(range(n_pages))
        rng.shuffle(ids)
        lens, table, refs = [], [], [0] * n_pages
        for b in range(B):
            n = rng.randint(0, longest if longest is not None else page * M // 2)
            row = [ids.pop() for _ in range(min(-(-n // page), len(ids)))]
            n = min(n, len(row) * page)
            for p in row:
                refs[p] += 1
            lens.append(n)
            table.append(row + [-1] * (M - len(row)))
        self.set(table, refs, lens)

    def set(self, table, refs, lens):
        i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.table, self.refs, self.lengths = i(table), i(refs), i(lens)
        self.books = Books(self.k, self.v, self.table, self.refs, self.lengths)

    def rows(self, T):
        L, _, h, _, d = self.k.shape
        return tuple(torch.randn(L, self.B, h, T, d, generator=self.gen, device="cuda").to(self.k.dtype) for _ in range(2))

    def check(self, what=""):
        b = self.books
        assert self.table.tolist() == b.table, f"{what}: tables"
        assert self.refs.tolist() == b.refs, f"{what}: counts"
        assert self.lengths.tolist() == b.lens, f"{what}: lengths"
        same = torch.equal(self.k.cpu(), b.k) and torch.equal(self.v.cpu(), b.v)
        assert same, f"{what}: rows"

    def reserve(self, rows):
        got = tk.pages_reserve(self.k, self.v, self.table, self.refs, self.lengths,
                               torch.tensor(rows, dtype=torch.int32, device="cuda") if isinstance(rows, list) else rows)
        want = self.books.reserve(rows)
        assert int(got) == want
        self.check("reserve")
        return want

    def append(self, T):
        k, v = self.rows(T)
        tk.pages_append(k, v, self.k, self.v, self.table, self.lengths)
        self.books.append(k.cpu(), v.cpu())
        self.check("append")

    def keep(self, kept):
        new = tk.pages_keep(self.k, self.v, self.table, self.lengths, torch.tensor(kept, dtype=torch.int32, device="cuda"))
        self.books.lens = self.books.keep(kept)
        self.lengths.copy_(new)
        self.check("keep")

    def fork(self, parents):
        tk.pages_fork(self.table, self.refs, self.lengths, torch.tensor(parents, dtype=torch.int32, device="cuda"), self.page)
        self.books.fork(parents)
        self.check("fork")

    def release(self):
        tk.pages_release(self.table, self.refs, self.lengths, self.page)
        self.books.release()
        self.check("release")


SHAPES = {
    # name: B, M, page, n_pages, layers, heads, d, dtype
    "one": (1, 1, 1, 1, 1, 1, 8, torch.bfloat16),
    "small": (5, 6, 4, 40, 1, 2, 64, torch.bfloat16),
    "odd_pages": (7, 9, 3, 80, 3, 1, 24, torch.float32),
    "layers": (9, 8, 16, 100, 4, 3, 128, torch.bfloat16),
    "single_rows": (6, 40, 1, 300, 2, 2, 64, torch.float32),
    "large_pages": (3, 3, 100, 12, 2, 5, 64, torch.bfloat16),
    "wide_rows": (4, 5, 7, 30, 1, 2, 1024, torch.float32),
    "many_pages": (13, 30, 5, 9001, 1, 1, 16, torch.bfloat16),
}


@pytest.mark.parametrize("name", sorted(SHAPES))
@pytest.mark.parametrize("seed", [0, 1])
def test_a_run_of_steps(name, seed):
    """Beams, drafts and ends in turn, as a decoder makes them, compared after every call."""
    B, M, page, n, layers, heads, d, dtype = SHAPES[name]
    c = Cache(B, M, page, n, layers, heads, d, dtype, seed)
    rng = c.rng
    for step in range(6):
        c.fork([rng.choice([b, rng.randrange(B), rng.randrange(B), -1 if step % 3 == 2 else b]) for b in range(B)])
        T = rng.randint(1, min(64, 2 * page + 1))
        if c.reserve(T if step % 2 else [T + rng.randint(0, T) for _ in range(B)]):  # (two requests must not append to one page)
            c.lengths.zero_()
            c.books.lens = [0] * B
            c.release()
            continue
        c.append(T)
        kept = [sorted(rng.sample(range(T), rng.randint(0, min(T, 5)))) for _ in range(B)]
        c.keep([k + [-1] * (5 - len(k)) for k in kept])
        c.release()


def test_more_requests_than_a_workgroup_takes_at_once():
    c = Cache(2500, 3, 4, 12000, 1, 1, 8, seed=3, longest=8)
    assert c.reserve(3) == 0
    c.fork([b // 3 * 3 for b in range(2500)])
    assert c.reserve([b % 4 for b in range(2500)]) == 0
    c.append(2)
    c.release()


@pytest.mark.parametrize("B,M", [(3000, 3), (700, 40), (9000, 1), (2, 5000)])
def test_forks_of_large_tables(B, M):
    """More entries than one workgroup takes: cycles, chains and ends of requests at once."""
    c = Cache(B, M, 4, 3 * B + 50, 1, 1, 8, seed=B, longest=8 if M > 1 else 4)
    rng = c.rng
    for _ in range(2):
        c.fork([rng.choice([b, (b + 1) % B, rng.randrange(B), -1, b // 7 * 7]) for b in range(B)])
    c.release()
    c.fork([-1] * B)
    assert not c.refs.any()


@pytest.mark.parametrize("B,M,n,held", [(40, 400, 16384, 0), (40, 400, 16385, 1), (40, 1000, 50000, 0.9), (1500, 6, 41000, 0.5),
                                        (3, 30000, 70001, 0.3)])
def test_large_pools(B, M, n, held):
    """Pools whose free pages are listed by blocks: the lowest numbers all the same, most of the first ones held by
    somebody else."""
    c = Cache(B, M, 2, n, 1, 1, 8, seed=n, longest=20 if M > 6 else 6)
    refs = c.refs.tolist()
    for p in range(n // 2 if held < 1 else n - B // 2):
        if refs[p] == 0 and c.rng.random() < held:
            refs[p] = 1
    c.set(c.table.tolist(), refs, c.lengths.tolist())
    for _ in range(2):
        c.fork([c.rng.choice([b, c.rng.randrange(B)]) for b in range(B)])
        rows = 3 if M == 6 else 100 if held == 0 else 40 if M < 30000 else [30000, 0, 20011]
        missing = c.reserve(rows)
        assert (missing > 0) == (held == 1)
        if not missing:  # (else several would write to one page)
            c.append(2)
    c.release()
    live = sum(r > 0 for r in c.books.refs)
    kt, vt = (torch.full((1, live, 1, 2, 8), 7.0, dtype=c.k.dtype, device="cuda") for _ in range(2))
    table, new, missing = tk.pages_compact(c.k, c.v, c.table, c.refs, kt, vt)
    at = c.refs > 0
    same = torch.equal(kt, c.k[:, at]) and torch.equal(vt, c.v[:, at]) and torch.equal(new, c.refs[at])
    assert int(missing) == 0 and same
    number = torch.where(at, at.cumsum(0) - 1, -1).int()
    assert torch.equal(table, torch.where(c.table >= 0, number[c.table.long().clamp(min=0)], -1))


@pytest.mark.parametrize("page,heads,layers", [(64, 8, 3), (130, 5, 40)])
def test_many_copies(page, heads, layers):
    """Copies of more pieces than there are workgroups."""
    c = Cache(60, 4, page, 200, layers, heads, 64, seed=page, longest=3 * page)
    c.fork([b // 3 * 3 for b in range(60)])
    assert c.reserve(1) == 0
    c.append(1)


def test_a_long_reservation():
    """More entries a request than a workgroup takes at once."""
    c = Cache(3, 4000, 2, 9000, 1, 1, 8, seed=4, longest=100)
    assert c.reserve([3000, 0, 7000]) == 0


def test_too_few_pages_change_nothing():
    c = Cache(4, 8, 4, 20, 2, 1, 8, seed=5, longest=14)
    c.fork([0, 0, 0, 0])
    before = [t.clone() for t in (c.table, c.refs, c.lengths, c.k, c.v)]
    assert c.reserve(4 * 8) > 0
    assert all(torch.equal(a, b) for a, b in zip(before, (c.table, c.refs, c.lengths, c.k, c.v)))
    assert c.reserve(1) == 0


@pytest.mark.parametrize("rows", [1, 5])
def test_where_all_holders_write_the_first_keeps(rows):
    c = Cache(6, 6, 4, 30, 1, 1, 8, seed=6)
    c.set([[7, 3, -1, -1, -1, -1]] * 4 + [[9, 3, -1, -1, -1, -1], [1, 2, -1, -1, -1, -1]],
          [1 if p in (1, 2, 9) else 4 if p == 7 else 5 if p == 3 else 0 for p in range(30)], [6, 6, 6, 6, 6, 7])
    assert c.reserve(rows) == 0
    assert c.table[0, 1] == 3 and c.refs[3] == 1 and c.refs[7] == 4
    # one that does not write goes on holding it
    c.set([[3, -1], [3, -1], [3, -1]] + [[-1, -1]] * 3, [3 if p == 3 else 0 for p in range(30)], [2, 2, 2, 0, 0, 0])
    assert c.reserve([1, 0, 1, 0, 0, 0]) == 0
    assert c.table[1, 0] == 3 and c.refs[3] == 1


def test_entries_that_name_no_page():
    """Numbers outside the pool, and negative lengths: nothing is read or written for them."""
    c = Cache(5, 4, 4, 12, 2, 2, 8, seed=7)
    c.set([[2, 12, -7, 3], [2 ** 31 - 1, 1, -1, -1], [-2 ** 31, -1, -1, -1], [4, 5, -1, -1], [0, -1, -1, -1]],
          [1, 1, 1, 1, 1, 1] + [0] * 6, [5, 6, 3, 7, -3])
    c.append(3)
    c.keep([[1, 0], [0, 1], [1, -1], [2, 1], [0, 1]])
    c.books.lens = [5, 6, 3, 7, -3]
    c.lengths.copy_(torch.tensor(c.books.lens))
    c.fork([1, 0, 3, 3, 9])
    assert c.reserve(2) == 0
    c.release()


def test_keep_in_any_order():
    """Rows change places: all are read before one is written."""
    c = Cache(2, 5, 8, 20, 2, 2, 128, seed=8)
    c.set([[3, 5, 1, -1, -1], [2, 4, 6, 7, -1]], [1 if 1 <= p <= 7 else 0 for p in range(20)], [3, 9])
    c.append(20)
    c.keep([[4, 0, 1, 1, 3, 2], [5, 4, 3, 2, 1, 0]])
    c2 = Cache(1, 10, 16, 20, 1, 1, 1024, torch.float32, seed=9)
    c2.set([list(range(10))], [1] * 10 + [0] * 10, [5])
    c2.keep([list(range(63, -1, -1))])


def test_packed_rows():
    """Packed prompts into pages, tokens outside every request left out."""
    B, M, page, h, d = 4, 6, 5, 2, 64
    c = Cache(B, M, page, 40, 1, h, d, seed=10, longest=10)
    lens = [7, 0, 12, 1]
    assert c.reserve(lens) == 0
    off = [3, 10, 10, 22, 23]
    gen = torch.Generator(device="cuda").manual_seed(0)
    k, v = (torch.randn(30, h, d, generator=gen, device="cuda").bfloat16().transpose(0, 1) for _ in range(2))
    tk.pages_append(k, v, c.k[0], c.v[0], c.table, c.lengths, torch.tensor(off, dtype=torch.int32, device="cuda"))
    for b in range(B):
        for t in range(lens[b]):
            c.books.write(b, c.books.lens[b] + t, k[:, off[b] + t].cpu()[None], v[:, off[b] + t].cpu()[None])
    c.check("packed")


@pytest.mark.parametrize("shape", [(4, 6, 4, 40, 1, 2, 64), (9, 8, 16, 100, 4, 3, 128), (3, 40, 1, 5000, 2, 1, 8)])
def test_compact(shape):
    c = Cache(*shape, seed=11)
    c.fork([b // 2 * 2 for b in range(c.B)])
    refs = c.refs.tolist()
    live = [p for p, r in enumerate(refs) if r > 0]
    for n_to in (len(live), len(live) + 5):
        kt, vt = (torch.full((shape[4], n_to, *c.k.shape[2:]), 7.0, dtype=c.k.dtype, device="cuda") for _ in range(2))
        table, new, missing = tk.pages_compact(c.k, c.v, c.table, c.refs, kt, vt)
        number = {p: i for i, p in enumerate(live)}
        assert int(missing) == 0
        assert table.tolist() == [[number.get(p, -1) for p in row] for row in c.table.tolist()]
        assert new.tolist() == [refs[p] for p in live] + [0] * (n_to - len(live))
        same = torch.equal(kt[:, :len(live)], c.k[:, live]) and torch.equal(vt[:, :len(live)], c.v[:, live])
        assert same
        assert bool((kt[:, len(live):] == 7).all()) and bool((vt[:, len(live):] == 7).all())
    c.check("the old pool")
    if len(live) > 1:
        kt, vt = (torch.full((shape[4], len(live) - 1, *c.k.shape[2:]), 7.0, dtype=c.k.dtype, device="cuda") for _ in range(2))
        table, new, missing = tk.pages_compact(c.k, c.v, c.table, c.refs, kt, vt)
        assert int(missing) == 1 and not new.any() and bool((table == -1).all()) and bool((kt == 7).all())


@pytest.mark.parametrize("page,heads,d,dtype", [(16, 8, 128, torch.bfloat16), (50, 6, 256, torch.float32), (3, 5, 24, torch.bfloat16)])
@pytest.mark.parametrize("strided", ["from", "to", "both", "layers"])
def test_compact_of_strided_pools(page, heads, d, dtype, strided):
    """Pools whose rows of all heads lie together, and pools cut from larger ones; pages of few and of many pieces."""
    c = Cache(5, 4, page, 30, 2, heads, d, dtype, seed=page)
    live = [p for p, r in enumerate(c.refs.tolist()) if r > 0]
    turned = lambda t: t.permute(0, 1, 3, 2, 4).contiguous().permute(0, 1, 3, 2, 4)  # noqa: E731
    k, v = (turned(t) if strided in ("from", "both") else t for t in (c.k, c.v))
    kt, vt = (torch.full((2, len(live) + 3, heads, page, d), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    if strided in ("to", "both"):
        kt, vt = turned(kt), turned(vt)
    if strided == "layers":  # every other layer of larger pools, with more pages
        k, v, kt, vt = (torch.full((4, t.shape[1] + 2, heads, page, d), 7.0, dtype=dtype, device="cuda")[::2, :-2].copy_(t) for t in (k, v, kt, vt))
    table, new, missing = tk.pages_compact(k, v, c.table, c.refs, kt, vt)
    assert int(missing) == 0 and new.tolist() == [1] * len(live) + [0] * 3
    same = torch.equal(kt[:, :len(live)], c.k[:, live]) and torch.equal(vt[:, :len(live)], c.v[:, live])
    assert same and bool((kt[:, len(live):] == 7).all()) and bool((vt[:, len(live):] == 7).all())


def test_strided_pools_tables_and_rows():
    """Pools with the rows of all heads together, a table cut from a wider one, rows from a projection."""
    c = Cache(4, 5, 6, 30, 2, 3, 64, seed=12)
    wide = torch.full((4, 9), -5, dtype=torch.int32, device="cuda")
    wide[:, 2:7] = c.table
    kp, vp = (t.permute(0, 1, 3, 2, 4).contiguous().permute(0, 1, 3, 2, 4) for t in (c.k, c.v))
    c.k, c.v, c.table = kp, vp, wide[:, 2:7]
    c.fork([1, 1, 1, 3])
    assert c.reserve(7) == 0
    x = torch.randn(2, 4, 7, 3, 3 * 64, generator=c.gen, device="cuda").bfloat16()
    k, v = x[..., 64:128].transpose(2, 3), x[..., 128:].transpose(2, 3)
    tk.pages_append(k, v, c.k, c.v, c.table, c.lengths)
    c.books.append(k.cpu(), v.cpu())
    c.check("append")
    c.keep([[2, 5], [0, 1], [-1, 3], [6, -1]])
    c.release()
    assert bool((wide[:, :2] == -5).all()) and bool((wide[:, 7:] == -5).all())


@pytest.mark.parametrize("far", ["pages", "layers", "heads"])
def test_pools_larger_than_32_bits_reach(far):
    """Layers, pages or heads of a pool that lie far apart."""
    c = Cache(3, 6, 4, 20, 2, 2, 64, seed=15, longest=12)
    st = {"pages": (512, 1 << 27, 256, 64), "layers": ((1 << 31) + 512, 512, 256, 64), "heads": (20 * 512, 256, (1 << 31) + 8, 64)}[far]
    for name in ("k", "v"):
        t = getattr(c, name)
        size = sum((n - 1) * s for n, s in zip(t.shape, (*st, 1))) + 1
        setattr(c, name, torch.zeros(size, dtype=t.dtype, device="cuda").as_strided(t.shape, (*st, 1)).copy_(t))
    c.fork([1, 1, 2])
    assert c.reserve(3) == 0
    c.append(3)
    c.keep([[2], [0], [1]])
    c.release()
    live = c.refs > 0
    to = [torch.zeros(2, int(live.sum()), 2, 4, 64, dtype=c.k.dtype, device="cuda") for _ in range(2)]
    assert int(tk.pages_compact(c.k, c.v, c.table, c.refs, *to)[2]) == 0
    same = torch.equal(to[0], c.k[:, live]) and torch.equal(to[1], c.v[:, live])
    assert same
    # and back, to the first pages
    used = to[0].shape[1]
    pages = torch.arange(used, dtype=torch.int32, device="cuda")[None]
    table, _, missing = tk.pages_compact(*to, pages, c.refs[live], c.k, c.v)
    same = torch.equal(table, pages) and torch.equal(c.k[:, :used], to[0]) and torch.equal(c.v[:, :used], to[1])
    assert same and int(missing) == 0


def test_streams_and_graphs():
    """A decoding step's calls, captured: the books change on every replay, on the GPU alone."""
    a, b = Cache(6, 8, 4, 60, 2, 2, 64, seed=13, longest=8), Cache(6, 8, 4, 60, 2, 2, 64, seed=13, longest=8)
    parents, kept = [0, 0, 2, 2, 5, 5], [[0, 2, -1], [1, -1, -1], [0, 1, 2], [-1, 0, 0], [2, -1, 0], [0, 1, -1]]
    par, kp = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (parents, kept))
    k, v = a.rows(3)

    def step(c):
        tk.pages_fork(c.table, c.refs, c.lengths, par, c.page)
        tk.pages_reserve(c.k, c.v, c.table, c.refs, c.lengths, 3)
        tk.pages_append(k, v, c.k, c.v, c.table, c.lengths)
        c.lengths.copy_(tk.pages_keep(c.k, c.v, c.table, c.lengths, kp))
        tk.pages_release(c.table, c.refs, c.lengths, c.page)

    start = [t.clone() for t in (a.table, a.refs, a.lengths, a.k, a.v)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(a)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(a)
    for t, x in zip((a.table, a.refs, a.lengths, a.k, a.v), start):
        t.copy_(x)
    for _ in range(4):
        g.replay()
        torch.cuda.synchronize()
        step(b)
        b.books.fork(parents)
        assert b.books.reserve(3) == 0
        b.books.append(k.cpu(), v.cpu())
        b.books.lens = b.books.keep(kept)
        b.books.release()
        b.check("eager")
        for x, y in zip((a.table, a.refs, a.lengths, a.k, a.v), (b.table, b.refs, b.lengths, b.k, b.v)):
            same = torch.equal(x, y)
            assert same


def test_refused_on_the_gpu():
    c = Cache(2, 3, 4, 10, 1, 1, 8, seed=14)
    with pytest.raises(ValueError):
        tk.pages_reserve(c.k, c.k, c.table, c.refs, c.lengths, 1)
    with pytest.raises(ValueError):
        tk.pages_reserve(c.k, c.v, c.table, c.refs[:5], c.lengths, 1)
    with pytest.raises(ValueError):
        tk.pages_reserve(c.k, c.v, c.table[:1].expand(2, -1), c.refs, c.lengths, 1)
    with pytest.raises(ValueError):
        tk.pages_reserve(c.k[:, :1].expand(-1, 10, -1, -1, -1), c.v, c.table, c.refs, c.lengths, 1)
    with pytest.raises(TypeError):
        tk.pages_fork(c.table.long(), c.refs, c.lengths, c.lengths, 4)
    with pytest.raises(tk.TopkError):
        tk.pages_reserve(c.k, c.v, c.table, c.refs, c.lengths, -1)
    with pytest.raises(tk.TopkError):
        tk.pages_release(c.table, c.refs, c.lengths, 0)
    with pytest.raises(tk.TopkError):
        tk.pages_keep(c.k, c.v, c.table, c.lengths, torch.zeros(2, 65, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        tk.pages_compact(c.k, c.v, c.table, c.refs, c.k[:, 2:], c.v[:, 2:])
    with pytest.raises(ValueError):
        tk.pages_append(c.k[:, :2], c.v[:, :2], c.k, c.v, c.table[:, :1], c.lengths, c.lengths)
    c.check("nothing")
