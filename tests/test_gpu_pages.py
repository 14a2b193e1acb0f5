"""Pages shared by rows, against a model of the calls on the host: counts, tables, lengths and contents are equal."""
import pytest
import torch

from paper_2602_00397_amd import binding as B
from test_gpu_attention import DEV, _gen, _int32, _refused, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


class Pool:
    """A pool and its model: lists on the host."""

    def __init__(self, n_pages, n_rows, stride, page_size=16, parts=((4, torch.bfloat16), (3, torch.uint8), (1, torch.float32)), seed=1):
        gen = _gen(seed)
        self.page_size, self.stride, self.n_pages, self.n_rows = page_size, stride, n_pages, n_rows
        self.refs, self.lens = torch.zeros(n_pages, dtype=torch.int32, device=DEV), torch.zeros(n_rows, dtype=torch.int32, device=DEV)
        self.table = torch.full((n_rows, stride), -1, dtype=torch.int32, device=DEV)
        self.parts = [torch.randint(0, 100, (n_pages, *((n,) if isinstance(n, int) else n)), device=DEV, generator=gen).to(t) for n, t in parts]
        self.pool = B.page_pool(self.refs, self.table, self.lens, page_size, self.parts)
        self.result = _int32([-7])
        self.m_refs, self.m_lens, self.m_table = [0] * n_pages, [0] * n_rows, [[-1] * stride for _ in range(n_rows)]
        self.m_parts = [p.cpu().clone() for p in self.parts]

    def pages(self, n):
        n = min(max(n, 0), self.stride * self.page_size)
        return -(-n // self.page_size)

    def is_row(self, r):
        return 0 <= r < self.n_rows

    def is_page(self, p):
        return 0 <= p < self.n_pages

    def winners(self, entries):
        return {r: i for i, r in enumerate(entries) if self.is_row(r)}

    def copy(self, ctx, sources, targets):
        ctx.pages_copy(self.pool, _int32(sources), _int32(targets))
        for a, b in zip(sources, targets):
            if self.is_page(a) and self.is_page(b):
                for p in self.m_parts:
                    p[b] = p[a]

    def fork(self, ctx, sources, targets):
        ctx.ensure_pages_workspace(self.pool, len(sources))
        ctx.pages_fork(self.pool, _int32(sources), _int32(targets), self.result)
        win, ps = self.winners(targets), self.page_size
        free, rows, moves = [p for p in range(self.n_pages) if self.m_refs[p] == 0], {}, []
        for i, (a, b) in enumerate(zip(sources, targets)):
            if self.is_row(a) and self.is_row(b) and win[b] == i:
                n = min(max(self.m_lens[a], 0), self.stride * ps)
                row, last = self.m_table[a][:self.pages(n)], n // ps
                own = n % ps and self.is_page(row[last]) and (a != b or self.m_refs[row[last]] > 1)
                if a == b and not own:
                    continue
                if own:
                    moves.append((row[last], len(moves)))
                    row = row[:last] + [("new", len(moves) - 1)]
                rows[b] = (row, n)
        if len(moves) > len(free):
            return len(moves) - len(free)
        for b, (row, n) in rows.items():
            for p in self.m_table[b][:self.pages(self.m_lens[b])]:
                if self.is_page(p):
                    self.m_refs[p] -= 1
        for b, (row, n) in rows.items():
            row = [free[p[1]] if isinstance(p, tuple) else p for p in row]
            for p in row:
                if self.is_page(p):
                    self.m_refs[p] += 1
            had = self.pages(self.m_lens[b])
            self.m_table[b] = row + [-1] * max(0, had - len(row)) + self.m_table[b][max(had, len(row)):]
            self.m_lens[b] = n
        held = [[p[a].clone() for p in self.m_parts] for a, _ in moves]
        for (_, k), contents in zip(moves, held):
            for p, x in zip(self.m_parts, contents):
                p[free[k]] = x
        return 0

    def grow(self, ctx, rows, lens):
        ctx.ensure_pages_workspace(self.pool, len(rows))
        ctx.pages_grow(self.pool, _int32(rows), _int32(lens), self.result)
        win, free = self.winners(rows), [p for p in range(self.n_pages) if self.m_refs[p] == 0]
        each = [(r, min(max(n, 0), self.stride * self.page_size)) for i, (r, n) in enumerate(zip(rows, lens)) if self.is_row(r) and win[r] == i]
        want = sum(max(0, self.pages(n) - self.pages(self.m_lens[r])) for r, n in each)
        if want > len(free):
            return want - len(free)
        for r, n in each:
            had, gets = self.pages(self.m_lens[r]), self.pages(n)
            for j in range(had, gets):
                self.m_table[r][j] = free.pop(0)
                self.m_refs[self.m_table[r][j]] = 1
            for j in range(gets, had):
                if self.is_page(self.m_table[r][j]):
                    self.m_refs[self.m_table[r][j]] -= 1
                self.m_table[r][j] = -1
            self.m_lens[r] = n
        return 0

    def free(self, ctx, rows):
        ctx.pages_free(self.pool, _int32(rows))
        for r in rows:
            if self.is_row(r):
                for j in range(self.pages(self.m_lens[r])):
                    if self.is_page(self.m_table[r][j]):
                        self.m_refs[self.m_table[r][j]] -= 1
                    self.m_table[r][j] = -1
                self.m_lens[r] = 0

    def compact(self, ctx):
        ctx.ensure_pages_workspace(self.pool, 1)
        ctx.pages_compact(self.pool, self.result)
        live = sum(n > 0 for n in self.m_refs)
        holes = [p for p in range(live) if self.m_refs[p] <= 0]
        place = {p: holes.pop(0) for p in range(live, self.n_pages) if self.m_refs[p] > 0}
        for a, b in place.items():
            self.m_refs[b], self.m_refs[a] = self.m_refs[a], 0
            for p in self.m_parts:
                p[b] = p[a]
        for r in range(self.n_rows):
            for j in range(self.pages(self.m_lens[r])):
                self.m_table[r][j] = place.get(self.m_table[r][j], self.m_table[r][j])
        return live

    def check(self, what, result=None):
        if result is not None:
            assert int(self.result) == result, f"{what}: {int(self.result)} said, {result} expected"
        assert self.refs.tolist() == self.m_refs, f"{what}: counts"
        assert self.lens.tolist() == self.m_lens, f"{what}: lengths"
        assert self.table.tolist() == self.m_table, f"{what}: table"
        for i, (x, m) in enumerate(zip(self.parts, self.m_parts)):
            assert torch.equal(x.cpu(), m), f"{what}: part {i}"

    def counts_match(self):
        """The calls' promise: a page's count is how many rows' entries hold it."""
        want = [0] * self.n_pages
        for r in range(self.n_rows):
            for p in self.m_table[r][:self.pages(self.m_lens[r])]:
                want[p] += 1
        return want == self.m_refs


def test_a_search(ctx):  # noqa: F811
    """Prompts, beams that fork, go on in each other's places, grow by tokens and end."""
    p = Pool(200, 12, 20, seed=2)
    for step in [lambda: p.grow(ctx, [0, 1], [37, 64]), lambda: p.fork(ctx, [0, 0, 0, 1, 1], [2, 3, 4, 5, 6]), lambda: p.grow(ctx, [0, 2, 3, 4, 1, 5, 6], [38] * 4 + [65] * 3),
                 lambda: p.fork(ctx, [2, 0, 2, 4], [0, 2, 3, 4]), lambda: p.grow(ctx, [0, 2, 3, 4], [48, 49, 60, 10]), lambda: p.fork(ctx, [5, 6, 1], [6, 1, 5]),
                 lambda: p.free(ctx, [1, 3]), lambda: p.fork(ctx, [0, 5], [11, 7])]:
        missing = step()
        p.check("search", missing)
        assert p.counts_match()
    p.check("compact", p.compact(ctx))
    assert p.counts_match() and all(n > 0 for n in p.m_refs[:int(p.result)])
    p.check("compact again", p.compact(ctx))


def test_rows_that_are_cut_inside_a_shared_page(ctx):  # noqa: F811
    """Tokens taken back behind a fork: the row shares the page that it was cut in until it is forked onto itself."""
    p = Pool(30, 6, 8, seed=11)
    for step in [lambda: p.grow(ctx, [0], [64]), lambda: p.fork(ctx, [0, 0, 0], [1, 2, 3]), lambda: p.grow(ctx, [1, 2, 3], [41, 48, 60])]:
        p.check("shared", step())
    assert p.m_table[1][2] == p.m_table[0][2] == p.m_table[2][2] and p.m_table[3][3] == p.m_table[0][3]
    p.check("own", p.fork(ctx, [1, 2, 3, 0, 4], [1, 2, 3, 0, 4]))
    assert p.m_table[1][2] != p.m_table[0][2] and p.m_table[2][2] == p.m_table[0][2] and p.m_table[3][3] != p.m_table[0][3] and p.counts_match()
    held = p.table.clone()
    p.check("own already", p.fork(ctx, [1, 3], [1, 3]))
    assert torch.equal(held, p.table)
    # the last two that hold a page, both forked; one forked onto itself and into another row; too few pages
    for step in [lambda: p.grow(ctx, [4], [16]), lambda: p.fork(ctx, [4], [5]), lambda: p.grow(ctx, [4, 5], [9, 5]), lambda: p.fork(ctx, [4, 5], [4, 5]),
                 lambda: p.fork(ctx, [4], [5]), lambda: p.grow(ctx, [4, 5], [16, 16]), lambda: p.fork(ctx, [4], [5]), lambda: p.grow(ctx, [4], [3]),
                 lambda: p.fork(ctx, [4, 4], [4, 1]), lambda: p.grow(ctx, [1, 4], [16 * (2 + sum(n == 0 for n in p.m_refs)), 16]), lambda: p.fork(ctx, [1], [4]),
                 lambda: p.grow(ctx, [1], [10]), lambda: p.grow(ctx, [4], [12])]:
        p.check("again", step())
        assert p.counts_match()


@pytest.mark.parametrize("parts", [(), ((1, torch.uint8),), ((7, torch.uint8), (6, torch.uint8)), (((2, 16, 64), torch.bfloat16),) * 3,
                                   (((2, 5000), torch.float32), (8, torch.bfloat16), (16385, torch.uint8)), ((2, torch.bfloat16),) * 150],
                         ids=["none", "a byte", "odd", "keys and values", "long", "150 parts"])
def test_parts_of_every_kind(ctx, parts):  # noqa: F811
    p = Pool(60, 6, 8, parts=parts, seed=3)
    p.check("grow", p.grow(ctx, [3, 0, 5], [33, 100, 16]))
    p.check("fork", p.fork(ctx, [3, 0, 5, 0], [1, 2, 4, 5]))
    p.free(ctx, [3, 0])
    p.check("free")
    p.check("compact", p.compact(ctx))
    if parts:
        p.copy(ctx, [0, 59, 3, 7, -1, 60, 5], [50, 51, 52, 7, 53, 54, 1 << 30])
        p.check("copy")


def test_random_steps(ctx):  # noqa: F811
    """Calls of every kind, rows out of range and listed twice among them, in pools that run out of pages."""
    import random
    for seed in range(6):
        r = random.Random(seed)
        p = Pool(r.choice([9, 40, 300, 2500]), r.choice([1, 5, 40]), r.choice([1, 7, 40]), page_size=r.choice([8, 16, 64]), seed=seed)
        row = lambda: r.randint(-1, p.n_rows)  # noqa: E731
        for _ in range(25):
            kind, n = r.choice(["fork", "fork", "grow", "grow", "grow", "free", "compact"]), r.choice([1, 2, 3, 20])
            if kind == "fork":
                p.check(f"{seed} fork", p.fork(ctx, [row() for _ in range(n)], [row() for _ in range(n)]))
            elif kind == "grow":
                p.check(f"{seed} grow", p.grow(ctx, [row() for _ in range(n)], [r.randint(-5, p.stride * p.page_size + 50) for _ in range(n)]))
            elif kind == "free":
                p.free(ctx, [row() for _ in range(n)])
                p.check(f"{seed} free")
            else:
                p.check(f"{seed} compact", p.compact(ctx))
            assert p.counts_match(), seed


def test_too_few_pages_change_nothing(ctx):  # noqa: F811
    p = Pool(10, 8, 9, seed=4)
    p.check("grow", p.grow(ctx, [0, 1], [5 * 16, 3 * 16 - 1]))
    assert p.grow(ctx, [2, 3], [33, 16]) == 2
    p.check("too long", 2)
    p.check("fork", p.fork(ctx, [1, 1], [2, 3]))
    assert p.fork(ctx, [1, 0, 1], [4, 5, 6]) == 2
    p.check("no page for the last parts", 2)
    p.check("full pages only", p.fork(ctx, [0], [5]))
    assert p.grow(ctx, [5, 6, 7], [1 << 30, 2147483647, -(1 << 31)]) == 13
    p.check("far too long", 13)
    p.check("shorter", p.grow(ctx, [0, 5], [0, 17]))


def test_pages_in_use_by_their_thousands(ctx):  # noqa: F811
    """More entries, rows and pages than a workgroup has threads, lists that end within four pages."""
    p = Pool(9001, 1500, 8, parts=((2, torch.float32),), seed=5)
    rows = list(range(0, 1500, 2)) + list(range(1, 1500, 2))
    p.check("grow", p.grow(ctx, rows, [1 + (i * 37) % 100 for i in range(1500)]))
    p.free(ctx, list(range(0, 1500, 3)))
    p.check("free")
    p.check("fork", p.fork(ctx, [1 + 3 * (i % 400) for i in range(500)], [3 * i for i in range(500)]))
    p.free(ctx, list(range(1, 1500, 3)) + [1, 4, 4])
    p.check("free")
    p.check("compact", p.compact(ctx))
    assert p.counts_match()
    n = 1200
    p.check("many entries of few rows", p.fork(ctx, [(7 * i) % 1500 for i in range(n)], [i % 3 for i in range(n)]))
    assert p.counts_match()


def test_more_rows_than_are_marked_in_lds(ctx):  # noqa: F811
    """Entries of one row among few and many entries, in tables of some thousand rows; rows that change by many pages beside those by one."""
    p = Pool(6000, 5000, 60, parts=((2, torch.float32),), seed=10)
    p.check("grow", p.grow(ctx, [4999, 3, 4999, 7, 3], [5, 900, 40, 16, 33]))
    p.check("fork", p.fork(ctx, [4999, 3, 7, 3], [8, 4500, 8, 9]))
    rows = [(13 * i) % 5000 for i in range(1100)] + [(13 * i) % 5000 for i in range(50)]
    p.check("grow many", p.grow(ctx, rows, [1 + i % 70 for i in range(1150)]))
    p.check("fork many", p.fork(ctx, rows, [(13 * i + 1) % 5000 for i in range(1150)]))
    p.free(ctx, rows[:600])
    p.check("free")
    p.check("compact", p.compact(ctx))
    assert p.counts_match()
    p.check("grow in LDS", p.grow(ctx, list(range(0, 1000)), [(i * 7) % 40 for i in range(1000)]))
    p.check("long rows", p.grow(ctx, [4000, 4001, 4002], [960, 1, 500]))
    p.check("short again", p.grow(ctx, [4000, 4001, 4002], [1, 960, 0]))
    assert p.counts_match()


def test_tables_that_hold_no_pages(ctx):  # noqa: F811
    """Entries out of range are not counted, not followed and not copied; lengths are cut to what a row can have."""
    p = Pool(50, 6, 6, seed=6)
    p.grow(ctx, [0, 1, 2], [90, 40, 33])
    for r, j, v in ((0, 2, -5), (1, 2, 1 << 30), (2, 0, 50)):
        p.m_refs[p.m_table[r][j]] -= 1
        p.m_table[r][j] = v
        p.table[r, j] = v
    p.refs.copy_(_int32(p.m_refs))
    p.check("fork", p.fork(ctx, [0, 1, 2], [3, 4, 5]))
    p.check("compact", p.compact(ctx))
    p.free(ctx, [1, 4])
    p.check("free")
    for r, n in ((3, 1 << 30), (5, -7)):
        p.m_lens[r] = n
        p.lens[r] = n
    p.check("fork of odd lengths", p.fork(ctx, [3, 5], [1, 2]))
    p.free(ctx, [3, 5])
    p.check("free")


def test_parts_behind_32_bit_offsets(ctx):  # noqa: F811
    part = torch.zeros((70000, 65536), dtype=torch.uint8, device=DEV)           # 4.3 GiB
    refs, table, lens = torch.zeros(70000, dtype=torch.int32, device=DEV), torch.full((4, 4), -1, dtype=torch.int32, device=DEV), _int32([0] * 4)
    pool, result = B.page_pool(refs, table, lens, 16, [part]), _int32([0])
    refs.fill_(1)
    refs[69990:] = 0
    part[69990:] = torch.arange(10, dtype=torch.uint8, device=DEV)[:, None]
    ctx.ensure_pages_workspace(pool, 4)
    ctx.pages_grow(pool, _int32([0]), _int32([40]), result)
    part[69992, 5:9] = 77
    ctx.pages_fork(pool, _int32([0]), _int32([1]), result)
    assert table[:2].tolist() == [[69990, 69991, 69992, -1], [69990, 69991, 69993, -1]] and int(result) == 0
    assert torch.equal(part[69993], part[69992]) and int(part[69993, 5]) == 77
    ctx.pages_copy(pool, _int32([69992]), _int32([69999]))
    assert torch.equal(part[69999], part[69992])
    refs[:3] = 0
    refs[3] = 7
    ctx.pages_compact(pool, result)
    # pages 0 to 2 are free, 3 to 69993 in use: the last three go to the first three
    assert int(result) == 69991 and table[:2].tolist() == [[69990, 0, 1, -1], [69990, 0, 2, -1]]
    assert int(part[0, 0]) == 1 and int(part[1, 5]) == 77


def test_a_pool_under_a_cache_in_8_bits(ctx):  # noqa: F811
    """A sequence forked in two; both get a token of their own, and attention sees each its own."""
    h = B.Attention(8, 2, 64, True, 0, 0.125)
    gen, n_pages, ps = _gen(7), 30, 16
    codes = [torch.zeros((n_pages, 2, ps, 64), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.ones((n_pages, 2, 2), device=DEV) for _ in range(2)]
    refs, table, lens = torch.zeros(n_pages, dtype=torch.int32, device=DEV), torch.full((3, 8), -1, dtype=torch.int32, device=DEV), _int32([0] * 3)
    pool, missing = B.page_pool(refs, table, lens, ps, codes + scales), _int32([0])
    cache = B.paged_cache8(*codes, *scales)
    ctx.ensure_pages_workspace(pool, 3)
    ctx.ensure_attention_workspace(h, 64, 3)
    k, v = (torch.randn((43, 128), device=DEV, generator=gen).to(torch.bfloat16) for _ in range(2))
    ctx.pages_grow(pool, _int32([0]), _int32([40]), missing)
    ctx.cache8_append(h, k[:40], v[:40], _int32([0, 40, 40, 40]), lens, cache, table)
    ctx.pages_fork(pool, _int32([0, 0]), _int32([2, 1]), missing)
    ctx.pages_grow(pool, _int32([0, 1, 2]), _int32([41, 41, 41]), missing)
    ctx.cache8_append(h, k[40:], v[40:], _int32([0, 1, 2, 3]), lens, cache, table)
    q = torch.randn((3, 512), device=DEV, generator=gen).to(torch.bfloat16)
    o = torch.empty_like(q)
    ctx.chunk_attention8(h, q, _int32([0, 1, 2, 3]), lens, 1, cache, table, o)
    from test_gpu_attention import _check, _reference
    from test_gpu_cache8 import _decode
    for r in range(3):
        page = table[r, :3].long()
        kk, vv = (_decode(c.view(torch.uint8)[page], s[page]).transpose(1, 2).reshape(-1, 2, 64)[:41] for c, s in zip(codes, scales))
        rows = torch.cat([torch.arange(40), torch.tensor([40 + r])]).to(DEV)
        for got, want in ((kk, k), (vv, v)):
            assert bool(((got - want[rows].double().reshape(41, 2, 64)).abs() <= 2.0 ** -4 * want[rows].double().reshape(41, 2, 64).abs() + 2.0 ** -14).all())
        _check(o[r:r + 1], None, _reference(h, q[r:r + 1].unflatten(1, (-1, 64)), kk, vv), 64, 41, f"row {r}")
    assert refs.tolist()[:6] == [3, 3, 1, 1, 1, 0]


def test_captured_steps():
    """A step of a search captured once and replayed on other rows and lengths, with eager calls between."""
    stream = torch.cuda.Stream()
    ctx = B.Context(0, stream)  # noqa: F811
    try:
        p = Pool(400, 10, 30, seed=8)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            p.check("grow", p.grow(ctx, [0, 1, 2], [33, 90, 64]))
        src, dst, rows, lens, ended = _int32([0, 1]), _int32([3, 4]), _int32([0, 3]), _int32([50, 60]), _int32([9])
        graph = torch.cuda.CUDAGraph()
        ctx.ensure_pages_workspace(p.pool, 4)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            ctx.pages_fork(p.pool, src, dst, p.result)
            ctx.pages_grow(p.pool, rows, lens, p.result)
            ctx.pages_free(p.pool, ended)
            ctx.pages_compact(p.pool, p.result)

        class Host:
            """Takes the calls that the graph makes."""
            def __getattr__(self, name):
                return lambda *a: None
        for rep, (a, b, r, n, e) in enumerate((([0, 1], [3, 4], [0, 3], [50, 60], [9]), ([3, 4], [0, 1], [1, 2], [200, 3], [4]), ([1, 1], [5, 5], [5, 0], [77, 0], [2]))):
            for x, y in ((src, a), (dst, b), (rows, r), (lens, n), (ended, e)):
                x.copy_(_int32(y))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            p.fork(Host(), a, b)
            p.grow(Host(), r, n)
            p.free(Host(), e)
            p.check(f"replay {rep}", p.compact(Host()))
            with torch.cuda.stream(stream):
                p.check(f"eager {rep}", p.fork(ctx, [0], [8]))
            torch.cuda.synchronize()
    finally:
        torch.cuda.synchronize()
        ctx.close()


def test_refusals(ctx):  # noqa: F811
    p = Pool(20, 4, 5, seed=9)
    p.check("grow", p.grow(ctx, [0, 1], [20, 40]))
    one, two = _int32([0]), _int32([1])
    calls = (lambda q: ctx.pages_fork(q, one, two, p.result), lambda q: ctx.pages_grow(q, one, two, p.result), lambda q: ctx.pages_free(q, one),
             lambda q: ctx.pages_compact(q, p.result), lambda q: B.pages_workspace_bytes(q, 1))
    for field, value, status in (("n_pages", 0, 2), ("n_pages", 1 << 29, 2), ("page_size", 12, 2), ("page_size", 4, 2), ("n_rows", 0, 2), ("table_stride", 0, 2),
                                 ("table_stride", 1 << 21, 2), ("n_parts", -1, 2), ("n_parts", 5000, 2), ("refs", None, 1), ("page_table", None, 1), ("lens", None, 1),
                                 ("refs", p.pool.refs + 4, 3)):
        for call in calls:
            bad = B.PagePool(*(getattr(p.pool, n) for n, _ in p.pool._fields_))
            setattr(bad, field, value)
            _refused(status, call, bad)
    for data, size, status in ((None, 16, 1), (p.parts[0].data_ptr() + 8, 16, 3), (p.parts[0].data_ptr(), 0, 2), (p.parts[0].data_ptr(), (1 << 32) + 1, 2)):
        bad = B.PagePool(*(getattr(p.pool, n) for n, _ in p.pool._fields_))
        bad.parts, bad.n_parts = (B.PagePart * 1)(B.PagePart(data, size)), 1
        for call in calls + (lambda q: ctx.pages_copy(q, one, two),):
            _refused(status, call, bad)
    bad = B.PagePool(*(getattr(p.pool, n) for n, _ in p.pool._fields_))
    bad.n_parts = 0
    _refused(1, ctx.pages_copy, bad, one, two)
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    for call in (lambda: ctx.pages_fork(p.pool, none, none, p.result), lambda: ctx.pages_free(p.pool, none)):
        with pytest.raises(B.FFError):
            call()
    lib = ctx.lib
    assert lib.ff_pages_fork(ctx._h, p.pool, 1, one.data_ptr(), two.data_ptr(), None) == 1
    assert lib.ff_pages_compact(ctx._h, p.pool, None) == 1
    for bad in (lambda: B.page_pool(p.refs, p.table, p.lens, 16, [p.parts[0][:-1]]), lambda: B.page_pool(p.refs, p.table, p.lens[:-1], 16, []),
                lambda: ctx.pages_fork(p.pool, one, _int32([1, 2]), p.result), lambda: ctx.pages_grow(p.pool, one, one.long(), p.result)):
        with pytest.raises(AssertionError):
            bad()
    fresh = B.Context(0)
    try:
        _refused(5, fresh.pages_fork, p.pool, one, two, p.result)
        _refused(5, fresh.pages_compact, p.pool, p.result)
        fresh.pages_free(p.pool, _int32([3]))                     # needs none
        torch.cuda.synchronize()
    finally:
        fresh.close()
    p.check("after refusals")


def _room(pool, n):
    """What grow asks for with n entries, and compact with 1."""
    return 4 * max(pool.n_rows + 3 * n + 64, pool.n_pages + pool.n_rows + 2 * n + 65, 3 * pool.n_pages + 64)


@pytest.mark.parametrize("n_rows,stride,page_size", [(40, 300, 8), (5000, 70, 16)])
def test_calls_that_keep_no_rows_need_no_room_for_them(ctx, n_rows, stride, page_size):  # noqa: F811
    """Exactly what the header says is enough for each call, nothing behind it is written, and a byte less is refused."""
    p = Pool(3000, n_rows, stride, page_size=page_size, seed=12)
    n = 300
    most = B.pages_workspace_bytes(p.pool, n)
    buf = torch.full((most + 4096,), 0x5a, dtype=torch.uint8, device=DEV)
    need = {"grow": _room(p.pool, n), "fork": most, "compact": _room(p.pool, 1)}
    assert max(need["grow"], need["compact"]) < most
    own = B.Context(0)  # noqa: F811
    try:
        own.ensure_pages_workspace = lambda pool, entries: None
        rows = [(i * 7) % n_rows for i in range(n)]
        for name, call in (("grow", lambda: p.grow(own, rows, [1 + (i * 31) % 140 for i in range(n)])),
                           ("fork", lambda: p.fork(own, rows, [(r + 1) % n_rows for r in rows])),
                           ("compact", lambda: p.compact(own))):
            size = need[name]
            own.set_workspace(buf[:size - 1])
            one = _int32([0] * n)
            _refused(5, *((own.pages_compact, p.pool, p.result) if name == "compact" else (getattr(own, "pages_" + name), p.pool, one, one, p.result)))
            p.check("refused")
            buf.fill_(0x5a)
            own.set_workspace(buf[:size])
            p.check(name, call())
            assert bool((buf[size:] == 0x5a).all()), f"{name} wrote behind its workspace"
            assert p.counts_match()
    finally:
        torch.cuda.synchronize()
        own.close()


def test_a_pool_at_the_limits_grows(ctx):  # noqa: F811
    """Entries and tables for which a fork would take tebibytes: the calls that keep no rows are not refused."""
    stride, n = 1 << 20, 1 << 20
    refs, lens = torch.zeros(64, dtype=torch.int32, device=DEV), _int32([0] * 4)
    table = torch.full((4, stride), -1, dtype=torch.int32, device=DEV)
    pool, missing = B.page_pool(refs, table, lens, 16, []), _int32([-1])
    rows = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    rows[77], rows[n - 1] = 2, 3
    new = torch.full((n,), 40, dtype=torch.int32, device=DEV)
    own = B.Context(0)  # noqa: F811
    try:
        assert B.pages_workspace_bytes(pool, n) > 1 << 42
        own.set_workspace(torch.zeros(_room(pool, n), dtype=torch.uint8, device=DEV))
        own.pages_grow(pool, rows, new, missing)
        assert int(missing) == 0 and lens.tolist() == [0, 0, 40, 40] and table[2:, :4].tolist() == [[0, 1, 2, -1], [3, 4, 5, -1]]
        _refused(5, own.pages_fork, pool, rows, new, missing)
        own.pages_free(pool, _int32([2]))
        own.pages_compact(pool, missing)
        assert int(missing) == 3 and table[3, :4].tolist() == [0, 1, 2, -1] and refs[:4].tolist() == [1, 1, 1, 0]
    finally:
        torch.cuda.synchronize()
        own.close()


@pytest.mark.parametrize("page_size", [0, -1, -(1 << 31), 24, (1 << 30) + 1, (1 << 31) - 1])
def test_copies_of_pages_of_any_size(ctx, page_size):  # noqa: F811
    """A copy takes the parts alone: what else the pool says does not matter to it."""
    p = Pool(20, 2, 3, seed=13)
    p.pool.page_size, p.pool.n_rows, p.pool.table_stride, p.pool.refs, p.pool.page_table, p.pool.lens = page_size, 0, -1, None, None, None
    p.copy(ctx, [3, 0, 19, 7], [4, 1, 18, 7])
    p.check(f"pages of {page_size}")


def test_the_validate_option(ctx):  # noqa: F811
    """Lengths that a row cannot have are refused before anything is changed; rows that are not there are passed over."""
    p = Pool(40, 5, 6, seed=14)
    ctx.ensure_pages_workspace(p.pool, 300)
    ctx.set_option("validate", 1)
    try:
        p.check("grow", p.grow(ctx, [0, 1, -1, 5], [96, 3, 1 << 30, -1]))
        for rows, lens in (([0, 1, 2], [96, 97, 5]), ([3], [-1]), ([3], [2147483647]), (list(range(-295, 5)), [7] * 299 + [97])):
            _refused(4, ctx.pages_grow, p.pool, _int32(rows), _int32(lens), p.result)
            p.check("refused")
        p.check("fork", p.fork(ctx, [0, 1], [2, 3]))
        p.check("longest", p.grow(ctx, [0, 1, 2, 3], [96, 96, 0, 96]))
    finally:
        ctx.set_option("validate", 0)
    p.check("cut", p.grow(ctx, [4], [97]))
