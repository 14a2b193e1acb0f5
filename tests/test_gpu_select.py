"""Attention over selected pages: means of pages to the bit, the choice of pages against a model in float64 (equal lists), and
attention over the lists against softmax(scale q k^T) v in float64.

A mean is a float64 sum of at most 4096 bf16 numbers of a few powers of two, which is exact, divided and rounded once: no bar.  A
score is a float64 sum of some hundred products, off by 2^-45 of their size at most; the scores of random pages lie further
apart, and those of equal pages are equal because their sums run alike.  Attention's bars are those of test_gpu_attention."""
import math

import pytest
import torch

from paper_2602_00397_amd import binding as B
from test_gpu_attention import DEV, H1B, H7B, H8B, MHA, MQA, TINY, _bf16, _check, _clamped, _gen, _heads, _int32, _reference, _refused, _starts, ctx  # noqa: F401
from test_gpu_cache8 import Cache8, _decode

pytestmark = pytest.mark.gpu


class Cache16:
    """Sequences' keys and values in bf16 pages in shuffled order; places without a key are NaN."""

    def __init__(self, h, lens, page_size, gen, far=0):
        self.h, self.lens, self.page_size = h, lens, page_size
        used = [-(-n // page_size) for n in lens]
        n_pages = sum(used) + 3 + far
        self.k_pages, self.v_pages = (torch.full((n_pages, h.n_kv_heads, page_size, h.head_dim), math.nan, dtype=torch.bfloat16, device=DEV)
                                      for _ in range(2))
        order = (torch.randperm(n_pages - far, device=DEV, generator=gen) + far).to(torch.int32)
        self.table = torch.full((len(lens), max(used + [1]) + 1), -1, dtype=torch.int32, device=DEV)
        at = 0
        for i, n in enumerate(lens):
            self.table[i, :used[i]] = order[at:at + used[i]]
            at += used[i]
            j = torch.arange(n, device=DEV)
            for pages in (self.k_pages, self.v_pages):
                pages[self.table[i].long()[j // page_size], :, j % page_size] = _bf16(gen, n, h.n_kv_heads, h.head_dim)
        self.cache = B.paged_cache(self.k_pages, self.v_pages)

    def values(self, which, pages):
        """All places of these pages, float64."""
        return (self.k_pages if which == "k" else self.v_pages)[pages].double()


class Cache8Values(Cache8):
    def values(self, which, pages):
        codes, scale = (self.k_pages, self.k_scale) if which == "k" else (self.v_pages, self.v_scale)
        return _decode(codes.view(torch.uint8)[pages], scale[pages])


class Step:
    """A layer's step over selected pages."""

    def __init__(self, h, new, lens, query_block, keep, first=1, page_size=16, eight=False, seed=1, behind=0, far=0):
        gen = _gen(seed)
        self.c = Cache8Values(h, lens, page_size, 8, gen, far) if eight else Cache16(h, lens, page_size, gen, far)
        self.h, self.new, self.sel = h, new, B.selection(query_block, keep, first)
        t, self.n_pages = sum(new) + behind, self.c.k_pages.shape[0]
        self.q = _bf16(gen, t, h.n_heads * h.head_dim)
        self.starts, self.lens, self.table = _int32(_starts(new)), _int32(lens), self.c.table
        self.means = torch.full((self.n_pages, h.n_kv_heads, h.head_dim), 5.0, device=DEV)
        self.n_blocks, self.width = B.selection_blocks(self.sel, t, len(new)), B.selection_pages(self.sel, page_size)
        self.block_starts, self.block_lens = _int32([-9] * (self.n_blocks + 1)), _int32([-9] * self.n_blocks)
        self.tables = torch.full((self.n_blocks, h.n_kv_heads, self.width), -9, dtype=torch.int32, device=DEV)
        self.o = torch.full((t, h.n_heads * h.head_dim), 7.0, dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((t, h.n_heads), 7.0, device=DEV)

    def all_means(self):
        """As calls for the earlier tokens would have left them."""
        for i, n in enumerate(self.c.lens):
            for j in range(0, n, self.c.page_size):
                page = int(self.table[i, j // self.c.page_size])
                if 0 <= page < self.n_pages:
                    self.means[page] = self.c.values("k", page)[:, :min(self.c.page_size, n - j)].mean(dim=1).float()

    def update(self, ctx):
        ctx.page_means(self.h, self.q.shape[0], self.starts, self.lens, self.c.cache, self.table, self.means)

    def select(self, ctx):
        ctx.ensure_selection_workspace(self.h, self.n_blocks, self.table.shape[1])
        ctx.select_pages(self.h, self.sel, self.q, self.starts, self.lens, self.c.page_size, self.means, self.table, self.block_starts,
                         self.block_lens, self.tables)

    def attend(self, ctx):
        ctx.ensure_attention_workspace(self.h, self.q.shape[0], self.n_blocks)
        ctx.selected_attention(self.h, self.q, self.block_starts, self.block_lens, max(1, min(self.sel.query_block, max(self.new))), self.c.cache,
                               self.tables, self.o, lse=self.lse)

    def run(self, ctx):
        self.update(ctx)
        self.select(ctx)
        self.attend(ctx)

    def model(self):
        """The block arrays, from the definition."""
        ps, h, qb, t = self.c.page_size, self.h, self.sel.query_block, self.q.shape[0]
        q = self.q.double().reshape(t, h.n_kv_heads, -1, h.head_dim).sum(dim=2)
        starts, lens = self.starts.tolist(), self.lens.tolist()
        table = self.table.tolist()
        b_starts, b_lens, b_tables = [], [], []
        for s in range(len(lens)):
            t0, t1 = _clamped(starts, s, t)
            keys = min(max(lens[s], 0), self.table.shape[1] * ps)
            for a in range(t0, t1, qb):
                b = min(t1, a + qb)
                last = keys - (t1 - b) - 1
                b_starts.append(a)
                if last < 0:
                    b_lens.append(0)
                    b_tables.append([[-1] * self.width] * h.n_kv_heads)
                    continue
                earlier = max(0, last - (b - a) + 1) // ps
                kept = min(earlier, self.sel.keep)
                own = table[s][earlier:last // ps + 1]
                b_lens.append((kept + len(own) - 1) * ps + last % ps + 1)
                pages = torch.tensor([p if 0 <= p < self.n_pages else 0 for p in table[s][:earlier]], dtype=torch.long, device=DEV)
                rows = []
                for g in range(h.n_kv_heads):
                    score = (self.means[pages, g].double() * q[a:b, g].sum(dim=0)).sum(dim=1)
                    score[:self.sel.first] = math.inf
                    best = sorted(sorted(range(earlier), key=lambda i, x=score.tolist(): (-x[i], i))[:kept])
                    rows.append([table[s][i] for i in best] + own + [-1] * (self.width - kept - len(own)))
                b_tables.append(rows)
        end = _clamped(starts + [1 << 40], len(lens), t)[0]
        b_starts += [end] * (self.n_blocks + 1 - len(b_starts))
        b_tables += [[[-1] * self.width] * h.n_kv_heads] * (self.n_blocks - len(b_lens))
        b_lens += [0] * (self.n_blocks - len(b_lens))
        return b_starts, b_lens, b_tables

    def check_selection(self, what):
        starts, lens, tables = self.model()
        assert self.block_starts.tolist() == starts, f"{what}: block starts"
        assert self.block_lens.tolist() == lens, f"{what}: block lengths"
        got = self.tables.tolist()
        for b in range(self.n_blocks):
            assert got[b] == tables[b], f"{what}: pages of block {b}"

    def check_attention(self, what):
        h, hd, ps = self.h, self.h.head_dim, self.c.page_size
        group = h.n_heads // h.n_kv_heads
        one = B.Attention(group, 1, hd, True, 0, h.scale)
        starts, lens = self.block_starts.tolist(), self.block_lens.tolist()
        left = torch.ones(self.q.shape[0], dtype=torch.bool, device=DEV)
        for b in range(self.n_blocks):
            a, e = starts[b], starts[b + 1]
            if a == e:
                continue
            left[a:e] = False
            refs = []
            for g in range(h.n_kv_heads):
                pages = self.tables[b, g, :-(-lens[b] // ps)].long()
                k, v = (self.c.values(x, pages)[:, g].reshape(-1, 1, hd)[:lens[b]] for x in ("k", "v"))
                refs.append(_reference(one, self.q[a:e].reshape(e - a, h.n_heads, hd)[:, g * group:(g + 1) * group], k, v))
            ref = [torch.cat([r[i] for r in refs], dim=1) for i in range(4)]
            _check(self.o[a:e], self.lse[a:e], ref, hd, lens[b], f"{what}, block {b}: {e - a} over {lens[b]}")
        assert bool((self.o[left] == 7.0).all()) and bool((self.lse[left] == 7.0).all()), f"{what}: rows of no block"

    def check(self, what):
        self.check_selection(what)
        self.check_attention(what)


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "8 bits"])
@pytest.mark.parametrize("h", [H8B, H7B, H1B, TINY, MHA, MQA], ids=lambda h: "%d_%d_%d" % h)
def test_means_of_the_pages_with_new_tokens(ctx, h, eight):  # noqa: F811
    for ps in (16, 64, 256):
        s = Step(_heads(h), [1, 0, 33, 300, 1, 5], [700, 20, 33, 900, 1, 260], 1, 1, page_size=ps, eight=eight, behind=2)
        want = s.means.clone()
        for i, (n, keys) in enumerate(zip(s.new, s.c.lens)):
            for j in range((keys - n) // ps, -(-keys // ps) if n else 0):
                page = int(s.table[i, j])
                want[page] = s.c.values("k", page)[:, :min(ps, keys - j * ps)].mean(dim=1).float()
        s.update(ctx)
        assert torch.equal(s.means, want), f"{h} pages of {ps}"


@pytest.mark.parametrize("n_seqs", [64, 65, 300, 4100])
@pytest.mark.parametrize("most", [1, 40])
def test_means_of_many_ragged_sequences(ctx, n_seqs, most):  # noqa: F811
    """One call against calls of 50 sequences, to the bit, with empty sequences throughout."""
    new = [(i * i * 7 + i // 64) % (most + 1) for i in range(n_seqs)]
    s = Step(_heads(TINY), new, [n + (37 * i) % 30 for i, n in enumerate(new)], 1, 1, page_size=16, behind=2)
    s.starts += 1                                  # (a row in front of the first sequence's)
    before = s.means.clone()
    for a in range(0, n_seqs, 50):
        e = min(n_seqs, a + 50)
        ctx.page_means(s.h, s.q.shape[0], s.starts[a:e + 1].clone(), s.lens[a:e].clone(), s.c.cache, s.table[a:e].clone(), s.means)
    want = s.means.clone()
    s.means.copy_(before)
    s.update(ctx)
    assert torch.equal(s.means, want) and not torch.equal(want, before)


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "8 bits"])
@pytest.mark.parametrize("h", [H8B, H7B, H1B, TINY, MHA, MQA], ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("query_block,keep,first", [(1, 4, 1), (16, 8, 0), (7, 3, 3), (64, 1, 0), (200, 40, 2)])
def test_steps(ctx, h, query_block, keep, first, eight):  # noqa: F811
    for new, lens in (([1] * 4, [700, 1, 333, 16]), ([300], [1000]), ([1, 90, 0, 40, 7], [500, 90, 40, 777, 650])):
        s = Step(_heads(h), new, lens, query_block, keep, first, eight=eight, seed=len(new), behind=3)
        s.all_means()
        s.run(ctx)
        s.check(f"{h} {new} over {lens}")


@pytest.mark.parametrize("page_size", [8, 16, 64, 128, 4096])
def test_page_sizes(ctx, page_size):  # noqa: F811
    for query_block in (1, 30, 128):
        s = Step(_heads(H8B), [1, 130, 5], [2000, 600, 77], query_block, 2, 0, page_size=page_size, seed=3)
        s.all_means()
        s.run(ctx)
        s.check(f"pages of {page_size}, blocks of {query_block}")


@pytest.mark.parametrize("keep", [1, 5, 64, 1000, 3000])
def test_long_contexts(ctx, keep):  # noqa: F811
    """Numbers in LDS and made again, pages shared out among workgroups."""
    for h, lens, new in ((TINY, [100000], [1]), (TINY, [30000, 66000], [3, 40]), (H8B, [20000, 500, 9000], [1, 1, 1])):
        s = Step(_heads(h), new, lens, 16, keep, min(keep, 4), seed=4)
        s.means.normal_(generator=_gen(5))
        s.update(ctx)
        s.select(ctx)
        s.check_selection(f"{h} {lens} keep {keep}")


def test_equal_scores_go_to_the_earlier_page(ctx):  # noqa: F811
    for n in (300, 5000):
        s = Step(_heads(TINY), [1, 9], [16 * n, 16 * n - 7], 4, 37, 2, seed=6)
        s.means.zero_()
        s.select(ctx)
        s.check_selection("all equal")
        s.means.copy_(torch.randint(0, 3, (s.n_pages, 1, 1), device=DEV, generator=_gen(7)).float().expand_as(s.means))
        s.q.copy_(torch.randint(-2, 3, s.q.shape, device=DEV, generator=_gen(8)).to(torch.bfloat16))
        s.select(ctx)
        s.check_selection("a few values")
        s.means *= -0.0
        s.select(ctx)
        s.check_selection("zeros of both signs")


def test_scores_far_apart(ctx):  # noqa: F811
    """Over hundreds of powers of two, of either sign, and with infinities: the order is the numbers'."""
    s = Step(_heads(TINY), [1, 3], [16 * 2500, 16 * 1800], 1, 100, 0, seed=9)
    gen = _gen(10)
    s.q.fill_(1.0)
    size = torch.exp2(torch.randint(-60, 61, (s.n_pages, 2, 1), device=DEV, generator=gen).float())
    sign = torch.randint(0, 2, (s.n_pages, 2, 1), device=DEV, generator=gen).float() * 2 - 1
    s.means.copy_((size * sign).expand_as(s.means))
    s.select(ctx)
    s.check_selection("far apart")
    used = s.table[0, :2500].long()
    s.means[used[:60]] = math.inf
    s.means[used[100:2490]] = -math.inf
    s.select(ctx)
    s.check_selection("infinities")
    s.means[used[5]] = math.nan                       # ranks by its bits: lists stay within what there is
    s.means[used[200]] = -math.nan
    s.select(ctx)
    for row in s.tables[0].tolist():
        at = [s.table[0].tolist().index(p) for p in row[:101]]
        assert at == sorted(set(at)) and at[-1] == 2499 and row[101:] == [-1] * (s.width - 101)


def test_keeping_all_pages_is_attention_over_the_cache(ctx):  # noqa: F811
    for h, new, lens in ((H8B, [1, 1], [900, 2000]), (H8B, [200, 1], [900, 30]), (H1B, [70], [70])):
        s = Step(_heads(h), new, lens, 32, 200, 0, page_size=64, seed=11)
        s.run(ctx)                                    # (no score decides: means of earlier pages do not matter)
        s.check("all pages")
        t0 = 0
        for i, n in enumerate(new):
            page = s.table[i, :-(-lens[i] // 64)].long()
            k, v = (s.c.values(x, page).transpose(1, 2).reshape(-1, h[1], h[2])[:lens[i]] for x in ("k", "v"))
            _check(s.o[t0:t0 + n], s.lse[t0:t0 + n], _reference(s.h, s.q[t0:t0 + n].unflatten(1, (-1, h[2])), k, v), h[2], lens[i], f"{h} {new}")
            t0 += n


def test_fewer_keys_than_tokens_or_none(ctx):  # noqa: F811
    for qb in (1, 5, 64):
        s = Step(_heads(H8B), [12, 3, 40, 9], [0, 2, 33, 9], qb, 2, seed=12, behind=1)
        s.all_means()
        s.run(ctx)
        s.check(f"short contexts, blocks of {qb}")


def test_many_sequences_and_blocks(ctx):  # noqa: F811
    new = [i % 4 for i in range(150)]
    s = Step(_heads(TINY), new, [n + (53 * i) % 400 for i, n in enumerate(new)], 2, 5, seed=13)
    s.all_means()
    s.run(ctx)
    s.check("150 sequences")
    s = Step(_heads(TINY), [3000], [3000], 3, 4, seed=14)
    s.all_means()
    s.run(ctx)
    s.check_selection("1001 blocks")


def test_rows_apart(ctx):  # noqa: F811
    s = Step(_heads(H7B), [1, 50], [700, 300], 16, 4, seed=15)
    s.all_means()
    s.run(ctx)
    first = s.tables.clone(), s.o.clone()
    w = s.q.shape[1]
    wide = torch.zeros((s.q.shape[0], w + 24), dtype=torch.bfloat16, device=DEV)
    wide[:, 16:16 + w] = s.q
    s.q, s.tables = wide[:, 16:16 + w], s.tables.fill_(-9)
    out = torch.full((s.q.shape[0], w + 16), 7.0, dtype=torch.bfloat16, device=DEV)
    s.o = out[:, 8:8 + w]
    s.run(ctx)
    assert torch.equal(s.tables, first[0]) and torch.equal(s.o.contiguous().view(torch.int16), first[1].view(torch.int16))
    assert bool((out[:, :8] == 7.0).all()) and bool((out[:, 8 + w:] == 7.0).all())


@pytest.mark.parametrize("new", [[1, 1], [40, 70]], ids=str)
@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "8 bits"])
def test_what_is_out_of_range_is_clamped(ctx, new, eight):  # noqa: F811
    for what, change in (("page", lambda s: s.table[1, 0].fill_(1 << 30)), ("negative page", lambda s: s.table[1, 1].fill_(-5)),
                         ("length", lambda s: s.lens[0].fill_(1 << 30)), ("negative length", lambda s: s.lens[0].fill_(-3)),
                         ("end", lambda s: s.starts[2].fill_(1 << 30)), ("descending starts", lambda s: s.starts[1].fill_(-9)),
                         ("all behind", lambda s: s.starts.fill_(2147483647))):
        s = Step(_heads(H8B), new, [200, 180], 16, 3, eight=eight, behind=3, seed=16)
        if eight:
            for x in (s.c.k_pages, s.c.v_pages):
                codes = x.view(torch.uint8)
                codes[codes == 0x7f] = 0x30
            for x in (s.c.k_scale, s.c.v_scale):
                x.nan_to_num_(0.25)
        else:
            s.c.k_pages.nan_to_num_(0.5)
            s.c.v_pages.nan_to_num_(0.5)
        s.all_means()
        change(s)
        held = s.means.clone()
        s.update(ctx)
        touched = (s.means != held).flatten(1).any(dim=1).nonzero()[:, 0].tolist()
        assert set(touched) <= set(s.table.flatten().tolist()), what
        s.select(ctx)
        s.check_selection(what)
        s.attend(ctx)
        torch.cuda.synchronize()
        s.tables = torch.where((s.tables < 0) | (s.tables >= s.n_pages), 0, s.tables)
        s.check_attention(what)


def test_pages_behind_32_bit_offsets(ctx):  # noqa: F811
    """Means and keys of pages behind more than 4 GiB of each."""
    s = Step(_heads((8, 8, 128)), [1, 40], [900, 300], 16, 5, page_size=16, seed=17, far=1 << 20)
    assert int(s.table[0, 0]) * 8 * 128 * 4 >= 1 << 32
    s.all_means()
    s.run(ctx)
    s.check("far pages")


def test_captured_steps():
    """A step captured once, replayed while lengths, tables, queries and keys change, with eager calls between."""
    stream = torch.cuda.Stream()
    ctx = B.Context(0, stream)  # noqa: F811
    try:
        a = Step(_heads(H8B), [1, 1, 1], [900, 40, 2000], 1, 4, seed=18)
        b = Step(_heads(H8B), [90, 1, 37], [900, 700, 64], 16, 6, seed=19, eight=True)
        for s in (a, b):
            s.all_means()
        torch.cuda.synchronize()
        for s in (a, b):
            s.run(ctx)
        stream.synchronize()
        g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g1, stream=stream):
            a.run(ctx)
        with torch.cuda.graph(g2, stream=stream):
            b.run(ctx)
        gen = _gen(20)
        for rep in range(4):
            for s in (a, b):
                s.q.copy_(_bf16(gen, *s.q.shape))
                s.lens.copy_(_int32([max(1, n - 13 * rep) for n in s.c.lens]))
                s.o.fill_(7.0)
                s.lse.fill_(7.0)
            torch.cuda.synchronize()
            g1.replay()
            g2.replay()
            torch.cuda.synchronize()
            for s in (a, b):
                s.check(f"replay {rep}")
            tables = [s.tables.clone() for s in (a, b)]
            for s in (a, b):
                s.run(ctx)
            stream.synchronize()
            assert all(torch.equal(s.tables, t) for s, t in zip((a, b), tables))
    finally:
        torch.cuda.synchronize()
        ctx.close()


def test_refusals(ctx):  # noqa: F811
    s = Step(_heads(TINY), [3, 1], [400, 90], 2, 2)
    s.run(ctx)

    def select(h=None, sel=None, page_size=16, starts=None):
        ctx.select_pages(h or s.h, sel or s.sel, s.q, s.starts, s.lens, page_size, s.means, s.table, s.block_starts if starts is None else starts,
                         s.block_lens, s.tables)

    def attend(h=None, max_chunk=2, cache=None):
        ctx.selected_attention(h or s.h, s.q, s.block_starts, s.block_lens, max_chunk, cache or s.c.cache, s.tables, s.o)

    for qb, keep, first in ((0, 2, 0), (-1, 2, 0), (2, 0, 0), (2, 2, 3), (2, 2, -1), (1 << 21, 2, 0), (2, 1 << 21, 0)):
        if qb > 0 and keep > 0 and (qb > 1 << 20 or keep > 1 << 20):
            with pytest.raises(B.FFError):
                B.selection_blocks(B.selection(qb, keep, first), 4, 2)
            continue
        _refused(2, select, sel=B.selection(qb, keep, first))
    for page_size in (4, 12, 8192):
        s.tables = torch.empty((s.n_blocks, 2, 2 + (2 + page_size - 2) // page_size + 1), dtype=torch.int32, device=DEV)
        _refused(2, select, page_size=page_size)
    s.tables = torch.zeros((s.n_blocks, 2, s.width), dtype=torch.int32, device=DEV)
    s.run(ctx)
    for h in (_heads(TINY, causal=False), _heads(TINY, window=4)):
        _refused(1, select, h)
        _refused(1, attend, h)
    for max_chunk in (0, 5):
        _refused(1, attend, max_chunk=max_chunk)
    lib, null = ctx.lib, None
    args = (ctx._h, s.h, 4, 2, s.starts.data_ptr(), s.lens.data_ptr())
    tail = (s.table.data_ptr(), s.table.shape[1], s.means.data_ptr())
    assert lib.ff_page_means(*args, null, null, *tail) == 1                       # neither cache
    c8 = Cache8Values(s.h, [400, 90], 16, 8, _gen(2))
    assert lib.ff_page_means(*args, s.c.cache, c8.cache, *tail) == 1              # both
    assert lib.ff_page_means(*args, s.c.cache, null, *tail[:2], null) == 1
    for bad in (lambda: select(starts=s.block_starts[:-1]), lambda: select(sel=B.selection(2, 3)), lambda: select(_heads(H8B)),
                lambda: ctx.page_means(s.h, 4, s.starts, s.lens, s.c.cache, s.table, s.means[:-1])):
        with pytest.raises(AssertionError):
            bad()
    fresh = B.Context(0)
    try:
        with pytest.raises(B.FFError) as e:
            fresh.select_pages(s.h, s.sel, s.q, s.starts, s.lens, 16, s.means, s.table, s.block_starts, s.block_lens, s.tables)
        assert e.value.status == 5
    finally:
        torch.cuda.synchronize()
        fresh.close()
    ctx.set_option("validate", 1)
    try:
        s.attend(ctx)
        s.check("validated")
        s.tables[1, 1, 0] = 1 << 30
        _refused(4, s.attend, ctx)
    finally:
        ctx.set_option("validate", 0)


@pytest.mark.parametrize("n_seqs", [5, 70])
def test_means_behind_the_end_of_the_table(ctx, n_seqs):  # noqa: F811
    """New tokens that the table has no place for change no mean: only pages with tokens in front of its end are made anew."""
    over = [(1, 97), (5, 98), (40, 130), (3, 96), (9, (1 << 30) - 1)]
    new, lens = ([over[i % len(over)][j] for i in range(n_seqs)] for j in (0, 1))
    s = Step(_heads(TINY), new, [96] * n_seqs, 1, 1, page_size=16, seed=n_seqs)
    s.table = s.table[:, :6].contiguous()
    s.lens = _int32(lens)
    want = s.means.clone()
    for i in range(n_seqs):
        for j in range(max(0, min(lens[i] - new[i], 96)) // 16, 6 if lens[i] - new[i] < 96 else 0):
            page = int(s.table[i, j])
            want[page] = s.c.values("k", page).mean(dim=1).float()
    s.update(ctx)
    assert torch.equal(s.means, want)


def test_the_validate_option_of_means_and_selection(ctx):  # noqa: F811
    s = Step(_heads(TINY), [3, 20], [400, 90], 2, 2)
    s.all_means()
    s.run(ctx)
    most = s.table.shape[1] * 16
    ctx.set_option("validate", 1)
    try:
        for what, change in (("longer than the table", lambda: s.lens[0].fill_(most + 1)), ("negative length", lambda: s.lens[1].fill_(-1)),
                             ("end", lambda: s.starts[2].fill_(24)), ("descending starts", lambda: s.starts[1].fill_(-1))):
            starts, lens, means, tables = s.starts.clone(), s.lens.clone(), s.means.clone(), s.tables.clone()
            change()
            _refused(4, s.update, ctx)
            _refused(4, s.select, ctx)
            assert torch.equal(s.means, means) and torch.equal(s.tables, tables), what
            s.starts.copy_(starts)
            s.lens.copy_(lens)
        s.run(ctx)
        s.check("validated")
        s.table[1, 1] = -5                                      # (passed over by the means, scored as page 0, listed as it is)
        s.update(ctx)
        s.select(ctx)
        s.check_selection("a page out of range")
    finally:
        ctx.set_option("validate", 0)
