"""The calls on pages together, as a server makes them: prompts in blocks and generated tokens through a pool of pages with an 8-bit cache
and means, sequences forked, ended and compacted between, every step's selection and attention against float64."""
import pytest
import torch

from paper_2602_00397_amd import binding as B
from test_gpu_attention import DEV, _bf16, _gen, _heads, _int32, _starts, ctx  # noqa: F401
from test_gpu_cache8 import Append, Cache8, _append_model, _same_codes
from test_gpu_select import Cache8Values, Step

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


class Server:
    """One layer's cache in 8 bits and its means, in a pool, for up to `rows` sequences."""

    def __init__(self, ctx, h, n_pages, rows, stride, page_size, scale_tokens, query_block, keep, most_tokens):  # noqa: F811
        self.ctx, self.h, self.ps, self.gen = ctx, h, page_size, _gen(3)
        shape = (n_pages, h.n_kv_heads, page_size, h.head_dim)
        # (what no token was written to may be anything)
        self.k, self.v = (torch.full(shape, 0x7f, dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2))
        self.ks, self.vs = (torch.full((n_pages, h.n_kv_heads, page_size // scale_tokens), float("nan"), device=DEV) for _ in range(2))
        self.means = torch.full((n_pages, h.n_kv_heads, h.head_dim), float("nan"), device=DEV)
        self.refs, self.lens = torch.zeros(n_pages, dtype=torch.int32, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV)
        self.table = torch.full((rows, stride), -1, dtype=torch.int32, device=DEV)
        self.cache = B.paged_cache8(self.k, self.v, self.ks, self.vs)
        self.pool = B.page_pool(self.refs, self.table, self.lens, page_size, [self.k, self.v, self.ks, self.vs, self.means])
        self.sel, self.rot = B.selection(query_block, keep, 1), B.rotary(h.head_dim, 10000.0 ** (-torch.arange(h.head_dim // 2, device=DEV) / (h.head_dim // 2)))
        self.missing, self.scale_tokens, self.n = _int32([0]), scale_tokens, [0] * rows
        ctx.ensure_pages_workspace(self.pool, rows)
        ctx.ensure_attention_workspace(h, most_tokens, B.selection_blocks(self.sel, most_tokens, rows))
        ctx.ensure_selection_workspace(h, B.selection_blocks(self.sel, most_tokens, rows), stride)

    def step(self, new, what):
        """new[r] tokens of each row."""
        ctx, h, rows = self.ctx, self.h, len(new)  # noqa: F811
        self.n = [a + b for a, b in zip(self.n, new)]
        want = _int32(self.n)
        ctx.pages_grow(self.pool, _int32(list(range(rows))), want, self.missing)
        assert int(self.missing) == 0 and torch.equal(self.lens, want)
        t, qw, kw = sum(new), h.n_heads * h.head_dim, h.n_kv_heads * h.head_dim
        qkv = _bf16(self.gen, t, qw + 2 * kw)
        q, k, v = qkv[:, :qw], qkv[:, qw:qw + kw], qkv[:, qw + kw:]
        positions = _int32([list(p for a, b in zip(self.n, new) for p in range(a - b, a))])
        ctx.rotary(h, self.rot, q, k, v, positions, q, k_out=k)
        starts = _int32(_starts(new))
        model = Cache8.__new__(Cache8)
        model.h, model.page_size, model.scale_tokens, model.table, model.k_pages = h, self.ps, self.scale_tokens, self.table, self.k
        held = [x.clone() for x in (self.k.view(torch.uint8), self.v.view(torch.uint8), self.ks, self.vs)]
        ctx.cache8_append(h, k, v, starts, self.lens, self.cache, self.table)
        want = _append_model(model, k, v, starts.tolist(), self.n, held)
        got = (self.k.view(torch.uint8), self.v.view(torch.uint8), self.ks, self.vs)
        assert all(_same_codes(a, b) for a, b in zip(got[:2], want[:2])), what
        assert all(torch.equal(a.nan_to_num(-1.0), b.nan_to_num(-1.0)) for a, b in zip(got[2:], want[2:])), what
        s = Step.__new__(Step)
        s.c = Cache8Values.__new__(Cache8Values)
        s.c.h, s.c.page_size, s.c.k_pages, s.c.v_pages, s.c.k_scale, s.c.v_scale, s.c.lens = h, self.ps, self.k, self.v, self.ks, self.vs, self.n
        s.c.cache, s.h, s.new, s.sel, s.n_pages, s.q, s.starts, s.lens, s.table, s.means = self.cache, h, new, self.sel, self.k.shape[0], q, starts, self.lens, self.table, self.means
        s.n_blocks, s.width = B.selection_blocks(self.sel, t, rows), B.selection_pages(self.sel, self.ps)
        s.block_starts, s.block_lens = _int32([-9] * (s.n_blocks + 1)), _int32([-9] * s.n_blocks)
        s.tables = torch.full((s.n_blocks, h.n_kv_heads, s.width), -9, dtype=torch.int32, device=DEV)
        s.o, s.lse = torch.full((t, qw), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((t, h.n_heads), 7.0, device=DEV)
        s.run(ctx)
        for i, n in enumerate(self.n):
            for j in range(0, n, self.ps):
                page = int(self.table[i, j // self.ps])
                mean = s.c.values("k", page)[:, :min(self.ps, n - j)].mean(dim=1).float()
                assert torch.equal(self.means[page], mean), f"{what}: mean of page {j // self.ps} of row {i}"
        s.check(what)


@pytest.mark.parametrize("h", [(8, 2, 128), (4, 4, 64)], ids=lambda h: "%d_%d_%d" % h)
def test_a_server(ctx, h):  # noqa: F811
    s = Server(ctx, _heads(h), 120, 6, 40, 16, 8, 8, 3, 200)
    s.step([40, 0, 90, 0, 0, 0], "first prompts")
    s.step([40, 33, 1, 0, 0, 0], "a prompt's next block, a new prompt, a token")
    for i in range(3):
        s.step([1, 1, 1, 0, 0, 0], f"token {i}")
    ctx.pages_fork(s.pool, _int32([0, 0, 2]), _int32([3, 4, 5]), s.missing)
    s.n[3:6] = [s.n[0], s.n[0], s.n[2]]
    assert int(s.missing) == 0
    for i in range(2):
        s.step([1, 1, 2, 1, 1, 1], f"forked, token {i}")
    ctx.pages_free(s.pool, _int32([0, 2]))
    s.n[0] = s.n[2] = 0
    live = _int32([0])
    ctx.pages_compact(s.pool, live)
    assert int(live) == int((s.refs > 0).sum()) and bool((s.refs[:int(live)] > 0).all())
    s.step([20, 1, 0, 1, 1, 3], "after two ended and the pages moved together")
    # a beam goes on in the place of another
    ctx.pages_fork(s.pool, _int32([4, 3]), _int32([3, 4]), s.missing)
    s.n[3], s.n[4] = s.n[4], s.n[3]
    s.step([1, 1, 17, 1, 1, 1], "beams changed places")


def test_append_on_another_stream_than_the_current_one():
    """A context's calls run on its stream, whatever torch's current one is; a second context beside it on the same device."""
    own, other = torch.cuda.Stream(), torch.cuda.Stream()
    a, b = B.Context(0, own), B.Context(0, other)
    try:
        x, y = Append((32, 8, 128), [3, 40], [130, 40], seed=1), Append((4, 2, 64), [70], [70], seed=2)
        torch.cuda.synchronize()
        held = x.held(), y.held()
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            x.run(a)
        y.run(b)
        torch.cuda.synchronize()
        x.check(held[0], "own stream")
        y.check(held[1], "other stream")
    finally:
        torch.cuda.synchronize()
        a.close()
        b.close()


def test_rows_that_outgrow_their_table_or_the_pool(ctx):  # noqa: F811
    """A step's lengths as the program wants them, whatever the pool could give: tokens without a page are dropped, and what is cached stays,
    of the row and of the rows that share its pages."""
    h, ps = _heads((8, 2, 64)), 16
    n_pages, stride, kw = 8, 3, 128
    k, v = (torch.zeros((n_pages, 2, ps, 64), dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2))
    ks, vs = (torch.ones((n_pages, 2, 2), device=DEV) for _ in range(2))
    refs, lens, table = torch.zeros(n_pages, dtype=torch.int32, device=DEV), _int32([0] * 3), torch.full((3, stride), -1, dtype=torch.int32, device=DEV)
    cache, pool, missing = B.paged_cache8(k, v, ks, vs), B.page_pool(refs, table, lens, ps, [k, v, ks, vs]), _int32([0])
    ctx.ensure_pages_workspace(pool, 3)
    gen, rows = _gen(9), _int32([0, 1, 2])
    x, y = _bf16(gen, 100, kw), _bf16(gen, 100, kw)

    def step(new, wanted):
        wanted = _int32(wanted)
        ctx.pages_grow(pool, rows, wanted, missing)
        ctx.cache8_append(h, x[:sum(new)], y[:sum(new)], _int32(_starts(new)), wanted, cache, table)

    def held():
        return [t.clone() for t in (k.view(torch.uint8), v.view(torch.uint8), ks, vs)]

    step([48, 0, 5], [48, 0, 5])
    ctx.pages_fork(pool, _int32([0]), _int32([1]), missing)
    assert lens.tolist() == [48, 48, 5] and refs.tolist()[:4] == [2, 2, 2, 1] and int(missing) == 0
    before = held()
    # a token behind the full row 0, then another: row 1 shares its pages, and nothing of them changes
    for n in (49, 50):
        step([1, 0, 0], [n, 48, 5])
        assert lens.tolist() == [48, 48, 5] and int(missing) == 0
        assert all(torch.equal(a, b) for a, b in zip(held(), before))
    # three tokens for row 2 that has a place for one of them
    step([0, 0, 42], [48, 48, 47])
    before = held()
    step([0, 0, 3], [48, 48, 50])
    after, last = held(), int(table[2, 2])
    same = torch.ones((n_pages, ps), dtype=torch.bool, device=DEV)
    same[last, 8:] = False                                    # (the block of the token, whose scale may have grown)
    for a, b in zip(after[:2], before[:2]):
        assert torch.equal(a.transpose(1, 2)[same], b.transpose(1, 2)[same]) and bool((a[last, :, 15] != b[last, :, 15]).any())
    # too few pages: nothing is grown, and the tokens of the pages that are missing are dropped
    refs[refs == 0] = 1
    ctx.pages_free(pool, _int32([2]))
    ctx.pages_grow(pool, _int32([2]), _int32([16]), missing)
    refs[refs == 0] = 1
    before, tables = held(), table.clone()
    step([0, 0, 20], [48, 48, 36])
    assert int(missing) == 2 and torch.equal(table, tables) and lens.tolist() == [48, 48, 16]
    assert all(torch.equal(a, b) for a, b in zip(held(), before))
