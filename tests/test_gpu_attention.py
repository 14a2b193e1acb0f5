"""Attention over prompts and over a paged cache, against softmax(scale q k^T) v in float64.

The bars follow from the roundings.  A row's output is off by its own rounding, half a bf16 step (2^-8 of its value), and
by the softmax weights' rounding to bf16, at most 2^-8 of each weight, so 2^-8 of sum_j p_j |v_j|; fp32 products and
sums, the exponentials and the normalisation stay below a sixteenth of that.  lse is fp32: head_dim products, the sum
over the keys and the logarithm, each with half a step of 2^-23."""
import math

import pytest
import torch

from paper_2602_00397_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
H8B, H7B, H1B, TINY, MHA, MQA = (32, 8, 128), (28, 4, 128), (32, 8, 64), (4, 2, 64), (3, 3, 64), (20, 1, 128)


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = B.Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


def _gen(seed=1):
    return torch.Generator(device=DEV).manual_seed(seed)


def _bf16(gen, *shape):
    return torch.randn(shape, device=DEV, generator=gen).to(torch.bfloat16)


def _heads(h, causal=True, window=0, scale=None):
    return B.Attention(h[0], h[1], h[2], causal, window, scale or h[2] ** -0.5)


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _starts(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _reference(h, q, k, v):
    """One sequence, new tokens q [n][heads][hd] behind keys - n earlier ones: o, sum p |v|, lse, largest sum |q k|."""
    n, keys, group = q.shape[0], k.shape[0], h.n_heads // h.n_kv_heads
    q, k, v = q.double(), k.double(), v.double()
    pos = torch.arange(keys - n, keys, device=DEV)[:, None]
    j = torch.arange(keys, device=DEV)[None]
    seen = (j <= pos if h.causal else j < keys + 0 * pos) & ((j > pos - h.window) if h.window else (j >= 0))
    o, spread = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full((n, h.n_heads), -math.inf, dtype=torch.float64, device=DEV)
    size = torch.zeros((n, h.n_heads), dtype=torch.float64, device=DEV)
    if n == 0 or keys == 0:
        return o, spread, lse, size
    for a in range(h.n_heads):
        ka, va = k[:, a // group], v[:, a // group]
        # (what a row does not see may be anything)
        x = torch.where(seen, q[:, a] @ ka.t() * h.scale, torch.full((), -math.inf, dtype=torch.float64, device=DEV))
        m = x.amax(dim=1, keepdim=True)
        p = torch.exp(x - torch.where(m == -math.inf, torch.zeros_like(m), m))
        l = p.sum(dim=1, keepdim=True)
        p = p / torch.where(l == 0, torch.ones_like(l), l)
        clean = torch.where(torch.isfinite(va), va, torch.zeros_like(va))
        o[:, a], spread[:, a] = p @ clean, p @ clean.abs()
        for bad in torch.nonzero(~torch.isfinite(va)).tolist():
            o[:, a, bad[1]] += torch.where(seen[:, bad[0]], va[bad[0], bad[1]], torch.zeros_like(l[:, 0]))
        lse[:, a] = (m + torch.log(l))[:, 0]
        size[:, a] = torch.where(seen, q[:, a].abs() @ torch.nan_to_num(ka, 0, 0, 0).abs().t() * h.scale, torch.zeros_like(x)).amax(dim=1)
    return o, spread, lse, size


def _check(got, lse, ref, hd, keys, what=""):
    o, spread, ref_lse, size = ref
    got = got.double().reshape(o.shape)
    finite = torch.isfinite(o)
    assert torch.equal(torch.isfinite(got), finite), f"{what}: finite where the reference is not, or the other way round"
    assert torch.equal(torch.isnan(got), torch.isnan(o)) and torch.equal(got[torch.isinf(o)], o[torch.isinf(o)]), what
    # fp32 under the softmax: logits to hd half steps of the largest |q k| sum, the same again for exponent and sums
    fine = (2.0 ** -23) * (hd * size + 64)[:, :, None]
    bar = 2.0 ** -8 * o.abs() + (2.0 ** -8 + fine) * 1.01 * spread + 1e-30
    off = ((got - o).abs() / bar)[finite]
    worst = float(off.max()) if off.numel() else 0.0
    print(f"[attention] {what}: worst error {worst:.3f} of its bar", flush=True)
    assert worst <= 1.0, what
    if lse is not None:
        seen = ref_lse > -math.inf
        assert torch.equal(lse == -math.inf, ~seen), f"{what}: lse of rows without keys"
        bar = 2.0 ** -23 * (hd * size + keys + 64 + ref_lse.abs())
        assert bool(((lse.double() - ref_lse).abs() <= bar)[seen].all()), f"{what}: lse"


# ------------------------------------------------------------------ whole prompts

class Prompt:
    def __init__(self, h, lengths, seed=1, behind=0, strided=False):
        gen = _gen(seed)
        self.h, self.lengths = h, lengths
        t = sum(lengths) + behind
        qw, kw = h.n_heads * h.head_dim, h.n_kv_heads * h.head_dim
        if strided:
            qkv = _bf16(gen, t, qw + 2 * kw + 24)
            self.q, self.k, self.v = qkv[:, :qw], qkv[:, qw:qw + kw], qkv[:, qw + kw:qw + 2 * kw]
        else:
            self.q, self.k, self.v = _bf16(gen, t, qw), _bf16(gen, t, kw), _bf16(gen, t, kw)
        self.starts = _int32(_starts(lengths))
        out = torch.full((t, qw + 40 if strided else qw), 7.0, dtype=torch.bfloat16, device=DEV)
        self.out, self.o = out, out[:, 8:8 + qw] if strided else out
        self.lse = torch.full((t, h.n_heads), 7.0, device=DEV)

    def run(self, ctx):
        ctx.prompt_attention(self.h, self.q, self.k, self.v, self.starts, self.o, lse=self.lse)

    def check(self, what):
        h, hd, t0 = self.h, self.h.head_dim, 0
        for n in self.lengths:
            part = [x[t0:t0 + n].unflatten(1, (-1, hd)) for x in (self.q, self.k, self.v)]
            _check(self.o[t0:t0 + n], self.lse[t0:t0 + n], _reference(h, *part), hd, n, f"{what}, {n} tokens at {t0}")
            t0 += n
        assert bool((self.o[t0:] == 7.0).all()) and bool((self.lse[t0:] == 7.0).all()), "rows behind the last sequence changed"
        if self.out.shape[1] != self.o.shape[1]:
            assert bool((self.out[:, :8] == 7.0).all()) and bool((self.out[:, 8 + self.o.shape[1]:] == 7.0).all()), "beside the rows"


@pytest.mark.parametrize("h", [H8B, H7B, H1B, TINY, MHA, MQA], ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("lengths", [[1], [2], [63, 0, 64, 1, 65], [129], [300, 1, 31]], ids=str)
def test_prompts_of_small_and_odd_lengths(ctx, h, lengths):
    p = Prompt(_heads(h), lengths, behind=3)
    p.run(ctx)
    p.check(f"{h} {lengths}")


@pytest.mark.parametrize("causal,window", [(False, 0), (True, 1), (True, 50), (True, 64), (True, 257), (True, 100000)])
@pytest.mark.parametrize("h", [H7B, H1B], ids=lambda h: "%d_%d_%d" % h)
def test_prompts_with_windows_and_without_a_causal_mask(ctx, h, causal, window):
    p = Prompt(_heads(h, causal, window), [517, 40, 0, 3, 129], seed=2)
    p.run(ctx)
    p.check(f"{h} causal {causal} window {window}")


def test_prompt_rows_apart(ctx):
    for h in (H8B, H1B):
        p = Prompt(_heads(h), [70, 141], seed=3, behind=2, strided=True)
        p.run(ctx)
        p.check(f"strided {h}")


def test_long_prompt_and_many_sequences(ctx):
    p = Prompt(_heads((8, 2, 128)), [3001], seed=4)
    p.run(ctx)
    p.check("3001 tokens")
    p = Prompt(_heads(TINY), [(7 * i) % 23 for i in range(150)], seed=5, behind=1)     # more sequences than lanes
    p.run(ctx)
    p.check("150 sequences")


@pytest.mark.parametrize("h", [(64, 64, 64), (64, 64, 128), (80, 40, 64), (48, 16, 128)], ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 300)])
def test_prompts_with_work_for_every_cu_in_large_tiles(ctx, h, causal, window):
    """Enough rows that tiles have 256 of them: whole, ragged and part-filled ones, and values that are not finite."""
    group = h[0] // h[1]
    t = -(-256 * 500 // h[0])                              # rows / 256 * key heads above 384
    lengths = [t - 517, 1, 0, 300, 63, 31, 129]
    p = Prompt(_heads(h, causal, window), lengths, seed=30, behind=3)
    for row, ch, val in ((t - 518, 5, math.inf), (t - 400, 0, math.nan), (t - 390, 9, -math.inf), (70, 64, math.inf)):
        p.v[row, ch] = val
    assert sum(lengths) * group // 256 * h[1] > 384
    p.run(ctx)
    p.check(f"{h} causal {causal} window {window}")


def test_more_sequences_than_a_launch_has_threads_across(ctx):
    """2^24 tiles of one row: a single token's output is its value."""
    n = 16384
    gen = _gen(31)
    h = _heads((1024, 1024, 64))
    q, v = _bf16(gen, n, 65536), _bf16(gen, n, 65536)
    o = torch.zeros_like(q)
    ctx.prompt_attention(h, q, q, v, torch.arange(n + 1, dtype=torch.int32, device=DEV), o)
    assert torch.equal(o.view(torch.int16), v.view(torch.int16))


def test_prompt_scale_and_large_logits(ctx):
    # logits up to some thousands: the running maximum moves all the time, and most weights vanish
    p = Prompt(_heads(H8B, scale=3.0), [400], seed=6)
    p.q *= 4.0
    p.run(ctx)
    p.check("large logits")
    p.q.zero_()                                            # all equal: the mean of what a row sees
    p.run(ctx)
    p.check("zero logits")


@pytest.mark.parametrize("h", [H8B, H1B], ids=lambda h: "%d_%d_%d" % h)
def test_prompt_what_a_row_does_not_see_never_reaches_it(ctx, h):
    """Keys and values of later tokens hold NaN, infinities and the type's lowest value: rows before them stay clean, rows
    that see such a value get it."""
    p = Prompt(_heads(h), [200, 30], seed=7)
    p.k[150:160] = float("nan")
    p.k[170] = torch.finfo(torch.bfloat16).min
    p.v[180, 5] = float("inf")
    p.v[181, 6] = float("nan")
    p.v[222, 3] = -float("inf")
    p.run(ctx)
    hd = p.h.head_dim
    for a, b in ((0, 150), (200, 230)):
        t0 = 0 if a < 200 else 200
        part = [x[t0:b].unflatten(1, (-1, hd)) for x in (p.q, p.k, p.v)]
        _check(p.o[a:b], p.lse[a:b], [x[a - t0:] for x in _reference(p.h, *part)], hd, b - t0, f"{h} rows {a} to {b}")
    assert bool(torch.isnan(p.o[160:200].float()).all())   # these see the keys that are NaN


# ------------------------------------------------------------------ chunks over a paged cache

class Chunks:
    def __init__(self, h, new, ctx_lens, page_size=16, seed=1, behind=0, extra_pages=3, max_chunk=None, unused=float("nan")):
        gen = _gen(seed)
        self.h, self.new, self.lens = h, new, ctx_lens
        t, hd = sum(new) + behind, h.head_dim
        self.q = _bf16(gen, t, h.n_heads * hd)
        used = [-(-n // page_size) for n in ctx_lens]
        n_pages = sum(used) + extra_pages
        # places that hold no key hold anything
        self.k_pages, self.v_pages = (torch.full((n_pages, h.n_kv_heads, page_size, hd), unused, dtype=torch.bfloat16, device=DEV)
                                      for _ in range(2))
        order = torch.randperm(n_pages, device=DEV, generator=gen).to(torch.int32)
        self.table = torch.full((len(new), max(used + [1]) + 1), -1, dtype=torch.int32, device=DEV)
        self.k, self.v, at = [], [], 0
        for i, n in enumerate(ctx_lens):
            self.table[i, :used[i]] = order[at:at + used[i]]
            at += used[i]
            for pages, keep in ((self.k_pages, self.k), (self.v_pages, self.v)):
                x = _bf16(gen, n, h.n_kv_heads, hd)
                j = torch.arange(n, device=DEV)
                pages[self.table[i].long()[j // page_size], :, j % page_size] = x
                keep.append(x)
        self.starts, self.ctx_lens = _int32(_starts(new)), _int32(ctx_lens)
        self.max_chunk = max_chunk or max(max(new), 1)
        self.cache = B.paged_cache(self.k_pages, self.v_pages)
        self.o = torch.full((t, h.n_heads * hd), 7.0, dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((t, h.n_heads), 7.0, device=DEV)

    def run(self, ctx):
        ctx.ensure_attention_workspace(self.h, self.q.shape[0], len(self.new))
        ctx.chunk_attention(self.h, self.q, self.starts, self.ctx_lens, self.max_chunk, self.cache, self.table, self.o, lse=self.lse)

    def check(self, what):
        hd, t0 = self.h.head_dim, 0
        for i, n in enumerate(self.new):
            ref = _reference(self.h, self.q[t0:t0 + n].unflatten(1, (-1, hd)), self.k[i], self.v[i])
            _check(self.o[t0:t0 + n], self.lse[t0:t0 + n], ref, hd, self.lens[i], f"{what}, sequence {i}: {n} over {self.lens[i]}")
            t0 += n
        assert bool((self.o[t0:] == 7.0).all()) and bool((self.lse[t0:] == 7.0).all()), "rows behind the last sequence changed"


@pytest.mark.parametrize("h", [H8B, H7B, H1B, TINY, MHA, MQA], ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("lens", [[1], [2, 33], [64, 1, 700, 31, 32], [5000]], ids=str)
def test_single_tokens(ctx, h, lens):
    c = Chunks(_heads(h), [1] * len(lens), lens, behind=2)
    c.run(ctx)
    c.check(f"tokens {h}")


@pytest.mark.parametrize("h", [H8B, H7B, H1B, MHA], ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("n", [2, 5, 8, 13, 16, 17, 33, 64, 65, 130, 257])
def test_chunks_of_every_kernel(ctx, h, n):
    c = Chunks(_heads(h), [n], [n + 400], page_size=64, seed=n)
    c.run(ctx)
    c.check(f"chunk {h} {n}")


@pytest.mark.parametrize("h", [(64, 64, 64), (64, 64, 128), (48, 16, 128)], ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 300)])
def test_chunks_with_work_for_every_cu_in_large_tiles(ctx, h, causal, window):
    t = -(-256 * 500 // h[0])
    new = [t - 60, 1, 40, 0, 19]
    c = Chunks(_heads(h, causal, window), new, [t + 200, 333, 40, 5, 7], page_size=32, seed=32, behind=2)
    for i, key, ch, val in ((0, t + 199, 3, math.inf), (0, t + 100, 7, math.nan), (1, 332, 0, -math.inf), (2, 5, 60, math.inf)):
        c.v[i][key, 0, ch] = val
        c.v_pages[c.table[i, key // 32].long(), 0, key % 32, ch] = val
    c.run(ctx)
    c.check(f"{h} causal {causal} window {window}")


@pytest.mark.parametrize("h", [H8B, H7B, H1B, MQA], ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("n", [1, 3, 4])
def test_few_rows_over_many_keys_with_values_that_are_not_finite(ctx, h, n):
    """Pieces joined by the last one of them or by a launch of their own: infinities and NaN reach the rows that see them."""
    c = Chunks(_heads(h), [n, 1], [9000, 4001], page_size=64, seed=33)
    for i, key, ch, val in ((0, 8999, 3, math.inf), (0, 9000 - n, 7, math.nan), (0, 17, 0, -math.inf), (0, 5000, 0, math.inf), (1, 4000, 60, math.inf)):
        c.v[i][key, 0, ch] = val
        c.v_pages[c.table[i, key // 64].long(), 0, key % 64, ch] = val
    c.run(ctx)
    c.check(f"{h} {n} not finite")


def test_without_the_log_sums(ctx):
    for new in ([1, 1], [3, 1], [9, 8], [100, 1]):
        c = Chunks(_heads(H8B), new, [5000, 300], page_size=64, seed=34)
        c.run(ctx)
        first = c.o.clone()
        c.o.fill_(7.0)
        ctx.chunk_attention(c.h, c.q, c.starts, c.ctx_lens, c.max_chunk, c.cache, c.table, c.o)
        assert torch.equal(c.o.view(torch.int16), first.view(torch.int16))
    p = Prompt(_heads(H1B), [300, 5], seed=35)
    p.run(ctx)
    first = p.o.clone()
    p.o.fill_(7.0)
    ctx.prompt_attention(p.h, p.q, p.k, p.v, p.starts, p.o)
    assert torch.equal(p.o.view(torch.int16), first.view(torch.int16))


@pytest.mark.parametrize("page_size", [8, 16, 128, 4096])
@pytest.mark.parametrize("h", [H8B, H1B], ids=lambda h: "%d_%d_%d" % h)
def test_mixed_batches_and_page_sizes(ctx, h, page_size):
    c = Chunks(_heads(h), [1, 90, 1, 0, 200, 7, 1], [500, 90, 1, 77, 1000, 650, 2048], page_size=page_size, seed=9, behind=5)
    c.run(ctx)
    c.check(f"mixed {h} pages of {page_size}")


@pytest.mark.parametrize("new", [[1, 1, 1, 1], [12, 3, 40, 9], [150, 3, 300, 9]], ids=str)
def test_sequences_with_fewer_keys_than_tokens_or_none(ctx, new):
    """The first tokens of such a sequence see nothing: zeros, and a log sum of -inf."""
    c = Chunks(_heads(H8B), new, [0, 2, 33, 9], seed=10)
    c.run(ctx)
    c.check(f"short contexts {new}")


@pytest.mark.parametrize("causal,window", [(False, 0), (True, 1), (True, 37), (True, 64), (True, 500)])
@pytest.mark.parametrize("new", [[1, 1, 1], [6, 1, 3], [140, 1, 60]], ids=str)
def test_windows_and_no_causal_mask(ctx, new, causal, window):
    for h in (H7B, H1B):
        c = Chunks(_heads(h, causal, window), new, [1500, 64, 333], page_size=32, seed=11)
        c.run(ctx)
        c.check(f"{h} {new} causal {causal} window {window}")


def test_pages_before_a_window_may_be_gone(ctx):
    for new in ([1, 1], [40, 1], [100, 80]):
        c = Chunks(_heads(H8B, True, 100), new, [1000, 700], page_size=16, seed=12)
        for i, n in enumerate(new):
            c.table[i, :(c.lens[i] - n + 1 - 100) // 16] = -1
        c.run(ctx)
        c.check(f"freed pages {new}")


@pytest.mark.parametrize("hint", [1, 3, 30, 60, 300])
def test_other_lengths_than_the_host_expected(ctx, hint):
    c = Chunks(_heads(H8B), [1, 20, 0, 279], [600, 20, 5, 900], page_size=64, seed=13, max_chunk=hint)
    c.run(ctx)
    c.check(f"longest chunk taken for {hint}")


def test_values_that_are_not_finite(ctx):
    for new in ([1, 1], [9, 2], [100, 70]):
        for h in (H8B, H1B):
            c = Chunks(_heads(h), new, [333, 200], seed=14)
            n, ps = new[0], c.cache.page_size
            for key, ch, val in ((332, 4, math.inf), (333 - n, 7, math.nan), (330, 0, -math.inf), (332, 0, math.inf)):
                if key < 333:
                    c.v[0][key, 0, ch] = val
                    c.v_pages[c.table[0, key // ps].long(), 0, key % ps, ch] = val
            c.run(ctx)
            c.check(f"{h} {new} not finite")


def test_many_sequences(ctx):
    lens = [1 + (37 * i) % 800 for i in range(130)]
    c = Chunks(_heads(H1B), [1] * 130, lens, seed=15)
    c.run(ctx)
    c.check("130 sequences")


@pytest.mark.parametrize("h", [H8B, H7B, TINY], ids=lambda h: "%d_%d_%d" % h)
def test_many_sequences_of_every_kernel(ctx, h):
    """More sequences than a wavefront has lanes, with pieces joined in each way."""
    for n_seqs, new in ((70, lambda i: i % 5), (90, lambda i: (i * 29) % 61), (67, lambda i: 150 if i == 66 else 1)):
        new = [new(i) for i in range(n_seqs)]
        lens = [n + (53 * i) % 300 for i, n in enumerate(new)]
        lens[65] = new[65] + 5000
        c = Chunks(_heads(h), new, lens, page_size=32, seed=38, behind=1)
        c.run(ctx)
        c.check(f"{n_seqs} sequences of up to {max(new)} tokens")


def test_thousands_of_sequences(ctx):
    """Contexts of one key or none: a token's output is that key's value, or zeros; the second of two tokens sees it."""
    h, n_seqs, ps = _heads((4, 2, 64)), 9000, 8
    gen = _gen(39)
    for most in (1, 2, 40):
        new = [1 + (i % 2 if most > 1 else 0) for i in range(n_seqs)]
        if most == 40:
            new[8999] = 40
        lens = [(i // 2) % 2 for i in range(n_seqs)]
        t = sum(new)
        q = _bf16(gen, t, 256)
        k_pages, v_pages = _bf16(gen, n_seqs, 2, ps, 64), _bf16(gen, n_seqs, 2, ps, 64)
        table = torch.randperm(n_seqs, device=DEV, generator=gen).to(torch.int32)[:, None].contiguous()
        starts = _int32(_starts(new))
        o = torch.full((t + 1, 256), 7.0, dtype=torch.bfloat16, device=DEV)
        ctx.ensure_attention_workspace(h, t, n_seqs)
        ctx.chunk_attention(h, q, starts, _int32(lens), most, B.paged_cache(k_pages, v_pages), table, o[:t])
        last = (starts[1:] - 1).long()
        want = torch.zeros_like(o[:t])
        value = v_pages[table[:, 0].long(), :, 0].repeat_interleave(2, dim=1).reshape(n_seqs, 256)
        want[last] = torch.where(_int32(lens)[:, None] > 0, value, torch.zeros_like(value))
        assert torch.equal(o[:t].view(torch.int16), want.view(torch.int16)) and bool((o[t:] == 7.0).all()), most


def test_chunk_rows_apart(ctx):
    for h, new in ((H8B, [1, 1]), (H7B, [4, 2]), (H8B, [100, 3]), (H1B, [70, 1])):
        c = Chunks(_heads(h), new, [5000, 77], page_size=64, seed=40)
        w = c.q.shape[1]
        q, o = torch.zeros((c.q.shape[0], w + 24), dtype=torch.bfloat16, device=DEV), torch.full((c.q.shape[0], w + 40), 7.0, dtype=torch.bfloat16, device=DEV)
        q[:, 16:16 + w] = c.q
        ctx.ensure_attention_workspace(c.h, c.q.shape[0], 2)
        ctx.chunk_attention(c.h, q[:, 16:16 + w], c.starts, c.ctx_lens, c.max_chunk, c.cache, c.table, o[:, 8:8 + w], lse=c.lse)
        assert bool((o[:, :8] == 7.0).all()) and bool((o[:, 8 + w:] == 7.0).all())
        c.o = o[:, 8:8 + w].contiguous()
        c.check(f"{h} {new} rows apart")


@pytest.mark.parametrize("new", [[1, 1], [4, 2], [9, 8], [100, 3]], ids=str)
def test_chunks_with_large_logits(ctx, new):
    for h in (H8B, H1B):
        c = Chunks(_heads(h, scale=3.0), new, [3000, 500], page_size=64, seed=41)
        c.q *= 4.0
        c.run(ctx)
        c.check(f"{h} {new} large logits")


def test_queries_that_are_not_finite_spoil_their_own_rows_only(ctx):
    for h in (H8B, H1B):
        for new in ([1, 1], [5, 2], [100, 40]):
            c = Chunks(_heads(h), new, [3000, 500], page_size=64, seed=42)
            c.run(ctx)
            first, d = c.o.clone(), h[2]
            c.q[1, d:d + 3] = float("nan")                     # head 1 of a token
            c.q[-1, 5] = float("inf")                          # head 0 of another
            c.run(ctx)
            same = torch.ones_like(c.o, dtype=torch.bool)
            same[1, d:2 * d] = same[-1, :d] = False
            assert bool(torch.isnan(c.o[~same].float()).all()), f"{h} {new}"
            assert torch.equal(c.o[same].view(torch.int16), first[same].view(torch.int16)), f"{h} {new}"


def test_cache_beyond_32_bit_offsets(ctx):
    """Pages at the end of a cache of more than 4 GiB, in bytes and (2^31) in elements."""
    h, ps = _heads(H8B), 64
    per_page = 8 * ps * 128
    n_pages = (1 << 31) // per_page + 2000
    k_pages = torch.empty((n_pages, 8, ps, 128), dtype=torch.bfloat16, device=DEV)
    v_pages = torch.empty_like(k_pages)
    for new in (1, 150):
        c = Chunks(h, [new], [700], page_size=ps, seed=16)
        used = c.table[0, :11].clone().long()
        at = torch.arange(n_pages - 11, n_pages, device=DEV)
        k_pages[at], v_pages[at] = c.k_pages[used], c.v_pages[used]
        c.table[0, :11] = at.to(torch.int32)
        c.cache = B.paged_cache(k_pages, v_pages)
        c.run(ctx)
        c.check(f"far pages, {new} tokens")


def test_the_same_call_gives_the_same_bits(ctx):
    for new, lens in (([1] * 5, [4000, 3, 900, 77, 1]), ([128], [3000]), ([1, 200, 1], [900, 400, 2000])):
        c = Chunks(_heads(H8B), new, lens, page_size=64, seed=17)
        c.run(ctx)
        first = c.o.clone(), c.lse.clone()
        for _ in range(5):
            c.o.fill_(3.0)
            c.run(ctx)
            assert torch.equal(c.o.view(torch.int16), first[0].view(torch.int16)) and torch.equal(c.lse, first[1])


def test_captured_calls_follow_lengths_and_tables():
    """Two graphs that share a workspace, captured once and replayed while lengths, pages and queries change, with eager calls
    in between."""
    stream = torch.cuda.Stream()
    ctx = B.Context(0, stream)
    try:
        a = Chunks(_heads(H8B), [1, 1, 1], [900, 40, 2000], page_size=64, seed=18)
        b = Chunks(_heads(H8B), [90, 1, 37], [900, 700, 64], page_size=64, seed=19)
        p = Prompt(_heads(H8B), [70, 0, 130], seed=20)
        torch.cuda.synchronize()
        for x in (a, b, p):
            x.run(ctx)
        stream.synchronize()
        g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g1, stream=stream):
            a.run(ctx)
            p.run(ctx)
        with torch.cuda.graph(g2, stream=stream):
            b.run(ctx)
        gen = _gen(21)
        for rep in range(4):
            for x in (a, b):
                x.q.copy_(_bf16(gen, *x.q.shape))
                x.ctx_lens.copy_(_int32([max(1, n - 13 * rep) for n in x.lens]))
            p.starts.copy_(_int32([0, 70 - rep, 70 + 5 * rep, 200]))
            torch.cuda.synchronize()
            g1.replay()
            g2.replay()
            torch.cuda.synchronize()
            got = [x.o.clone() for x in (a, b, p)]
            for x in (a, b, p):
                x.o.fill_(5.0)
            torch.cuda.synchronize()
            for x in (a, b, p):
                x.run(ctx)
            stream.synchronize()
            for x, y in zip((a, b, p), got):
                assert torch.equal(x.o.view(torch.int16), y.view(torch.int16)), f"replay {rep}"
    finally:
        torch.cuda.synchronize()
        ctx.close()


def _refused(status, call, *args, **kw):
    with pytest.raises(B.FFError) as e:
        call(*args, **kw)
    assert e.value.status == status, e.value


def test_refusals(ctx):
    p = Prompt(_heads(TINY), [40])
    c = Chunks(_heads(TINY), [3, 1], [40, 9])

    def prompt(h, **kw):
        x = dict(dict(q=p.q, k=p.k, v=p.v, seq_starts=p.starts, o=p.o), **kw)
        ctx.prompt_attention(h, x["q"], x["k"], x["v"], x["seq_starts"], x["o"])

    def chunk(h=None, **kw):
        x = dict(dict(max_chunk=3, table=c.table, lens=c.ctx_lens, cache=c.cache), **kw)
        ctx.chunk_attention(h or c.h, c.q, c.starts, x["lens"], x["max_chunk"], x["cache"], x["table"], c.o)

    for field, value, status in (("scale", 0.0, 1), ("scale", -1.0, 1), ("scale", math.nan, 1), ("scale", math.inf, 1),
                                 ("window", -1, 1)):
        h = _heads(TINY)
        setattr(h, field, value)
        _refused(status, prompt, h)
        _refused(status, chunk, h)
    _refused(1, prompt, _heads(TINY, causal=False, window=4))
    _refused(1, chunk, max_chunk=0)
    _refused(1, chunk, max_chunk=5)
    small = B.PagedCache(c.cache.k, c.cache.v, c.cache.n_pages, 16)
    small.tensors = c.cache.tensors
    for field, value, status in (("n_pages", 0, 1), ("page_size", 12, 2), ("page_size", 4, 2), ("page_size", 8192, 2), ("k", None, 1)):
        bad = B.PagedCache(small.k, small.v, small.n_pages, small.page_size)
        bad.tensors = small.tensors
        setattr(bad, field, value)
        _refused(status, chunk, cache=bad)
    q96 = torch.zeros((40, 4 * 96), dtype=torch.bfloat16, device=DEV)
    kv96 = torch.zeros((40, 2 * 96), dtype=torch.bfloat16, device=DEV)
    _refused(2, prompt, _heads((4, 2, 96)), q=q96, k=kv96, v=kv96, o=torch.zeros_like(q96))
    odd = torch.zeros((40, 4 * 64 + 4), dtype=torch.bfloat16, device=DEV)
    _refused(3, prompt, p.h, q=odd[:, :256])                         # rows that are no multiple of 16 bytes apart
    fresh = B.Context(0)
    try:
        big = Chunks(_heads(H8B), [1], [4000])
        with pytest.raises(B.FFError) as e:                          # no workspace
            fresh.chunk_attention(big.h, big.q, big.starts, big.ctx_lens, 1, big.cache, big.table, big.o)
        assert e.value.status == 5
        p8 = Prompt(_heads(H8B), [40])
        fresh.prompt_attention(p8.h, p8.q, p8.k, p8.v, p8.starts, p8.o)   # needs none
        torch.cuda.synchronize()
    finally:
        fresh.close()


def test_lengths_and_pages_out_of_range(ctx):
    """Nothing outside the tensors is touched; with the validate option such a call is an error."""
    for new in ([1, 1], [40, 70]):
        for what, change in (("page", lambda c: c.table[1, 0].fill_(1 << 30)), ("negative page", lambda c: c.table[1, 0].fill_(-5)),
                             ("length", lambda c: c.ctx_lens[0].fill_(1 << 30)), ("negative length", lambda c: c.ctx_lens[0].fill_(-3)),
                             ("starts", lambda c: c.starts[2].fill_(1 << 30)), ("descending starts", lambda c: c.starts[1].fill_(-9))):
            c = Chunks(_heads(H8B), new, [100, 80], unused=0.0)
            change(c)
            ctx.set_option("validate", 1)
            try:
                _refused(4, c.run, ctx)
                assert bool((c.o == 7.0).all())
            finally:
                ctx.set_option("validate", 0)
            c.run(ctx)                                               # (clamped: finishes, with no access out of range)
            torch.cuda.synchronize()
    c = Chunks(_heads(H8B), [1, 40], [100, 80])
    ctx.set_option("validate", 1)
    try:
        c.run(ctx)
        c.check("validated")
    finally:
        ctx.set_option("validate", 0)


def test_a_call_after_chunks_that_overlap(ctx):
    """Chunks that overlap are more work than there is room for: whatever such a call leaves in its own rows, the next one is right."""
    t, n_seqs = 64, 200
    bad = Chunks(_heads(H8B), [1] * t, [3000] * t, page_size=64, seed=36)
    lens, table = _int32([3000] * n_seqs), bad.table[:1].repeat(n_seqs, 1).contiguous()
    ends = [0, t] * (n_seqs // 2) + [0]                     # every other sequence has all the rows
    ctx.ensure_attention_workspace(bad.h, t, n_seqs)
    ctx.chunk_attention(bad.h, bad.q, _int32(ends), lens, 1, bad.cache, table, bad.o)
    for _ in range(2):
        good = Chunks(_heads(H8B), [1, 1], [9000, 5000], page_size=64, seed=37)
        good.run(ctx)
        good.check("after overlapping chunks")


@pytest.mark.parametrize("h", [H8B, H7B, H1B, MHA], ids=lambda h: "%d_%d_%d" % h)
def test_a_workspace_for_the_largest_call_is_enough_for_smaller_ones(h):
    """Sized once, for calls that are not split themselves; a call of fewer tokens or sequences finds enough, and the workspace stays."""
    ctx = B.Context(0)
    try:
        ctx.ensure_attention_workspace(_heads(h), 16384, 48)
        ws = ctx._ws
        for new, lens in (([1], [9000]), ([5], [3000]), ([130], [4000]), ([1] * 20, list(range(100, 2100, 100))), ([60, 1, 1], [2000, 900, 3000])):
            c = Chunks(_heads(h), new, lens, page_size=64, seed=41)
            ctx.chunk_attention(c.h, c.q, c.starts, c.ctx_lens, c.max_chunk, c.cache, c.table, c.o, lse=c.lse)
            c.check(f"{h} in a workspace for more")
            c.run(ctx)
            assert ctx._ws is ws
    finally:
        torch.cuda.synchronize()
        ctx.close()


def test_creating_a_context_waits_for_no_other_stream(ctx):
    """Nor does it wait for its own; the counters are zero when its first call comes."""
    tick = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    tick[0].record()
    torch.cuda._sleep(1000000)
    tick[1].record()
    torch.cuda.synchronize()
    cycles = int(1000000 * 300.0 / tick[0].elapsed_time(tick[1]))          # 0.3 s
    c = Chunks(_heads(H8B), [1], [4000], seed=42)
    torch.cuda.synchronize()
    for busy, own in ((torch.cuda.Stream(), torch.cuda.Stream()), (torch.cuda.Stream(),) * 2, (torch.cuda.default_stream(),) * 2):
        with torch.cuda.stream(busy):
            torch.cuda._sleep(cycles)
            done = torch.cuda.Event()
            done.record()
        fresh = B.Context(0, stream=own)
        waited = done.query()
        torch.cuda.synchronize()
        assert not waited
        with torch.cuda.stream(own):
            c.o.fill_(7.0)
            c.run(fresh)
        torch.cuda.synchronize()
        c.check("in a fresh context")
        fresh.close()


def test_a_context_created_while_its_stream_is_captured(ctx):
    """In the mode that allows allocations; the graph holds nothing of it, and its first call may come before a replay."""
    c, x = Chunks(_heads(H8B), [1], [4000], seed=43), torch.ones(1000, device=DEV)
    graph, own = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=own, capture_error_mode="relaxed"):
        x.add_(1)
        fresh = B.Context(0, stream=own)
    try:
        for rep in range(3):
            with torch.cuda.stream(own):
                c.o.fill_(7.0)
                c.run(fresh)
                graph.replay()
            torch.cuda.synchronize()
            c.check(f"before replay {rep}")
            assert bool((x == 2 + rep).all())
    finally:
        torch.cuda.synchronize()
        fresh.close()


@pytest.mark.parametrize("nats", [60.0, 320.0], ids=["weights of e^-60", "weights of e^-320"])
@pytest.mark.parametrize("h", [H8B, H1B], ids=lambda h: "%d_%d_%d" % h)
def test_infinities_of_keys_with_small_weights(ctx, h, nats):
    """One key takes nearly all the weight.  An infinity among the others' values is in the rows that see it, as itself where its weight
    is 2^-87 and as itself or NaN where that underflows, in tiles that all rows see whole, at their edges, before and behind that key and in pieces
    without it; other channels and rows are as without it."""
    hd, inf = h[2], float("inf")

    def check(o, lse, heads, q, k, v, what):
        ref = _reference(heads, *(x.unflatten(1, (-1, hd)) if x.dim() == 2 else x for x in (q, k, v)))
        got = o.double().reshape(ref[0].shape)
        if nats > 88:
            got = torch.where(torch.isnan(got) & torch.isinf(ref[0]), ref[0], got)
        _check(got, lse, ref, hd, k.shape[0], what)

    for causal, window in ((True, 0), (True, 300), (False, 0)):
        p = Prompt(_heads(h, causal=causal, window=window, scale=1.0), [900], seed=44)
        p.q.zero_()
        p.k.zero_()
        p.q[:, ::hd] = 1.0
        p.k[400, ::hd] = nats
        for channel, (key, x) in enumerate(((10, inf), (390, -inf), (399, inf), (401, inf), (600, -inf), (899, inf))):
            p.v[key, channel::hd] = x
        p.run(ctx)
        check(p.o, p.lse, p.h, p.q, p.k, p.v, f"prompt, causal {causal}, window {window}")
    for new, keys, window in ((1, 9000, 0), (3, 5000, 0), (8, 6000, 1500), (40, 4000, 0), (200, 4000, 0), (200, 4000, 1500)):
        c = Chunks(_heads(h, window=window, scale=1.0), [new], [keys], page_size=64, seed=45)
        c.q.zero_()
        c.q[:, ::hd] = 1.0
        c.k[0].zero_()
        c.k[0][keys - 700, :, 0] = nats
        for channel, key in enumerate((10, keys - 1400, keys - 701, keys - 699, keys - 300, keys - new - 1, keys - new, keys - 1)):
            c.v[0][key, :, channel] = inf if channel % 2 else -inf
        j = torch.arange(keys, device=DEV)
        for pages, x in ((c.k_pages, c.k[0]), (c.v_pages, c.v[0])):
            pages[c.table[0].long()[j // 64], :, j % 64] = x
        c.run(ctx)
        check(c.o, c.lse, c.h, c.q.unflatten(1, (-1, hd)), c.k[0], c.v[0], f"{new} tokens over {keys} keys, window {window}")


def _clamped(starts, s, t):
    t0 = min(max(starts[s], 0), t)
    return t0, min(max(starts[s + 1], t0), t)


@pytest.mark.parametrize("h", [H8B, H1B], ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("new", [[1, 1], [7, 6], [40, 70], [200, 300]], ids=str)
def test_what_is_out_of_range_is_clamped_and_touches_nothing_else(ctx, h, new):
    """Starts, lengths and pages out of range against the clamped ones in float64; margins around the outputs and the cache stay."""
    hd, qw, lens, t = h[2], h[0] * h[2], [100, 80], sum(new) + 3
    for what, change in (("nothing", lambda c: None), ("page", lambda c: c.table[1, 0].fill_(1 << 30)), ("negative page", lambda c: c.table[1, 1].fill_(-5)),
                         ("length", lambda c: c.ctx_lens[0].fill_(1 << 30)), ("negative length", lambda c: c.ctx_lens[0].fill_(-3)),
                         ("end", lambda c: c.starts[2].fill_(1 << 30)), ("descending starts", lambda c: c.starts[1].fill_(-9)),
                         ("start", lambda c: c.starts[0].fill_(-(1 << 31))), ("all behind", lambda c: c.starts.fill_(2147483647))):
        c = Chunks(_heads(h), new, lens, unused=0.0, behind=3, seed=46)
        change(c)
        out, lse = torch.full((t + 16, qw + 16), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((t + 16, h[0]), 7.0, device=DEV)
        c.o, c.lse = out[8:8 + t, 8:8 + qw], lse[8:8 + t]
        pages = c.k_pages.clone(), c.v_pages.clone()
        c.run(ctx)
        torch.cuda.synchronize()
        starts, n_keys, table = c.starts.tolist(), c.ctx_lens.tolist(), c.table.long()
        table = torch.where((table < 0) | (table >= c.k_pages.shape[0]), 0, table)
        left = torch.ones(t, dtype=torch.bool, device=DEV)
        for s in range(2):
            t0, t1 = _clamped(starts, s, t)
            j = torch.arange(min(max(n_keys[s], 0), table.shape[1] * 16), device=DEV)
            k, v = (x[table[s][j // 16], :, j % 16] for x in pages)
            _check(c.o[t0:t1], c.lse[t0:t1], _reference(c.h, c.q[t0:t1].unflatten(1, (-1, hd)), k, v), hd, len(j), f"{h} {new} {what}, sequence {s}")
            left[t0:t1] = False
        assert bool((c.o[left] == 7.0).all()) and bool((c.lse[left] == 7.0).all()), f"{what}: rows of no sequence"
        c.o.fill_(7.0)
        c.lse.fill_(7.0)
        assert bool((out == 7.0).all()) and bool((lse == 7.0).all()), f"{what}: around the outputs"
        assert torch.equal(c.k_pages, pages[0]) and torch.equal(c.v_pages, pages[1]), f"{what}: the cache"


@pytest.mark.parametrize("h", [H8B, H1B], ids=lambda h: "%d_%d_%d" % h)
def test_prompts_with_starts_out_of_range(ctx, h):
    hd, qw, t = h[2], h[0] * h[2], 330
    for starts in ([-5, 130, 330], [0, 130, 1 << 30], [100, 40, 330], [-(1 << 31), 2147483647, 2147483647], [330, 400, 500], [200, 100, 50]):
        p = Prompt(_heads(h), [130, 200], seed=47)
        p.starts.copy_(_int32(starts))
        out, lse = torch.full((t + 16, qw + 16), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((t + 16, h[0]), 7.0, device=DEV)
        p.o, p.lse = out[8:8 + t, 8:8 + qw], lse[8:8 + t]
        p.run(ctx)
        torch.cuda.synchronize()
        left = torch.ones(t, dtype=torch.bool, device=DEV)
        for s in range(2):
            t0, t1 = _clamped(starts, s, t)
            part = [x[t0:t1].unflatten(1, (-1, hd)) for x in (p.q, p.k, p.v)]
            _check(p.o[t0:t1], p.lse[t0:t1], _reference(p.h, *part), hd, t1 - t0, f"{h} starts {starts}, sequence {s}")
            left[t0:t1] = False
        assert bool((p.o[left] == 7.0).all()) and bool((p.lse[left] == 7.0).all()), f"{starts}: rows of no sequence"
        p.o.fill_(7.0)
        p.lse.fill_(7.0)
        assert bool((out == 7.0).all()) and bool((lse == 7.0).all()), f"{starts}: around the outputs"


def test_a_workspace_that_grows_leaves_calls_in_flight_alone():
    """Its memory comes back when the context's stream is through with it, whatever stream it was allocated on."""
    own = torch.cuda.Stream()
    ctx = B.Context(0, stream=own)
    try:
        c = Chunks(_heads(H8B), [130], [4000], page_size=64, seed=48)
        ctx.ensure_attention_workspace(c.h, 130, 1)
        size = ctx._ws.numel()
        torch.cuda.synchronize()
        with torch.cuda.stream(own):
            torch.cuda._sleep(20000000)
        ctx.chunk_attention(c.h, c.q, c.starts, c.ctx_lens, c.max_chunk, c.cache, c.table, c.o, lse=c.lse)
        ctx.ensure_attention_workspace(c.h, 2048, 32)
        assert ctx._ws.numel() > size
        others = [torch.full((size,), 255, dtype=torch.uint8, device=DEV) for _ in range(2)]
        torch.cuda.synchronize()
        c.check("while the workspace grew")
        del others
    finally:
        torch.cuda.synchronize()
        ctx.close()


def test_no_memory_for_a_larger_workspace(ctx):
    """The one that there was is gone; a call that needs one is refused and does not write where it was."""
    fresh = B.Context(0)
    try:
        c = Chunks(_heads(H8B), [1], [4000], seed=49)
        c.run(fresh)
        with pytest.raises(torch.OutOfMemoryError):
            fresh._ensure(1 << 45)
        _refused(5, fresh.chunk_attention, c.h, c.q, c.starts, c.ctx_lens, 1, c.cache, c.table, c.o)
        c.o.fill_(7.0)
        c.run(fresh)
        c.check("in a workspace of its own again")
    finally:
        torch.cuda.synchronize()
        fresh.close()
