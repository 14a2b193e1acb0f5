"""A cache in 8 bits: the write of new tokens against a model of it in float64, to the bit, and attention over it against
softmax(scale q k^T) v in float64 of the values that the codes and scales stand for.

Those values are bf16 numbers, so attention's bars are the ones of test_gpu_attention.  The write rounds each value once, to
the nearest code (ties to even): no bar."""
import math

import pytest
import torch

from paper_2602_00397_amd import binding as B
from test_gpu_attention import DEV, H1B, H7B, H8B, MHA, MQA, TINY, _bf16, _check, _clamped, _gen, _heads, _int32, _reference, _refused, _starts, ctx  # noqa: F401

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def _table():
    """What each code stands for, from the format: sign, four bits of exponent (bias 7), three of mantissa; no infinities."""
    c = torch.arange(256, dtype=torch.float64)
    e, m = (c // 8) % 16, c % 8
    x = torch.where(e > 0, (8 + m) * 2.0 ** (e - 10), m * 2.0 ** -9)
    x[127] = math.nan
    return torch.where(c < 128, x, -torch.cat([x[:128], x[:128]])).to(DEV)


def _decode(codes, scales):
    """Pages of codes and their scales -> float64 values."""
    x = _table()[codes.view(torch.uint8).long()]
    return x * scales.double().repeat_interleave(codes.shape[-2] // scales.shape[-1], dim=-1)[..., None]


def _encode(x):
    """float64 values within +-448 -> codes, to nearest, ties to the even code; infinities and NaN -> NaN (a code of 127, whatever the sign)."""
    steps = _table()[:127]
    a = x.abs().clamp(max=448.0)
    hi = torch.searchsorted(steps, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = steps[hi] - a, a - steps[lo]
    code = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = torch.where(torch.isfinite(x), code, torch.full_like(code, 127))
    return (code + 128 * torch.signbit(x)).to(torch.uint8)


class Cache8:
    """Sequences' keys and values in pages of 8 bits in shuffled order; places and blocks without a key are NaN."""

    def __init__(self, h, lens, page_size, scale_tokens, gen, far=0):
        self.h, self.lens, self.page_size, self.scale_tokens = h, lens, page_size, scale_tokens
        used = [-(-n // page_size) for n in lens]
        n_pages = sum(used) + 3 + far
        shape = (n_pages, h.n_kv_heads, page_size, h.head_dim)
        order = (torch.randperm(n_pages - far, device=DEV, generator=gen) + far).to(torch.int32)
        self.table = torch.full((len(lens), max(used + [1]) + 1), -1, dtype=torch.int32, device=DEV)
        at = 0
        for i, n in enumerate(used):
            self.table[i, :n] = order[at:at + n]
            at += n
        self.k_pages, self.v_pages = (torch.full(shape, 0x7f, dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2))
        self.k_scale, self.v_scale = (torch.full((n_pages, h.n_kv_heads, page_size // scale_tokens), math.nan, device=DEV) for _ in range(2))
        for codes, scale in ((self.k_pages, self.k_scale), (self.v_pages, self.v_scale)):
            for i, n in enumerate(lens):
                j = torch.arange(n, device=DEV)
                page = self.table[i].long()[j // page_size]
                # one code in 50 is NaN's neighbour 448, as a block's largest value is
                x = (torch.randn((n, h.n_kv_heads, h.head_dim), device=DEV, generator=gen) * 100).clamp(-448, 448)
                codes.view(torch.uint8)[page, :, j % page_size] = x.to(E4M3).view(torch.uint8)
                scale[page, :, j % page_size // scale_tokens] = torch.exp2(
                    torch.randint(-9, -5, (-(-n // scale_tokens), h.n_kv_heads), device=DEV, generator=gen).float())[j // scale_tokens]
        self.cache = B.paged_cache8(self.k_pages, self.v_pages, self.k_scale, self.v_scale)

    def value(self, which, i, n):
        """The first n keys or values of sequence i, float64 [n][kv_heads][hd]."""
        page = self.table[i, :-(-n // self.page_size)].long()
        page = torch.where((page < 0) | (page >= self.k_pages.shape[0]), 0, page)
        pages, scale = (self.k_pages, self.k_scale) if which == "k" else (self.v_pages, self.v_scale)
        x = _decode(pages.view(torch.uint8)[page].view(E4M3), scale[page])
        return x.transpose(1, 2).reshape(-1, self.h.n_kv_heads, self.h.head_dim)[:n]

    def put(self, i, key, head, channel, code, which="v"):
        pages = self.k_pages if which == "k" else self.v_pages
        pages.view(torch.uint8)[self.table[i, key // self.page_size].long(), head, key % self.page_size, channel] = code


class Chunks8(Cache8):
    def __init__(self, h, new, lens, page_size=64, scale_tokens=32, seed=1, behind=0, max_chunk=None, far=0):
        gen = _gen(seed)
        super().__init__(h, lens, page_size, scale_tokens, gen, far)
        self.new, t = new, sum(new) + behind
        self.q = _bf16(gen, t, h.n_heads * h.head_dim)
        self.starts, self.ctx_lens = _int32(_starts(new)), _int32(lens)
        self.max_chunk = max_chunk or max(max(new), 1)
        self.o = torch.full((t, h.n_heads * h.head_dim), 7.0, dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((t, h.n_heads), 7.0, device=DEV)

    def run(self, ctx):
        ctx.ensure_attention_workspace(self.h, self.q.shape[0], len(self.new))
        ctx.chunk_attention8(self.h, self.q, self.starts, self.ctx_lens, self.max_chunk, self.cache, self.table, self.o, lse=self.lse)

    def check(self, what):
        hd, t0 = self.h.head_dim, 0
        for i, n in enumerate(self.new):
            ref = _reference(self.h, self.q[t0:t0 + n].unflatten(1, (-1, hd)), self.value("k", i, self.lens[i]), self.value("v", i, self.lens[i]))
            _check(self.o[t0:t0 + n], self.lse[t0:t0 + n], ref, hd, self.lens[i], f"{what}, sequence {i}: {n} over {self.lens[i]}")
            t0 += n
        assert bool((self.o[t0:] == 7.0).all()) and bool((self.lse[t0:] == 7.0).all()), "rows behind the last sequence changed"


# ------------------------------------------------------------------ attention

@pytest.mark.parametrize("h", [H8B, H7B, H1B, TINY, MHA, MQA], ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("lens", [[1], [2, 33], [64, 1, 700, 31, 32], [5000]], ids=str)
def test_single_tokens(ctx, h, lens):  # noqa: F811
    c = Chunks8(_heads(h), [1] * len(lens), lens, behind=2)
    c.run(ctx)
    c.check(f"tokens {h}")


@pytest.mark.parametrize("h", [H8B, H7B, H1B, MHA], ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("n", [2, 5, 8, 13, 16, 17, 33, 64, 65, 130, 257])
def test_chunks_of_every_kernel(ctx, h, n):  # noqa: F811
    c = Chunks8(_heads(h), [n], [n + 400], seed=n)
    c.run(ctx)
    c.check(f"chunk {h} {n}")


@pytest.mark.parametrize("page_size,scale_tokens", [(16, 8), (16, 16), (32, 8), (64, 64), (128, 128), (256, 32), (4096, 128)])
@pytest.mark.parametrize("h", [H8B, H1B], ids=lambda h: "%d_%d_%d" % h)
def test_mixed_batches_page_sizes_and_scales(ctx, h, page_size, scale_tokens):  # noqa: F811
    c = Chunks8(_heads(h), [1, 90, 1, 0, 200, 7, 1], [500, 90, 1, 77, 1000, 650, 2048], page_size=page_size, scale_tokens=scale_tokens,
                seed=9, behind=5)
    c.run(ctx)
    c.check(f"mixed {h} pages of {page_size}, scales of {scale_tokens}")


@pytest.mark.parametrize("h", [(64, 64, 64), (64, 64, 128), (48, 16, 128)], ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 300)])
def test_work_for_every_cu_in_large_tiles(ctx, h, causal, window):  # noqa: F811
    t = -(-256 * 500 // h[0])
    new = [t - 60, 1, 40, 0, 19]
    c = Chunks8(_heads(h, causal, window), new, [t + 200, 333, 40, 5, 7], page_size=32, seed=32, behind=2)
    for i, key, ch in ((0, t + 199, 3), (0, t + 100, 7), (1, 332, 0), (2, 5, 60)):
        c.put(i, key, 0, ch, 0x7f)
    c.run(ctx)
    c.check(f"{h} causal {causal} window {window}")


@pytest.mark.parametrize("new", [[1, 1, 1, 1], [12, 3, 40, 9], [150, 3, 300, 9]], ids=str)
def test_fewer_keys_than_tokens_or_none(ctx, new):  # noqa: F811
    for h in (H8B, H1B):
        c = Chunks8(_heads(h), new, [0, 2, 33, 9], seed=10)
        c.run(ctx)
        c.check(f"short contexts {new}")


@pytest.mark.parametrize("causal,window", [(False, 0), (True, 1), (True, 37), (True, 64), (True, 500)])
@pytest.mark.parametrize("new", [[1, 1, 1], [6, 1, 3], [140, 1, 60]], ids=str)
def test_windows_and_no_causal_mask(ctx, new, causal, window):  # noqa: F811
    for h in (H7B, H1B):
        c = Chunks8(_heads(h, causal, window), new, [1500, 64, 333], page_size=32, scale_tokens=8, seed=11)
        c.run(ctx)
        c.check(f"{h} {new} causal {causal} window {window}")


@pytest.mark.parametrize("new", [[1, 1], [4, 2], [9, 2], [100, 70]], ids=str)
def test_values_that_are_not_finite(ctx, new):  # noqa: F811
    """NaN codes, and a block whose scale makes infinities: both reach the rows that see them and no others."""
    for h in (H8B, H7B, H1B):
        c = Chunks8(_heads(h), new, [9000, 200], scale_tokens=8, seed=14)
        for key, ch in ((8999, 4), (9000 - new[0], 7), (17, 0), (5000, 1)):
            c.put(0, key, 0, ch, 0x7f if ch else 0xff)
        # 2^122 * 448 is beyond bf16, and so is 2^122 * 64; the block's other values are 0
        page, block = c.table[1, 199 // 64].long(), 199 % 64 // 8
        c.v_pages.view(torch.uint8)[page, :, block * 8:block * 8 + 8] = 0
        c.v_scale[page, :, block] = 2.0 ** 122
        c.put(1, 199, 0, 9, 0x7e)
        c.put(1, 198, 0, 10, 0x80 | 0x68)
        ref_v = c.value("v", 1, 200)
        assert bool((ref_v.abs() > 3.4e38).any())
        big = c.value
        c.value = lambda which, i, n: big(which, i, n).float().to(torch.bfloat16).double()
        c.run(ctx)
        c.check(f"{h} {new} not finite")


@pytest.mark.parametrize("n_seqs,new", [(70, 5), (130, 1), (67, 150)])
def test_many_sequences(ctx, n_seqs, new):  # noqa: F811
    for h in (H8B, TINY):
        lens_new = [1 if new == 150 and i < 66 else min(new, i % (new + 1)) for i in range(n_seqs)]
        lens = [n + (53 * i) % 300 for i, n in enumerate(lens_new)]
        lens[65] = lens_new[65] + 5000
        c = Chunks8(_heads(h), lens_new, lens, page_size=32, scale_tokens=16, seed=38, behind=1)
        c.run(ctx)
        c.check(f"{n_seqs} sequences of up to {new} tokens")


@pytest.mark.parametrize("hint", [1, 3, 30, 300])
def test_other_lengths_than_the_host_expected(ctx, hint):  # noqa: F811
    c = Chunks8(_heads(H8B), [1, 20, 0, 279], [600, 20, 5, 900], seed=13, max_chunk=hint)
    c.run(ctx)
    c.check(f"longest chunk taken for {hint}")


def test_rows_apart_and_without_log_sums(ctx):  # noqa: F811
    for h, new in ((H8B, [1, 1]), (H7B, [4, 2]), (H8B, [100, 3]), (H1B, [70, 1])):
        c = Chunks8(_heads(h), new, [5000, 77], seed=40)
        w = c.q.shape[1]
        q, o = torch.zeros((c.q.shape[0], w + 24), dtype=torch.bfloat16, device=DEV), torch.full((c.q.shape[0], w + 40), 7.0, dtype=torch.bfloat16, device=DEV)
        q[:, 16:16 + w] = c.q
        c.run(ctx)
        c.check(f"{h} {new}")
        ctx.chunk_attention8(c.h, q[:, 16:16 + w], c.starts, c.ctx_lens, c.max_chunk, c.cache, c.table, o[:, 8:8 + w])
        assert bool((o[:, :8] == 7.0).all()) and bool((o[:, 8 + w:] == 7.0).all())
        assert torch.equal(o[:, 8:8 + w].contiguous().view(torch.int16), c.o.view(torch.int16))


def test_scales_over_their_whole_range(ctx):  # noqa: F811
    """A scale's exponent is all that counts; values of the least and the largest scales are exact.  (Larger ones are outside what the
    cache is defined for: a row's sum is kept before it is divided by the sum of its weights, which are up to 2^8 each, so with 256
    keys of 448 * 2^119 it may pass fp32's 2^128; with 2^80 it stays below 2^(9 + 80 + 8 + 8).)"""
    for h, new in ((H8B, [1]), (H8B, [40]), (H1B, [1]), (H1B, [90])):
        c = Chunks8(_heads(h), new, [256], scale_tokens=8, seed=50)
        page, block = c.table[0, 1].long(), 3
        c.v_scale[c.table[0, 0].long(), :, 2] = 2.0 ** -110
        c.v_scale[page, :, block] = 2.0 ** 80
        c.run(ctx)
        c.check(f"{h} {new} scales from 2^-110 to 2^80")
        first = c.o.clone()
        c.k_scale *= 1.75
        c.v_scale[c.table[0, 2].long()] *= 1.25
        c.run(ctx)
        assert torch.equal(c.o.view(torch.int16), first.view(torch.int16)), "a scale's mantissa counts"


def test_cache_beyond_32_bit_offsets(ctx):  # noqa: F811
    """Pages behind more than 4 GiB of codes."""
    for new in (1, 150):
        c = Chunks8(_heads(H8B), [new], [700], seed=16, far=66000)
        assert int(c.table[0, 0]) * 8 * 64 * 128 > 1 << 32
        c.run(ctx)
        c.check(f"far pages, {new} tokens")
        del c


def test_the_same_call_gives_the_same_bits(ctx):  # noqa: F811
    for new, lens in (([1] * 5, [4000, 3, 900, 77, 1]), ([128], [3000]), ([1, 200, 1], [900, 400, 2000])):
        c = Chunks8(_heads(H8B), new, lens, seed=17)
        c.run(ctx)
        first = c.o.clone(), c.lse.clone()
        for _ in range(5):
            c.o.fill_(3.0)
            c.run(ctx)
            assert torch.equal(c.o.view(torch.int16), first[0].view(torch.int16)) and torch.equal(c.lse, first[1])


@pytest.mark.parametrize("h", [H8B, H1B], ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("new", [[1, 1], [7, 6], [40, 70], [200, 300]], ids=str)
def test_what_is_out_of_range_is_clamped_and_touches_nothing_else(ctx, h, new):  # noqa: F811
    hd, qw, lens, t = h[2], h[0] * h[2], [100, 80], sum(new) + 3
    for what, change in (("nothing", lambda c: None), ("page", lambda c: c.table[1, 0].fill_(1 << 30)), ("negative page", lambda c: c.table[1, 1].fill_(-5)),
                         ("length", lambda c: c.ctx_lens[0].fill_(1 << 30)), ("negative length", lambda c: c.ctx_lens[0].fill_(-3)),
                         ("end", lambda c: c.starts[2].fill_(1 << 30)), ("descending starts", lambda c: c.starts[1].fill_(-9))):
        c = Chunks8(_heads(h), new, lens, page_size=16, scale_tokens=8, behind=3, seed=46)
        for x in (c.k_pages, c.v_pages):                           # (unused pages and places are read here)
            codes = x.view(torch.uint8)
            codes[codes == 0x7f] = 0x30
        for x in (c.k_scale, c.v_scale):
            x.nan_to_num_(0.25)
        change(c)
        out, lse = torch.full((t + 16, qw + 16), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((t + 16, h[0]), 7.0, device=DEV)
        c.o, c.lse = out[8:8 + t, 8:8 + qw], lse[8:8 + t]
        held = [x.clone() for x in (c.k_pages.view(torch.uint8), c.v_pages.view(torch.uint8), c.k_scale, c.v_scale)]
        c.run(ctx)
        torch.cuda.synchronize()
        starts, n_keys = c.starts.tolist(), c.ctx_lens.tolist()
        left = torch.ones(t, dtype=torch.bool, device=DEV)
        for s in range(2):
            t0, t1 = _clamped(starts, s, t)
            keys = min(max(n_keys[s], 0), c.table.shape[1] * 16)
            _check(c.o[t0:t1], c.lse[t0:t1], _reference(c.h, c.q[t0:t1].unflatten(1, (-1, hd)), c.value("k", s, keys), c.value("v", s, keys)), hd,
                   keys, f"{h} {new} {what}, sequence {s}")
            left[t0:t1] = False
        assert bool((c.o[left] == 7.0).all()) and bool((c.lse[left] == 7.0).all()), f"{what}: rows of no sequence"
        c.o.fill_(7.0)
        c.lse.fill_(7.0)
        assert bool((out == 7.0).all()) and bool((lse == 7.0).all()), f"{what}: around the outputs"
        assert all(torch.equal(x, y) for x, y in zip(held, (c.k_pages.view(torch.uint8), c.v_pages.view(torch.uint8), c.k_scale, c.v_scale)))


# ------------------------------------------------------------------ the write

def _append_model(c, k, v, starts, lens, held):
    """What the pages and scales hold after the write, in float64, block by block, from what they held."""
    st, ps, out = c.scale_tokens, c.page_size, []
    n_pages, stride = c.k_pages.shape[0], c.table.shape[1]
    for x, codes, scales in ((k, held[0], held[2]), (v, held[1], held[3])):
        codes, scales = codes.clone(), scales.clone()
        x = x.double().unflatten(1, (c.h.n_kv_heads, -1))
        for s in range(len(lens)):
            t0, t1 = _clamped(starts, s, x.shape[0])
            keys = min(max(lens[s], 0), stride * ps)
            at = max(0, keys - (t1 - t0))
            while t1 > t0 and at < keys:
                end = min(keys, at // st * st + st)
                page, block, p = int(c.table[s, at // ps]), at % ps // st, at % ps
                rows = x[t1 - (keys - at):t1 - (keys - at) + end - at].transpose(0, 1)
                if 0 <= page < n_pages:
                    top = torch.where(torch.isfinite(rows), rows.abs(), 0.0).amax(dim=(1, 2))
                    need = torch.full_like(top, 2.0 ** -110)
                    for e in range(-110, 80):
                        need = torch.where(top > 448.0 * 2.0 ** e, 2.0 ** (e + 1), need)
                    if at % st:
                        old = scales[page, :, block].double()
                        need = torch.maximum(need, old)
                        older = codes[page, :, block * st:p]
                        again = _encode(_table()[older.long()] * (old / need)[:, None, None])
                        nan = older % 128 == 127
                        same = (need == old)[:, None, None]
                        codes[page, :, block * st:p] = torch.where(nan | same, older, again)
                    codes[page, :, p:p + end - at] = _encode(rows / need[:, None, None])
                    scales[page, :, block] = need.float()
                at = end
        out += [codes, scales]
    return out[0], out[2], out[1], out[3]


def _same_codes(got, want):
    """Equal but for the sign of NaN."""
    a, b = got.view(torch.uint8), want.view(torch.uint8)
    return bool(((a == b) | ((a % 128 == 127) & (b % 128 == 127))).all())


class Append:
    """New tokens behind what a cache holds."""

    def __init__(self, h, new, lens, page_size=64, scale_tokens=32, seed=1, behind=0, strided=True):
        gen = _gen(seed)
        self.c = Cache8(_heads(h), lens, page_size, scale_tokens, gen)
        kw, t = h[1] * h[2], sum(new) + behind
        kv = _bf16(gen, t, 2 * kw + 24)
        self.k, self.v = (kv[:, 8:8 + kw], kv[:, 16 + kw:16 + 2 * kw]) if strided else (kv[:, :kw].contiguous(), kv[:, kw:2 * kw].contiguous())
        self.starts, self.lens = _int32(_starts(new)), _int32(lens)

    def held(self):
        c = self.c
        return [x.clone() for x in (c.k_pages.view(torch.uint8), c.v_pages.view(torch.uint8), c.k_scale, c.v_scale)]

    def run(self, ctx):
        ctx.cache8_append(self.c.h, self.k, self.v, self.starts, self.lens, self.c.cache, self.c.table)

    def check(self, held, what):
        want = _append_model(self.c, self.k, self.v, self.starts.tolist(), self.lens.tolist(), held)
        got = self.held()
        for name, a, b in zip(("k", "v"), got[:2], want[:2]):
            assert _same_codes(a, b), f"{what}: codes of {name}, {int((a != b).sum())} of {a.numel()} differ"
        for name, a, b in zip(("k", "v"), got[2:], want[2:]):
            assert torch.equal(a.nan_to_num(-1.0), b.nan_to_num(-1.0)), f"{what}: scales of {name}"

    def run_and_check(self, ctx, what):
        held = self.held()
        self.run(ctx)
        self.check(held, what)


@pytest.mark.parametrize("page_size,scale_tokens", [(16, 8), (16, 16), (32, 8), (64, 64), (128, 128), (256, 32), (4096, 128)])
@pytest.mark.parametrize("h", [H8B, TINY, MHA, MQA], ids=lambda h: "%d_%d_%d" % h)
def test_append_is_the_model_to_the_bit(ctx, h, page_size, scale_tokens):  # noqa: F811
    for new, lens in (([1], [1]), ([1] * 5, [1, 64, 65, 700, 129]), ([300], [300]), ([7, 0, 250, 1, 33], [300, 9, 251, 17, 33]), ([5, 3], [3, 0])):
        a = Append(h, new, lens, page_size, scale_tokens, seed=len(new), behind=2)
        a.run_and_check(ctx, f"{h} {new} behind {lens}, pages of {page_size}, scales of {scale_tokens}")


def test_append_token_by_token_and_in_one_call(ctx):  # noqa: F811
    """A scale that grows with its block's values: older codes are rounded again, each time as the model does."""
    for h in (H8B, H1B):
        a = Append(h, [70], [70], page_size=32, scale_tokens=16, seed=3)
        a.k *= torch.exp2(torch.arange(70, device=DEV) % 16 // 3)[:, None].to(torch.bfloat16)      # grows within blocks
        a.v[5::7] *= 64
        for t in range(70):
            held = a.held()
            one = Append.__new__(Append)
            one.c, one.k, one.v, one.starts, one.lens = a.c, a.k[t:t + 1], a.v[t:t + 1], _int32([0, 1]), _int32([t + 1])
            one.run(ctx)
            one.check(held, f"{h} token {t}")


def test_append_values_of_every_size(ctx):  # noqa: F811
    """Zeros, the least and the largest bf16 numbers, infinities and NaN."""
    for h in (TINY, H8B):
        a = Append(h, [160], [160], page_size=32, scale_tokens=16, seed=4)
        kw = h[1] * h[2]
        bits = torch.randint(0, 65536, (160, kw), device=DEV, generator=_gen(5), dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
        a.k[:16] = 0
        a.k[16:32] = bits[16:32]                               # with infinities and NaN
        a.k[32:48] = 3.3895e38
        a.k[48:64] = 1e-38
        a.k[64:80] = float("inf")
        a.k[80:96] = float("nan")
        a.k[96:112] = bits[96:112].nan_to_num(0, 0, 0)
        a.k[112] = 448.0
        a.k[113:128] = torch.linspace(-448, 448, 15, device=DEV)[:, None].to(torch.bfloat16)
        a.v.copy_(bits)
        a.run_and_check(ctx, f"{h} values of every size")


def test_append_where_pages_are_out_of_range(ctx):  # noqa: F811
    """Nothing is written for those tokens, nor anywhere else."""
    for h in (H8B, H1B):
        for what, change in (("page", lambda a: a.c.table[1, 0].fill_(1 << 30)), ("negative page", lambda a: a.c.table[0, 6].fill_(-5)),
                             ("length", lambda a: a.lens[0].fill_(1 << 30)), ("negative length", lambda a: a.lens[0].fill_(-3)),
                             ("fewer keys", lambda a: a.lens.copy_(_int32([3, 20]))),
                             ("end", lambda a: a.starts[2].fill_(1 << 30)), ("descending starts", lambda a: a.starts[1].fill_(-9)),
                             ("no rows", lambda a: a.starts.fill_(-1))):
            a = Append(h, [40, 30], [100, 80], page_size=16, scale_tokens=8, seed=6, behind=3)
            for x in (a.c.k_scale, a.c.v_scale):
                x.nan_to_num_(0.25)
            change(a)
            a.run_and_check(ctx, f"{h} {what}")


def test_append_to_many_sequences(ctx):  # noqa: F811
    """More than a wavefront looks at together."""
    new = [i % 4 for i in range(200)]
    a = Append(TINY, new, [n + (37 * i) % 60 for i, n in enumerate(new)], page_size=16, scale_tokens=8, seed=7)
    a.run_and_check(ctx, "200 sequences")
    n, ps = 3000, 16
    h = _heads(TINY)
    gen = _gen(8)
    k, v = _bf16(gen, n, 128), _bf16(gen, n, 128)
    pages = [torch.zeros((n, 2, ps, 64), dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2)]
    scales = [torch.zeros((n, 2, 2), device=DEV) for _ in range(2)]
    table = torch.randperm(n, device=DEV, generator=gen).to(torch.int32)[:, None].contiguous()
    ctx.cache8_append(h, k, v, _int32(list(range(n + 1))), _int32([1] * n), B.paged_cache8(*pages, *scales), table)
    for x, codes, scale in zip((k, v), pages, scales):
        got = _decode(codes, scale)[table[:, 0].long(), :, 0].reshape(n, 128)
        assert bool(((got - x.double()).abs() <= x.double().abs() * 2.0 ** -4 + scale[table[:, 0].long(), :, 0].double().repeat_interleave(64, dim=1) * 2.0 ** -10).all())
        assert not codes.view(torch.uint8)[:, :, 1:].any() and not scale[:, :, 1].any()


@pytest.mark.parametrize("n_seqs", [64, 65, 300, 4100])
@pytest.mark.parametrize("most", [2, 40])
def test_append_to_many_ragged_sequences(ctx, n_seqs, most):  # noqa: F811
    """One call against calls of 50 sequences, to the bit: few tokens to a sequence and many, with empty sequences throughout."""
    new = [(i * i * 7 + i // 64) % (most + 1) for i in range(n_seqs)]
    a = Append(TINY, new, [n + (37 * i) % 30 for i, n in enumerate(new)], page_size=16, scale_tokens=8, seed=17, behind=2)
    a.starts += 1                                  # (a row in front of the first sequence's)
    before = a.held()
    for s in range(0, n_seqs, 50):
        e = min(n_seqs, s + 50)
        ctx.cache8_append(a.c.h, a.k, a.v, a.starts[s:e + 1].clone(), a.lens[s:e].clone(), a.c.cache, a.c.table[s:e].clone())
    want = a.held()
    assert any(not torch.equal(x, y) for x, y in zip(before, want))
    for x, held in zip((a.c.k_pages.view(torch.uint8), a.c.v_pages.view(torch.uint8), a.c.k_scale, a.c.v_scale), before):
        x.copy_(held)
    a.run(ctx)
    for x, y in zip(a.held(), want):
        assert torch.equal(x.nan_to_num(-1.0), y.nan_to_num(-1.0)) if x.is_floating_point() else torch.equal(x, y)


def test_append_to_many_sequences_whose_starts_do_not_ascend(ctx):  # noqa: F811
    """What is written is of the call's tokens, at its places: nothing else changes."""
    new = [3] * 200
    for what, change in (("one", lambda a: a.starts[100].fill_(-9)), ("far", lambda a: a.starts[30:40].fill_(1 << 30)), ("none", lambda a: a.starts.fill_(-1)),
                         ("all", lambda a: a.starts.copy_(a.starts.flip(0)))):
        a = Append(TINY, new, [3 + (37 * i) % 60 for i in range(200)], page_size=16, scale_tokens=8, seed=18)
        change(a)
        before = a.held()
        a.run(ctx)
        rows = a.starts.tolist()
        may = torch.zeros(before[0].shape[0], 16, dtype=torch.bool, device=DEV)
        for s in range(200):
            t0, t1 = _clamped(rows, s, 600)
            for j in range(max(0, int(a.lens[s]) - (t1 - t0)) // 8 * 8 if t1 > t0 else int(a.lens[s]), int(a.lens[s])):
                may[int(a.c.table[s, j // 16]), j % 16] = True
        for x, y in zip(a.held()[:2], before[:2]):
            assert not ((x != y).any(dim=3).any(dim=1) & ~may).any(), what
        for x, y in zip(a.held()[2:], before[2:]):
            assert not ((x.nan_to_num(-1.0) != y.nan_to_num(-1.0)).any(dim=1) & ~may.unflatten(1, (2, 8)).any(dim=2)).any(), what


def test_append_beyond_32_bit_offsets(ctx):  # noqa: F811
    a = Append(H8B, [3, 40], [130, 40], seed=9)
    big = Cache8(_heads(H8B), [130, 40], 64, 32, _gen(9), far=66000)
    a.c = big
    held = a.held()
    a.run(ctx)
    got, used = a.held(), torch.cat([big.table[0, :3], big.table[1, :1]]).long()
    small = Cache8.__new__(Cache8)
    small.h, small.page_size, small.scale_tokens = big.h, 64, 32
    small.k_pages = big.k_pages[:4]                       # (for its number of pages)
    small.table = _int32([[0, 1, 2, -1], [3, -1, -1, -1]])
    want = _append_model(small, a.k, a.v, a.starts.tolist(), a.lens.tolist(), [x[used] for x in held])
    for g, x, w in zip(got, held, want):
        assert torch.equal(g[used].nan_to_num(-1.0) if g.is_floating_point() else g[used], w.nan_to_num(-1.0) if w.is_floating_point() else w)
        x[used] = g[used]
        assert torch.equal(g.view(torch.uint8), x.view(torch.uint8)), "pages that got nothing"


def test_append_then_attention(ctx):  # noqa: F811
    """A prompt in blocks, then tokens: written, and attended over, as a layer does."""
    h = _heads(H8B)
    gen = _gen(10)
    t, ps, st = 330, 64, 32
    k, v, q = _bf16(gen, t, 1024), _bf16(gen, t, 1024), _bf16(gen, t, 4096)
    c = Cache8(h, [t], ps, st, gen)
    o, lse = torch.empty_like(q), torch.empty((t, 32), device=DEV)
    ctx.ensure_attention_workspace(h, 128, 1)
    for a, b in [(0, 128), (128, 256), (256, 320)] + [(i, i + 1) for i in range(320, 330)]:
        starts, lens = _int32([0, b - a]), _int32([b])
        ctx.cache8_append(h, k[a:b], v[a:b], starts, lens, c.cache, c.table)
        ctx.chunk_attention8(h, q[a:b], starts, lens, b - a, c.cache, c.table, o[a:b], lse=lse[a:b])
        ref = _reference(h, q[a:b].unflatten(1, (-1, 128)), c.value("k", 0, b), c.value("v", 0, b))
        _check(o[a:b], lse[a:b], ref, 128, b, f"rows {a} to {b}")
    # and what was cached is what was given, within half a step of four bits of mantissa or of e4m3's least step
    for which, x, scale in (("k", k, c.k_scale), ("v", v, c.v_scale)):
        got, want = c.value(which, 0, t), x.double().unflatten(1, (8, 128))
        page = c.table[0, :-(-t // ps)].long()
        step = scale[page].repeat_interleave(st, dim=2).transpose(1, 2).reshape(-1, 8)[:t].double()[..., None] * 2.0 ** -9
        # (blocks that grew token by token were rounded once for each time their scale grew)
        assert bool(((got - want).abs() <= 2.0 ** -4 * want.abs() * (1 + 2.0 ** -4) + step * 2).all())


def test_captured_appends_and_attention():
    """Two graphs captured once and replayed while lengths, starts and tables change, with eager calls between."""
    stream = torch.cuda.Stream()
    ctx = B.Context(0, stream)  # noqa: F811
    try:
        a = Append(H8B, [1, 1, 1], [900, 40, 2000], seed=18)
        x = Chunks8(_heads(H8B), [90, 1, 37], [900, 700, 64], seed=19)
        y = Chunks8(_heads(H8B), [1, 1, 1], [900, 40, 2000], seed=18)
        y.cache, y.table = a.c.cache, a.c.table
        torch.cuda.synchronize()
        a.run(ctx)
        x.run(ctx)
        y.run(ctx)
        stream.synchronize()
        g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g1, stream=stream):
            a.run(ctx)
            y.run(ctx)
        with torch.cuda.graph(g2, stream=stream):
            x.run(ctx)
        gen = _gen(21)
        for rep in range(4):
            a.k.copy_(_bf16(gen, *a.k.shape))
            a.v.copy_(_bf16(gen, *a.v.shape))
            a.lens.copy_(_int32([900 - 13 * rep, 40 - 3 * rep, 2000 - 100 * rep]))
            y.ctx_lens.copy_(a.lens)
            x.ctx_lens.copy_(_int32([max(1, n - 13 * rep) for n in x.lens]))
            torch.cuda.synchronize()
            held = a.held()
            g1.replay()
            g2.replay()
            torch.cuda.synchronize()
            a.check(held, f"replay {rep}")
            got = [z.o.clone() for z in (x, y)]
            for z in (x, y):
                z.o.fill_(5.0)
            torch.cuda.synchronize()
            for z in (x, y):
                z.run(ctx)
            stream.synchronize()
            for z, o in zip((x, y), got):
                assert torch.equal(z.o.view(torch.int16), o.view(torch.int16)), f"replay {rep}"
    finally:
        torch.cuda.synchronize()
        ctx.close()


def test_refusals(ctx):  # noqa: F811
    a, c = Append(TINY, [3, 1], [40, 9]), Chunks8(_heads(TINY), [3, 1], [40, 9])

    def append(h=None, cache=None, table=None):
        ctx.cache8_append(h or a.c.h, a.k, a.v, a.starts, a.lens, cache or a.c.cache, a.c.table if table is None else table)

    def attend(h=None, cache=None, max_chunk=3):
        ctx.chunk_attention8(h or c.h, c.q, c.starts, c.ctx_lens, max_chunk, cache or c.cache, c.table, c.o)

    for field, value, status in (("n_pages", 0, 1), ("page_size", 48, 2), ("page_size", 8, 2), ("page_size", 8192, 2), ("k", None, 1), ("v_scale", None, 1),
                                 ("scale_tokens", 4, 2), ("scale_tokens", 24, 2), ("scale_tokens", 256, 2), ("scale_tokens", 0, 2),
                                 ("k", a.c.cache.k + 8, 3), ("k_scale", a.c.cache.k_scale + 4, 3)):
        for call, cache in ((append, a.c.cache), (attend, c.cache)):
            bad = B.PagedCache8(*(getattr(cache, n) for n, _ in cache._fields_))
            bad.tensors = cache.tensors
            setattr(bad, field, value)
            _refused(status, call, cache=bad)
    small = B.PagedCache8(*(getattr(c.cache, n) for n, _ in c.cache._fields_))
    small.tensors, small.page_size, small.scale_tokens = c.cache.tensors, 16, 32        # more than a page
    _refused(2, attend, cache=small)
    for field, value in (("scale", 0.0), ("scale", math.nan), ("window", -1)):
        h = _heads(TINY)
        setattr(h, field, value)
        _refused(1, attend, h)
        append(h)                                                                      # (of these only the heads count there)
    _refused(1, attend, max_chunk=0)
    _refused(1, attend, max_chunk=5)
    for bad in (lambda: B.paged_cache8(c.k_pages, c.v_pages, c.k_scale, c.v_scale.double()),
                lambda: B.paged_cache8(c.k_pages.view(torch.uint8), c.v_pages, c.k_scale, c.v_scale),
                lambda: B.paged_cache8(c.k_pages, c.v_pages, c.k_scale[:-1], c.v_scale[:-1]),
                lambda: ctx.cache8_append(_heads(H8B), a.k, a.v, a.starts, a.lens, a.c.cache, a.c.table),
                lambda: ctx.cache8_append(a.c.h, a.k[:2], a.v, a.starts, a.lens, a.c.cache, a.c.table)):
        with pytest.raises(AssertionError):
            bad()
    fresh = B.Context(0)
    try:
        big = Chunks8(_heads(H8B), [1], [4000])
        _refused(5, fresh.chunk_attention8, big.h, big.q, big.starts, big.ctx_lens, 1, big.cache, big.table, big.o)
        a.run(fresh)                                                                   # needs no workspace
        torch.cuda.synchronize()
    finally:
        fresh.close()


def test_the_validate_option(ctx):  # noqa: F811
    c = Chunks8(_heads(H8B), [1, 40], [100, 80])
    ctx.set_option("validate", 1)
    try:
        c.run(ctx)
        c.check("validated")
        c.table[1, 0] = 1 << 30
        _refused(4, c.run, ctx)
    finally:
        ctx.set_option("validate", 0)


# ------------------------------------------------------------------ sequences that outgrow their page table

def _placed(new, lens, most):
    """How many of each sequence's new tokens have a place in a table of `most` keys: the first ones."""
    return [min(n, max(0, n - max(0, keys - most))) for n, keys in zip(new, lens)]


def _placed_model(c, k, v, starts, lens, held):
    """The write of the tokens that have a place, as if the others were not in the call."""
    most, new = c.table.shape[1] * c.page_size, [b - a for a, b in zip(starts, starts[1:])]
    n = _placed(new, lens, most)
    rows = torch.tensor([t for a, m in zip(starts, n) for t in range(a, a + m)], dtype=torch.long, device=DEV)
    return _append_model(c, k[rows], v[rows], _starts(n), [min(x, most) for x in lens], held)


@pytest.mark.parametrize("h", [H8B, H1B], ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("n_seqs", [6, 64, 65, 200])
def test_append_behind_the_end_of_the_table(ctx, h, n_seqs):  # noqa: F811
    """Tokens that the table has no place for are not written, and nor is any earlier key or scale changed; up to there they are."""
    most = 6 * 16
    over = [(1, 97), (5, 98), (5, 101), (5, 102), (40, 130), (3, 96), (0, 97), (1, 500), (9, (1 << 30) - 1), (2, 95), (20, 110)]
    new, lens = ([over[i % len(over)][j] for i in range(n_seqs)] for j in (0, 1))
    a = Append(h, new, [min(n, most - 1) for n in lens], page_size=16, scale_tokens=8, seed=n_seqs, behind=2)
    # a full table: each row has its pages and no column more
    c = a.c
    c.table = torch.randperm(c.k_pages.shape[0], device=DEV, generator=_gen(3))[:n_seqs * 6].to(torch.int32).view(n_seqs, 6).contiguous()
    for x in (c.k_pages, c.v_pages):
        codes = x.view(torch.uint8)
        codes.copy_(torch.randint(0, 127, codes.shape, device=DEV, generator=_gen(4)))
    for x in (c.k_scale, c.v_scale):
        x.copy_(torch.exp2(torch.randint(-9, -5, x.shape, device=DEV, generator=_gen(5)).float()))
    a.lens = _int32(lens)
    held = a.held()
    a.run(ctx)
    want = _placed_model(c, a.k, a.v, a.starts.tolist(), lens, held)
    for x, y in zip(a.held(), want):
        assert torch.equal(x, y)
    # of a token behind a full row there is no trace
    full = [i for i in range(n_seqs) if lens[i] - new[i] >= most]
    pages = c.table[full].long().flatten()
    assert full and all(torch.equal(x[pages], y[pages]) for x, y in zip(a.held(), held))


def test_the_validate_option_of_the_write(ctx):  # noqa: F811
    """Starts and lengths out of range are refused and nothing is written; pages out of range are passed over as without it."""
    ctx.set_option("validate", 1)
    try:
        a = Append(H8B, [40, 30], [100, 80], page_size=16, scale_tokens=8, seed=6, behind=3)
        most = a.c.table.shape[1] * 16
        for what, change in (("longer than the table", lambda: a.lens[0].fill_(most + 1)), ("negative length", lambda: a.lens[1].fill_(-3)),
                             ("end", lambda: a.starts[2].fill_(74)), ("descending starts", lambda: a.starts[1].fill_(-9))):
            starts, lens, held = a.starts.clone(), a.lens.clone(), a.held()
            change()
            _refused(4, a.run, ctx)
            assert all(torch.equal(x.nan_to_num(-1.0), y.nan_to_num(-1.0)) if x.is_floating_point() else torch.equal(x, y) for x, y in zip(a.held(), held)), what
            a.starts.copy_(starts)
            a.lens.copy_(lens)
        a.run_and_check(ctx, "validated")
        a.lens[0] = most
        a.run_and_check(ctx, "a full table")
        a.c.table[1, 0] = 1 << 30
        a.c.table[0, 6] = -5
        a.run_and_check(ctx, "pages passed over")
    finally:
        ctx.set_option("validate", 0)
