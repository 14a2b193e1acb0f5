"""Norms around a block and rotary positions, against their formulas in float64, and the calls of a layer together.

A bf16 output is off by half a step of its own rounding (2^-8 of its value) and by the fp32 arithmetic before it: some tens of
half steps of 2^-24 of the sizes that went into it, taken as 2^-18 of them."""
import math

import numpy as np
import pytest
import torch

from oracle import ff_oracle as O
from paper_2602_00397_amd import binding as B
from paper_2602_00397_amd import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = B.Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


def _gen(seed=1):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(gen, *shape):
    return torch.randn(shape, device=DEV, generator=gen)


def _bf16(gen, *shape):
    return _randn(gen, *shape).to(torch.bfloat16)


def _close(got, ref, size, what):
    """size: what the fp32 arithmetic's errors are relative to, elementwise."""
    bar = 2.0 ** -8 * ref.abs() + 2.0 ** -18 * size + 1e-38
    worst = float(((got.double() - ref).abs() / bar).max())
    print(f"[layer] {what}: worst error {worst:.3f} of its bar", flush=True)
    assert worst <= 1.0, what


# ------------------------------------------------------------------ norms

def _norm(gen, kind, d, gain=True, bias=False, offset=0.0, eps=EPS):
    g = (1.0 - offset + 0.2 * _randn(gen, d)).to(torch.bfloat16) if gain else None
    b = _bf16(gen, d) if bias else None
    return B.norm(kind, eps, gain=g, bias=b, gain_offset=offset)


def _normed(v, n):
    """The norm of the rows of v and the size of what went into it (float64)."""
    if n is None:
        return v, v.abs()
    gain, bias = (None if t is None else t.double() for t in n.tensors)
    c = v.mean(dim=1, keepdim=True) if n.kind == B.NORM["layer"] else torch.zeros_like(v[:, :1])
    inv = 1.0 / torch.sqrt(((v - c) ** 2).mean(dim=1, keepdim=True) + n.eps)
    g = gain + n.gain_offset if gain is not None else torch.ones_like(v[0])
    b = bias if bias is not None else torch.zeros_like(v[0])
    # an error of the mean moves every channel by its fraction of the row's size, one of the statistics scales them all
    return (v - c) * inv * g + b, (v.abs() + v.abs().mean(dim=1, keepdim=True)) * inv * g.abs() + b.abs()


def _norm_reference(h, y, post, gate, gate_tokens, scale, pre):
    s = size = h.double()
    size = size.abs()
    if y is not None:
        p, p_size = _normed(y.double(), post)
        g = gate.double()[torch.arange(h.shape[0], device=DEV) // gate_tokens] if gate is not None else torch.ones_like(p)
        s, size = s + scale * g * p, size + abs(scale) * g.abs() * p_size
    if pre is None:
        return s, size, None, None
    x, _ = _normed(s, pre)
    # errors of s, relative to size, go through the norm with its factor
    _, x_size = _normed(size, pre)
    gain = pre.tensors[0]
    g = (gain.double() + pre.gain_offset).abs() if gain is not None else torch.ones_like(s[0])
    c = s.mean(dim=1, keepdim=True) if pre.kind == B.NORM["layer"] else torch.zeros_like(s[:, :1])
    inv = 1.0 / torch.sqrt(((s - c) ** 2).mean(dim=1, keepdim=True) + pre.eps)
    return s, size, x, (size + size.mean(dim=1, keepdim=True)) * inv * g + x.abs() * (1 + (size * size).mean(dim=1, keepdim=True) * inv * inv)


def _run_norm(ctx, t, d, y_dtype=torch.bfloat16, post=None, pre=None, gate_tokens=None, scale=1.0, in_place=False, seed=1):
    gen = _gen(seed)
    h = _bf16(gen, t, d)
    y = (_randn(gen, t, d) * 2.0).to(y_dtype) if y_dtype is not None else None
    gate = _bf16(gen, -(-t // gate_tokens), d) if gate_tokens else None
    s, s_size, x_ref, x_size = _norm_reference(h, y, post, gate, gate_tokens, scale, pre)
    h_out = None if y is None else (h if in_place else torch.full_like(h, 7.0))
    x = torch.full_like(h, 7.0) if pre is not None else None
    ctx.norm_residual(h, y, h_out, x, post=post, gate=gate, gate_tokens=gate_tokens or 1, scale=scale, pre=pre)
    what = f"{t} x {d}"
    if h_out is not None:
        _close(h_out, s, s_size, what + " h")
    if x is not None:
        _close(x, x_ref, x_size, what + " x")


@pytest.mark.parametrize("d", [8, 64, 256, 512, 520, 2040, 2048, 3584, 4096, 4104, 8192, 8200, 16384])
@pytest.mark.parametrize("t", [1, 5, 130])
def test_norm_sizes(ctx, t, d):
    gen = _gen(3)
    _run_norm(ctx, t, d, pre=_norm(gen, "rms", d))
    _run_norm(ctx, t, d, torch.float32, post=_norm(gen, "layer", d, bias=True), pre=_norm(gen, "layer", d, bias=True), gate_tokens=2, scale=0.3)


@pytest.mark.parametrize("t,d", [(3, 256), (1500, 2048), (4099, 3584)])
def test_norm_variants(ctx, t, d):
    gen = _gen(4)
    for in_place in (False, True):
        _run_norm(ctx, t, d, in_place=in_place)                                                  # a residual add alone
        _run_norm(ctx, t, d, pre=_norm(gen, "rms", d, gain=False), in_place=in_place)
        _run_norm(ctx, t, d, post=_norm(gen, "rms", d, offset=1.0), gate_tokens=1, scale=-2.5, in_place=in_place)
        _run_norm(ctx, t, d, torch.float32, post=_norm(gen, "rms", d, gain=False, bias=True), pre=_norm(gen, "rms", d, offset=1.0, bias=True),
                  gate_tokens=128, scale=0.22, in_place=in_place)
        _run_norm(ctx, t, d, pre=_norm(gen, "layer", d, gain=False), gate_tokens=t, in_place=in_place)
        _run_norm(ctx, t, d, pre=_norm(gen, "layer", d, gain=False), gate_tokens=2 * t + 1, in_place=in_place)   # one row for more tokens than there are
    for kind in ("rms", "layer"):
        _run_norm(ctx, t, d, None, pre=_norm(gen, kind, d, bias=True))                            # no block before: the norm alone


def test_norm_agrees_with_the_stack_glue(ctx):
    """gain 1, no gate, scale 1: the residual add and the norm that ff_residual_add and ff_rmsnorm do one after the other.  Those
    round the sum before its norm, so only the sum has the same bits."""
    gen = _gen(5)
    h, y = _bf16(gen, 300, 4096), _bf16(gen, 300, 4096)
    h2, x, h_out = h.clone(), torch.empty_like(h), torch.empty_like(h)
    ctx.residual_add(h2, y)
    ctx.norm_residual(h, y, h_out, x, pre=B.norm("rms", EPS))
    assert torch.equal(h2.view(torch.int16), h_out.view(torch.int16))


def test_norm_of_constant_and_extreme_rows(ctx):
    """A constant row has no deviation; large and tiny rows keep their statistics in range."""
    d = 2048
    h = torch.zeros((6, d), dtype=torch.bfloat16, device=DEV)
    h[1] = 3.0
    h[2] = 1e15
    h[3] = 1e-15
    h[4, 7] = 1e18
    h[5] = float("nan")
    x = torch.empty_like(h)
    ctx.norm_residual(h, None, None, x, pre=B.norm("layer", 1e-5))
    assert bool((x[:2] == 0).all()) and bool((x[3] == 0).all()) and bool(torch.isnan(x[5].float()).all())
    ctx.norm_residual(h, None, None, x, pre=B.norm("rms", 0.0))
    ref = h.double() / torch.sqrt((h.double() ** 2).mean(dim=1, keepdim=True))
    _close(x[[1, 2, 3, 4]], ref[[1, 2, 3, 4]], ref[[1, 2, 3, 4]].abs(), "extreme rows")


def _refused(status, call, *args, **kw):
    with pytest.raises(B.FFError) as e:
        call(*args, **kw)
    assert e.value.status == status, e.value


def test_more_tokens_than_a_launch_has_threads_across(ctx):
    """Above 2^24 rows, of a norm and of rotary positions: the last ones and some between."""
    t = (1 << 24) + 70
    gen = _gen(10)
    some = torch.cat([torch.arange(0, t, 99991, device=DEV), torch.arange(t - 200, t, device=DEV)])
    h = _bf16(gen, t, 8)
    h_out, x = torch.empty_like(h), torch.empty_like(h)
    n = _norm(gen, "rms", 8)
    ctx.norm_residual(h, h, h_out, x, pre=n)
    s, s_size, x_ref, x_size = _norm_reference(h[some], h[some], None, None, 1, 1.0, n)
    _close(h_out[some], s, s_size, "rows above 2^24, h")
    _close(x[some], x_ref, x_size, "rows above 2^24, x")
    del h, h_out, x
    q = _bf16(gen, t, 64)
    q_out, k_out = torch.zeros_like(q), torch.zeros_like(q)
    pos, freqs = torch.arange(t, dtype=torch.int32, device=DEV)[None].contiguous(), _freqs(64)
    ctx.rotary(B.Attention(1, 1, 64, 1, 0, 1.0), B.rotary(64, freqs), q, q, None, pos, q_out, k_out=k_out)
    ref, size = _turned(q[some], 64, 64, pos[:, some], [0] * 32, freqs, False)
    _close(q_out[some].unflatten(1, (-1, 64)), ref, size, "tokens above 2^24")
    assert torch.equal(q_out.view(torch.int16), k_out.view(torch.int16))


def test_norm_refusals(ctx):
    h = torch.zeros((4, 64), dtype=torch.bfloat16, device=DEV)
    x, n = torch.empty_like(h), B.norm("rms", EPS)
    _refused(1, ctx.norm_residual, h, h, x, None, pre=n)                       # a norm without its output
    _refused(1, ctx.norm_residual, h, h, None, x)                              # an output without its norm
    _refused(1, ctx.norm_residual, h, None, x, None)                           # a sum of nothing
    _refused(1, ctx.norm_residual, h, None, None, x, pre=n, post=n)
    _refused(1, ctx.norm_residual, h, h, None, None)
    _refused(1, ctx.norm_residual, h, h, x, None, scale=math.nan)
    _refused(1, ctx.norm_residual, h, h, x, None, gate=h, gate_tokens=0)
    for kind, eps, offset in ((0, EPS, 0.0), (3, EPS, 0.0), (1, -1.0, 0.0), (1, math.nan, 0.0), (1, math.inf, 0.0), (1, EPS, math.nan)):
        bad = B.Norm(kind, eps, offset, None, None)
        bad.tensors = (None, None)
        _refused(1, ctx.norm_residual, h, None, None, x, pre=bad)
    for d in (60, 16392):
        w = torch.zeros((2, d), dtype=torch.bfloat16, device=DEV)
        _refused(2, ctx.norm_residual, w, w, torch.empty_like(w), None)
    flat = torch.zeros(4 * 64 + 4, dtype=torch.bfloat16, device=DEV)
    _refused(3, ctx.norm_residual, flat[4:].view(4, 64), None, None, x, pre=n)
    with pytest.raises(AssertionError):                                        # weights of another width
        ctx.norm_residual(h, None, None, x, pre=B.norm("rms", EPS, gain=torch.ones(32, dtype=torch.bfloat16, device=DEV)))


# ------------------------------------------------------------------ rotary positions

def _turned(v, hd, rot, positions, axis, inv_freq, interleaved):
    """(reference, size) [t][heads][hd] in float64."""
    v = v.double().unflatten(1, (-1, hd))
    pairs = rot // 2
    i = torch.arange(pairs, device=DEV)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
    angle = (positions.double()[torch.tensor(axis, device=DEV)] * inv_freq.double()[:, None]).t()[:, None]
    out, size = v.clone(), v.abs()
    out[:, :, a] = v[:, :, a] * torch.cos(angle) - v[:, :, b] * torch.sin(angle)
    out[:, :, b] = v[:, :, b] * torch.cos(angle) + v[:, :, a] * torch.sin(angle)
    size[:, :, a] = size[:, :, b] = v[:, :, a].abs() + v[:, :, b].abs()
    return out, size


def _freqs(rot):
    return (500000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))).float().to(DEV)


@pytest.mark.parametrize("h", [(32, 8, 128), (28, 4, 128), (4, 2, 64), (3, 3, 64), (5, 1, 128)], ids=str)
@pytest.mark.parametrize("t", [1, 7, 1030])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary(ctx, h, t, interleaved):
    gen = _gen(7)
    hd, ps = h[2], 16
    heads = B.Attention(h[0], h[1], hd, 1, 0, 1.0)
    for rot, n_axes in ((hd, 1), (hd // 2, 3), (16, 2)):
        axis = [(5 * i) % n_axes for i in range(rot // 2)]
        freqs = _freqs(rot)
        spec = B.rotary(rot, freqs, axis=axis, interleaved=interleaved, n_axes=n_axes)
        qkv = _bf16(gen, t, (h[0] + 2 * h[1]) * hd + 16)
        q, k, v = qkv[:, :h[0] * hd], qkv[:, h[0] * hd:(h[0] + h[1]) * hd], qkv[:, (h[0] + h[1]) * hd:(h[0] + 2 * h[1]) * hd]
        pos = torch.randint(0, 2 ** 31 - 1, (n_axes, t), device=DEV, dtype=torch.int32, generator=gen)
        n_pages = -(-t // ps) + 2
        pages = [torch.full((n_pages, h[1], ps, hd), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        slots = torch.randperm(n_pages * ps, device=DEV, generator=gen)[:t].to(torch.int32)
        slots[t // 2] = -1                                            # a padded token
        if t > 3:
            slots[3], slots[1] = n_pages * ps, 2 ** 31 - 1            # slots behind the cache
        q_out, k_out = torch.full((t, h[0] * hd), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((t, h[1] * hd + 8), 7.0, dtype=torch.bfloat16, device=DEV)
        ctx.rotary(heads, spec, q, k, v, pos, q_out, k_out=k_out[:, :h[1] * hd], cache=B.paged_cache(*pages), slots=slots)
        what = f"{h} {t} tokens rot {rot} axes {n_axes}"
        ref_q, size_q = _turned(q, hd, rot, pos, axis, freqs, interleaved)
        ref_k, size_k = _turned(k, hd, rot, pos, axis, freqs, interleaved)
        _close(q_out.unflatten(1, (-1, hd)), ref_q, size_q, what + " q")
        _close(k_out[:, :h[1] * hd].unflatten(1, (-1, hd)), ref_k, size_k, what + " k")
        assert bool((k_out[:, h[1] * hd:] == 7.0).all())
        # the cache: k as it was given back, v as it came, everything else as it was
        want = [torch.full_like(p, 7.0) for p in pages]
        kept = (slots >= 0) & (slots < n_pages * ps)
        s = slots[kept].long()
        want[0][s // ps, :, s % ps] = k_out[:, :h[1] * hd].unflatten(1, (-1, hd))[kept]
        want[1][s // ps, :, s % ps] = v.unflatten(1, (-1, hd))[kept]
        for name, p, w in zip("kv", pages, want):
            assert torch.equal(p.view(torch.int16), w.view(torch.int16)), f"{what}: {name} pages"
        # in the inputs' place; without k_out; without a cache
        only_q, only_pages = torch.empty_like(q_out), [torch.full_like(p, 7.0) for p in pages]
        ctx.rotary(heads, spec, q, k, v, pos, only_q, cache=B.paged_cache(*only_pages), slots=slots)
        assert torch.equal(only_q.view(torch.int16), q_out.view(torch.int16)) and all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(only_pages, pages))
        ctx.rotary(heads, spec, q, k, None, pos, q, k_out=k)
        assert torch.equal(q.contiguous().view(torch.int16), q_out.view(torch.int16))
        assert torch.equal(k.contiguous().view(torch.int16), k_out[:, :h[1] * hd].contiguous().view(torch.int16))


def test_rotary_of_far_and_negative_positions(ctx):
    """Angles of positions up to 2^31 - 1 at a frequency of 1: the reduction keeps their digits."""
    gen = _gen(8)
    heads, freqs = B.Attention(2, 2, 64, 1, 0, 1.0), torch.ones(32, device=DEV)
    pos = torch.tensor([[0, 1, -1, 2 ** 31 - 1, 2 ** 24 + 1, -2 ** 31]], dtype=torch.int32, device=DEV)
    q = _bf16(gen, 6, 128)
    out, k_out = torch.empty_like(q), torch.empty_like(q)
    ctx.rotary(heads, B.rotary(64, freqs), q, q, None, pos, out, k_out=k_out)
    ref, size = _turned(q, 64, 64, pos, [0] * 32, freqs, False)
    _close(out.unflatten(1, (-1, 64)), ref, size, "far positions")
    assert torch.equal(out, k_out) and torch.equal(out[0], q[0])


def test_rotary_refusals(ctx):
    heads = B.Attention(4, 2, 64, 1, 0, 1.0)
    q, k = torch.zeros((3, 256), dtype=torch.bfloat16, device=DEV), torch.zeros((3, 128), dtype=torch.bfloat16, device=DEV)
    pos, slots = torch.zeros((1, 3), dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    pages = [torch.zeros((2, 2, 16, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    cache, spec = B.paged_cache(*pages), B.rotary(64, _freqs(64))
    _refused(1, ctx.rotary, heads, spec, q, k, k, pos, q)                                    # nowhere to put k
    _refused(1, ctx.rotary, heads, spec, q, k, k, pos, q, cache=cache)                       # no slots
    _refused(1, ctx.rotary, heads, spec, q, k, k, pos, q, k_out=k, slots=slots)
    _refused(1, ctx.rotary, heads, spec, q, k, None, pos, q, cache=cache, slots=slots)       # no values
    _refused(1, ctx.rotary, heads, B.rotary(64, _freqs(64), axis=[1] * 32), q, k, k, pos, q, k_out=k)
    _refused(1, ctx.rotary, heads, B.rotary(64, _freqs(64), axis=[-1] * 32), q, k, k, pos, q, k_out=k)
    for rot in (8, 24, 128):
        _refused(2, ctx.rotary, heads, B.rotary(rot, _freqs(rot)), q, k, k, pos, q, k_out=k)
    five = B.rotary(64, _freqs(64), axis=[0] * 32, n_axes=5)
    _refused(2, ctx.rotary, heads, five, q, k, k, torch.zeros((5, 3), dtype=torch.int32, device=DEV), q, k_out=k)
    _refused(2, ctx.rotary, B.Attention(4, 3, 64, 1, 0, 1.0), spec, q, torch.zeros((3, 192), dtype=torch.bfloat16, device=DEV), None, pos, q,
             k_out=torch.zeros((3, 192), dtype=torch.bfloat16, device=DEV))
    _refused(2, ctx.rotary, B.Attention(4, 2, 32, 1, 0, 1.0), spec, q[:, :128], k[:, :64], None, pos, q[:, :128], k_out=k[:, :64])
    wide = torch.zeros((3, 512), dtype=torch.bfloat16, device=DEV)
    _refused(1, ctx.rotary, heads, spec, wide[:, :256], k, k, pos, wide.view(-1)[:768].view(3, 256), k_out=k)   # the input's place, other rows


def test_captured_norms_and_rotary_positions_follow_their_inputs():
    """Norm, rotary positions with the cache write and norm again on a stream of their own, captured once and replayed while
    inputs, positions and slots change, with eager calls in between."""
    stream = torch.cuda.Stream()
    ctx = B.Context(0, stream)
    try:
        gen, t, d = _gen(11), 37, 512
        heads, spec = B.Attention(4, 2, 64, 1, 0, 1.0), B.rotary(64, _freqs(64), interleaved=True)
        h, y, qkv = _bf16(gen, t, d), _randn(gen, t, d), _bf16(gen, t, 512)
        h_out, x, q_out, n = torch.zeros_like(h), torch.zeros_like(h), torch.zeros((t, 256), dtype=torch.bfloat16, device=DEV), _norm(gen, "layer", d, bias=True)
        pages = [torch.zeros((6, 2, 8, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        cache, pos, slots = B.paged_cache(*pages), torch.zeros((1, t), dtype=torch.int32, device=DEV), torch.zeros(t, dtype=torch.int32, device=DEV)
        out = (h_out, x, q_out, *pages)

        def run():
            ctx.norm_residual(h, y, h_out, x, post=n, gate=h, pre=n, scale=0.5)
            ctx.rotary(heads, spec, qkv[:, :256], qkv[:, 256:384], qkv[:, 384:], pos, q_out, cache=cache, slots=slots)

        def draw():
            for v in (h, y, qkv):
                v.copy_(_randn(gen, *v.shape))
            pos.copy_(torch.randint(0, 1 << 20, (1, t), device=DEV, generator=gen))
            slots.copy_(torch.randperm(48, device=DEV, generator=gen)[:t])
            for v in out:
                v.zero_()
            torch.cuda.synchronize()

        draw()
        run()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run()
        for rep in range(4):
            draw()
            graph.replay()
            torch.cuda.synchronize()
            got = [v.clone() for v in out]
            for v in out:
                v.zero_()
            torch.cuda.synchronize()
            run()
            stream.synchronize()
            assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(got, out)), f"replay {rep}"
    finally:
        torch.cuda.synchronize()
        ctx.close()


# ------------------------------------------------------------------ a layer's calls together

def test_a_layer_chunk_by_chunk_equals_the_whole_prompt_and_float64(ctx):
    """One decoder layer over a prompt: norm, projections, rotary positions, attention, projection, gate and residual with the norm
    before the FFN, predictor, sparse FFN, residual.  Once over the whole prompt with prompt attention, once block by block over
    a paged cache (the last block of one token), and in float64."""
    shp = W.CONFIGS["c0"]
    d, block, T = shp.d_model, shp.block, 3 * shp.block + 1
    n_h, n_kv, hd, ps = 4, 2, 64, 16
    gen = _gen(9)
    heads = B.Attention(n_h, n_kv, hd, 1, 0, hd ** -0.5)
    lt = W.make_layer(shp)
    dev, pred, w, comp = B.make_structs(lt, DEV)
    w_qkv = (_randn(gen, (n_h + 2 * n_kv) * hd, d) * 0.06).to(torch.bfloat16)
    w_o = (_randn(gen, d, n_h * hd) * 0.06).to(torch.bfloat16)
    gate = torch.tanh(_randn(gen, 1, d)).to(torch.bfloat16)
    n1, n2, n3 = (_norm(gen, "rms", d) for _ in range(3))
    freqs = _freqs(hd)
    spec = B.rotary(hd, freqs)
    h0 = B.to_device_bf16(W.make_hidden(shp, n_tokens=T), DEV)
    k_keep = O.k_from_sparsity(shp.d_ffn, 0.5)

    def layer(h, positions, attend):
        n = h.shape[0]
        shape = B.Shape(d, shp.d_ffn, n, block, shp.r_pred, shp.r_comp)
        nb = -(-n // block)
        x, h1, x2, h2 = (torch.empty_like(h) for _ in range(4))
        y = torch.empty((n, d), dtype=torch.float32, device=DEV)
        idx = torch.empty((nb, k_keep), dtype=torch.int32, device=DEV)
        ctx.norm_residual(h, None, None, x, pre=n1)
        qkv = x @ w_qkv.t()
        o = attend(qkv, positions)
        ctx.norm_residual(h, o @ w_o.t(), h1, x2, post=n2, gate=gate, gate_tokens=n, scale=0.7, pre=n3)
        ctx.ensure_workspace(shape, k_keep)
        ctx.predict(shape, x2, pred, [k_keep] * nb, k_keep, idx)
        ctx.sparse_ffn(shape, x2, w, comp, idx, [k_keep] * nb, k_keep, y, B.OUT_F32)
        ctx.norm_residual(h1, y, h2, None)
        return h2, idx, x2, h1

    def parts(qkv):
        a, b = n_h * hd, (n_h + n_kv) * hd
        return qkv[:, :a], qkv[:, a:b], qkv[:, b:]

    def whole(qkv, positions):
        q, k, v = parts(qkv)
        o = torch.empty((q.shape[0], n_h * hd), dtype=torch.bfloat16, device=DEV)
        ctx.rotary(heads, spec, q, k, None, positions, q, k_out=k)
        ctx.prompt_attention(heads, q, k, v, torch.tensor([0, q.shape[0]], dtype=torch.int32, device=DEV), o)
        return o

    pages = [torch.full((20, n_kv, ps, hd), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    cache = B.paged_cache(*pages)
    table = torch.randperm(20, device=DEV, generator=gen)[None].to(torch.int32)

    def over_cache(qkv, positions):
        q, k, v = parts(qkv)
        n = q.shape[0]
        o, q_out = (torch.empty((n, n_h * hd), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        j = positions[0]
        slots = (table[0][(j // ps).long()] * ps + j % ps).to(torch.int32)
        ctx.rotary(heads, spec, q, k, v, positions, q_out, cache=cache, slots=slots)
        ctx.ensure_attention_workspace(heads, n, 1)
        ctx.chunk_attention(heads, q_out, torch.tensor([0, n], dtype=torch.int32, device=DEV), j[-1:].clone() + 1, n, cache, table, o)
        return o

    pos = torch.arange(T, dtype=torch.int32, device=DEV)[None]
    h_whole, idx, x2, h1 = layer(h0, pos, whole)
    chunks = [layer(h0[a:a + block], pos[:, a:a + block].contiguous(), over_cache) for a in range(0, T, block)]
    h_chunks, x2_chunks = torch.cat([c[0] for c in chunks]), torch.cat([c[2] for c in chunks])
    # float64, with the library's own lists (its score margins are not this test's subject)
    hd64 = h0.double()
    x, _ = _normed(hd64, n1)
    q, k, v = parts(x @ w_qkv.double().t())
    q, k = (_turned(t, hd, hd, pos, [0] * (hd // 2), freqs, False)[0] for t in (q, k))
    v = v.unflatten(1, (-1, hd))
    o = torch.zeros((T, n_h, hd), dtype=torch.float64, device=DEV)
    for a in range(n_h):
        s = (q[:, a] @ k[:, a // 2].t() * hd ** -0.5).masked_fill(torch.ones((T, T), device=DEV).triu(1).bool(), -math.inf)
        o[:, a] = torch.softmax(s, dim=1) @ v[:, a // 2]
    s1, _, x_ref, _ = _norm_reference(h0, o.flatten(1) @ w_o.double().t(), n2, gate, T, 0.7, n3)
    f = {n: W.bf16_to_f32(getattr(lt, n)) for n in ("w_gate", "w_up", "w_down", "w1", "w2", "wc1", "wc2")}
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())
    # norm, projections, rotary, attention, projection: about six roundings to bf16 on the way, each 2^-9.5 rms at most
    bar = math.sqrt(6) * 2.0 ** -9 * 2
    assert rel(h1, s1) <= bar and rel(x2, x_ref) <= bar, (rel(h1, s1), rel(x2, x_ref))
    assert rel(x2_chunks, x2.double()) <= bar
    for got, x_in, res, lists in ((h_whole, x2, h1, idx), (h_chunks, x2_chunks, torch.cat([c[3] for c in chunks]), torch.cat([c[1] for c in chunks]))):
        ref = O.fastforward_layer(x_in.float().cpu().numpy(), f["w_gate"], f["w_up"], f["w_down"].T, f["w1"], f["w2"], block,
                                  [k_keep] * lists.shape[0], wc1=f["wc1"].T, wc2=f["wc2"], comp_act="silu",
                                  indices_override=list(lists.cpu().numpy()))
        want = res.double() + torch.from_numpy(np.ascontiguousarray(ref.y)).to(DEV)
        assert rel(got, want) <= 1e-2
    print("[layer] h1 %.2e, x %.2e, chunks against the whole %.2e" % (rel(h1, s1), rel(x2, x_ref), rel(x2_chunks, x2.double())), flush=True)
