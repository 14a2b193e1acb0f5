"""A cache in 8 bits, attention over the pages that a cheap score selects, and the handling of a cache's pages, as measurable cases.

A case is a dict of plain values.  By its "op":

  "append"  ff_cache8_append: n_seqs sequences bring up to `chunk` new tokens each (mixed: about half of them bring one) behind
            what their caches hold, up to `context` tokens with the new ones (spread: the others' lengths lie below the
            first's); page_size, scale_tokens, kv_heads, head_dim
  "chunk8"  ff_chunk_attention8 of such sequences: also heads, causal, window, lse
  "select"  one layer's step of sparse attention: ff_page_means of the pages that have new tokens, ff_select_pages for blocks of
            query_block tokens (`keep` earlier pages to a block and key head, the first `first` of them always), and
            ff_selected_attention, over a bf16 cache (scale_tokens 0) or one in 8 bits
  "fork"    a step of a search: n_rows sequences of a page pool forked `beams` times each (ff_pages_fork), all of them grown by a
            token (ff_pages_grow); `layers` of parts to a page: bf16 keys and values, or (eight) codes, scales and means
  "compact" sequences end (ff_pages_free, every `ended`-th of n_rows) and the pages in use move together (ff_pages_compact)

The last two begin each pass with the counts, tables and lengths that the program had before it.  Sizes are those of the benchmark
configurations' models (workloads.CONFIGS) and generic ones.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
E4M3 = torch.float8_e4m3fn
# heads, kv_heads, head_dim of the configurations' models
TINY, M1B, M8B, M7B = (4, 2, 64), (32, 8, 64), (32, 8, 128), (28, 4, 128)


def _heads(m):
    return {"heads": m[0], "kv_heads": m[1], "head_dim": m[2]}


def _sequences_case(op, m, n_seqs, chunk, context, mixed, spread, page_size, scale_tokens, **more):
    return dict(_heads(m), op=op, n_seqs=n_seqs, chunk=chunk, context=context, mixed=mixed, spread=spread, page_size=page_size,
                scale_tokens=scale_tokens, **more)


def _append_case(m, n_seqs, chunk, context, mixed=False, spread=True, page_size=64, scale_tokens=64):
    return _sequences_case("append", m, n_seqs, chunk, context, mixed, spread, page_size, scale_tokens)


def _chunk8_case(m, n_seqs, chunk, context, mixed=False, spread=True, page_size=64, scale_tokens=64, causal=True, window=0, lse=False):
    return _sequences_case("chunk8", m, n_seqs, chunk, context, mixed, spread, page_size, scale_tokens, causal=causal, window=window, lse=lse)


def _select_case(m, n_seqs, chunk, context, query_block, keep, first=1, mixed=False, spread=True, page_size=64, scale_tokens=0):
    return _sequences_case("select", m, n_seqs, chunk, context, mixed, spread, page_size, scale_tokens, query_block=query_block,
                           keep=keep, first=first)


def _pool_case(op, m, n_rows, context, layers, page_size=64, eight=False, beams=0, ended=0):
    return dict(_heads(m), op=op, n_rows=n_rows, context=context, layers=layers, page_size=page_size, eight=eight, beams=beams, ended=ended)


def listed():
    return [
        # 48 sequences generating: a token each into its cache, latency
        dict(_append_case(M8B, 48, 1, 16384), name="append_tokens48_8b"),
        # a long prompt's keys and values into an empty cache, finer scales
        dict(_append_case(M7B, 1, 9001, 9001, page_size=128, scale_tokens=32), name="append_prompt9001_7b"),
        # one sequence generating one token
        dict(_chunk8_case(M8B, 1, 1, 8191), name="chunk8_token_8b"),
        # 48 sequences generating together
        dict(_chunk8_case(M8B, 48, 1, 16384, lse=True), name="chunk8_tokens48_8b"),
        # a server's step: some sequences generate, the others bring a piece of their prompt, narrow heads
        dict(_chunk8_case(M1B, 12, 500, 6000, mixed=True, page_size=16, scale_tokens=16), name="chunk8_mixed_1b"),
        # one token over a very long context, 64 earlier pages of it
        dict(_select_case(M8B, 1, 1, 131072, 1, 64), name="select_token_8b"),
        # 48 sequences generating, a cache in 8 bits
        dict(_select_case(M8B, 48, 1, 32768, 1, 32, scale_tokens=64), name="select_tokens48_8b"),
        # the headline configuration's prompt in its blocks of 128
        dict(_select_case(M8B, 1, 8192, 8192, 128, 16), name="select_prompt8192_8b"),
        # a search of four beams begins: a small model's cache in 8 bits
        dict(_pool_case("fork", M1B, 1, 777, 2, eight=True, beams=3), name="fork_beams4_1b"),
        # 64 sequences of a server forked in three each, all of eight layers' pages
        dict(_pool_case("fork", M7B, 64, 4096, 8, beams=3), name="fork_64x3_7b"),
        # two of eight short sequences end
        dict(_pool_case("compact", M1B, 8, 500, 1, page_size=16, ended=4), name="compact_8_1b"),
        # half of 96 sequences end and the cache is to shrink
        dict(_pool_case("compact", M8B, 96, 4096, 4, ended=2), name="compact_96_8b"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw(rng):
    op = rng.choice(["append"] * 2 + ["chunk8"] * 4 + ["select"] * 3 + ["fork"] + ["compact"])
    m = rng.choice([TINY, M1B, M1B, M8B, M8B, M8B, M7B, M7B])
    page_size = rng.choice([16, 64, 128])
    if op in ("fork", "compact"):
        eight, layers = rng.random() < 0.4, _log_int(rng, 1, 8)
        rows, context = _log_int(rng, 1, 96), _log_int(rng, 1, 4096)
        if op == "fork":
            return _pool_case(op, m, rows, context, layers, page_size, eight, beams=rng.randint(1, 4))
        return _pool_case(op, m, rows, context, layers, page_size, eight, ended=rng.randint(1, 5))
    scale_tokens = rng.choice([t for t in (8, 16, 32, 64, 128) if t <= page_size])
    kind = rng.choice(["tokens", "tokens", "chunk", "mixed"])
    if kind == "tokens":
        n_seqs, chunk = _log_int(rng, 1, 96), rng.choice([1, 1, 1, rng.randint(1, 8)])
    elif kind == "chunk":
        n_seqs, chunk = rng.choice([1, 1, rng.randint(1, 6)]), _log_int(rng, 2, 1024)
    else:
        n_seqs, chunk = rng.randint(2, 48), _log_int(rng, 2, 700)
    spread = rng.random() < 0.8
    if op == "append":
        if kind == "chunk" and n_seqs == 1:
            chunk = _log_int(rng, 2, 9001)
        context = chunk if rng.random() < 0.3 else _log_int(rng, chunk, max(chunk, 16384))
        return _append_case(m, n_seqs, chunk, context, kind == "mixed", spread, page_size, scale_tokens)
    if op == "chunk8":
        context = _log_int(rng, chunk, 32768)
        causal = rng.random() < 0.9
        window = _log_int(rng, 1, 8192) if causal and rng.random() < 0.25 else 0
        return _chunk8_case(m, n_seqs, chunk, context, kind == "mixed", spread, page_size, scale_tokens, causal, window, rng.random() < 0.3)
    if kind == "chunk" and n_seqs == 1:
        chunk = _log_int(rng, 2, 8192)
    context = _log_int(rng, chunk, 65536)
    block = 1 if kind == "tokens" and chunk == 1 else rng.choice([16, 64, 128, rng.randint(2, 200)])
    keep = _log_int(rng, 1, 64)
    return _select_case(m, n_seqs, chunk, context, block, keep, rng.randint(0, min(keep, 4)), kind == "mixed", spread, page_size,
                        rng.choice([0, scale_tokens]))


def draw(rng):
    # (no more work than the largest listed case of any operator)
    most = [work(c) for c in listed()]
    flops, bytes_ = max(w["flops"] for w in most), max(w["bytes"] for w in most)
    while True:
        c = _draw(rng)
        w = work(c)
        if w["flops"] <= flops and w["bytes"] <= bytes_:
            return c


# ---- lengths, by the case alone ------------------------------------------------------------------------------------------

def _lengths(c):
    """New tokens and cached tokens (the new ones included) of every sequence; the first has the most of both."""
    r = random.Random("%d %d %d" % (c["n_seqs"], c["chunk"], c["context"]))
    new, ctx = [c["chunk"]], [c["context"]]
    for _ in range(c["n_seqs"] - 1):
        n = c["chunk"] if not c["mixed"] else (1 if r.random() < 0.5 else r.randint(1, c["chunk"]))
        new.append(n)
        ctx.append(_log_int(r, n, c["context"]) if c["spread"] else c["context"])
    return new, ctx


def _rows_of(c):
    """Lengths of a pool's rows."""
    r = random.Random("%d rows %d" % (c["n_rows"], c["context"]))
    return [c["context"]] + [r.randint(1, c["context"]) for _ in range(c["n_rows"] - 1)]


def _pages(n, page_size):
    return -(-n // page_size)


def _blocks(c):
    """Blocks of query_block tokens: (sequence, first position, position behind the last, earlier pages kept, pages of its own)."""
    out = []
    for s, (n, keys) in enumerate(zip(*_lengths(c))):
        for a in range(keys - n, keys, c["query_block"]):
            b = min(keys, a + c["query_block"])
            earlier = a // c["page_size"]
            out.append((s, a, b, min(c["keep"], earlier), (b - 1) // c["page_size"] - earlier + 1))
    return out


def _block_keys(c, block):
    _, _, b, kept, own_pages = block
    return (kept + own_pages) * c["page_size"] - (-b % c["page_size"])


def _pairs(n, keys, causal, window):
    """How many (token, key) pairs a sequence's mask leaves."""
    if not causal:
        return n * keys
    seen = [keys - n + i + 1 for i in range(n)]
    return sum(min(s, window) if window else s for s in seen)


def _part_bytes(c):
    """Bytes of one page in every part of a layer."""
    n = c["kv_heads"] * c["page_size"] * c["head_dim"]
    return [n, n, c["kv_heads"] * 4, c["kv_heads"] * 4, c["kv_heads"] * c["head_dim"] * 4] if c["eight"] else [2 * n, 2 * n]


def _pool_tables(c):
    """Counts, table and lengths of a pool whose rows came and went in turn, with a prefix that every fourth row shares with the row
    before it, and room for what a pass takes."""
    lens, ps = _rows_of(c), c["page_size"]
    r = random.Random("%d pool %d" % (c["n_rows"], c["context"]))
    rows = c["n_rows"] * (1 + c["beams"])
    used = sum(_pages(n, ps) for n in lens)
    n_pages = used + used // 4 + 2 * rows + 3
    order = list(range(n_pages))
    r.shuffle(order)
    stride = _pages(c["context"] + 1, ps) + 1
    refs, table = [0] * n_pages, [[-1] * stride for _ in range(rows)]
    at = 0
    for i, n in enumerate(lens):
        for j in range(_pages(n, ps)):
            shared = i % 4 == 3 and (j + 1) * ps <= min(n, lens[i - 1]) // 2
            if not shared:
                at += 1
            page = table[i - 1][j] if shared else order[at - 1]
            table[i][j] = page
            refs[page] += 1
    return refs, table, lens + [0] * (rows - len(lens))


def _fork_rows(c):
    sources = [i for i in range(c["n_rows"]) for _ in range(c["beams"])]
    return sources, list(range(c["n_rows"], c["n_rows"] * (1 + c["beams"])))


def work(case):
    c = case
    if c["op"] in ("fork", "compact"):
        page = c["layers"] * sum(_part_bytes(c))
        refs, table, lens = _pool_tables(c)
        if c["op"] == "fork":
            copies = sum(lens[i] % c["page_size"] != 0 for i in _fork_rows(c)[0])
            small = 4 * sum(_pages(lens[i], c["page_size"]) for i in _fork_rows(c)[0])
        else:
            live = set()
            for i, row in enumerate(table):
                if i % c["ended"] != c["ended"] - 1:
                    live.update(p for p in row if p >= 0)
            copies, small = sum(p >= len(live) for p in live), 4 * len(refs)
        return {"bytes": 2 * copies * page + 3 * small + 64, "flops": small + 64}
    n_h, n_kv, hd = c.get("heads", 0), c["kv_heads"], c["head_dim"]
    new, ctx = _lengths(c)
    t = sum(new)
    if c["op"] == "append":
        return {"bytes": t * n_kv * hd * 6, "flops": 8 * t * n_kv * hd}
    code = 1 if c["scale_tokens"] else 2
    scales = 8 * n_kv / c["scale_tokens"] if c["scale_tokens"] else 0
    if c["op"] == "chunk8":
        keys = sum(min(k, n + c["window"] - 1) if c["window"] else k for n, k in zip(new, ctx))
        pairs = sum(_pairs(n, k, c["causal"], c["window"]) for n, k in zip(new, ctx))
        return {"bytes": int(4 * hd * n_h * t + keys * (2 * hd * n_kv * code + scales)) + (4 * n_h * t if c["lse"] else 0),
                "flops": 4 * hd * n_h * pairs}
    # what all blocks of a sequence select is at most the sequence; the earlier pages' means, once
    keys, pairs, scores, means = [0] * len(new), 0, 0, sum((k - n) // c["page_size"] for n, k in zip(new, ctx))
    for b in _blocks(c):
        own_keys = _block_keys(c, b)
        keys[b[0]] += own_keys
        pairs += _pairs(b[2] - b[1], own_keys, True, 0)
        scores += b[1] // c["page_size"]
    keys = sum(min(a, k) for a, k in zip(keys, ctx))
    return {"bytes": int(4 * hd * n_h * t + keys * (2 * hd * n_kv * code + scales) + means * n_kv * hd * 4),
            "flops": 4 * hd * n_h * pairs + 2 * hd * n_kv * scores}


# ---- inputs ----------------------------------------------------------------------------------------------------------------

def _randn(gen, *shape):
    return torch.randn(shape, device=DEV, generator=gen)


def _hidden(gen, t, d):
    # (some channels are far larger than the others, as in a trained model)
    return (_randn(gen, t, d) * torch.exp(0.5 * _randn(gen, d))).to(torch.bfloat16)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _starts(lengths):
    s = [0]
    for n in lengths:
        s.append(s[-1] + n)
    return s


def _codes(values):
    return values.clamp(-448.0, 448.0).to(E4M3)


def _prepare_sequences(c, gen, s):
    new, ctx = _lengths(c)
    t, n_h, n_kv, hd, ps, st = sum(new), c["heads"], c["kv_heads"], c["head_dim"], c["page_size"], c["scale_tokens"]
    # the projections come as one product's output
    qkv = _hidden(gen, t, (n_h + 2 * n_kv) * hd)
    s["q"], s["k"], s["v"] = qkv[:, :n_h * hd], qkv[:, n_h * hd:(n_h + n_kv) * hd], qkv[:, (n_h + n_kv) * hd:]
    s["starts"], s["lens"] = _int32(_starts(new)), _int32(ctx)
    used = [_pages(n, ps) for n in ctx]
    n_pages = sum(used) + 5
    # (keys of one page are alike, as neighbouring tokens' are)
    keys = _randn(gen, n_pages, n_kv, ps, hd).add_(_randn(gen, n_pages, n_kv, 1, hd)) * torch.exp(0.5 * _randn(gen, hd))
    values = _randn(gen, n_pages, n_kv, ps, hd)
    if st:
        # a block's scale is the power of two that its largest value asks for
        for name, x in (("k", keys), ("v", values)):
            x = x.view(n_pages, n_kv, ps // st, st * hd)
            m, e = torch.frexp(x.abs().amax(dim=3))
            e = e - 9 + (m > 0.875).int()
            s[name + "_pages"] = _codes(x * torch.exp2(-e.float())[..., None]).view(n_pages, n_kv, ps, hd)
            s[name + "_scale"] = torch.exp2(e.float())
    else:
        s["k_pages"], s["v_pages"] = keys.to(torch.bfloat16), values.to(torch.bfloat16)
    order = torch.randperm(n_pages, device=DEV, generator=gen).to(torch.int32)
    table = torch.full((len(ctx), max(used)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for i, n in enumerate(used):
        table[i, :n] = order[at:at + n]
        at += n
    s["table"], s["max_chunk"] = table, max(new)
    if c["op"] == "select":
        s["means"] = _means_of(c, s, torch.arange(n_pages, device=DEV), torch.full((n_pages,), ps, device=DEV))


def _prepare_pool(c, gen, s):
    refs, table, lens = _pool_tables(c)
    s["first"] = {"refs": _int32(refs), "table": _int32(table), "lens": _int32(lens)}
    for name, x in s["first"].items():
        s[name] = x.clone()
    n_kv, hd, ps, n_pages = c["kv_heads"], c["head_dim"], c["page_size"], len(refs)
    parts = []
    for _ in range(c["layers"]):
        for _ in range(2):
            x = torch.empty((n_pages, n_kv, ps, hd), dtype=torch.bfloat16, device=DEV).normal_(generator=gen)
            parts.append(_codes(x * 64) if c["eight"] else x)
        if c["eight"]:
            parts += [torch.exp2(torch.randint(-17, -2, (n_pages, n_kv, 1), device=DEV, generator=gen).float()) for _ in range(2)]
            parts.append(_randn(gen, n_pages, n_kv, hd))
    s["parts"] = parts
    s["missing"] = _int32([-1])
    if c["op"] == "fork":
        sources, targets = _fork_rows(c)
        s["sources"], s["targets"] = _int32(sources), _int32(targets)
        rows = list(range(c["n_rows"])) + targets
        s["rows"] = _int32(rows)
        s["grown"] = _int32([lens[i] + 1 for i in list(range(c["n_rows"])) + sources])
    else:
        s["rows"] = _int32([i for i in range(c["n_rows"]) if i % c["ended"] == c["ended"] - 1] or [0])
        s["live"] = _int32([-1])


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    s = {"case": c}
    (_prepare_pool if c["op"] in ("fork", "compact") else _prepare_sequences)(c, gen, s)
    if own:
        _prepare_own(c, s)
    return s


def _prepare_own(c, s):
    from paper_2602_00397_amd import binding as B
    ctx = s["ctx"] = B.Context(0)
    if c["op"] in ("fork", "compact"):
        s["pool"] = B.page_pool(s["refs"], s["table"], s["lens"], c["page_size"], s["parts"])
        s["grow_missing"] = _int32([-1])
        ctx.ensure_pages_workspace(s["pool"], s["rows"].numel())
        return
    n_tokens, n_seqs = s["q"].shape[0], c["n_seqs"]
    s["shape"] = B.Attention(c["heads"], c["kv_heads"], c["head_dim"], c.get("causal", True), c.get("window", 0), c["head_dim"] ** -0.5)
    if c["scale_tokens"]:
        s["cache"] = B.paged_cache8(s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"])
    else:
        s["cache"] = B.paged_cache(s["k_pages"], s["v_pages"])
    if c["op"] == "append":
        return
    s["o"] = torch.empty((n_tokens, s["q"].shape[1]), dtype=torch.bfloat16, device=DEV)
    if c["op"] == "chunk8":
        ctx.ensure_attention_workspace(s["shape"], n_tokens, n_seqs)
        s["lse"] = torch.empty((n_tokens, c["heads"]), dtype=torch.float32, device=DEV) if c["lse"] else None
        return
    s["selection"] = B.selection(c["query_block"], c["keep"], c["first"])
    n_blocks, width = B.selection_blocks(s["selection"], n_tokens, n_seqs), B.selection_pages(s["selection"], c["page_size"])
    ctx.ensure_attention_workspace(s["shape"], n_tokens, n_blocks)
    ctx.ensure_selection_workspace(s["shape"], n_blocks, s["table"].shape[1])
    s["block_starts"], s["block_lens"] = (torch.empty(n_blocks + i, dtype=torch.int32, device=DEV) for i in (1, 0))
    s["block_tables"] = torch.empty((n_blocks, c["kv_heads"], width), dtype=torch.int32, device=DEV)


# ---- one pass --------------------------------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if c["op"] in ("fork", "compact"):
        # the program's own counts, tables and lengths, as they were before the pass
        for name, x in s["first"].items():
            s[name].copy_(x)
    if own:
        return _run_own(c, s)
    return {"append": _plain_append, "chunk8": _plain_chunk8, "select": _plain_select, "fork": _plain_fork, "compact": _plain_compact}[c["op"]](c, s)


def _cache_of(s):
    return {x: s[x] for x in ("k_pages", "v_pages", "k_scale", "v_scale")}


def _pool_of(s):
    return dict({x: s[x] for x in ("refs", "table", "lens", "missing")}, parts=s["parts"])


def _run_own(c, s):
    ctx = s["ctx"]
    if c["op"] == "append":
        ctx.cache8_append(s["shape"], s["k"], s["v"], s["starts"], s["lens"], s["cache"], s["table"])
        return _cache_of(s)
    if c["op"] == "chunk8":
        ctx.chunk_attention8(s["shape"], s["q"], s["starts"], s["lens"], s["max_chunk"], s["cache"], s["table"], s["o"], lse=s["lse"])
        return {"o": s["o"], "lse": s["lse"]} if c["lse"] else {"o": s["o"]}
    if c["op"] == "select":
        ctx.page_means(s["shape"], s["q"].shape[0], s["starts"], s["lens"], s["cache"], s["table"], s["means"])
        ctx.select_pages(s["shape"], s["selection"], s["q"], s["starts"], s["lens"], c["page_size"], s["means"], s["table"],
                         s["block_starts"], s["block_lens"], s["block_tables"])
        ctx.selected_attention(s["shape"], s["q"], s["block_starts"], s["block_lens"], min(c["query_block"], s["max_chunk"]), s["cache"],
                               s["block_tables"], s["o"])
        return {x: s[x] for x in ("o", "means", "block_starts", "block_lens", "block_tables")}
    if c["op"] == "fork":
        # (each call says how many pages it was short of; a program looks at both)
        ctx.pages_fork(s["pool"], s["sources"], s["targets"], s["missing"])
        ctx.pages_grow(s["pool"], s["rows"], s["grown"], s["grow_missing"])
        s["missing"].add_(s["grow_missing"])
        return _pool_of(s)
    ctx.pages_free(s["pool"], s["rows"])
    ctx.pages_compact(s["pool"], s["live"])
    return dict(_pool_of(s), live=s["live"])


# ---- the plain forms -------------------------------------------------------------------------------------------------------

def _tokens(c, s):
    """Sequence and position of every new token."""
    new = (s["starts"][1:] - s["starts"][:-1]).long()
    t = s["k"].shape[0]
    seq = torch.repeat_interleave(torch.arange(c["n_seqs"], device=DEV), new, output_size=t)
    return seq, torch.arange(t, device=DEV) + (s["lens"].long() - s["starts"][1:].long())[seq]


def _plain_append(c, s):
    st, hd, n_kv = c["scale_tokens"], c["head_dim"], c["kv_heads"]
    per_page = c["page_size"] // st
    seq, pos = _tokens(c, s)
    page = s["table"][seq, pos // c["page_size"]].long()
    block, place = page * per_page + pos % c["page_size"] // st, pos % st
    n_blocks = s["k_scale"].shape[0] * per_page
    # the new tokens' first place in each block that gets some
    first = torch.full((n_blocks,), st, device=DEV).scatter_reduce_(0, block, place, "amin")
    touched = torch.nonzero(first < st)[:, 0]
    tp, tb, tf = touched // per_page, touched % per_page, first[touched]
    for name in ("k", "v"):
        x = s[name].reshape(-1, n_kv, hd).float()
        codes, scales = s[name + "_pages"].view(-1, n_kv, per_page, st, hd), s[name + "_scale"]
        top = torch.zeros((n_blocks, n_kv), device=DEV).scatter_reduce_(0, block[:, None].expand(-1, n_kv), x.abs().amax(dim=2), "amax")[touched]
        m, e = torch.frexp(top)
        need = torch.where(top > 0, e - 9 + (m > 0.875).int(), torch.full_like(e, -110)).clamp(-110, 80)
        need, old = torch.exp2(need.float()), scales[tp, :, tb]
        now = torch.where((tf == 0)[:, None], need, torch.maximum(old, need))
        # older tokens of a block whose scale grows
        raw = codes.view(torch.uint8)[tp, :, tb].view(E4M3)
        again = _codes(raw.float() * (old / now)[:, :, None, None])
        kept = torch.arange(st, device=DEV) < tf[:, None]
        codes.view(torch.uint8)[tp, :, tb] = torch.where(kept[:, None, :, None], again.view(torch.uint8), raw.view(torch.uint8))
        scales[tp, :, tb] = now
        scale = scales[page, :, block % per_page]
        codes.view(torch.uint8)[page, :, block % per_page, place] = _codes(x / scale[:, :, None]).view(torch.uint8)
    return _cache_of(s)


def _gathered(c, s, name, pages):
    """Keys or values of pages [...][n], float32 [...][n * page_size][kv_heads][head_dim] (entries below 0: any page)."""
    pages = pages.clamp(min=0).long()
    if c["scale_tokens"]:
        codes, scales = s[name + "_pages"].view(torch.uint8)[pages].view(E4M3).float(), s[name + "_scale"][pages]
        shape = codes.shape
        x = codes.view(*shape[:-2], -1, c["scale_tokens"], shape[-1]) * scales[..., None, None]
        x = x.view(shape)
    else:
        x = s[name + "_pages"][pages].float()
    return x.transpose(-3, -2).reshape(*pages.shape[:-1], -1, c["kv_heads"], c["head_dim"])


def _plain_attend(c, q, k, v, seen):
    """q [b][n][heads][hd]; k, v [b][keys][kv_heads][hd] (or [b][kv_heads][keys][hd], already by head); seen [b][n][keys] -> o, lse."""
    b, n, n_h, hd = q.shape
    n_kv, group = c["kv_heads"], n_h // c["kv_heads"]
    q = q.view(b, n, n_kv, group, hd).permute(0, 2, 1, 3, 4).reshape(b, n_kv, n * group, hd)
    x = (q @ k.transpose(2, 3).contiguous()).mul_(hd ** -0.5).view(b, n_kv, n, group, -1)
    x.masked_fill_(~seen[:, None, :, None], -math.inf)
    m = x.amax(dim=4, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = x.sub_(m).exp_()
    l = p.sum(dim=4, keepdim=True)
    o = (p.view(b, n_kv, n * group, -1) @ v).view(b, n_kv, n, group, hd) / torch.where(l > 0, l, torch.ones_like(l))
    lse = (m + torch.log(l))[..., 0]
    return o.permute(0, 2, 1, 3, 4).reshape(b, n, n_h, hd), lse.permute(0, 2, 1, 3).reshape(b, n, n_h)


def _padded(s, starts, n_rows, t):
    """Which row of q stands at each place of [sequences][n_rows], and whether there is one."""
    at = starts[:-1].long()[:, None] + torch.arange(n_rows, device=DEV)
    return at.clamp(max=t - 1), at < starts[1:].long()[:, None]


def _at_once(n, values_each):
    """How many of n sequences to take at a time."""
    return max(1, min(n, (1 << 30) // max(1, values_each)))


def _plain_chunk8(c, s):
    t, n, ps, n_kv = s["q"].shape[0], s["max_chunk"], c["page_size"], c["kv_heads"]
    q = s["q"].reshape(t, -1, c["head_dim"])
    o, lse = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV), torch.empty((t, c["heads"]), device=DEV)
    at, is_row = _padded(s, s["starts"], n, t)
    new = (s["starts"][1:] - s["starts"][:-1])[:, None, None]
    keys = s["table"].shape[1] * ps
    step = _at_once(c["n_seqs"], keys * max(n * c["heads"], 4 * n_kv * c["head_dim"]))
    j = torch.arange(keys, device=DEV)
    for a in range(0, c["n_seqs"], step):
        b = slice(a, a + step)
        k, v = (_gathered(c, s, x, s["table"][b]).transpose(1, 2).contiguous() for x in ("k", "v"))
        lens = s["lens"][b, None, None]
        if c["causal"]:
            pos = lens - new[b] + torch.arange(n, device=DEV)[:, None]
            seen = (j <= pos) & (j > pos - (c["window"] or 1 << 30))
        else:
            seen = (j < lens).expand(-1, n, -1)
        part, l = _plain_attend(c, q[at[b]].float(), k, v, seen)
        o[at[b][is_row[b]]] = part[is_row[b]].to(torch.bfloat16)
        lse[at[b][is_row[b]]] = l[is_row[b]]
    o = o.reshape(t, -1)
    return {"o": o, "lse": lse} if c["lse"] else {"o": o}


def _means_of(c, s, pages, live):
    """Mean key of the first `live` places of each page, float32 [n][kv_heads][head_dim]."""
    x = _gathered(c, s, "k", pages[:, None]).double()
    on = torch.arange(c["page_size"], device=DEV) < live[:, None]
    return ((x * on[:, :, None, None]).sum(dim=1) / live.double()[:, None, None]).float()


def _plain_select(c, s):
    ps, qb, n_kv, hd, t, n_seqs = c["page_size"], c["query_block"], c["kv_heads"], c["head_dim"], s["q"].shape[0], c["n_seqs"]
    seq, pos = _tokens(c, s)
    # pages with new tokens
    ends = (pos % ps == ps - 1) | (pos == s["lens"].long()[seq] - 1)
    at = torch.nonzero(ends)[:, 0]
    changed = s["table"][seq[at], pos[at] // ps].long()
    s["means"][changed] = _means_of(c, s, changed, pos[at] % ps + 1)
    # blocks
    new, lens = (s["starts"][1:] - s["starts"][:-1]).long(), s["lens"].long()
    of_seq = (new + qb - 1) // qb
    n_blocks, most = min(t, t // qb + n_seqs), int(t // qb + n_seqs)
    owner = torch.repeat_interleave(torch.arange(n_seqs + 1, device=DEV), torch.cat([of_seq, (most - of_seq.sum())[None]]), output_size=most)[:n_blocks]
    is_block = owner < n_seqs
    owner = owner.clamp(max=n_seqs - 1)
    number = torch.arange(n_blocks, device=DEV) - (of_seq.cumsum(0) - of_seq)[owner]
    t0 = torch.where(is_block, s["starts"].long()[owner] + number * qb, torch.full_like(number, t))
    t1 = torch.where(is_block, torch.minimum(t0 + qb, s["starts"].long()[owner + 1]), t0)
    p0 = lens[owner] - s["starts"].long()[owner + 1] + t0
    p1 = p0 + t1 - t0
    earlier, last = torch.where(is_block, p0 // ps, 0), torch.where(is_block, (p1 - 1) // ps, -1)
    kept, own_pages = earlier.clamp(max=c["keep"]), last - torch.where(is_block, earlier, 0) + 1
    block_starts = torch.cat([t0, t0.new_full((1,), t)]).int()
    block_lens = torch.where(is_block, (kept + own_pages) * ps - (-p1) % ps, 0).int()
    # scores of the earlier pages: the block's queries of a key head, summed, times the page's mean key
    rows, is_row = _padded(s, block_starts, qb, t)
    q = s["q"].reshape(t, n_kv, -1, hd).double().sum(dim=2)
    q = torch.where(is_row[:, :, None, None], q[rows], torch.zeros((), dtype=torch.float64, device=DEV)).sum(dim=1)
    width, stride = c["keep"] + (qb + ps - 2) // ps + 1, s["table"].shape[1]
    scores = torch.empty((n_blocks, n_kv, stride), dtype=torch.float64, device=DEV)
    step = _at_once(n_blocks, stride * n_kv * hd)
    for a in range(0, n_blocks, step):
        b = slice(a, a + step)
        means = s["means"][s["table"][owner[b]].clamp(min=0).long()].double()      # [b][pages][kv_heads][hd]
        scores[b] = (means * q[b, None]).sum(dim=3).transpose(1, 2)
    page = torch.arange(stride, device=DEV)
    scores.masked_fill_(page < c["first"], math.inf)
    scores.masked_fill_(page >= earlier[:, None, None], -math.inf)
    best = torch.sort(scores, dim=2, descending=True, stable=True).indices[:, :, :c["keep"]]
    place = torch.arange(width, device=DEV)
    best = torch.nn.functional.pad(best, (0, width - best.shape[2]))
    chosen = torch.where(place < kept[:, None, None], best, stride + 1)
    chosen = torch.sort(chosen, dim=2).values
    mine = earlier[:, None, None] + place - kept[:, None, None]
    chosen = torch.where(place < kept[:, None, None], chosen, mine)
    listed_ = (place < (kept + own_pages)[:, None, None]).expand_as(chosen)
    block_tables = torch.where(listed_, s["table"][owner[:, None, None], chosen.clamp(max=stride - 1)], -1).int()
    # attention over what is selected
    n, keys = min(qb, s["max_chunk"]), width * ps
    o = torch.empty((t, c["heads"], hd), dtype=torch.bfloat16, device=DEV)
    qr = s["q"].reshape(t, -1, hd)
    step = _at_once(n_blocks, keys * max(n * c["heads"], 4 * n_kv * n_kv * hd))
    j, head = torch.arange(keys, device=DEV), torch.arange(n_kv, device=DEV)
    for a in range(0, n_blocks, step):
        b = slice(a, a + step)
        k, v = (_of_own_head(c, s, x, block_tables[b], head) for x in ("k", "v"))
        limit = block_lens[b, None, None] - (t1 - t0)[b, None, None] + torch.arange(n, device=DEV)[:, None]
        part, _ = _plain_attend(c, qr[rows[b, :n]].float(), k, v, j <= limit)
        o[rows[b, :n][is_row[b, :n]]] = part[is_row[b, :n]].to(torch.bfloat16)
    return {"o": o.reshape(t, -1), "means": s["means"], "block_starts": block_starts, "block_lens": block_lens, "block_tables": block_tables}


def _of_own_head(c, s, name, tables, head):
    """Keys or values of tables [b][kv_heads][n], each head its own pages, float32 [b][kv_heads][n * page_size][hd]."""
    pages, h = tables.clamp(min=0).long(), head[:, None]
    if c["scale_tokens"]:
        x = s[name + "_pages"].view(torch.uint8)[pages, h].view(E4M3).float()
        shape = x.shape
        scale = s[name + "_scale"][pages, h]
        x = (x.view(*shape[:3], -1, c["scale_tokens"], shape[-1]) * scale[..., None, None]).view(shape)
    else:
        x = s[name + "_pages"][pages, h].float()
    return x.reshape(*tables.shape[:2], -1, c["head_dim"])


def _move(s, origin, target):
    for x in s["parts"]:
        x = x.view(torch.uint8) if x.dtype == E4M3 else x
        x[target] = x[origin]


def _free_pages(s, n):
    """The first n free pages, in order, and how many there are."""
    order = torch.sort((s["refs"] != 0).int(), stable=True).indices
    return order[:n], (s["refs"] == 0).sum()


def _plain_fork(c, s):
    ps, stride = c["page_size"], s["table"].shape[1]
    src, dst = s["sources"].long(), s["targets"].long()
    rows, lens = s["table"][src], s["lens"][src]
    col = torch.arange(stride, device=DEV)
    partial = lens % ps != 0
    free, n_free = _free_pages(s, src.numel())
    rank = partial.long().cumsum(0) - 1
    page = free[rank.clamp(min=0)]
    last = (lens // ps).long().clamp(max=stride - 1)
    origin = rows.gather(1, last[:, None])[:, 0].clamp(min=0).long()
    rows = torch.where((col == last[:, None]) & partial[:, None], page[:, None].int(), rows)
    held = torch.where(rows >= 0, 1, 0).int()
    # (the rows that are written held nothing before)
    s["refs"].index_add_(0, rows.clamp(min=0).reshape(-1).long(), held.reshape(-1))
    s["table"][dst], s["lens"][dst] = rows, lens
    _move(s, origin[partial], page[partial])
    missing = (partial.sum() - n_free).clamp(min=0)
    # one more token each
    r, want = s["rows"].long(), s["grown"]
    have, need = (s["lens"][r] + ps - 1) // ps, (want + ps - 1) // ps
    more = (need > have).long()
    free, n_free = _free_pages(s, r.numel())
    page = free[(more.cumsum(0) - 1).clamp(min=0)]
    at = have.long().clamp(max=stride - 1)
    s["table"][r, at] = torch.where(more > 0, page.int(), s["table"][r, at])
    s["refs"].index_add_(0, page, more.int())
    s["lens"][r] = want
    s["missing"].copy_(missing + (more.sum() - n_free).clamp(min=0))
    return _pool_of(s)


def _plain_compact(c, s):
    r = s["rows"].long()
    rows = s["table"][r]
    s["refs"].index_add_(0, rows.clamp(min=0).reshape(-1).long(), -(rows >= 0).int().reshape(-1))
    s["table"][r] = -1
    s["lens"][r] = 0
    used = s["refs"] > 0
    live = used.sum()
    page = torch.arange(used.numel(), device=DEV)
    holes = torch.sort((used | (page >= live)).int(), stable=True).indices     # the free pages below `live` first
    moves = used & (page >= live)
    target = torch.where(moves, holes[(moves.long().cumsum(0) - 1).clamp(min=0)], page)
    origin = torch.nonzero(moves)[:, 0]
    s["table"].copy_(torch.where(s["table"] >= 0, target[s["table"].clamp(min=0).long()].int(), s["table"]))
    _move(s, origin, target[origin])
    s["refs"][target[origin]] = s["refs"][origin]
    s["refs"][origin] = 0
    s["live"].copy_(live)
    return dict(_pool_of(s), live=s["live"])


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    return {"append": _exact_append, "chunk8": _exact_chunk8, "select": _exact_select, "fork": _exact_pool, "compact": _exact_pool}[c["op"]](c, s)


def _decoded(s, name):
    """The values that a cache stands for, from the codes' bits, float64 [n_pages][kv_heads][page_size][hd]."""
    if name + "_scale" not in s:
        return s[name + "_pages"].double()
    byte = s[name + "_pages"].view(torch.uint8).int()
    sign, e, m = 1 - 2 * (byte >> 7), (byte >> 3) & 15, byte & 7
    x = torch.ldexp(torch.where(e > 0, 8 + m, m).double() * sign, e.clamp(min=1) - 10)
    scales = s[name + "_scale"].double()
    return x * scales.repeat_interleave(x.shape[2] // scales.shape[2], dim=2)[..., None]


def _exact_append(c, s):
    """Codes before they are rounded to 8 bits, and the scales."""
    st, hd, ps = c["scale_tokens"], c["head_dim"], c["page_size"]
    out = {}
    table = s["table"].tolist()
    for name in ("k", "v"):
        exps = torch.frexp(s[name + "_scale"])[1] - 1
        values = torch.ldexp(_decoded(s, name), -exps.repeat_interleave(st, dim=2)[..., None])
        new_all = s[name].double().reshape(-1, c["kv_heads"], hd).transpose(0, 1)
        t = 0
        for i, (n, keys) in enumerate(zip(*_lengths(c))):
            at = keys - n
            while at < keys:
                end = min(keys, at // st * st + st)
                page, b, p = table[i][at // ps], at % ps // st, at % ps
                x = new_all[:, t:t + end - at]
                top = x.abs().amax(dim=(1, 2))
                need = torch.where(top > 0, torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0)), -110.0).clamp(-110, 80).int()
                old = exps[page, :, b]
                now = need if at % st == 0 else torch.maximum(old, need)
                if at % st:
                    values[page, :, b * st:p] = torch.ldexp(values[page, :, b * st:p], (old - now)[:, None, None])
                values[page, :, p:p + end - at] = torch.ldexp(x, -now[:, None, None])
                exps[page, :, b] = now
                t += end - at
                at = end
        out[name + "_pages"], out[name + "_scale"] = values, torch.ldexp(torch.ones_like(exps, dtype=torch.float64), exps)
    return out


def _exact_rows(c, q, k, v, first, window):
    """Rows q [n][hd] of one head, the first at place `first` of keys k, v [keys][hd]; first None: every row sees every key."""
    o = torch.zeros_like(q)
    lse = torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=DEV)
    for a in range(0, q.shape[0], 2048):
        b = min(q.shape[0], a + 2048)
        logits = q[a:b] @ k.t() / math.sqrt(c["head_dim"])
        if first is not None:
            distance = torch.arange(first + a, first + b, device=DEV)[:, None] - torch.arange(k.shape[0], device=DEV)
            logits = torch.where((distance >= 0) & (distance < (window or 1 << 40)), logits, -math.inf)
        lse[a:b] = torch.logsumexp(logits, dim=1)
        o[a:b] = torch.exp(logits - lse[a:b, None]) @ v
    return o, lse


def _exact_chunk8(c, s):
    t, hd, ps, group = s["q"].shape[0], c["head_dim"], c["page_size"], c["heads"] // c["kv_heads"]
    o = torch.zeros((t, c["heads"], hd), dtype=torch.float64, device=DEV)
    lse = torch.zeros((t, c["heads"]), dtype=torch.float64, device=DEV)
    k_all, v_all = _decoded(s, "k"), _decoded(s, "v")
    q = s["q"].double().reshape(t, -1, hd)
    row = 0
    for i, (n, keys) in enumerate(zip(*_lengths(c))):
        pages = s["table"][i, :_pages(keys, ps)].long()
        for h in range(c["heads"]):
            k, v = (x[pages, h // group].reshape(-1, hd)[:keys] for x in (k_all, v_all))
            o[row:row + n, h], lse[row:row + n, h] = _exact_rows(c, q[row:row + n, h], k, v, keys - n if c["causal"] else None, c["window"])
        row += n
    o = o.reshape(t, -1)
    return {"o": o, "lse": lse} if c["lse"] else {"o": o}


def _exact_select(c, s):
    blocks = _blocks(c)
    ps, hd, n_kv, group, t = c["page_size"], c["head_dim"], c["kv_heads"], c["heads"] // c["kv_heads"], s["q"].shape[0]
    if len(blocks) * c["heads"] > 20000:
        return None
    new, ctx = _lengths(c)
    k_all, v_all, means = _decoded(s, "k"), _decoded(s, "v"), s["means"].double()
    for i, (n, keys) in enumerate(zip(new, ctx)):
        for j in range((keys - n) // ps, _pages(keys, ps)):
            page = int(s["table"][i, j])
            means[page] = k_all[page, :, :min(ps, keys - j * ps)].mean(dim=1)
    rounded = means.float().double()
    width, n_blocks = c["keep"] + (c["query_block"] + ps - 2) // ps + 1, min(t, t // c["query_block"] + len(new))
    starts, lens = torch.full((n_blocks + 1,), t, dtype=torch.int32), torch.zeros(n_blocks, dtype=torch.int32)
    tables = torch.full((n_blocks, n_kv, width), -1, dtype=torch.int32, device=DEV)
    o = torch.zeros((t, c["heads"], hd), dtype=torch.float64, device=DEV)
    row = 0
    for x, (i, a, b, kept, own_pages) in enumerate(blocks):
        starts[x], lens[x] = row, _block_keys(c, (i, a, b, kept, own_pages))
        q = s["q"][row:row + b - a].double().reshape(b - a, n_kv, group, hd)
        earlier = s["table"][i, :a // ps].long()
        for g in range(n_kv):
            score = rounded[earlier, g] @ q[:, g].sum(dim=(0, 1))
            score[:c["first"]] = math.inf
            best = torch.topk(score, kept).indices.sort().values if kept else torch.zeros(0, dtype=torch.long, device=DEV)
            pages = torch.cat([earlier[best], s["table"][i, a // ps:a // ps + own_pages].long()])
            tables[x, g, :kept + own_pages] = pages.int()
            k, v = (z[pages, g].reshape(-1, hd)[:int(lens[x])] for z in (k_all, v_all))
            for h in range(group):
                o[row:row + b - a, g * group + h], _ = _exact_rows(c, q[:, g, h], k, v, int(lens[x]) - (b - a), 0)
        row += b - a
    return {"o": o.reshape(t, -1), "means": means, "block_starts": starts.to(DEV), "block_lens": lens.to(DEV), "block_tables": tables}


def _exact_pool(c, s):
    """The counts, tables and lengths, one page after another on the host; the parts are copies of what is given."""
    ps = c["page_size"]
    refs, table, lens = s["refs"].tolist(), s["table"].tolist(), s["lens"].tolist()
    free = [p for p, n in enumerate(refs) if n == 0]
    out = {}
    if c["op"] == "fork":
        for a, b in zip(s["sources"].tolist(), s["targets"].tolist()):
            for j, page in enumerate(table[a]):
                if page >= 0 and j == lens[a] // ps:
                    page = free.pop(0)
                if page >= 0:
                    refs[page] += 1
                table[b][j] = page
            lens[b] = lens[a]
        for a, n in zip(s["rows"].tolist(), s["grown"].tolist()):
            for j in range(_pages(lens[a], ps), _pages(n, ps)):
                table[a][j] = free.pop(0)
                refs[table[a][j]] = 1
            lens[a] = n
        out["missing"] = _int32([0])
    else:
        for a in s["rows"].tolist():
            for page in table[a]:
                refs[page] -= page >= 0
            table[a], lens[a] = [-1] * len(table[a]), 0
        live = sum(n > 0 for n in refs)
        holes = [p for p in range(live) if refs[p] == 0]
        place = {}
        for p in range(live, len(refs)):
            if refs[p] > 0:
                place[p] = holes.pop(0)
                refs[place[p]], refs[p] = refs[p], 0
        table = [[place.get(p, p) for p in row] for row in table]
        out["missing"], out["live"] = s["missing"], _int32([live])
    return dict(out, refs=_int32(refs), table=_int32(table), lens=_int32(lens), parts=None)
