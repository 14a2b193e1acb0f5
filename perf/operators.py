"""The attention half of a layer and the norms around it, as measurable cases.

A case is a dict of plain values.  By its "op":

  "norm"    ff_norm_residual: n_tokens, d_model, y ("bf16" or "f32"), post, pre ("none", "rms", "layer"), gate ("none" or
            how many tokens share a row of it), scale
  "rotary"  ff_rotary: n_tokens, heads, kv_heads, head_dim, rot_dim, interleaved, axes, page_size; "prompt" says whether the
            tokens are one prompt (positions in order, k kept beside the cache) or one of many sequences each
  "prompt"  ff_prompt_attention: n_tokens in n_seqs packed sequences, heads, kv_heads, head_dim, causal, window, lse
  "chunk"   ff_chunk_attention: n_seqs sequences with up to `chunk` new tokens each (mixed: about half of them generate one
            token) over up to `context` cached ones (spread: the others' lengths lie below the first's), page_size, and
            heads, kv_heads, head_dim, causal, window, lse

Sizes are those of the benchmark configurations' models (workloads.CONFIGS) and generic ones.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
# heads, kv_heads, head_dim of the configurations' models
TINY, M1B, M8B, M7B = (4, 2, 64), (32, 8, 64), (32, 8, 128), (28, 4, 128)
D_MODEL = {TINY: 256, M1B: 2048, M8B: 4096, M7B: 3584}
EPS = 1e-6
THETA = 500000.0


def _heads(m):
    return {"heads": m[0], "kv_heads": m[1], "head_dim": m[2]}


def _norm_case(d_model, n_tokens, y="bf16", post="none", pre="rms", gate="none", scale=1.0):
    return {"op": "norm", "d_model": d_model, "n_tokens": n_tokens, "y": y, "post": post, "pre": pre,
            "gate": gate if gate == "none" else int(gate), "scale": scale}


def _rotary_case(m, n_tokens, prompt, rot_dim=None, interleaved=False, axes=1, page_size=64):
    return dict(_heads(m), op="rotary", n_tokens=n_tokens, prompt=prompt, rot_dim=rot_dim or m[2], interleaved=interleaved,
                axes=axes, page_size=page_size)


def _prompt_case(m, n_tokens, n_seqs=1, causal=True, window=0, lse=False):
    return dict(_heads(m), op="prompt", n_tokens=n_tokens, n_seqs=n_seqs, causal=causal, window=window, lse=lse)


def _chunk_case(m, n_seqs, chunk, context, mixed=False, spread=True, page_size=64, causal=True, window=0, lse=False):
    return dict(_heads(m), op="chunk", n_seqs=n_seqs, chunk=chunk, context=context, mixed=mixed, spread=spread,
                page_size=page_size, causal=causal, window=window, lse=lse)


def listed():
    return [
        # between the halves of a layer, one sequence generating: latency
        dict(_norm_case(4096, 1), name="norm_token_8b"),
        # a prompt of odd length through a layer-normed model, the FFN's fp32 output
        dict(_norm_case(2048, 777, y="f32", pre="layer", scale=0.5), name="norm_prompt777_1b"),
        # the stack configuration's long prompt, norms before and after the block, a gate row for each block of 128 tokens
        dict(_norm_case(3584, 16384, post="rms", gate=128), name="norm_prompt16384_7b"),
        # 64 sequences generating one token each, far into their contexts
        dict(_rotary_case(M8B, 64, False), name="rotary_tokens64_8b"),
        # an image prompt: time, height and width positions, half of the pairs for the first
        dict(_rotary_case(M7B, 9001, True, axes=3), name="rotary_image9001_7b"),
        # packed prompts of all lengths, narrow heads
        dict(_prompt_case(M1B, 4099, n_seqs=13, lse=True), name="prompts4099_packed_1b"),
        # the headline configuration's prompt
        dict(_prompt_case(M8B, 8192), name="prompt8192_8b"),
        # the stack configuration's long prompt through a layer with a window
        dict(_prompt_case(M7B, 16384, window=4096), name="prompt16384_window_7b"),
        # one sequence generating one token
        dict(_chunk_case(M8B, 1, 1, 8191), name="chunk_token_8b"),
        # 48 sequences generating together
        dict(_chunk_case(M8B, 48, 1, 16384, lse=True), name="chunk_tokens48_8b"),
        # one block of the chunked prefill over a long context
        dict(_chunk_case(M8B, 1, 128, 8192, page_size=128), name="chunk_block128_8b"),
        # a server's step: some sequences generate, the others bring a piece of their prompt
        dict(_chunk_case(M1B, 12, 500, 6000, mixed=True, page_size=16), name="chunk_mixed_1b"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw(rng):
    op = rng.choice(["norm"] * 2 + ["rotary"] * 2 + ["prompt"] * 3 + ["chunk"] * 4)
    m = rng.choice([TINY, M1B, M1B, M8B, M8B, M8B, M7B, M7B])
    if op == "norm":
        t = _log_int(rng, 1, 16384)
        gate = rng.choice(["none", "none", 1, 128, t])
        return _norm_case(rng.choice([D_MODEL[m], 8 * _log_int(rng, 8, 1024)]), t, y=rng.choice(["bf16", "bf16", "f32"]),
                          post=rng.choice(["none", "none", "rms", "layer"]), pre=rng.choice(["rms", "rms", "layer"]),
                          gate=gate, scale=rng.choice([1.0, 1.0, 0.22, round(rng.uniform(0.1, 2.0), 3)]))
    if op == "rotary":
        rot = rng.choice([m[2], m[2], m[2], m[2] // 2, m[2] // 4])
        return _rotary_case(m, _log_int(rng, 1, 9001), rng.random() < 0.5, rot_dim=rot, interleaved=rng.random() < 0.3,
                            axes=rng.choice([1, 1, 1, 2, 3]), page_size=rng.choice([16, 64, 128]))
    causal = rng.random() < 0.9
    window = _log_int(rng, 1, 8192) if causal and rng.random() < 0.25 else 0
    lse = rng.random() < 0.3
    if op == "prompt":
        t = _log_int(rng, 1, 16384)
        n_seqs = 1 if rng.random() < 0.4 else _log_int(rng, 2, 64)
        return _prompt_case(m, t, n_seqs=n_seqs, causal=causal, window=window, lse=lse)
    kind = rng.choice(["tokens", "tokens", "chunk", "mixed"])
    page_size = rng.choice([16, 64, 128])
    context = _log_int(rng, 1, 32768)
    if kind == "tokens":
        n_seqs, chunk = _log_int(rng, 1, 96), rng.choice([1, 1, 1, rng.randint(1, 8)])
    elif kind == "chunk":
        n_seqs, chunk = rng.choice([1, 1, rng.randint(1, 6)]), _log_int(rng, 2, 1024)
    else:
        n_seqs, chunk = rng.randint(2, 48), _log_int(rng, 2, 700)
    return _chunk_case(m, n_seqs, min(chunk, context), context, mixed=kind == "mixed", spread=rng.random() < 0.8,
                       page_size=page_size, causal=causal, window=window, lse=lse)


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

def _prompt_lengths(c):
    r = random.Random("%d in %d" % (c["n_tokens"], c["n_seqs"]))
    cuts = sorted(r.randint(0, c["n_tokens"]) for _ in range(c["n_seqs"] - 1))
    ends = cuts + [c["n_tokens"]]
    return [b - a for a, b in zip([0] + cuts, ends)]


def _chunk_lengths(c):
    """New tokens and cached tokens (the new ones included) of every sequence; the first has the most of both."""
    r = random.Random("%d %d %d" % (c["n_seqs"], c["chunk"], c["context"]))
    new, ctx = [c["chunk"]], [c["context"]]
    for _ in range(c["n_seqs"] - 1):
        n = c["chunk"] if not c["mixed"] else (1 if r.random() < 0.5 else r.randint(1, c["chunk"]))
        new.append(n)
        ctx.append(_log_int(r, n, c["context"]) if c["spread"] else c["context"])
    return new, ctx


def _sequences(c):
    """(new tokens, keys) of every sequence."""
    if c["op"] == "prompt":
        return [(n, n) for n in _prompt_lengths(c)]
    return list(zip(*_chunk_lengths(c)))


def _pairs(n, keys, causal, window):
    """How many (token, key) pairs a sequence's mask leaves."""
    if not causal:
        return n * keys
    seen = [keys - n + i + 1 for i in range(n)]
    return sum(min(max(s, 0), window) if window else max(s, 0) for s in seen)


def _keys_read(n, keys, window):
    return min(keys, n + window - 1) if window else keys


def work(case):
    c = case
    if c["op"] == "norm":
        t, d = c["n_tokens"], c["d_model"]
        gate_rows = 0 if c["gate"] == "none" else -(-t // c["gate"])
        return {"bytes": t * d * (6 + (4 if c["y"] == "f32" else 2)) + gate_rows * d * 2, "flops": 12 * t * d}
    n_h, n_kv, hd = c["heads"], c["kv_heads"], c["head_dim"]
    if c["op"] == "rotary":
        t = c["n_tokens"]
        writes = n_h + (3 if c["prompt"] else 2) * n_kv
        return {"bytes": t * (hd * 2 * (n_h + 2 * n_kv + writes) + 4 * c["axes"] + 4), "flops": 3 * t * c["rot_dim"] * (n_h + n_kv)}
    seqs = _sequences(c)
    t = sum(n for n, _ in seqs)
    pairs = sum(_pairs(n, k, c["causal"], c["window"]) for n, k in seqs)
    keys = sum(_keys_read(n, k, c["window"]) for n, k in seqs)
    return {"bytes": 4 * hd * (n_h * t + n_kv * keys) + (4 * n_h * t if c["lse"] else 0), "flops": 4 * hd * n_h * pairs}


# ---- inputs ----------------------------------------------------------------------------------------------------------------

def _randn(gen, *shape):
    return torch.randn(shape, device=DEV, generator=gen)


def _hidden(gen, t, d, dtype=torch.bfloat16):
    # (some channels are far larger than the others, as in a trained model)
    return (_randn(gen, t, d) * torch.exp(0.5 * _randn(gen, d))).to(dtype)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _starts(lengths):
    s = [0]
    for n in lengths:
        s.append(s[-1] + n)
    return s


def _prepare_norm(c, gen, s):
    t, d = c["n_tokens"], c["d_model"]
    s["h"] = _hidden(gen, t, d)
    s["y"] = _hidden(gen, t, d, torch.float32 if c["y"] == "f32" else torch.bfloat16)
    for which in ("post", "pre"):
        s[which] = None
        if c[which] != "none":
            gain = (1.0 + 0.1 * _randn(gen, d)).to(torch.bfloat16)
            bias = (0.1 * _randn(gen, d)).to(torch.bfloat16) if c[which] == "layer" else None
            s[which] = (gain, bias)
    s["gate"] = None if c["gate"] == "none" else torch.tanh(_randn(gen, -(-t // c["gate"]), d)).to(torch.bfloat16)
    if own:
        s["h_out"], s["x"] = torch.empty_like(s["h"]), torch.empty_like(s["h"])


def _prepare_rotary(c, gen, s):
    t, n_h, n_kv, hd, ps = c["n_tokens"], c["heads"], c["kv_heads"], c["head_dim"], c["page_size"]
    # the projections come as one product's output
    qkv = _hidden(gen, t, (n_h + 2 * n_kv) * hd)
    s["q"], s["k"], s["v"] = qkv[:, :n_h * hd], qkv[:, n_h * hd:(n_h + n_kv) * hd], qkv[:, (n_h + n_kv) * hd:]
    pairs = c["rot_dim"] // 2
    s["inv_freq"] = (THETA ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).float().to(DEV)
    # the first axis (time) has half of the pairs, the others share the rest
    s["axis"] = [0] * pairs if c["axes"] == 1 else [max(0, 2 * i - pairs) * (c["axes"] - 1) // pairs + (2 * i >= pairs) for i in range(pairs)]
    if c["prompt"]:
        pos = [torch.arange(t, dtype=torch.int32, device=DEV)]
        side = max(1, math.isqrt(t))
        pos += [pos[0] // side, pos[0] % side][:c["axes"] - 1]
        s["positions"] = torch.stack(pos)
    else:
        s["positions"] = torch.randint(0, 131072, (c["axes"], t), device=DEV, dtype=torch.int32, generator=gen)
    n_pages = -(-t // ps) + 3 if c["prompt"] else t + 3
    s["k_pages"], s["v_pages"] = (_randn(gen, n_pages, n_kv, ps, hd).to(torch.bfloat16) for _ in range(2))
    page = torch.randperm(n_pages, device=DEV, generator=gen)
    i = torch.arange(t, device=DEV)
    slots = page[i // ps] * ps + i % ps if c["prompt"] else page[i] * ps + s["positions"][0] % ps
    s["slots"] = slots.to(torch.int32)
    if own:
        s["q_out"] = torch.empty((t, n_h * hd), dtype=torch.bfloat16, device=DEV)
        s["k_out"] = torch.empty((t, n_kv * hd), dtype=torch.bfloat16, device=DEV) if c["prompt"] else None


def _prepare_prompt(c, gen, s):
    t, n_h, n_kv, hd = c["n_tokens"], c["heads"], c["kv_heads"], c["head_dim"]
    s["q"], s["k"] = _hidden(gen, t, n_h * hd), _hidden(gen, t, n_kv * hd)
    # (v stays where the projection left it, behind q and k)
    s["v"] = _hidden(gen, t, (n_h + 2 * n_kv) * hd)[:, (n_h + n_kv) * hd:]
    s["starts"] = _int32(_starts(_prompt_lengths(c)))


def _prepare_chunk(c, gen, s):
    new, ctx = _chunk_lengths(c)
    n_h, n_kv, hd, ps = c["heads"], c["kv_heads"], c["head_dim"], c["page_size"]
    s["q"] = _hidden(gen, sum(new), n_h * hd)
    s["starts"], s["lens"] = _int32(_starts(new)), _int32(ctx)
    used = [-(-n // ps) for n in ctx]
    n_pages = sum(used) + 5
    s["k_pages"], s["v_pages"] = (torch.empty((n_pages, n_kv, ps, hd), dtype=torch.bfloat16, device=DEV).normal_(generator=gen)
                                  for _ in range(2))
    s["k_pages"] *= torch.exp(0.5 * _randn(gen, hd)).to(torch.bfloat16)
    order = torch.randperm(n_pages, device=DEV, generator=gen).to(torch.int32)
    table = torch.full((len(ctx), max(used)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for i, n in enumerate(used):
        table[i, :n] = order[at:at + n]
        at += n
    s["table"] = table


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    s = {"case": c}
    {"norm": _prepare_norm, "rotary": _prepare_rotary, "prompt": _prepare_prompt, "chunk": _prepare_chunk}[c["op"]](c, gen, s)
    if own:
        _prepare_own(c, s)
    return s


def _prepare_own(c, s):
    from paper_2602_00397_amd import binding as B
    ctx = s["ctx"] = B.Context(0)
    if c["op"] == "norm":
        for which in ("post", "pre"):
            s[which + "_norm"] = None if s[which] is None else B.norm(c[which], EPS, gain=s[which][0], bias=s[which][1])
        return
    causal, window = (True, 0) if c["op"] == "rotary" else (c["causal"], c["window"])
    s["shape"] = B.Attention(c["heads"], c["kv_heads"], c["head_dim"], causal, window, c["head_dim"] ** -0.5)
    if c["op"] == "rotary":
        s["rot"] = B.rotary(c["rot_dim"], s["inv_freq"], axis=s["axis"], interleaved=c["interleaved"], n_axes=c["axes"])
    if c["op"] in ("rotary", "chunk"):
        s["cache"] = B.paged_cache(s["k_pages"], s["v_pages"])
    if c["op"] in ("prompt", "chunk"):
        ctx.ensure_attention_workspace(s["shape"], s["q"].shape[0], s["starts"].numel() - 1)
        s["o"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((s["q"].shape[0], c["heads"]), dtype=torch.float32, device=DEV) if c["lse"] else None


# ---- one pass --------------------------------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if own:
        return _run_own(c, s)
    return {"norm": _plain_norm, "rotary": _plain_rotary, "prompt": _plain_prompt, "chunk": _plain_chunk}[c["op"]](c, s)


def _run_own(c, s):
    ctx = s["ctx"]
    if c["op"] == "norm":
        ctx.norm_residual(s["h"], s["y"], s["h_out"], s["x"], post=s["post_norm"], gate=s["gate"],
                          gate_tokens=1 if c["gate"] == "none" else c["gate"], scale=c["scale"], pre=s["pre_norm"])
        return {"h": s["h_out"], "x": s["x"]}
    if c["op"] == "rotary":
        ctx.rotary(s["shape"], s["rot"], s["q"], s["k"], s["v"], s["positions"], s["q_out"], k_out=s["k_out"], cache=s["cache"],
                   slots=s["slots"])
        out = {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
        return dict(out, k=s["k_out"]) if c["prompt"] else out
    if c["op"] == "prompt":
        ctx.prompt_attention(s["shape"], s["q"], s["k"], s["v"], s["starts"], s["o"], lse=s["lse"])
    else:
        ctx.chunk_attention(s["shape"], s["q"], s["starts"], s["lens"], c["chunk"], s["cache"], s["table"], s["o"], lse=s["lse"])
    return {"o": s["o"], "lse": s["lse"]} if c["lse"] else {"o": s["o"]}


def _plain_normed(v, kind, params):
    if params is None:
        return v
    if kind == "layer":
        v = v - v.mean(dim=-1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(dim=-1, keepdim=True) + EPS) * params[0].float()
    return v if params[1] is None else v + params[1].float()


def _plain_norm(c, s):
    y = _plain_normed(s["y"].float(), c["post"], s["post"]) * c["scale"]
    if s["gate"] is not None:
        row = torch.arange(c["n_tokens"], device=DEV) // c["gate"]
        y = y * s["gate"].float()[row]
    h = s["h"].float() + y
    return {"h": h.to(torch.bfloat16), "x": _plain_normed(h, c["pre"], s["pre"]).to(torch.bfloat16)}


def _pair_channels(c):
    i = torch.arange(c["rot_dim"] // 2, device=DEV)
    return (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + c["rot_dim"] // 2)


def _plain_rotary(c, s):
    t, hd = c["n_tokens"], c["head_dim"]
    # far positions' angles need more than 24 bits
    pos = s["positions"].double()[torch.tensor(s["axis"], device=DEV)]
    angle = pos.t() * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    a, b = _pair_channels(c)

    def turned(v):
        v = v.reshape(t, -1, hd).float()
        out = v.clone()
        out[:, :, a] = v[:, :, a] * cos - v[:, :, b] * sin
        out[:, :, b] = v[:, :, b] * cos + v[:, :, a] * sin
        return out.to(torch.bfloat16)

    q, k = turned(s["q"]), turned(s["k"])
    page, at = s["slots"].long() // c["page_size"], s["slots"].long() % c["page_size"]
    s["k_pages"][page, :, at] = k
    s["v_pages"][page, :, at] = s["v"].reshape(t, -1, hd)
    out = {"q": q.reshape(t, -1), "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    return dict(out, k=k.reshape(t, -1)) if c["prompt"] else out


def _plain_attend(c, q, k, v):
    """One sequence: q [n][heads][hd], k and v [keys][kv_heads][hd], float32 -> o [n][heads][hd], lse [n][heads]."""
    n, keys, group = q.shape[0], k.shape[0], c["heads"] // c["kv_heads"]
    o, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, device=DEV)
    if keys == 0:
        return o, lse
    rows = max(1, min(n, (1 << 27) // (keys * group)))
    for g in range(c["kv_heads"]):
        kt, vg = k[:, g].t().contiguous(), v[:, g].contiguous()
        for r0 in range(0, n, rows):
            r1 = min(n, r0 + rows)
            x = q[r0:r1, g * group:(g + 1) * group].reshape(-1, q.shape[2]) @ kt * c["head_dim"] ** -0.5
            if c["causal"]:
                pos = torch.arange(keys - n + r0, keys - n + r1, device=DEV).repeat_interleave(group)[:, None]
                j = torch.arange(keys, device=DEV)[None]
                out = j > pos
                if c["window"]:
                    out |= j <= pos - c["window"]
                x.masked_fill_(out, -math.inf)
            m = x.amax(dim=1, keepdim=True)
            m = torch.where(m == -math.inf, torch.zeros_like(m), m)
            p = torch.exp_(x.sub_(m))
            l = p.sum(dim=1, keepdim=True)
            o[r0:r1, g * group:(g + 1) * group] = (p @ vg / torch.where(l > 0, l, torch.ones_like(l))).reshape(r1 - r0, group, -1)
            lse[r0:r1, g * group:(g + 1) * group] = (m + torch.log(l)).reshape(r1 - r0, group)
    return o, lse


def _plain_sequences(c, s, keys_of):
    t, hd = s["q"].shape[0], c["head_dim"]
    q = s["q"].reshape(t, -1, hd)
    o, lse = torch.empty_like(q), torch.empty((t, c["heads"]), device=DEV)
    t0 = 0
    for i, (n, _) in enumerate(_sequences(c)):
        if n:
            k, v = keys_of(i, t0, t0 + n)
            part, l = _plain_attend(c, q[t0:t0 + n].float(), k.float(), v.float())
            o[t0:t0 + n] = part.to(torch.bfloat16)
            lse[t0:t0 + n] = l
        t0 += n
    return {"o": o.reshape(t, -1), "lse": lse} if c["lse"] else {"o": o.reshape(t, -1)}


def _plain_prompt(c, s):
    k, v = (s[x].reshape(c["n_tokens"], -1, c["head_dim"]) for x in ("k", "v"))
    return _plain_sequences(c, s, lambda i, a, b: (k[a:b], v[a:b]))


def _cached(c, s, i, n):
    """The first n cached keys and values of sequence i, [n][kv_heads][hd]."""
    pages = s["table"][i, :-(-n // c["page_size"])].long()
    return tuple(s[x][pages].transpose(1, 2).reshape(-1, c["kv_heads"], c["head_dim"])[:n] for x in ("k_pages", "v_pages"))


def _plain_chunk(c, s):
    lens = [k for _, k in _sequences(c)]
    return _plain_sequences(c, s, lambda i, a, b: _cached(c, s, i, lens[i]))


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    return {"norm": _exact_norm, "rotary": _exact_rotary, "prompt": _exact_attention, "chunk": _exact_attention}[c["op"]](c, s)


def _exact_statistics(v, kind, params):
    if params is None:
        return v
    centre = v.sum(1) / v.shape[1] if kind == "layer" else torch.zeros(v.shape[0], dtype=torch.float64, device=DEV)
    dev = v - centre[:, None]
    out = dev * torch.rsqrt(dev.square().sum(1) / v.shape[1] + EPS)[:, None] * params[0].double()
    return out + (0.0 if params[1] is None else params[1].double())


def _exact_norm(c, s):
    y = _exact_statistics(s["y"].double(), c["post"], s["post"])
    if s["gate"] is not None:
        y = y * torch.repeat_interleave(s["gate"].double(), c["gate"], dim=0)[:c["n_tokens"]]
    h = torch.add(s["h"].double(), y, alpha=c["scale"])
    return {"h": h, "x": _exact_statistics(h, c["pre"], s["pre"])}


def _exact_rotary(c, s):
    t, hd, pairs = c["n_tokens"], c["head_dim"], c["rot_dim"] // 2
    q, k = (s[x].double().reshape(t, -1, hd).clone() for x in ("q", "k"))
    for i in range(pairs):
        a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + pairs)
        turn = torch.polar(torch.ones(t, dtype=torch.float64, device=DEV), s["positions"][s["axis"][i]].double() * s["inv_freq"][i].double())
        for x in (q, k):
            z = torch.complex(x[:, :, a].clone(), x[:, :, b].clone()) * turn[:, None]
            x[:, :, a], x[:, :, b] = z.real, z.imag
    k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
    flat = s["slots"].long()
    k_pages.transpose(1, 2)[flat // c["page_size"], flat % c["page_size"]] = k
    v_pages.transpose(1, 2)[flat // c["page_size"], flat % c["page_size"]] = s["v"].double().reshape(t, -1, hd)
    out = {"q": q.reshape(t, -1), "k_pages": k_pages, "v_pages": v_pages}
    return dict(out, k=k.reshape(t, -1)) if c["prompt"] else out


def _exact_attention(c, s):
    t, hd, group, scale = s["q"].shape[0], c["head_dim"], c["heads"] // c["kv_heads"], 1.0 / math.sqrt(c["head_dim"])
    o = torch.zeros((t, c["heads"], hd), dtype=torch.float64, device=DEV)
    lse = torch.full((t, c["heads"]), -math.inf, dtype=torch.float64, device=DEV)
    first = 0
    for i, (n, keys) in enumerate(_sequences(c)):
        if c["op"] == "prompt":
            k, v = (s[x][first:first + n].reshape(n, -1, hd) for x in ("k", "v"))
        else:
            k, v = _cached(c, s, i, keys)
        for h in range(c["heads"]):
            kh, vh = k[:, h // group].double(), v[:, h // group].double()
            for a in range(0, n, 2048):
                b = min(n, a + 2048)
                # keys [lo, hi) are seen by some token of [a, b)
                hi = keys - n + b if c["causal"] else keys
                lo = max(0, keys - n + a - c["window"] + 1) if c["window"] else 0
                logits = s["q"][first + a:first + b, h * hd:(h + 1) * hd].double() @ kh[lo:hi].t() * scale
                if c["causal"]:
                    distance = (torch.arange(a, b, device=DEV)[:, None] + (keys - n)) - torch.arange(lo, hi, device=DEV)[None]
                    seen = (distance >= 0) & (distance < (c["window"] or keys + 1))
                    logits = torch.where(seen, logits, torch.full_like(logits, -math.inf))
                total = torch.logsumexp(logits, dim=1)
                o[first + a:first + b, h] = torch.exp(logits - total[:, None]) @ vh[lo:hi]
                lse[first + a:first + b, h] = total
        first += n
    return {"o": o.reshape(t, -1), "lse": lse} if c["lse"] else {"o": o.reshape(t, -1)}
