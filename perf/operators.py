"""The operators that work on KV caches outside the decoder layer, and what is measured of them.

A serving worker that computes its own projections (another rotary form, adapters, the tokens that follow the prompt) does
with a layer's caches:

  append    rotates the new tokens' queries and keys (halves or interleaved pairs, the whole head or its first part, plain
            or with frequencies scaled for long contexts) and stores keys and values into the caches
            (Context.kv_append).  Outputs: the rotated queries and the cache memory.
  attend    attention of the new tokens - one per request, a few drafted ones, or a chunk - over all that is cached
            (Context.attend).  Output: the attention rows.
  bounds    bounds on the keys of every finished 64-token block, as 8-bit codes and a power of two (Context.bounds_update).
            Outputs: codes and units.
  blocks    attention over the blocks that a cheap score, taken from those bounds, selects for each new token and KV head
            (Context.attend_blocks).  Outputs: the attention rows and the selected blocks.

Where `own` is false, run() computes them in plain torch operations in 32 bits, on cache memory of the same layout.

Cache memory.  A block holds 64 tokens: K as [64][d], V transposed as [d][64].  A contiguous cache is
[K, V][KV head][block] of such tiles, a page of a pool [K, V][KV head] of one block.  Elements are bfloat16, or E4M3 codes
that stand for code * scale.

Block bounds.  Of every element of a block's keys the largest and smallest value over its 64 tokens (elements beyond
+-2^100 count as +-2^100, NaN as 0), in codes of `unit` = 2^e, e the smallest integer, at least -100, that keeps the largest
magnitude of the block and KV head within 127 units: ceil(high / unit), floor(low / unit).

Score of a block for a token and KV head.  The group's g query heads in codes of their common power of two, chosen in
the same way; the positive and the negative codes are added up over the heads, halved ceil(log2 g) times at once, rounding
half away from zero: p and n.  score = unit * sum_j (p_j high_j + n_j low_j), all of it exact in 32 bits.  A token in
block b0 attends to at most n_blocks blocks: the first n_first, the last n_last up to its own, and of the others the best
scores, ties to the lowest block.
"""
from __future__ import annotations

import math
import random

import torch

own = False

# q heads, KV heads, head dim of the layer shapes (synth/workloads.py: TINY, L7B, L72B)
SHAPES = {"tiny": (4, 2, 64), "7b": (28, 4, 128), "72b": (64, 8, 128)}
FP8_SCALE = 0.0625   # of 8-bit caches: E4M3 then spans +-28
LIMIT = 2.0 ** 100
MAX_POS, MAX_ROWS, MAX_REQUESTS = 131200, 4096, 64

# rotary forms: pair layout, part of the head that is turned, base, frequency scaling and its parameters
ROTARY = {
    "halves": dict(layout="halves", part=1.0, theta=1e6, scaling="none"),
    "interleaved_part": dict(layout="interleaved", part=0.5, theta=1e4, scaling="none"),
    "halves_linear": dict(layout="halves", part=1.0, theta=1e4, scaling="linear", factor=4.0),
    "halves_ramp": dict(layout="halves", part=1.0, theta=1e6, scaling="ramp", factor=4.0, original=32768),
    "interleaved_bands": dict(layout="interleaved", part=1.0, theta=5e5, scaling="bands", factor=8.0, original=8192),
}


# ------------------------------------------------------------------------------------------------ the cases
def _append(name, shape, rows, cached, requests, cache, rotary, split=0):
    return {"name": name, "kind": "append", "shape": shape, "rows": rows, "cached": cached, "requests": requests,
            "cache": cache, "rotary": rotary, "split": split}


def _attend(name, shape, rows, cached, requests, cache, split=0):
    return {"name": name, "kind": "attend", "shape": shape, "rows": rows, "cached": cached, "requests": requests,
            "cache": cache, "split": split}


def _bounds(name, shape, blocks, cached, requests, cache, split=0):
    return {"name": name, "kind": "bounds", "shape": shape, "blocks": blocks, "cached": cached, "requests": requests,
            "cache": cache, "split": split}


def _blocks(name, shape, rows, cached, requests, cache, n_blocks, split=0):
    return {"name": name, "kind": "blocks", "shape": shape, "rows": rows, "cached": cached, "requests": requests,
            "cache": cache, "n_blocks": n_blocks, "split": split}


def listed():
    return [
        # one request's next token: the call is all latency
        _append("append_1", "7b", 1, 500, 1, "contiguous", "halves"),
        # the next token of a full batch, on pages; half of each head turned in interleaved pairs
        _append("append_64x1", "7b", 64, 4000, 64, "paged", "interleaved_part", 1),
        # a full token budget of eight prompts into 8-bit pages, long-context frequencies
        _append("append_2048_fp8", "7b", 2048, 9000, 8, "paged_fp8", "halves_ramp", 2),
        # one request's next token on a short cache: latency again
        _attend("attend_1", "7b", 1, 2000, 1, "contiguous"),
        # the next token of a full batch, contexts ragged: bound by reading the caches
        _attend("attend_64x1", "7b", 64, 8000, 64, "paged", 3),
        # long contexts in 8-bit pages
        _attend("attend_16x1_fp8", "7b", 16, 32000, 16, "paged_fp8", 4),
        # a few drafted tokens per request, checked at once
        _attend("attend_24x3", "72b", 72, 6000, 24, "paged", 5),
        # a prompt's chunk: bound by the products
        _attend("attend_2048", "7b", 2048, 6144, 1, "contiguous"),
        # blocks that have just been filled: one of each of 32 requests
        _bounds("bounds_32x1", "7b", 1, 6000, 32, "paged", 6),
        # a whole prompt's blocks
        _bounds("bounds_32768", "7b", 512, 32768, 1, "contiguous"),
        # one token of a very long context: a sixty-fourth of it is read
        _blocks("blocks_1_of_131072", "7b", 1, 131000, 1, "paged_fp8", 32),
        # a chunk late in a long prompt, every token with blocks of its own
        _blocks("blocks_256_of_16384", "7b", 256, 16000, 1, "paged", 32),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choices(["append", "attend", "bounds", "blocks"], [3, 5, 2, 3])[0]
    shape = rng.choices(["tiny", "7b", "72b"], [1, 4, 1])[0]
    cache = rng.choice(["contiguous", "paged", "fp8", "paged_fp8"])
    one = cache in ("contiguous", "fp8")   # (the plain form keeps one contiguous cache, or a pool)
    split = rng.randint(0, 9999)
    if kind == "append":
        requests = 1 if one else rng.randint(2, 64)
        rows = requests if rng.random() < 0.4 else max(requests, _log_int(rng, 1, 2048))
        return dict(kind=kind, shape=shape, rows=rows, cached=_log_int(rng, 16, 4000), requests=requests, cache=cache,
                    rotary=rng.choice(sorted(ROTARY)), split=split)
    if kind == "attend":
        requests = 1 if one else rng.randint(2, 64)
        most = 8 * requests if requests > 1 else 800 if shape == "72b" else 2048
        rows = requests if rng.random() < 0.5 else max(requests, _log_int(rng, 1, most))
        cached = _log_int(rng, 16, 32000 if requests <= 8 and rows <= 64 else 6000)
        return dict(kind=kind, shape=shape, rows=rows, cached=cached, requests=requests, cache=cache, split=split)
    if kind == "bounds":
        requests = 1 if one else rng.randint(2, 32)
        cached = _log_int(rng, 200, 32000 if requests <= 8 else 6000)
        return dict(kind=kind, shape=shape, blocks=_log_int(rng, 1, 500), cached=cached, requests=requests, cache=cache, split=split)
    requests = 1 if one else rng.randint(2, 16)
    rows = requests if rng.random() < 0.5 else max(requests, _log_int(rng, 1, 128))
    cached = _log_int(rng, 1000, 100000 if requests == 1 else 20000)
    return dict(kind=kind, shape=shape, rows=rows, cached=cached, requests=requests, cache=cache,
                n_blocks=rng.choice([4, 8, 15, 32]), split=split)


# ------------------------------------------------------------------------------------------------ sizes
def _lengths(case):
    """(new rows, cached tokens) of every request.  One request has them all; of several, the rows are ragged (1 + a random
    share of the rest) and the cached lengths uniform in 0 .. `cached`."""
    r, rows = case["requests"], case.get("rows", 0)
    if r == 1:
        return [rows], [case["cached"]]
    rng = random.Random(case["split"])
    if case["kind"] == "bounds":
        return [0] * r, [rng.randint(64, case["cached"]) for _ in range(r)]
    w = [rng.expovariate(1.0) for _ in range(r)]
    lens = [1 + int((rows - r) * x / sum(w)) for x in w]
    lens[0] += rows - sum(lens)
    return lens, [rng.randint(0, case["cached"]) for _ in range(r)]


def _first_blocks(case):
    """The first block whose bounds are taken, of every request (the last `blocks` finished ones are)."""
    return [max(0, p // 64 - case["blocks"]) for p in _lengths(case)[1]]


def _budget(case):
    """n_blocks, n_first, n_last."""
    return case["n_blocks"], 1, 2


def work(case):
    hq, hkv, d = SHAPES[case["shape"]]
    lens, cached = _lengths(case)
    rows, el = sum(lens), 1 if "fp8" in case["cache"] else 2
    if case["kind"] == "append":
        return {"bytes": rows * d * (4 * hq + 4 * hkv + 2 * hkv * el), "flops": 3 * rows * d * (hq + hkv)}
    if case["kind"] == "attend":
        seen = sum(n * p + n * (n + 1) // 2 for n, p in zip(lens, cached))
        return {"bytes": 4 * rows * hq * d + 2 * hkv * d * el * sum(n + p for n, p in zip(lens, cached)), "flops": 4 * hq * d * seen}
    if case["kind"] == "bounds":
        blocks = sum(p // 64 - f for p, f in zip(cached, _first_blocks(case)))
        return {"bytes": blocks * hkv * (64 * d * el + 2 * d + 4), "flops": 2 * blocks * hkv * 64 * d}
    n_blocks = case["n_blocks"]
    scored = sum((p + n - 1) // 64 for n, p in zip(lens, cached))
    read = sum(min((p + n + 63) // 64, n * n_blocks) for n, p in zip(lens, cached))
    taken = sum(n * min((p + 64) // 64, n_blocks) for n, p in zip(lens, cached))
    return {"bytes": 4 * rows * hq * d + scored * hkv * (2 * d + 4) + read * 2 * hkv * 64 * d * el + 4 * rows * hkv * n_blocks,
            "flops": 4 * hq * d * 64 * taken + 4 * hkv * d * sum(n * ((p + n - 1) // 64) for n, p in zip(lens, cached))}


# ------------------------------------------------------------------------------------------------ inputs
class _State:
    pass


def _inverse_frequencies(spec, rd):
    """theta^(-2j/rd) in 64 bits, scaled: `linear` divides all by `factor`; `ramp` divides those that turn less than once
    over the original context and leaves those that turn more than 32 times, a linear ramp over the pairs between; `bands`
    divides the wavelengths beyond the original context, leaves those below a quarter of it, and blends between."""
    j = torch.arange(rd // 2, dtype=torch.float64)
    f = spec["theta"] ** (-2.0 * j / rd)
    if spec["scaling"] == "linear":
        return f / spec["factor"], 1.0
    if spec["scaling"] == "ramp":
        def pair_of(turns):
            return rd * math.log(spec["original"] / (turns * 2 * math.pi)) / (2 * math.log(spec["theta"]))
        low, high = max(math.floor(pair_of(32.0)), 0), min(math.ceil(pair_of(1.0)), rd - 1)
        share = ((j - low) / max(high - low, 1e-3)).clamp(0, 1)
        return f / spec["factor"] * share + f * (1 - share), 0.1 * math.log(spec["factor"]) + 1.0
    if spec["scaling"] == "bands":
        turns = spec["original"] * f / (2 * math.pi)
        keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return f / spec["factor"] * (1 - keep) + f * keep, 1.0
    return f, 1.0


def _inputs(case, seed):
    """Queries, new keys and values, and every request's cached keys and values [tokens, KV heads, d]: the keys drift from
    block to block, as those of a text's passages do, so that blocks differ."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    hq, hkv, d = SHAPES[case["shape"]]
    lens, cached = _lengths(case)
    rows = sum(lens)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    qkv = normal(rows, (hq + 2 * hkv) * d).to(torch.bfloat16)
    tokens = sum(cached) + (rows if case["kind"] in ("attend", "blocks") else 0)
    k = normal(tokens, hkv, d) * 0.8
    k += normal(tokens // 64 + 1, hkv, d).repeat_interleave(64, 0)[:tokens] * 0.6
    return qkv, k.to(torch.bfloat16), normal(tokens, hkv, d).to(torch.bfloat16)


def _e4m3(x, scale):
    return (x.float() * (1.0 / scale)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


_contexts, _rotaries = {}, {}


def _context(shape):
    """One context per layer shape, as a worker has."""
    from paper_2509_24381_amd.binding import Context, LayerConfig
    if shape not in _contexts:
        hq, hkv, d = SHAPES[shape]
        _contexts[shape] = Context(LayerConfig(hidden=hq * d, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, mlp_inter=1024,
                                               max_tokens_per_call=MAX_ROWS, max_requests=MAX_REQUESTS, max_pos=MAX_POS))
    return _contexts[shape]


def _rotary(shape, name):
    from paper_2509_24381_amd.binding import RotaryConfig
    if (shape, name) not in _rotaries:
        s, d = ROTARY[name], SHAPES[shape][2]
        _rotaries[shape, name] = _context(shape).rotary(RotaryConfig(
            rotary_dim=int(d * s["part"]), theta=s["theta"], max_pos=16384, layout=s["layout"], scaling=s["scaling"],
            factor=s.get("factor", 1.0), original_max_pos=s.get("original", 0)))
    return _rotaries[shape, name]


def prepare(case, seed):
    hq, hkv, d = SHAPES[case["shape"]]
    kind = case["kind"]
    s = _State()
    s.case, s.hq, s.hkv, s.d, s.g = case, hq, hkv, d, hq // hkv
    s.fp8, s.paged = "fp8" in case["cache"], case["cache"].startswith("paged")
    lens, cached = _lengths(case)
    s.lens, s.cached = lens, cached
    s.rows = rows = sum(lens)
    s.qkv, k, v = _inputs(case, seed)
    s.q, s.k, s.v = s.qkv.split([hq * d, hkv * d, hkv * d], dim=1)   # (rows of one projection: strided views)
    held = [p + (n if kind in ("attend", "blocks") else 0) for n, p in zip(lens, cached)]   # tokens cached before the call
    room = [p + n for n, p in zip(lens, cached)]                                            # and after it
    nb = [(t + 63) // 64 for t in room]
    s.out = torch.empty((rows, hq * d), dtype=torch.bfloat16, device="cuda")
    s.capb = max(nb)
    if kind in ("bounds", "blocks"):
        s.codes = torch.zeros((len(lens), hkv, s.capb, 2, d), dtype=torch.int8, device="cuda")
        s.units = torch.zeros((len(lens), hkv, s.capb), dtype=torch.float32, device="cuda")
    if kind == "blocks":
        s.chosen = torch.empty((rows, hkv, case["n_blocks"]), dtype=torch.int32, device="cuda")

    # pages of every request: those of what is cached, request by request, then those the call adds
    table, free = [], 0
    for t in held:
        table.append(list(range(free, free + (t + 63) // 64)))
        free += (t + 63) // 64
    for i, n in enumerate(nb):
        more = n - len(table[i])
        table[i] += list(range(free, free + more))
        free += more
    el = torch.uint8 if s.fp8 else torch.bfloat16
    if own:
        from paper_2509_24381_amd.binding import CacheSet, KVPool, int_array
        s.ctx = ctx = _context(case["shape"])
        if s.paged:
            s.pool = KVPool(ctx, free, fp8=s.fp8)
            slab = s.pool.slab
            slab.zero_()
            kvs = [s.pool.new_cache(1, FP8_SCALE, FP8_SCALE) for _ in lens]
        else:
            kvs = [ctx.kv_alloc_fp8(1, room[0], FP8_SCALE, FP8_SCALE) if s.fp8 else ctx.kv_alloc(1, room[0])]
            slab = kvs[0].slab
            slab.zero_()
        for kv, a, b in zip(kvs, k.split(held), v.split(held)):
            kv.import_(0, a, b)
        s.kvs, s.n, s.starts = CacheSet(kvs), int_array(lens), int_array(cached)
        if kind == "append":
            s.rotary = _rotary(case["shape"], case["rotary"])
        elif kind in ("attend", "blocks"):
            s.ws = ctx.attend_workspace(rows, len(lens), fp8_visible_tokens=sum(room) if s.fp8 else 0,
                                        n_blocks=case.get("n_blocks", 0))
        if kind in ("bounds", "blocks"):
            for kv, c, u in zip(kvs, s.codes, s.units):
                kv.attach_bounds(c, u)
            if kind == "bounds":
                s.firsts = int_array([64 * f for f in _first_blocks(case)])
            else:
                ctx.bounds_update(0, s.kvs)
        shape = (free, 2, hkv, 64 * d) if s.paged else (2, hkv, free, 64 * d)
        s.memory = slab.view(el)[: free * 2 * hkv * 64 * d].view(shape)
        torch.cuda.synchronize()
        return s

    # the same memory, written by torch
    s.memory = torch.zeros((free, 2, hkv, 64 * d) if s.paged else (2, hkv, free, 64 * d), dtype=el, device="cuda")
    at = [(table[i][t // 64], t % 64) for i, n in enumerate(held) for t in range(n)]
    if at:
        page, slot = torch.tensor(at, device="cuda").t()
        _store(s, page, slot, k, v)
    s.table = torch.tensor([row + [0] * (s.capb - len(row)) for row in table], device="cuda")
    where = [(i, p + t) for i, (n, p) in enumerate(zip(lens, cached)) for t in range(n)]   # request and position of every row
    if where:
        s.request, s.position = torch.tensor(where, device="cuda").t()
        tmax = max(lens)
        first = [sum(lens[:i]) for i in range(len(lens))]
        pad = [[f + min(t, n - 1) for t in range(tmax)] for f, n in zip(first, lens)]   # rows of every request, padded
        s.pad = torch.tensor(pad, device="cuda")
        s.unpad = torch.tensor([i * tmax + t for i, n in enumerate(lens) for t in range(n)], device="cuda")
    if kind == "append":
        spec = ROTARY[case["rotary"]]
        f, magnitude = _inverse_frequencies(spec, int(d * spec["part"]))
        angle = torch.arange(16384, dtype=torch.float64).cuda()[:, None] * f.cuda()
        s.cos, s.sin = (angle.cos() * magnitude).float(), (angle.sin() * magnitude).float()   # a table, as one keeps
    if kind in ("bounds", "blocks"):
        firsts = _first_blocks(case) if kind == "bounds" else [0] * len(lens)
        fresh = [(i, b) for i, (f, t) in enumerate(zip(firsts, held)) for b in range(f, t // 64)]
        s.fresh = torch.tensor(fresh, dtype=torch.int64, device="cuda").view(-1, 2).t()   # request and number of every block
        if kind == "blocks":
            _run_bounds(s)
    torch.cuda.synchronize()
    return s


# ------------------------------------------------------------------------------------------------ the plain forms
def _pages(s):
    """The cache memory as [page][K, V][KV head][64 d]."""
    return s.memory if s.paged else s.memory.permute(2, 0, 1, 3)


def _store(s, page, slot, k, v):
    """Tokens' keys and values [n, KV heads, d] into the memory."""
    if s.fp8:
        k, v = _e4m3(k, FP8_SCALE), _e4m3(v, FP8_SCALE)
    m = _pages(s)
    m.unflatten(-1, (64, s.d))[page, 0, :, slot, :] = k
    m.unflatten(-1, (s.d, 64))[page, 1, :, :, slot] = v


def _value(s, x):
    """What gathered elements stand for, in 32 bits."""
    return x.contiguous().view(torch.float8_e4m3fn).float() * FP8_SCALE if s.fp8 else x.float()


def _turn(s, x, layout, rd):
    """Rotates the first rd features of [rows, heads, d] by the rows' angles."""
    cos, sin = s.cos[s.position][:, None], s.sin[s.position][:, None]
    part, rest = x[..., :rd].float(), x[..., rd:].float()
    if layout == "halves":
        a, b = part[..., : rd // 2], part[..., rd // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1).to(torch.bfloat16)
    a, b = part[..., 0::2], part[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1).to(torch.bfloat16)


def _run_append(s):
    spec = ROTARY[s.case["rotary"]]
    rd = int(s.d * spec["part"])
    q = _turn(s, s.q.unflatten(1, (s.hq, s.d)), spec["layout"], rd)
    k = _turn(s, s.k.unflatten(1, (s.hkv, s.d)), spec["layout"], rd)
    _store(s, s.table[s.request, s.position // 64], s.position % 64, k, s.v.unflatten(1, (s.hkv, s.d)))
    return q.flatten(1)


def _softmax_rows(scores, seen, v):
    scores = scores.masked_fill(~seen, float("-inf"))
    e = (scores - scores.amax(-1, keepdim=True)).exp()
    return torch.matmul(e, v) / e.sum(-1, keepdim=True)


def _run_attend(s):
    r, tmax = s.pad.shape
    m, tokens = _pages(s), s.capb * 64
    k = _value(s, m[s.table, 0].unflatten(-1, (64, s.d))).transpose(1, 2).reshape(r, s.hkv, tokens, s.d)
    v = _value(s, m[s.table, 1].unflatten(-1, (s.d, 64))).permute(0, 2, 1, 4, 3).reshape(r, s.hkv, tokens, s.d)
    q = s.q[s.pad].float().view(r, tmax, s.hkv, s.g, s.d).transpose(1, 2).reshape(r, s.hkv, tmax * s.g, s.d)
    scores = torch.matmul(q, k.transpose(2, 3)) * s.d ** -0.5
    seen = torch.arange(tokens, device="cuda") <= s.position[s.pad][:, :, None]
    out = _softmax_rows(scores, seen.repeat_interleave(s.g, 1)[:, None], v)
    out = out.view(r, s.hkv, tmax, s.g, s.d).transpose(1, 2).reshape(r * tmax, s.hq * s.d)
    return out[s.unpad].to(torch.bfloat16)


def _exponent(largest, least=-100):
    """The smallest e >= least with largest <= 127 * 2^e."""
    m, x = torch.frexp(largest)
    return torch.where(largest == 0, torch.full_like(x, least), x - 7 + (m * 128 > 127)).clamp(min=least)


def _run_bounds(s):
    request, block = s.fresh
    k = _value(s, _pages(s)[s.table[request, block], 0].unflatten(-1, (64, s.d)))   # [blocks, KV heads, 64, d]
    k = k.nan_to_num(0.0, LIMIT, -LIMIT).clamp(-LIMIT, LIMIT)
    high, low = k.amax(2), k.amin(2)
    unit = torch.exp2(_exponent(torch.maximum(high, -low).amax(2)).float())
    s.codes[request, :, block] = torch.stack([(high / unit[..., None]).ceil(), (low / unit[..., None]).floor()], 2).to(torch.int8)
    s.units[request, :, block] = unit
    return s.codes, s.units


def _run_blocks(s):
    n_blocks, n_first, n_last = _budget(s.case)
    r, tmax = s.pad.shape
    q = s.q[s.pad].float().view(r, tmax, s.hkv, s.g, s.d).transpose(1, 2)   # [requests, KV heads, rows, g, d]
    at = s.position[s.pad]
    # scores
    finite = q.nan_to_num(0.0, LIMIT, -LIMIT).clamp(-LIMIT, LIMIT)
    code = (finite / torch.exp2(_exponent(finite.abs().amax((3, 4))).float())[..., None, None]).round()
    halvings = (s.g - 1).bit_length()
    half = (1 << halvings) // 2
    p = ((code.clamp(min=0).sum(3) + half) / (1 << halvings)).floor()
    n = -(((-code).clamp(min=0).sum(3) + half) / (1 << halvings)).floor()
    score = torch.matmul(torch.cat([p, n], -1), s.codes.float().flatten(3).transpose(2, 3)) * s.units[:, :, None]
    # selection: [requests, KV heads, rows, blocks]
    b, b0 = torch.arange(s.capb, device="cuda"), (at // 64)[:, None, :, None]
    score = torch.where((b < n_first) | (b > b0 - n_last), torch.full_like(score, float("inf")), score)
    score = torch.where(b <= b0, score, torch.full_like(score, float("-inf")))
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :n_blocks]
    best = torch.where(best <= b0, best, torch.full_like(best, s.capb))
    best = torch.nn.functional.pad(best, (0, n_blocks - best.shape[-1]), value=s.capb).sort(-1).values
    live = best < s.capb
    best = torch.where(live, best, torch.zeros_like(best))
    # attention over the selected blocks
    head = torch.arange(s.hkv, device="cuda")[:, None, None]
    page = s.table[torch.arange(r, device="cuda")[:, None, None, None], best]
    m = _pages(s)
    k = _value(s, m[page, 0, head].unflatten(-1, (64, s.d))).flatten(3, 4)
    v = _value(s, m[page, 1, head].unflatten(-1, (s.d, 64))).transpose(4, 5).flatten(3, 4)
    key = (best[..., None] * 64 + torch.arange(64, device="cuda")).flatten(3)
    seen = live.repeat_interleave(64, 3) & (key <= at[:, None, :, None])
    out = _softmax_rows(torch.matmul(q, k.transpose(3, 4)) * s.d ** -0.5, seen[:, :, :, None], v)
    out = out.transpose(1, 2).reshape(r * tmax, s.hq * s.d)[s.unpad].to(torch.bfloat16)
    chosen = torch.where(live, best, torch.full_like(best, -1)).transpose(1, 2).reshape(r * tmax, s.hkv, n_blocks)[s.unpad]
    return out, chosen.to(torch.int32)


def _memory(s):
    """The cache memory as numbers (8-bit caches: E4M3)."""
    return s.memory.view(torch.float8_e4m3fn) if s.fp8 else s.memory


def run(s):
    kind = s.case["kind"]
    if own:
        if kind == "append":
            s.ctx.kv_append(0, s.kvs, s.n, s.q, s.k, s.v, s.out, rotary=s.rotary, starts=s.starts)
            return s.out, _memory(s)
        if kind == "attend":
            return s.ctx.attend(0, s.kvs, s.n, s.q, s.out, s.ws)
        if kind == "bounds":
            s.ctx.bounds_update(0, s.kvs, firsts=s.firsts)
            return s.codes, s.units
        n_blocks, n_first, n_last = _budget(s.case)
        s.ctx.attend_blocks(0, s.kvs, s.n, s.q, s.out, s.ws, n_blocks, n_first=n_first, n_last=n_last, chosen=s.chosen)
        return s.out, s.chosen
    if kind == "append":
        return _run_append(s), _memory(s)
    if kind == "attend":
        return _run_attend(s)
    return _run_bounds(s) if kind == "bounds" else _run_blocks(s)


# ------------------------------------------------------------------------------------------------ 64 bits
def _stored(x, fp8):
    """The numbers that a cache holds of bfloat16 rows, in 64 bits."""
    if not fp8:
        return x.double()
    return _e4m3(x, FP8_SCALE).view(torch.float8_e4m3fn).double() * FP8_SCALE


def _turned(x, position, spec, d):
    rd = int(d * spec["part"])
    f, magnitude = _inverse_frequencies(spec, rd)
    turn = torch.polar(torch.full((len(position), rd // 2), magnitude, dtype=torch.float64, device="cuda"),
                       position.double()[:, None] * f.cuda())[:, None]
    y = x.double().clone()
    a, b = (slice(0, rd // 2), slice(rd // 2, rd)) if spec["layout"] == "halves" else (slice(0, rd, 2), slice(1, rd, 2))
    z = torch.complex(y[..., a].clone(), y[..., b].clone()) * turn
    y[..., a], y[..., b] = z.real, z.imag
    return y


def _code_of(x):
    """Integer codes of x in the smallest power of two (at least 2^-100) that keeps them within 127, and its exponent."""
    top, e = float(x.abs().max()), -100
    while top > 127 * 2.0 ** e:
        e += 1
    return x / 2.0 ** e, e


def exact(case, seed):
    hq, hkv, d = SHAPES[case["shape"]]
    g, kind, fp8 = hq // hkv, case["kind"], "fp8" in case["cache"]
    lens, cached = _lengths(case)
    qkv, k, v = _inputs(case, seed)
    q = qkv[:, : hq * d].view(-1, hq, d)
    if kind == "append":
        spec = ROTARY[case["rotary"]]
        position = torch.cat([torch.arange(p, p + n, device="cuda") for n, p in zip(lens, cached)])
        kn = _turned(qkv[:, hq * d: (hq + hkv) * d].view(-1, hkv, d), position, spec, d)
        vn = qkv[:, (hq + hkv) * d:].view(-1, hkv, d).double()
        blocks = [(p + 63) // 64 for p in cached]
        more = [(p + n + 63) // 64 - b for n, p, b in zip(lens, cached, blocks)]
        total = sum(blocks) + sum(more)
        tiles = torch.zeros((total, 2, hkv, 64 * d), dtype=torch.float64, device="cuda")
        old = new = row = 0
        added = sum(blocks)
        for n, p, b, extra in zip(lens, cached, blocks, more):
            pages = list(range(old, old + b)) + list(range(added, added + extra))
            old, added = old + b, added + extra
            for x, y, plane in ((k, kn, 0), (v, vn, 1)):
                if fp8:   # in units of the scale, beyond the format's range at its end
                    seq = torch.cat([_stored(x[new: new + p], True) / FP8_SCALE, (y[row: row + n] / FP8_SCALE).clamp(-448, 448)])
                else:
                    seq = torch.cat([x[new: new + p].double(), y[row: row + n]])
                seq = torch.nn.functional.pad(seq, (0, 0, 0, 0, 0, 64 * len(pages) - p - n)).view(len(pages), 64, hkv, d)
                seq = seq.permute(0, 2, 1, 3) if plane == 0 else seq.permute(0, 2, 3, 1)
                tiles[torch.tensor(pages, device="cuda"), plane] = seq.reshape(len(pages), hkv, 64 * d)
            new, row = new + p, row + n
        if not case["cache"].startswith("paged"):
            tiles = tiles.permute(1, 2, 0, 3).contiguous()
        return _turned(q, position, spec, d).flatten(1), tiles
    if kind == "bounds":
        capb = max((p + 63) // 64 for p in cached)
        codes = torch.zeros((len(lens), hkv, capb, 2, d), dtype=torch.int8, device="cuda")
        units = torch.zeros((len(lens), hkv, capb), dtype=torch.float32, device="cuda")
        for i, (x, first) in enumerate(zip(k.split(cached), _first_blocks(case))):
            n = len(x) // 64
            x = _stored(x[: n * 64], fp8).view(n, 64, hkv, d)
            high, low = x.max(1).values, x.min(1).values
            top = torch.maximum(high.abs(), low.abs()).amax(2)
            e = torch.ceil(torch.log2(top / 127.0)).clamp(min=-100.0)
            e = torch.where(top > 127 * 2.0 ** e, e + 1, torch.where(top <= 127 * 2.0 ** (e - 1), e - 1, e)).clamp(min=-100.0)
            unit = 2.0 ** e
            c = torch.stack([(high / unit[..., None]).ceil(), (low / unit[..., None]).floor()], 2)
            codes[i, :, first:n] = c.transpose(0, 1)[:, first:].to(torch.int8)
            units[i, :, first:n] = unit.t()[:, first:].float()
        return codes, units
    out = torch.empty((sum(lens), hq, d), dtype=torch.float64, device="cuda")
    n_sel = case.get("n_blocks", 0)
    chosen = torch.full((sum(lens), hkv, max(n_sel, 1)), -1, dtype=torch.int32)
    row = new = 0
    for n, p in zip(lens, cached):
        held = p + n
        position = torch.arange(p, held, device="cuda")
        for h in range(hkv):
            kk, vv = _stored(k[new: new + held, h], fp8), _stored(v[new: new + held, h], fp8)
            qh = q[row: row + n, h * g: (h + 1) * g].double()
            seen = torch.arange(held, device="cuda") <= position[:, None]
            if kind == "blocks":
                allowed = _allowed(case, qh, kk, position, chosen, row, h)
                seen = seen & allowed.repeat_interleave(64, 1)[:, :held]
            step = max(1, (1 << 28) // (held * g))
            for a in range(0, n, step):
                x = torch.matmul(qh[a: a + step], kk.t().contiguous()) / math.sqrt(d)
                x = torch.where(seen[a: a + step, None], x, torch.full_like(x, float("-inf")))
                out[row + a: row + min(n, a + step), h * g: (h + 1) * g] = torch.matmul(torch.softmax(x, -1), vv)
        row, new = row + n, new + held
    out = out.flatten(1)
    return (out, chosen) if kind == "blocks" else out


def _allowed(case, qh, kk, position, chosen, row, h):
    """Which blocks each row attends to, from the definition in whole numbers; noted in `chosen`."""
    n_blocks, n_first, n_last = _budget(case)
    n, g, d = qh.shape
    blocks = (len(kk) + 63) // 64
    full = len(kk) // 64
    high, low, unit = [], [], []
    for b in range(full):
        x = kk[64 * b: 64 * b + 64]
        pair, e = _code_of(torch.stack([x.max(0).values, x.min(0).values]))
        high.append(pair[0].ceil())
        low.append(pair[1].floor())
        unit.append(2.0 ** e)
    allowed = torch.zeros((n, blocks), dtype=torch.bool, device="cuda")
    marked = []
    for t in range(n):
        own_block = int(position[t]) // 64
        forced = [b for b in range(own_block + 1) if b < n_first or b > own_block - n_last]
        # (more that have to be taken than there is room for: the first ones)
        take = forced[:n_blocks]
        others = [b for b in range(own_block) if b not in set(forced)]
        if others and len(take) < n_blocks:
            code = _code_of(qh[t])[0].round().long()
            halvings = (g - 1).bit_length()
            half = (1 << halvings) >> 1
            p = (code.clamp(min=0).sum(0) + half) >> halvings
            m = -(((-code).clamp(min=0).sum(0) + half) >> halvings)
            at = torch.tensor(others, device="cuda")
            hi, lo = torch.stack(high)[at], torch.stack(low)[at]
            score = ((hi * p + lo * m).sum(1) * torch.tensor(unit, dtype=torch.float64, device="cuda")[at]).tolist()
            take = take + sorted(others, key=lambda b: (-score[b - others[0]], b))[: n_blocks - len(take)]
        take.sort()
        chosen[row + t, h, : len(take)] = torch.tensor(take, dtype=torch.int32)
        marked += [(t, b) for b in take]
    t, b = torch.tensor(marked, device="cuda").t()
    allowed[t, b] = True
    return allowed
