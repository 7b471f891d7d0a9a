"""GPU: the operators on KV caches (include/rserve_attend.h) against the 64-bit oracle.

Tolerances, from the number formats (significands of 8 bits in bfloat16, 4 in E4M3: roundings of up to 2^-8 and 2^-4):
  attention  the weights and the output are each rounded to bfloat16 once, scores are fp32 sums of exact products: every
             element within (2^-7 + 2^-12) sum_k w_k |v_k| of the 64-bit one.  Chunks on 8-bit caches also round each key and value
             to bfloat16 (exact for the power-of-two scales used there).
  append     rotated elements within 2^-8 |y| + 2^-21 (|a| + |b|), values equal to the bit; 8-bit codes those of the rounded rows
  bounds, selected blocks: equal
"""
import gc
import math

import numpy as np
import pytest
import torch

from oracle import cache_ops as O
from oracle.fp8_kv import e4m3_decode, e4m3_encode

pytestmark = pytest.mark.gpu

KINDS = ("contiguous", "paged", "fp8", "paged_fp8")
K_SCALE, V_SCALE = 0.0625, 0.03125
SLACK = 2.0 ** -7 + 2.0 ** -12


def context(hq=4, hkv=2, d=64, **kw):
    from paper_2509_24381_amd.binding import Context, LayerConfig
    args = dict(hidden=hq * d, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, mlp_inter=64, max_tokens_per_call=2048, max_requests=64, max_pos=40000)
    args.update(kw)
    return Context(LayerConfig(**args))


def caches(ctx, kind, capacities, n_layers=1, scales=(K_SCALE, V_SCALE)):
    from paper_2509_24381_amd.binding import KVPool
    if kind.startswith("paged"):
        pool = KVPool(ctx, n_layers * sum((c + 63) // 64 for c in capacities) + 3, fp8=kind == "paged_fp8")
        return [pool.new_cache(n_layers, *scales) for _ in capacities]
    if kind == "fp8":
        return [ctx.kv_alloc_fp8(n_layers, max(c, 1), *scales) for c in capacities]
    return [ctx.kv_alloc(n_layers, max(c, 1)) for c in capacities]


def fill(kvs, content, layer=0):
    """Imports every request's keys and values, in growing pieces by turns, so that the pages of paged caches lie scattered."""
    for part in (0.2, 0.6, 1.0):
        for kv, (k, v) in zip(kvs, content):
            n = int(part * len(k))
            kv.import_(layer, k[:n].contiguous(), v[:n].contiguous())


def normal(g, *shape, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def f64(t):
    return t.double().cpu().numpy()


def stored(t, kind, scale):
    """The numbers a cache holds of bfloat16 rows."""
    x = f64(t)
    if "fp8" not in kind:
        return x
    return e4m3_decode(e4m3_encode((x.astype(np.float32) * np.float32(1.0 / scale)).astype(np.float64))) * scale


def assert_attention(out, ref, mag, what=""):
    out = f64(out).reshape(ref.shape)
    off = np.abs(out - ref) - SLACK * mag
    worst = float(off.max())
    assert worst <= 0, f"{what}: {worst:.3e} beyond the bound at {np.unravel_index(off.argmax(), off.shape)}"   # (NaN fails too)


# ------------------------------------------------------------------------------------------------ append
ROTARY_FORMS = [
    dict(layout="halves", scaling="none", theta=1e6),
    dict(layout="interleaved", scaling="none", theta=1e4),
    dict(layout="halves", scaling="linear", theta=1e4, factor=4.0),
    dict(layout="halves", scaling="ramp", theta=1e6, factor=4.0, original_max_pos=4096),
    dict(layout="interleaved", scaling="bands", theta=5e5, factor=8.0, original_max_pos=2048),
]


def rotary_of(ctx, part, form, max_pos=2048):
    from paper_2509_24381_amd.binding import RotaryConfig
    return ctx.rotary(RotaryConfig(rotary_dim=part, max_pos=max_pos, **form))


def rotated(x, pos, part, form):
    f = O.rotary_frequencies(part, form["theta"], form["scaling"], form.get("factor", 1.0), form.get("original_max_pos", 0))
    return O.rotate(f64(x), pos, part, f, form["layout"], O.rotary_magnitude(form["scaling"], form.get("factor", 1.0)))


def rotation_bound(x, y, part, form):
    """2^-8 |y| + 2^-21 (|a| + |b|) of every element."""
    a = np.abs(f64(x))
    pair = a.copy()
    if form["layout"] == "halves":
        pair[..., :part] = np.roll(a[..., :part], part // 2, axis=-1)
    else:
        pair[..., :part] = a[..., :part].reshape(*a.shape[:-1], part // 2, 2)[..., ::-1].reshape(*a.shape[:-1], part)
    return 2.0 ** -8 * np.abs(y) + 2.0 ** -21 * 1.2 * (a + pair)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq, hkv, d, part, form", [
    (4, 2, 64, 64, 0), (4, 2, 64, 16, 1), (28, 4, 128, 128, 3), (8, 8, 128, 48, 0), (6, 2, 128, 128, 4), (4, 1, 64, 32, 2),
])
def test_append_rotates_and_stores(kind, hq, hkv, d, part, form):
    """Ragged requests - none, one, a few and more than a block of tokens, from slots inside and at the edge of blocks - as strided
    views of one projection's rows; the rotated queries and what the caches then hold."""
    form = ROTARY_FORMS[form]
    ctx = context(hq, hkv, d)
    rot = rotary_of(ctx, part, form)
    g = gen(1)
    before, lens = [0, 63, 64, 100, 0, 190], [1, 1, 130, 0, 70, 9]
    kvs = caches(ctx, kind, [b + n for b, n in zip(before, lens)])
    old = [(normal(g, b, hkv, d), normal(g, b, hkv, d)) for b in before]
    fill(kvs, old)
    rows = sum(lens)
    qkv = normal(g, rows, (hq + 2 * hkv) * d)
    q, k, v = qkv.split([hq * d, hkv * d, hkv * d], dim=1)
    out = torch.full((rows, hq * d + 8), float("nan"), device="cuda", dtype=torch.bfloat16)[:, : hq * d]   # (rows further apart than wide)
    ctx.kv_append(0, kvs, lens, q, k, v, out, rotary=rot)
    pos = np.concatenate([np.arange(b, b + n) for b, n in zip(before, lens)])
    qh = q.unflatten(1, (hq, d))
    ref = rotated(qh, pos, part, form)
    assert (np.abs(f64(out).reshape(ref.shape) - ref) <= rotation_bound(qh, ref, part, form)).all()
    kh, vh = k.unflatten(1, (hkv, d)), v.unflatten(1, (hkv, d))
    kref = rotated(kh, pos, part, form)
    kbound = rotation_bound(kh, kref, part, form)
    if "fp8" in kind:
        kbound = kbound * 1.1 + 2.0 ** -4 * np.abs(kref) + K_SCALE * 2.0 ** -10
    at = 0
    for kv, b, n, (ko, vo) in zip(kvs, before, lens, old):
        assert kv.length(0) == b + n
        ke, ve = kv.export(0)
        assert np.array_equal(f64(ke[:b]), stored(ko, kind, K_SCALE)) and np.array_equal(f64(ve[:b]), stored(vo, kind, V_SCALE))
        assert np.array_equal(f64(ve[b:]), stored(vh[at: at + n], kind, V_SCALE))
        assert (np.abs(f64(ke[b:]) - kref[at: at + n]) <= kbound[at: at + n]).all()
        at += n


@pytest.mark.parametrize("kind", KINDS)
def test_append_leaves_the_same_bits_however_tokens_come(kind):
    """One by one, in ragged pieces, or at once; and as the layer call's own append does from rotated rows (no rotation here: import)."""
    ctx = context(28, 4, 128)
    rot = rotary_of(ctx, 128, ROTARY_FORMS[0])
    g = gen(2)
    n = 150
    k, v = normal(g, n, 4 * 128), normal(g, n, 4 * 128)
    results = []
    for pieces in ([n], [1] * n, [40, 24, 1, 63, 22]):
        kv, = caches(ctx, kind, [n])
        at = 0
        for p in pieces:
            ctx.kv_append(0, [kv], [p], None, k[at: at + p], v[at: at + p], None, rotary=rot)
            at += p
        results.append(kv.export_codes(0) if "fp8" in kind else kv.export(0))
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))
    plain, imported = caches(ctx, kind, [n]) + caches(ctx, kind, [n])
    ctx.kv_append(0, [plain], [n], None, k, v, None)
    imported.import_(0, k.view(n, 4, 128), v.view(n, 4, 128))
    assert all(torch.equal(a, b) for a, b in zip(plain.export(0), imported.export(0)))


@pytest.mark.parametrize("kind", KINDS)
def test_append_from_an_earlier_slot_drops_what_was_behind(kind):
    """Drafted tokens that were not accepted: the cache is as if they had never come, to the zeros behind the newest value that the
    chunk kernels rely on, and its pages and bounds with it."""
    from paper_2509_24381_amd.binding import KVPool
    ctx = context(4, 2, 64)
    g = gen(3)
    k, v = normal(g, 200, 2, 64), normal(g, 200, 2, 64)
    pool = KVPool(ctx, 8, fp8=kind == "paged_fp8") if kind.startswith("paged") else None
    kv = pool.new_cache(1, K_SCALE, V_SCALE) if pool else caches(ctx, kind, [200])[0]
    kv.new_bounds(256)
    kv.slab.zero_()
    kv.import_(0, k, v)
    ctx.bounds_update(0, [kv])
    assert kv.bounded(0) == 3
    ctx.kv_append(0, [kv], [2], None, k[70:72].flatten(1), v[70:72].flatten(1), None, starts=[70])
    assert kv.length(0) == 72 and kv.bounded(0) == 1
    if pool:
        assert pool.free_pages == 8 - 2
    ke, ve = kv.export(0)
    assert np.array_equal(f64(ve), stored(v[:72], kind, V_SCALE)) and np.array_equal(f64(ke), stored(k[:72], kind, K_SCALE))
    # V^T tiles of block 1: [Hkv][d][64], zero from place 8 on
    el = torch.uint8 if "fp8" in kind else torch.bfloat16
    slab = kv.slab.view(el)
    if pool:
        tiles = slab[: 8 * 2 * 2 * 4096].view(8, 2, 2, 64, 64)[1, 1]
    else:
        tiles = slab[: 2 * 2 * 4 * 4096].view(2, 2, 4, 64, 64)[1, :, 1]
    assert not tiles[..., 8:].any() and tiles[..., :8].any()
    kv.truncate(0, 65)   # a stale tail that a later append has to clear
    ctx.kv_append(0, [kv], [1], None, k[65:66].flatten(1), v[65:66].flatten(1), None)
    assert not tiles[..., 2:].any()
    ctx.kv_append(0, [kv], [0], None, k[:0].flatten(1), v[:0].flatten(1), None, starts=[3])
    assert kv.length(0) == 3 and kv.bounded(0) == 0


def test_append_takes_explicit_positions_and_rotates_in_place():
    """Rotary positions other than the slots, more rows than one launch's arguments hold, queries turned where they are."""
    ctx = context(4, 2, 64)
    form = ROTARY_FORMS[0]
    rot = rotary_of(ctx, 64, form, max_pos=5000)
    g = gen(4)
    lens = [700, 1, 900]
    kvs = caches(ctx, "paged", lens)
    rows = sum(lens)
    q, k, v = normal(g, rows, 256), normal(g, rows, 128), normal(g, rows, 128)
    pos = np.random.default_rng(5).integers(0, 5000, rows)
    ref = rotated(q.view(rows, 4, 64), pos, 64, form)
    bound = rotation_bound(q.view(rows, 4, 64), ref, 64, form)
    kref = rotated(k.view(rows, 2, 64), pos, 64, form)
    ctx.kv_append(0, kvs, lens, q, k, v, q, rotary=rot, positions=pos)
    assert (np.abs(f64(q).reshape(ref.shape) - ref) <= bound).all()
    got = np.concatenate([f64(kv.export(0)[0]) for kv in kvs])
    assert (np.abs(got - kref) <= rotation_bound(k.view(rows, 2, 64), kref, 64, form)).all()


def test_append_of_more_blocks_than_one_launch_describes():
    ctx = context(4, 2, 64, max_tokens_per_call=8192)
    g = gen(6)
    k, v = normal(g, 6000, 2, 64), normal(g, 6000, 2, 64)
    lens = [100] * 20 + [4000]
    kvs = caches(ctx, "paged", lens)
    ctx.kv_append(0, kvs, lens, None, k.flatten(1), v.flatten(1), None)
    at = 0
    for kv, n in zip(kvs, lens):
        ke, ve = kv.export(0)
        assert torch.equal(ke, k[at: at + n]) and torch.equal(ve, v[at: at + n])
        at += n


# ------------------------------------------------------------------------------------------------ attention
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq, hkv, d", [(4, 2, 64), (28, 4, 128), (8, 8, 64), (24, 1, 128), (40, 1, 64), (16, 2, 128)])
def test_attend_single_tokens_and_drafts(kind, hq, hkv, d):
    """Few rows per request on caches of one token to many, ends inside and at the edge of tiles; queries strided, out wider than a row."""
    ctx = context(hq, hkv, d)
    g = gen(10)
    held = [1, 2, 63, 64, 65, 130, 700, 1500]
    lens = [1, 2, 1, 1, 3, 1, 2, 1]
    kvs = caches(ctx, kind, held)
    content = [(normal(g, n, hkv, d), normal(g, n, hkv, d)) for n in held]
    fill(kvs, content)
    rows = sum(lens)
    q = normal(g, rows, hq * d + 64, std=1.5)[:, 64:]
    out = torch.full((rows, hq * d + 16), float("nan"), device="cuda", dtype=torch.bfloat16)
    ws = ctx.attend_workspace(rows, len(held), fp8_visible_tokens=sum(held))
    ctx.attend(0, kvs, lens, q, out[:, 8: 8 + hq * d], ws)
    assert out[:, :8].isnan().all() and out[:, 8 + hq * d:].isnan().all()
    at = 0
    for n, t, (k, v) in zip(held, lens, content):
        ref, mag = O.attend(f64(q[at: at + t]).reshape(t, hq, d), stored(k, kind, K_SCALE), stored(v, kind, V_SCALE), n - t)
        assert_attention(out[at: at + t, 8: 8 + hq * d], ref, mag, f"{n} cached, {t} rows")
        at += t


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq, hkv, d", [(4, 2, 64), (28, 4, 128)])
def test_attend_mixes_single_tokens_and_chunks(kind, hq, hkv, d):
    """One call with a chunk, a few drafted tokens, an idle request and single tokens; a scale of the caller's."""
    ctx = context(hq, hkv, d)
    g = gen(11)
    held, lens = [300, 90, 50, 128, 9], [150, 4, 0, 128, 1]
    kvs = caches(ctx, kind, held)
    content = [(normal(g, n, hkv, d), normal(g, n, hkv, d)) for n in held]
    fill(kvs, content)
    rows = sum(lens)
    q = normal(g, rows, hq * d)
    out = torch.full_like(q, float("nan"))
    ctx.attend(0, kvs, lens, q, out, ctx.attend_workspace(rows, len(held), fp8_visible_tokens=sum(held)), scale=0.2)
    at = 0
    for n, t, (k, v) in zip(held, lens, content):
        ref, mag = O.attend(f64(q[at: at + t]).reshape(t, hq, d), stored(k, kind, K_SCALE), stored(v, kind, V_SCALE), n - t, scale=0.2)
        if t:
            assert_attention(out[at: at + t], ref, mag, f"{n} cached, {t} rows")
        at += t


@pytest.mark.parametrize("kind, held, lens", [("paged_fp8", [20011], [1]), ("contiguous", [9000, 333], [2, 1]), ("paged", [5000], [9]),
                                               ("paged", [4000 - 61 * i for i in range(40)], [1] * 40)])
def test_attend_joins_parts_of_long_caches(kind, held, lens):
    """Long key ranges are cut into parts; descriptors beyond the kernel arguments."""
    hq, hkv, d = 28, 4, 128
    ctx = context(hq, hkv, d)
    g = gen(12)
    kvs = caches(ctx, kind, held)
    content = [(normal(g, n, hkv, d), normal(g, n, hkv, d)) for n in held]
    fill(kvs, content)
    rows = sum(lens)
    q = normal(g, rows, hq * d, std=2.0)
    out = torch.empty_like(q)
    ctx.attend(0, kvs, lens, q, out, ctx.attend_workspace(rows, len(held)))
    at = 0
    for n, t, (k, v) in zip(held, lens, content):
        ref, mag = O.attend(f64(q[at: at + t]).reshape(t, hq, d), stored(k, kind, K_SCALE), stored(v, kind, V_SCALE), n - t)
        assert_attention(out[at: at + t], ref, mag, f"{n} cached")
        at += t


def test_attend_takes_scales_of_8_bit_caches_that_are_no_powers_of_two():
    """Few rows read code * scale without a rounding of its own."""
    hq, hkv, d = 4, 2, 64
    ctx = context(hq, hkv, d)
    g = gen(13)
    kv, = caches(ctx, "fp8", [777], scales=(0.0473, 0.0311))
    k, v = normal(g, 777, hkv, d), normal(g, 777, hkv, d)
    kv.import_(0, k, v)
    kc, vc = kv.export_codes(0)
    q = normal(g, 1, hq * d)
    out = torch.empty_like(q)
    ctx.attend(0, [kv], [1], q, out, ctx.attend_workspace(1))
    scales = [float(np.float32(s)) for s in (0.0473, 0.0311)]
    ref, mag = O.attend(f64(q).reshape(1, hq, d), e4m3_decode(kc.cpu().numpy()) * scales[0], e4m3_decode(vc.cpu().numpy()) * scales[1], 776)
    assert_attention(out, ref, mag)


def test_every_8_bit_code_is_read_as_its_value():
    """A cache of one token: the output is its value, whatever the code."""
    ctx = context(4, 2, 128)
    kv, = caches(ctx, "fp8", [1], scales=(1.0, 1.0))
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").view(1, 2, 128)
    kv.import_codes(0, torch.zeros_like(codes), codes)
    q, out = torch.zeros((1, 512), dtype=torch.bfloat16, device="cuda"), torch.empty((1, 512), dtype=torch.bfloat16, device="cuda")
    ctx.attend(0, [kv], [1], q, out, ctx.attend_workspace(1))
    ref = e4m3_decode(np.arange(256, dtype=np.uint8)).reshape(2, 128)
    for head in range(4):
        got, want = f64(out).reshape(4, 128)[head], ref[head // 2]
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)])


@pytest.mark.parametrize("kind", ["contiguous", "paged"])
@pytest.mark.parametrize("held, rows", [(100, 8), (1300, 8), (5000, 4), (400, 200), (3000, 130)])
def test_what_a_query_does_not_see_does_not_reach_it(kind, held, rows):
    """The last tokens' keys and values are infinite or NaN: earlier queries of the same call, few or a chunk, on whole and on
    split key ranges, are as without them; the queries that see them are not finite."""
    hq, hkv, d = 4, 2, 64
    ctx = context(hq, hkv, d)
    g = gen(14)
    kv, = caches(ctx, kind, [held])
    k, v = normal(g, held, hkv, d), normal(g, held, hkv, d)
    bad = 3
    k[-1, 0, 5], v[-1, 1, 7], v[-2, 0, 63], v[-3, 0, 2], v[-3, 1, 2] = float("inf"), float("nan"), float("-inf"), float("inf"), float("nan")
    kv.import_(0, k, v)
    q = normal(g, rows, hq * d)
    out = torch.empty_like(q)
    ctx.attend(0, [kv], [rows], q, out, ctx.attend_workspace(rows))
    ref, mag = O.attend(f64(q[: rows - bad]).reshape(-1, hq, d), f64(k), f64(v), held - rows)
    assert_attention(out[: rows - bad], ref, mag)
    assert not out[rows - bad:].isfinite().all(1).any()


def test_a_dropped_token_does_not_reach_later_reads():
    """Infinite values behind the newest token, left by tokens that were dropped, in the block that is read."""
    hq, hkv, d = 4, 2, 64
    ctx = context(hq, hkv, d)
    g = gen(15)
    kv, = caches(ctx, "contiguous", [200])
    k, v = normal(g, 200, hkv, d), normal(g, 200, hkv, d)
    k[140:], v[140:] = float("nan"), float("inf")
    kv.import_(0, k, v)
    kv.truncate(0, 140)
    for rows in (1, 100):
        q = normal(g, rows, hq * d)
        out = torch.empty_like(q)
        ctx.attend(0, [kv], [rows], q, out, ctx.attend_workspace(rows))
        ref, mag = O.attend(f64(q).reshape(rows, hq, d), f64(k[:140]), f64(v[:140]), 140 - rows)
        assert_attention(out, ref, mag)


def test_large_scores_and_keys_of_minus_infinity():
    """Scores of several hundred (weights of one and zero), and keys that score minus infinity among others."""
    hq, hkv, d = 4, 2, 64
    ctx = context(hq, hkv, d)
    g = gen(16)
    for rows in (1, 100):
        kv, = caches(ctx, "contiguous", [900])
        k, v = normal(g, 900, hkv, d, std=20.0), normal(g, 900, hkv, d)
        k[::3, :, 0] = float("-inf")
        q = normal(g, rows, hq * d, std=4.0).view(rows, hq, d)
        q[:, :, 0] = 1.0
        kv.import_(0, k, v)
        out = torch.empty((rows, hq * d), dtype=torch.bfloat16, device="cuda")
        ctx.attend(0, [kv], [rows], q.flatten(1), out, ctx.attend_workspace(rows))
        ref, mag = O.attend(f64(q), f64(k), f64(v), 900 - rows)
        # scores up to 2^10, fp32: their errors, up to 2^-11, are weights' relative errors
        off = np.abs(f64(out).reshape(ref.shape) - ref) - (SLACK + 2.0 ** -10) * mag
        assert off.max() <= 0


def test_attend_on_another_stream_and_twice_the_same_bits():
    hq, hkv, d = 28, 4, 128
    ctx = context(hq, hkv, d)
    g = gen(17)
    held, lens = [5000, 300, 2222], [1, 40, 3]
    kvs = caches(ctx, "paged", held)
    fill(kvs, [(normal(g, n, hkv, d), normal(g, n, hkv, d)) for n in held])
    q = normal(g, sum(lens), hq * d)
    ws = ctx.attend_workspace(sum(lens), 3)
    outs = [torch.empty_like(q) for _ in range(2)]
    ctx.attend(0, kvs, lens, q, outs[0], ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx.attend(0, kvs, lens, q, outs[1], ws)
    side.synchronize()
    assert torch.equal(outs[0], outs[1])


def test_pages_beyond_four_gigabytes():
    """A request whose pages lie beyond 2^32 bytes of the pool, filled and read by every operator."""
    from paper_2509_24381_amd.binding import KVPool
    hq, hkv, d = 28, 4, 128
    ctx = context(hq, hkv, d)
    page = 2 * hkv * 64 * d * 2
    pool = KVPool(ctx, (1 << 32) // page + 40)
    others, filler = [], torch.zeros((32768, hkv, d), dtype=torch.bfloat16, device="cuda")
    while pool.free_pages > 39:
        kv = pool.new_cache(1)
        n = min(32768, 64 * (pool.free_pages - 39))
        kv.import_(0, filler[:n], filler[:n])
        others.append(kv)
    g = gen(18)
    kv = pool.new_cache(1)
    kv.new_bounds(4096)
    n = 2000
    k, v = normal(g, n, hkv, d), normal(g, n, hkv, d)
    ctx.kv_append(0, [kv], [n], None, k.flatten(1), v.flatten(1), None)
    ke, ve = kv.export(0)
    assert torch.equal(ke, k) and torch.equal(ve, v)
    ref = None
    for rows in (1, 20):
        q = normal(g, rows, hq * d)
        out = torch.empty_like(q)
        ctx.attend(0, [kv], [rows], q, out, ctx.attend_workspace(rows))
        ref, mag = O.attend(f64(q).reshape(rows, hq, d), f64(k), f64(v), n - rows)
        assert_attention(out, ref, mag)
        ctx.attend_blocks(0, [kv], [rows], q, out, ctx.attend_workspace(rows, n_blocks=64), 64)
        assert_attention(out, ref, mag)
    del others, kv, pool
    gc.collect()


# ------------------------------------------------------------------------------------------------ bounds and selected blocks
def bounds_of(x):
    """Oracle bounds of every finished block and head of [n, Hkv, d]: codes [blocks, Hkv, 2, d], units [blocks, Hkv]."""
    blocks, hkv, d = len(x) // 64, x.shape[1], x.shape[2]
    codes, units = np.zeros((blocks, hkv, 2, d), dtype=np.int64), np.zeros((blocks, hkv))
    for b in range(blocks):
        for h in range(hkv):
            codes[b, h, 0], codes[b, h, 1], units[b, h] = O.block_bounds(x[64 * b: 64 * b + 64, h])
    return codes, units


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hkv, d", [(2, 64), (4, 128)])
def test_bounds_are_exact(kind, hkv, d):
    """Ordinary keys, and blocks of zeros, tiny, huge, infinite and NaN ones; several requests; a bound on every key."""
    ctx = context(hkv, hkv, d)
    g = gen(20)
    held = [700, 63, 64, 201]
    kvs = caches(ctx, kind, held)
    content = [(normal(g, n, hkv, d), normal(g, n, hkv, d)) for n in held]
    k = content[0][0]
    k[64:128] = 0.0
    k[128:192] *= 1e-30
    k[130, 0, 1] = 0.0
    if "fp8" not in kind:
        k[192:256] *= 1e35
        k[260, 0, 3], k[270, 1, 5], k[320, 0, 7] = float("inf"), float("-inf"), float("nan")
        k[384:448, :, 0] = float("nan")
        k[448:512] = 2.0 ** -133
    fill(kvs, content)
    room = 16
    memory = [kv.new_bounds(64 * room) for kv in kvs]
    for codes, units in memory:
        codes.fill_(77)
        units.fill_(-1)
    ctx.bounds_update(0, kvs)
    for kv, n, (x, _), (codes, units) in zip(kvs, held, content, memory):
        x = stored(x, kind, K_SCALE)
        want_codes, want_units = bounds_of(x)
        full = n // 64
        assert kv.bounded(0) == full
        got_codes, got_units = codes[0].cpu().numpy().astype(np.int64), f64(units[0])
        assert np.array_equal(got_codes[:, :full].transpose(1, 0, 2, 3), want_codes) and np.array_equal(got_units[:, :full].T, want_units)
        assert (got_codes[:, full:] == 77).all() and (got_units[:, full:] == -1).all()
        for b in range(full):
            keys = x[64 * b: 64 * b + 64]
            with np.errstate(invalid="ignore"):
                fine = np.isfinite(keys) & (np.abs(keys) <= O.LIMIT)
                assert (np.where(fine, keys - want_codes[b, :, 0] * want_units[b][:, None], 0) <= 0).all()
                assert (np.where(fine, keys - want_codes[b, :, 1] * want_units[b][:, None], 0) >= 0).all()


def test_bounds_follow_what_the_cache_holds():
    """Only new blocks are computed, or those from a slot on; dropping tokens and importing take bounds back."""
    ctx = context(4, 2, 64)
    g = gen(21)
    kv, = caches(ctx, "paged", [640])
    k, v = normal(g, 640, 2, 64), normal(g, 640, 2, 64)
    codes, units = kv.new_bounds(640)
    kv.import_(0, k[:200], v[:200])
    ctx.bounds_update(0, [kv])
    assert kv.bounded(0) == 3
    codes.zero_()
    ctx.kv_append(0, [kv], [440], None, k[200:].flatten(1), v[200:].flatten(1), None)
    assert kv.bounded(0) == 3
    ctx.bounds_update(0, [kv])
    assert kv.bounded(0) == 10 and not codes[0, :, :3].any() and codes[0, :, 3:].any(-1).all()
    ctx.bounds_update(0, [kv], firsts=[64])
    assert not codes[0, :, :1].any() and codes[0, :, 1:].any(-1).all()
    kv.truncate(0, 300)
    assert kv.bounded(0) == 4
    kv.import_(0, k[:100], v[:100])
    assert kv.bounded(0) == 0
    kv.reset()
    assert kv.bounded(0) == 0


def run_blocks(ctx, kvs, lens, q, n_blocks, n_first, n_last, scale=0.0):
    rows = sum(lens)
    out = torch.full_like(q, float("nan"))
    chosen = torch.full((rows, ctx.cfg.n_kv_heads, n_blocks), -7, dtype=torch.int32, device="cuda")
    ctx.attend_blocks(0, kvs, lens, q, out, ctx.attend_workspace(rows, len(lens), n_blocks=n_blocks), n_blocks, n_first, n_last, chosen=chosen, scale=scale)
    return out, chosen.cpu().numpy()


def check_blocks(ctx, kind, held, lens, content, q, out, chosen, n_blocks, n_first, n_last):
    hq, hkv, d = ctx.cfg.n_q_heads, ctx.cfg.n_kv_heads, ctx.cfg.head_dim
    g = hq // hkv
    at = 0
    for n, t, (k, v) in zip(held, lens, content):
        ks, vs = stored(k, kind, K_SCALE), stored(v, kind, V_SCALE)
        codes, units = bounds_of(ks)
        qh = f64(q[at: at + t]).reshape(t, hq, d)
        want = {}
        for i in range(t):
            for h in range(hkv):
                bounds = [(codes[b, h, 0], codes[b, h, 1], units[b, h]) for b in range(len(codes))]
                want[i, h] = O.select_blocks(qh[i, h * g: (h + 1) * g], bounds, n - t + i, n_blocks, n_first, n_last)
                got = chosen[at + i, h].tolist()
                assert got == want[i, h] + [-1] * (n_blocks - len(want[i, h])), (n, i, h)

        def allowed(i, h):
            m = np.zeros(n + 64, dtype=bool)
            for b in want[i, h]:
                m[64 * b: 64 * b + 64] = True
            return m

        if t:
            ref, mag = O.attend(qh, ks, vs, n - t, allowed=allowed)
            assert_attention(out[at: at + t], ref, mag, f"{n} cached, {t} rows")
        at += t


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq, hkv, d, n_blocks, n_first, n_last", [(4, 2, 64, 4, 1, 2), (28, 4, 128, 5, 0, 1), (8, 8, 64, 9, 2, 3), (24, 1, 128, 3, 1, 1), (40, 1, 64, 6, 1, 2)])
def test_selected_blocks_and_attention_over_them(kind, hq, hkv, d, n_blocks, n_first, n_last):
    """Single tokens, a few and more, on caches with fewer blocks than are taken, as many, and many more."""
    ctx = context(hq, hkv, d)
    g = gen(30)
    held, lens = [1, 64, 300, 1500, 777], [1, 2, 0, 1, 20]
    kvs = caches(ctx, kind, held)
    content = [(normal(g, n, hkv, d), normal(g, n, hkv, d)) for n in held]
    fill(kvs, content)
    for kv, n in zip(kvs, held):
        kv.new_bounds(n + 64)
    q = normal(g, sum(lens), hq * d, std=1.5)
    out, chosen = run_blocks(ctx, kvs, lens, q, n_blocks, n_first, n_last)
    check_blocks(ctx, kind, held, lens, content, q, out, chosen, n_blocks, n_first, n_last)
    assert [kv.bounded(0) for kv, t in zip(kvs, lens) if t] == [n // 64 for n, t in zip(held, lens) if t]


@pytest.mark.parametrize("rows", [1, 70])
def test_equal_scores_go_to_the_lowest_blocks(rows):
    """All blocks alike; and two kinds of them by turns."""
    hq, hkv, d = 4, 2, 64
    ctx = context(hq, hkv, d)
    g = gen(31)
    kv, = caches(ctx, "paged", [64 * 40])
    one, two = normal(g, 64, hkv, d), normal(g, 64, hkv, d)
    for blocks in ([one] * 40, [one, two] * 20):
        k = torch.cat(blocks)
        v = normal(g, 64 * 40, hkv, d)
        kv.import_(0, k, v)
        kv.new_bounds(64 * 40)
        q = normal(g, rows, hq * d)
        out, chosen = run_blocks(ctx, [kv], [rows], q, 7, 1, 2)
        check_blocks(ctx, "paged", [64 * 40], [rows], [(k, v)], q, out, chosen, 7, 1, 2)
        if blocks[1] is one and rows == 1:
            assert chosen[0].tolist() == [[0, 1, 2, 3, 4, 38, 39]] * hkv


@pytest.mark.parametrize("n_blocks, n_first, n_last", [(1, 0, 1), (3, 5, 2), (2, 0, 6), (40, 40, 1), (12, 0, 40)])
def test_first_and_last_blocks(n_blocks, n_first, n_last):
    """More forced blocks than there is room for, or than there are."""
    hq, hkv, d = 4, 2, 64
    ctx = context(hq, hkv, d)
    g = gen(32)
    held, lens = [1000, 130], [3, 1]
    kvs = caches(ctx, "contiguous", held)
    content = [(normal(g, n, hkv, d), normal(g, n, hkv, d)) for n in held]
    fill(kvs, content)
    for kv in kvs:
        kv.new_bounds(1024)
    q = normal(g, 4, hq * d)
    out, chosen = run_blocks(ctx, kvs, lens, q, n_blocks, n_first, n_last)
    check_blocks(ctx, "contiguous", held, lens, content, q, out, chosen, n_blocks, n_first, n_last)


def test_queries_and_keys_that_are_not_finite_are_scored_as_defined():
    """NaN, infinite, huge and zero queries select by the definition, and leave the other heads' outputs alone."""
    hq, hkv, d = 4, 2, 64
    ctx = context(hq, hkv, d)
    g = gen(33)
    kv, = caches(ctx, "contiguous", [1300])
    k, v = normal(g, 1300, hkv, d), normal(g, 1300, hkv, d)
    k[100, 0, 3], k[500, 0, 9] = float("nan"), float("inf")
    kv.import_(0, k, v)
    kv.new_bounds(1300)
    q = normal(g, 5, hq * d).view(5, hq, d)
    q[0, 0, 0], q[1, 1, 5], q[2, 0] = float("nan"), float("-inf"), 0.0
    q[3] *= 1e37
    out, chosen = run_blocks(ctx, [kv], [5], q.flatten(1), 4, 0, 1)
    codes, units = bounds_of(f64(k))
    for i in range(5):
        for h in range(hkv):
            bounds = [(codes[b, h, 0], codes[b, h, 1], units[b, h]) for b in range(20)]
            want = O.select_blocks(f64(q)[i, 2 * h: 2 * h + 2], bounds, 1295 + i, 4, 0, 1)
            assert chosen[i, h].tolist() == want
    # KV head 1 of row 2 has finite queries and keys
    allowed = np.zeros(1300, dtype=bool)
    for b in chosen[2, 1]:
        allowed[64 * b: 64 * b + 64] = True
    seen = np.nonzero(allowed[:1298])[0]
    for head in (2, 3):
        ref, mag = O.attend_row(f64(q)[2, head], f64(k)[seen, 1], f64(v)[seen, 1], 1 / math.sqrt(d))
        assert (np.abs(f64(out).reshape(5, hq, d)[2, head] - ref) <= SLACK * mag).all()


def test_selection_over_a_very_long_cache():
    """More blocks than a wavefront's registers or one thread's share; a long table of pages."""
    hq, hkv, d = 4, 2, 64
    ctx = context(hq, hkv, d, max_pos=300000)
    g = gen(34)
    n = 64 * 4100 + 17
    kv, = caches(ctx, "paged_fp8", [n])
    k, v = normal(g, n, hkv, d), normal(g, n, hkv, d)
    kv.import_(0, k, v)
    kv.new_bounds(n)
    for rows in (1, 6):
        q = normal(g, rows, hq * d)
        out, chosen = run_blocks(ctx, [kv], [rows], q, 33, 1, 2)
        check_blocks(ctx, "paged_fp8", [n], [rows], [(k, v)], q, out, chosen, 33, 1, 2)


# ------------------------------------------------------------------------------------------------ refusals
def test_calls_on_a_capturing_stream_are_refused_and_change_nothing():
    from paper_2509_24381_amd.binding import RsError
    ctx = context(4, 2, 64)
    kv, = caches(ctx, "contiguous", [256])
    g = gen(40)
    k, v, q = normal(g, 130, 2, 64), normal(g, 130, 2, 64), normal(g, 1, 256)
    kv.import_(0, k, v)
    kv.new_bounds(256)
    ws = ctx.attend_workspace(1, n_blocks=2)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    calls = [lambda: ctx.kv_append(0, [kv], [1], None, k[:1].flatten(1), v[:1].flatten(1), None), lambda: ctx.attend(0, [kv], [1], q, q, ws),
             lambda: ctx.bounds_update(0, [kv]), lambda: ctx.attend_blocks(0, [kv], [1], q, q, ws, 2)]
    x = torch.zeros(4, device="cuda")
    with torch.cuda.stream(side):
        graph.capture_begin()
        x += 1
        for call in calls:
            with pytest.raises(RsError) as e:
                call()
            assert e.value.status_name == "RS_ESTATE"
        graph.capture_end()
    torch.cuda.synchronize()
    assert kv.length(0) == 130 and kv.bounded(0) == 0
    out = torch.empty_like(q)
    ctx.attend(0, [kv], [1], q, out, ws)
    ref, mag = O.attend(f64(q).reshape(1, 4, 64), f64(k), f64(v), 129)
    assert_attention(out, ref, mag)
