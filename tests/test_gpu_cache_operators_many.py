"""GPU: the operators on caches with more requests, pages and blocks than one form of their descriptors holds, and lists of blocks that are
cut into parts, against the 64-bit oracle; tolerances as in test_gpu_cache_operators.py."""
import numpy as np
import pytest
import torch

import test_gpu_cache_operators as T
from oracle import cache_ops as O

pytestmark = pytest.mark.gpu


def filled(ctx, kind, held, seed, d=64, hkv=2):
    g = T.gen(seed)
    kvs = T.caches(ctx, kind, held)
    content = [(T.normal(g, n, hkv, d), T.normal(g, n, hkv, d)) for n in held]
    T.fill(kvs, content)
    return kvs, content, g


def check_attend(ctx, kind, kvs, content, held, lens, g):
    hq, hkv, d = ctx.cfg.n_q_heads, ctx.cfg.n_kv_heads, ctx.cfg.head_dim
    rows = sum(lens)
    q = T.normal(g, rows, hq * d, std=1.5)
    out = torch.full_like(q, float("nan"))
    ctx.attend(0, kvs, lens, q, out, ctx.attend_workspace(rows, len(held), fp8_visible_tokens=sum(held)))
    at = 0
    for n, t, (k, v) in zip(held, lens, content):
        if t:
            ref, mag = O.attend(T.f64(q[at: at + t]).reshape(t, hq, d), T.stored(k, kind, T.K_SCALE), T.stored(v, kind, T.V_SCALE), n - t)
            T.assert_attention(out[at: at + t], ref, mag, f"{n} cached, {t} rows")
        at += t


@pytest.mark.parametrize("kind", ["paged", "paged_fp8"])
@pytest.mark.parametrize("requests, longest", [(66, 60), (67, 60), (100, 40), (128, 700), (20, 3500)])
@pytest.mark.parametrize("chunk", [0, 60])
def test_attend_of_many_requests_and_pages(kind, requests, longest, chunk, monkeypatch):
    """Descriptors in the kernel arguments, page numbers beside them or in place, all of it in the workspace; with a chunk for the chunk
    kernel beside them, whose own descriptors are copied in the same launch."""
    monkeypatch.setenv("RS_ATTEND_FEW", "0")
    ctx = T.context(4, 2, 64, max_requests=160)
    held = [1 + (i * 37 + longest) % longest for i in range(requests)] + ([chunk + 130] if chunk else [])
    lens = [0 if i == 3 else 2 if n > 1 and i % 5 == 0 else 1 for i, n in enumerate(held)]
    if chunk:
        lens[-1] = chunk
    kvs, content, g = filled(ctx, kind, held, 60)
    check_attend(ctx, kind, kvs, content, held, lens, g)


@pytest.mark.parametrize("kind", T.KINDS)
def test_append_of_many_requests(kind):
    """A token for every one of 90 requests, with explicit positions: more than one launch's descriptors."""
    ctx = T.context(4, 2, 64, max_requests=160)
    held = [(i * 29) % 130 for i in range(90)]
    g = T.gen(61)
    kvs = T.caches(ctx, kind, [n + 1 for n in held])
    content = [(T.normal(g, n, 2, 64), T.normal(g, n, 2, 64)) for n in held]
    for kv, (k, v) in zip(kvs, content):
        if len(k):
            kv.import_(0, k, v)
    form = T.ROTARY_FORMS[1]
    rot = T.rotary_of(ctx, 32, form)
    pos = [(7 * i) % 2000 for i in range(90)]
    q, k, v = T.normal(g, 90, 256), T.normal(g, 90, 128), T.normal(g, 90, 128)
    out = torch.empty_like(q)
    ctx.kv_append(0, kvs, [1] * 90, q, k, v, out, rotary=rot, positions=pos)
    ref = T.rotated(q.view(90, 4, 64), np.array(pos), 32, form)
    assert (np.abs(T.f64(out).reshape(ref.shape) - ref) <= T.rotation_bound(q.view(90, 4, 64), ref, 32, form)).all()
    assert [kv.length(0) for kv in kvs] == [n + 1 for n in held]
    for i, (kv, n) in enumerate(zip(kvs, held)):
        _, ve = kv.export(0)
        assert np.array_equal(T.f64(ve[n]), T.stored(v[i].view(2, 64), kind, T.V_SCALE))


@pytest.mark.parametrize("kind", ["paged", "paged_fp8"])
def test_bounds_of_more_pages_than_one_launch_describes(kind):
    ctx = T.context(4, 2, 64, max_requests=160)
    held = [64 * (i % 60) + 5 * i for i in range(50)]
    kvs, content, _ = filled(ctx, kind, [max(n, 1) for n in held], 62)
    memory = [kv.new_bounds(64 * 64) for kv in kvs]
    ctx.bounds_update(0, kvs)
    for kv, (k, _), (codes, units) in zip(kvs, content, memory):
        want_codes, want_units = T.bounds_of(T.stored(k, kind, T.K_SCALE))
        full = len(want_codes)
        assert kv.bounded(0) == full == len(k) // 64
        assert np.array_equal(codes[0, :, :full].cpu().numpy().transpose(1, 0, 2, 3), want_codes)
        assert np.array_equal(T.f64(units[0, :, :full]).T, want_units)


@pytest.mark.parametrize("rows", [1, 3])
def test_blocks_of_many_requests(rows):
    """100 requests: more descriptors than one selection launch has, pages beyond the kernel arguments, bounds that are missing."""
    ctx = T.context(4, 2, 64, max_requests=160)
    held = [rows + (i * 91) % 900 for i in range(100)]
    lens = [0 if i % 9 == 4 else rows for i in range(100)]
    kvs, content, g = filled(ctx, "paged", held, 63)
    for kv, n in zip(kvs, held):
        kv.new_bounds(n + 64)
    q = T.normal(g, sum(lens), 256, std=1.5)
    out, chosen = T.run_blocks(ctx, kvs, lens, q, 5, 1, 2)
    T.check_blocks(ctx, "paged", held, lens, content, q, out, chosen, 5, 1, 2)


@pytest.mark.parametrize("kind", ["contiguous", "paged_fp8"])
@pytest.mark.parametrize("hq, hkv, d", [(14, 2, 128), (40, 1, 64)])
@pytest.mark.parametrize("held, lens, n_blocks", [([4500], [1], 48), ([2500, 4000, 600], [1, 3, 2], 33), ([3000], [70], 20), ([1700], [100], 17), ([1100], [200], 16)])
def test_lists_in_parts(kind, hq, hkv, d, held, lens, n_blocks):
    """Lists of more blocks than four wavefronts take alone are cut into parts by how many rows there are; shorter ones are not."""
    ctx = T.context(hq, hkv, d)
    kvs, content, g = filled(ctx, kind, held, 64, d, hkv)
    for kv, n in zip(kvs, held):
        kv.new_bounds(n + 64)
    q = T.normal(g, sum(lens), hq * d, std=1.5)
    out, chosen = T.run_blocks(ctx, kvs, lens, q, n_blocks, 1, 2)
    T.check_blocks(ctx, kind, held, lens, content, q, out, chosen, n_blocks, 1, 2)


def test_masked_values_that_are_not_finite_in_lists_in_parts():
    """What lies behind a row's own slot, in the block it is in, is infinite or NaN; lists in parts, and slots of rows that end in another part."""
    hq, hkv, d = 14, 2, 128
    ctx = T.context(hq, hkv, d)
    g = T.gen(65)
    n, rows = 64 * 40, 30
    k, v = T.normal(g, n, hkv, d), T.normal(g, n, hkv, d)
    kv, = T.caches(ctx, "paged", [n])
    dirty_k, dirty_v = k.clone(), v.clone()
    dirty_v[-4:, 0] = float("nan")
    dirty_k[-4:, 1] = float("inf")
    dirty_v[-8:-4, 1, :5] = float("-inf")
    kv.import_(0, dirty_k, dirty_v)
    kv.new_bounds(n)
    q = T.normal(g, rows, hq * d)
    out, chosen = T.run_blocks(ctx, [kv], [rows], q, 40, 1, 2)
    ref, mag = O.attend(T.f64(q).reshape(rows, hq, d), T.f64(k), T.f64(v), n - rows)
    T.assert_attention(out[:rows - 8], ref[:rows - 8], mag[:rows - 8])


@pytest.mark.parametrize("kind", T.KINDS)
@pytest.mark.parametrize("hq, hkv, d", [(64, 8, 64), (28, 4, 128), (40, 2, 128)])
def test_drafts_on_much_cache(kind, hq, hkv, d):
    """Requests of 33 to 64 rows and more in calls with so much to read that wavefronts have 32 rows, beside single tokens and few drafts."""
    ctx = T.context(hq, hkv, d)
    per_head = 2100 // hkv * 64 // 6
    lens = [5, 1, 12, 8, 3, 0, 7, 2, 1, 16]
    held = [per_head + 171 * i for i in range(6)] + [300, 40, 1, 16]
    kvs, content, g = filled(ctx, kind, held, 66, d, hkv)
    check_attend(ctx, kind, kvs, content, held, lens, g)


@pytest.mark.parametrize("kind", ["contiguous", "paged"])
def test_what_drafts_on_much_cache_do_not_see_does_not_reach_them(kind):
    """Infinities and NaN behind the rows' own slots, in their blocks; wavefronts of 32 rows."""
    hq, hkv, d = 64, 8, 64
    ctx = T.context(hq, hkv, d)
    g = T.gen(67)
    n, rows = 17011, 8
    kv, = T.caches(ctx, kind, [n])
    k, v = T.normal(g, n, hkv, d), T.normal(g, n, hkv, d)
    dirty_k, dirty_v = k.clone(), v.clone()
    dirty_v[-3:, 0] = float("nan")
    dirty_v[-2:, 1, 7] = float("inf")
    dirty_k[-1:, 2] = float("-inf")
    kv.import_(0, dirty_k, dirty_v)
    q = T.normal(g, rows, hq * d, std=1.5)
    out = torch.full_like(q, float("nan"))
    ctx.attend(0, [kv], [rows], q, out, ctx.attend_workspace(rows))
    ref, mag = O.attend(T.f64(q).reshape(rows, hq, d), T.f64(k), T.f64(v), n - rows)
    T.assert_attention(out[: rows - 3], ref[: rows - 3], mag[: rows - 3])
    group = hq // hkv * d   # (the other KV heads' rows are whole to the last)
    T.assert_attention(out[:, 3 * group:].reshape(rows, hq - 3 * (hq // hkv), d), ref[:, 3 * (hq // hkv):], mag[:, 3 * (hq // hkv):])


@pytest.mark.parametrize("rule", ["0", "1000000"])
def test_out_may_be_q(rule, monkeypatch):
    """The same bits whether the output goes to memory of its own or over the queries."""
    monkeypatch.setenv("RS_ATTEND_FEW", rule)
    hq, hkv, d = 28, 4, 128
    ctx = T.context(hq, hkv, d)
    held, lens = [3000, 700, 90, 400], [1, 5, 40, 150]
    kvs, content, g = filled(ctx, "paged", held, 68, d, hkv)
    q = T.normal(g, sum(lens), hq * d)
    ws = ctx.attend_workspace(sum(lens), len(held))
    out, over = torch.empty_like(q), q.clone()
    ctx.attend(0, kvs, lens, q, out, ws)
    ctx.attend(0, kvs, lens, over, over, ws)
    assert torch.equal(out, over)
    for kv, n in zip(kvs, held):
        kv.new_bounds(n + 64)
    ws = ctx.attend_workspace(sum(lens), len(held), n_blocks=20)
    over = q.clone()
    ctx.attend_blocks(0, kvs, lens, q, out, ws, 20)
    ctx.attend_blocks(0, kvs, lens, over, over, ws, 20)
    assert torch.equal(out, over)


@pytest.mark.parametrize("kind", ["contiguous", "paged_fp8"])
@pytest.mark.parametrize("held, rows, n_blocks", [(17000, 70, 6), (17000, 129, 19), (40000, 1, 33), (1100, 300, 5), (3000, 260, 24), (17000, 260, 4)])
def test_every_way_to_select(kind, held, rows, n_blocks):
    """Selection and attention in one kernel, with scores taken ahead and without, and in kernels of their own for few tokens and for many."""
    ctx = T.context(4, 2, 64)
    kvs, content, g = filled(ctx, kind, [held], 69)
    kvs[0].new_bounds(held + 64)
    q = T.normal(g, rows, 256, std=1.5)
    out, chosen = T.run_blocks(ctx, kvs, [rows], q, n_blocks, 1, 2)
    T.check_blocks(ctx, kind, [held], [rows], content, q, out, chosen, n_blocks, 1, 2)
    over = torch.empty_like(out)
    ctx.attend_blocks(0, kvs, [rows], q, over, ctx.attend_workspace(rows, 1, n_blocks=n_blocks), n_blocks)   # (the lists are not wanted)
    assert torch.equal(out, over)


@pytest.mark.parametrize("kind", ["paged", "paged_fp8"])
@pytest.mark.parametrize("rows, n_blocks", [(1, 9), (3, 40), (16, 9)])
def test_selection_from_many_pages(kind, rows, n_blocks):
    """More pages than the kernel arguments hold: a token or two select in a kernel of their own, more in the one that attends."""
    held = 70000
    ctx = T.context(4, 2, 64, max_pos=80000)
    kvs, content, g = filled(ctx, kind, [held], 70)
    kvs[0].new_bounds(held + 64)
    q = T.normal(g, rows, 256, std=1.5)
    out, chosen = T.run_blocks(ctx, kvs, [rows], q, n_blocks, 1, 2)
    T.check_blocks(ctx, kind, [held], [rows], content, q, out, chosen, n_blocks, 1, 2)
