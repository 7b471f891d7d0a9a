"""GPU: attention whose scores are far beyond 2^24 (in powers of two), and scales that make them so or make them vanish, against the 64-bit
oracle: a softmax of finite scores is finite, on whole and on split key ranges, of everything cached and of selected blocks.

A score is an fp32 sum of d exact products, so off by at most d 2^-23 sum_j |q_j k_j| in whatever order it is taken, and by as much again
where it is scaled; so is its difference from another one.  Where the best key of a row leads by more than that and 2^7 (in powers of two),
every other weight vanishes: the output is that key's value, rounded to bfloat16 (2^-8; the joining of parts adds less than 2^-20).
"""
import math

import numpy as np
import pytest
import torch

import test_gpu_cache_operators as T
from oracle import cache_ops as O

pytestmark = pytest.mark.gpu
ONE_KEY = 2.0 ** -8 + 2.0 ** -20


def check_winners(out, q, k, v, first, scale, least=0.9):
    """Rows whose best key leads are that key's value; all rows are finite and within the range of the values they see."""
    t_n, hq, d = q.shape
    g = hq // k.shape[1]
    got, led = T.f64(out).reshape(q.shape), 0
    assert np.isfinite(got).all(), f"{int((~np.isfinite(got)).sum())} elements of {got.size} are not finite"
    for t in range(t_n):
        n = first + t + 1
        for head in range(hq):
            kk, vv, c = k[:n, head // g], v[:n, head // g], scale * math.log2(math.e)
            s = kk @ q[t, head] * c
            off = 2 * d * 2.0 ** -23 * (np.abs(kk) @ np.abs(q[t, head])).max() * c
            best = int(s.argmax())
            near = s > s[best] - 2 * off - 128
            lo, hi = vv[near].min(0), vv[near].max(0)
            assert (got[t, head] >= lo - ONE_KEY * np.abs(lo)).all() and (got[t, head] <= hi + ONE_KEY * np.abs(hi)).all(), (n, t, head)
            led += near.sum() == 1
    assert led >= least * t_n * hq, f"only {led} of {t_n * hq} rows have a key that leads"


def run(ctx, kvs, lens, q, held, fp8=False, n_blocks=0, **kw):
    rows = sum(lens)
    out = torch.full((rows, q.shape[-2] * q.shape[-1]), float("nan"), device="cuda", dtype=torch.bfloat16)
    ws = ctx.attend_workspace(rows, len(lens), fp8_visible_tokens=sum(held) if fp8 and not n_blocks else 0, n_blocks=n_blocks)
    if n_blocks:
        ctx.attend_blocks(0, kvs, lens, q.flatten(1), out, ws, n_blocks, **kw)
    else:
        ctx.attend(0, kvs, lens, q.flatten(1), out, ws, **kw)
    return out


@pytest.mark.parametrize("kind", T.KINDS)
@pytest.mark.parametrize("hq, hkv, d", [(4, 2, 64), (28, 4, 128)])
@pytest.mark.parametrize("held, lens", [([1, 2, 5, 64, 900], [1, 1, 2, 1, 1]), ([9000], [1]), ([3000], [2]), ([5000, 40], [9, 3])])
def test_large_queries_and_keys(kind, hq, hkv, d, held, lens):
    """Elements of 1e5: scores of 2^30 to 2^42 powers of two."""
    ctx = T.context(hq, hkv, d)
    g = T.gen(60)
    scales = (256.0, 1.0)
    kvs = T.caches(ctx, kind, held, scales=scales)
    content = [(T.normal(g, n, hkv, d, std=3e4), T.normal(g, n, hkv, d)) for n in held]
    T.fill(kvs, content)
    q = T.normal(g, sum(lens), hq, d, std=1e5)
    out = run(ctx, kvs, lens, q, held, "fp8" in kind)
    at = 0
    for n, t, (k, v) in zip(held, lens, content):
        check_winners(out[at: at + t], T.f64(q[at: at + t]), T.stored(k, kind, scales[0]), T.stored(v, kind, scales[1]), n - t, d ** -0.5)
        at += t


@pytest.mark.parametrize("rows, n_blocks", [(1, 8), (1, 40), (70, 8)])
def test_large_queries_and_keys_over_selected_blocks(rows, n_blocks):
    """In one kernel, in parts, and with a selection of its own; against what the call says it chose."""
    hq, hkv, d = 4, 2, 64
    for n in (3000, 6000):
        ctx = T.context(hq, hkv, d)
        g = T.gen(61)
        kv, = T.caches(ctx, "paged", [n])
        k, v = T.normal(g, n, hkv, d, std=3e4), T.normal(g, n, hkv, d)
        kv.import_(0, k, v)
        kv.new_bounds(n)
        q = T.normal(g, rows, hq, d, std=1e5)
        chosen = torch.empty((rows, hkv, n_blocks), dtype=torch.int32, device="cuda")
        out = run(ctx, [kv], [rows], q, [n], n_blocks=n_blocks, chosen=chosen)
        kd, vd, qd, lists = T.f64(k), T.f64(v), T.f64(q), chosen.cpu().numpy()
        for t in range(rows):
            for h in range(hkv):
                slots = np.concatenate([np.arange(64 * b, min(64 * b + 64, n - rows + t + 1)) for b in lists[t, h] if b >= 0])
                check_winners(out[t].view(hq, d)[2 * h: 2 * h + 2], qd[t: t + 1, 2 * h: 2 * h + 2], kd[slots][:, h: h + 1], vd[slots][:, h: h + 1],
                              len(slots) - 1, d ** -0.5, least=0.0)


def longer_requests(kind, held, rows):
    hq, hkv, d = 4, 2, 64
    ctx = T.context(hq, hkv, d)
    g = T.gen(62)
    scales = (256.0, 1.0)
    kv, = T.caches(ctx, kind, [held], scales=scales)
    k, v = T.normal(g, held, hkv, d, std=3e4), T.normal(g, held, hkv, d)
    kv.import_(0, k, v)
    q = T.normal(g, rows, hq, d, std=1e5)
    out = run(ctx, [kv], [rows], q, [held], "fp8" in kind)
    check_winners(out, T.f64(q), T.stored(k, kind, scales[0]), T.stored(v, kind, scales[1]), held - rows, d ** -0.5)


@pytest.mark.parametrize("kind", ["contiguous", "paged", "fp8"])
@pytest.mark.parametrize("held, rows", [(130, 130), (3000, 70), (1700, 33)])
def test_large_queries_and_keys_in_row_groups(kind, held, rows, monkeypatch):
    monkeypatch.setenv("RS_ATTEND_FEW", "1000000")
    longer_requests(kind, held, rows)


SCALES = [2.0 ** -119, 1e-30, 1e6, 1e30]


def scaled(held, rows, scale):
    """A scale that makes all scores equal gives the plain average; one that sets them far apart gives the best key's value."""
    hq, hkv, d = 4, 2, 64
    ctx = T.context(hq, hkv, d)
    g = T.gen(63)
    kv, = T.caches(ctx, "contiguous", [held])
    k, v = T.normal(g, held, hkv, d), T.normal(g, held, hkv, d)
    kv.import_(0, k, v)
    q = T.normal(g, rows, hq, d)
    out = run(ctx, [kv], [rows], q, [held], scale=scale)
    if scale < 1:
        ref, mag = O.attend(T.f64(q), T.f64(k), T.f64(v), held - rows, scale=float(np.float32(scale)))
        T.assert_attention(out, ref, mag, f"scale {scale}")
    else:
        check_winners(out, T.f64(q), T.f64(k), T.f64(v), held - rows, float(np.float32(scale)))


@pytest.mark.parametrize("held, rows", [(1, 1), (70, 1), (9000, 1), (400, 100), (3000, 70)])
@pytest.mark.parametrize("scale", SCALES)
def test_scales_of_the_callers(held, rows, scale, monkeypatch):
    monkeypatch.setenv("RS_ATTEND_FEW", "1000000")
    scaled(held, rows, scale)
