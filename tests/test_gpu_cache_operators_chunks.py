"""GPU: rs_attend's chunk kernel on calls so small that the rule would not take it (RS_ATTEND_FEW=0), and row groups of the kernel for few rows
on requests that the rule would not give it, against the 64-bit oracle; tolerances as in test_gpu_cache_operators.py."""
import numpy as np
import pytest
import torch

import test_gpu_cache_operators as T
from oracle import cache_ops as O

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["0", "1000000"])
def rule(request, monkeypatch):
    monkeypatch.setenv("RS_ATTEND_FEW", request.param)
    return request.param


@pytest.mark.parametrize("kind", T.KINDS)
@pytest.mark.parametrize("hq, hkv, d", [(4, 2, 64), (28, 4, 128), (24, 1, 128)])
def test_mixed_calls(rule, kind, hq, hkv, d):
    ctx = T.context(hq, hkv, d)
    g = T.gen(50)
    held, lens = [300, 90, 50, 128, 9, 700], [150, 4, 0, 128, 1, 41]
    kvs = T.caches(ctx, kind, held)
    content = [(T.normal(g, n, hkv, d), T.normal(g, n, hkv, d)) for n in held]
    T.fill(kvs, content)
    rows = sum(lens)
    q = T.normal(g, rows, hq * d + 8, std=1.5)[:, : hq * d]
    out = torch.full((rows, hq * d), float("nan"), device="cuda", dtype=torch.bfloat16)
    ctx.attend(0, kvs, lens, q, out, ctx.attend_workspace(rows, len(held), fp8_visible_tokens=sum(held)))
    at = 0
    for n, t, (k, v) in zip(held, lens, content):
        if t:
            ref, mag = O.attend(T.f64(q[at: at + t]).reshape(t, hq, d), T.stored(k, kind, T.K_SCALE), T.stored(v, kind, T.V_SCALE), n - t)
            T.assert_attention(out[at: at + t], ref, mag, f"{n} cached, {t} rows")
        at += t


@pytest.mark.parametrize("kind", ["contiguous", "paged"])
@pytest.mark.parametrize("held, rows", [(400, 200), (3000, 130), (1700, 33)])
def test_what_a_query_does_not_see_does_not_reach_it(rule, kind, held, rows):
    """Infinite and NaN keys and values of the last tokens, on whole and split key ranges, and rows in several groups."""
    hq, hkv, d = 4, 2, 64
    ctx = T.context(hq, hkv, d)
    g = T.gen(51)
    kv, = T.caches(ctx, kind, [held])
    k, v = T.normal(g, held, hkv, d), T.normal(g, held, hkv, d)
    k[-1, 0, 5], v[-1, 1, 7], v[-2, 0, 63], v[-3, 0, 2], v[-3, 1, 2] = float("inf"), float("nan"), float("-inf"), float("inf"), float("nan")
    kv.import_(0, k, v)
    q = T.normal(g, rows, hq * d)
    out = torch.empty_like(q)
    ctx.attend(0, [kv], [rows], q, out, ctx.attend_workspace(rows))
    ref, mag = O.attend(T.f64(q[: rows - 3]).reshape(-1, hq, d), T.f64(k), T.f64(v), held - rows)
    T.assert_attention(out[: rows - 3], ref, mag)
    assert not out[rows - 3:].isfinite().all(1).any()


def test_dropped_tokens_and_large_scores(rule):
    hq, hkv, d = 4, 2, 64
    ctx = T.context(hq, hkv, d)
    g = T.gen(52)
    kv, = T.caches(ctx, "contiguous", [900])
    k, v = T.normal(g, 900, hkv, d, std=20.0), T.normal(g, 900, hkv, d)
    k[::3, :, 0] = float("-inf")
    k[840:], v[840:] = float("nan"), float("inf")
    kv.import_(0, k, v)
    kv.truncate(0, 840)
    q = T.normal(g, 100, hq * d, std=4.0).view(100, hq, d)
    q[:, :, 0] = 1.0
    out = torch.empty((100, hq * d), dtype=torch.bfloat16, device="cuda")
    ctx.attend(0, [kv], [100], q.flatten(1), out, ctx.attend_workspace(100))
    ref, mag = O.attend(T.f64(q), T.f64(k[:840]), T.f64(v[:840]), 740)
    # scores up to 2^10, fp32: their errors, up to 2^-11, are weights' relative errors
    assert (np.abs(T.f64(out).reshape(ref.shape) - ref) - (T.SLACK + 2.0 ** -10) * mag).max() <= 0
