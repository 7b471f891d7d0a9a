"""GPU: longer requests on 8-bit caches read what shorter ones read, code * scale, without a rounding of their own, with scales that are
no powers of two: against the 64-bit oracle, and where such a rounding would show."""
import numpy as np
import pytest
import torch

import test_gpu_cache_operators as T
from oracle import cache_ops as O
from oracle.fp8_kv import e4m3_decode, e4m3_encode

pytestmark = pytest.mark.gpu
SCALES = (0.0473, 0.0311)


@pytest.fixture(params=["0", "1000000"])
def rule(request, monkeypatch):
    monkeypatch.setenv("RS_ATTEND_FEW", request.param)
    return request.param


@pytest.mark.parametrize("kind", ["fp8", "paged_fp8"])
@pytest.mark.parametrize("hq, hkv, d", [(4, 2, 64), (28, 4, 128)])
@pytest.mark.parametrize("held, lens", [([200], [200]), ([1500, 70, 300], [60, 1, 140]), ([5000], [40])])
def test_scales_that_are_no_powers_of_two(rule, kind, hq, hkv, d, held, lens):
    ctx = T.context(hq, hkv, d)
    g = T.gen(80)
    kvs = T.caches(ctx, kind, held, scales=SCALES)
    T.fill(kvs, [(T.normal(g, n, hkv, d), T.normal(g, n, hkv, d)) for n in held])
    rows = sum(lens)
    q = T.normal(g, rows, hq * d, std=2.0)
    out = torch.full_like(q, float("nan"))
    ctx.attend(0, kvs, lens, q, out, ctx.attend_workspace(rows, len(held), fp8_visible_tokens=sum(held)))
    scales = [float(np.float32(s)) for s in SCALES]
    at = 0
    for kv, n, t in zip(kvs, held, lens):
        k, v = (e4m3_decode(c.cpu().numpy()) * s for c, s in zip(kv.export_codes(0), scales))
        qd = T.f64(q[at: at + t]).reshape(t, hq, d)
        for i in np.unique(np.linspace(0, t - 1, 30).astype(int)):
            ref, mag = O.attend(qd[i: i + 1], k, v, n - t + i)
            T.assert_attention(out[at + i], ref, mag, f"{n} cached, row {i}")
        at += t


@pytest.mark.parametrize("kind", ["fp8", "paged_fp8"])
@pytest.mark.parametrize("held, rows", [(200, 200), (1500, 60), (9000, 33)])
def test_keys_of_equal_scores_weigh_the_same(rule, kind, held, rows):
    """Two kinds of keys, 1 and 9/8 times the scale in one feature each, that a query with 9/8 and 1 there scores alike, some 2^9 high: every
    visible key weighs the same, so an output is the mean of values of +-1.  (The scale and 9/8 of it differ in how they round to
    bfloat16, by 2^-9.6 of themselves.)  The products are exact, and so are their scores' differences: the weights' and the output's roundings
    are left, 2^-8 each, and a part's weights' sum."""
    hq, hkv, d = 4, 2, 64
    ctx = T.context(hq, hkv, d)
    kv, = T.caches(ctx, kind, [held], scales=(SCALES[0], 1.0))
    rng = np.random.default_rng(81)
    first = rng.random((held, hkv)) < 0.5
    k, v = np.zeros((held, hkv, d)), np.zeros((held, hkv, d))
    k[..., 0], k[..., 1] = first, 1.125 * ~first
    v[:] = np.where(first, 1.0, -1.0)[..., None]
    kv.import_codes(0, *(torch.from_numpy(e4m3_encode(x).astype(np.uint8)).cuda() for x in (k, v)))
    q = torch.zeros((rows, hq, d), dtype=torch.bfloat16, device="cuda")
    q[..., 0], q[..., 1] = 1.125 * 2.0 ** 16, 2.0 ** 16
    out = torch.empty((rows, hq * d), dtype=torch.bfloat16, device="cuda")
    ctx.attend(0, [kv], [rows], q.flatten(1), out, ctx.attend_workspace(rows, fp8_visible_tokens=held))
    mean = v[..., 0].cumsum(0) / np.arange(1, held + 1)[:, None]
    got = T.f64(out).reshape(rows, hkv, hq // hkv, d)
    assert np.abs(got - mean[held - rows:, :, None, None]).max() <= T.SLACK
