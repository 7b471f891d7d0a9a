"""GPU: bounds of blocks whose features differ by many powers of two, against the 64-bit oracle (equal), and as bounds: on either side of
zero no code is nearer to zero than the keys are."""
import numpy as np
import pytest
import torch

import test_gpu_cache_operators as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["contiguous", "paged"])
@pytest.mark.parametrize("large, small", [(1e30, 1e-30), (1.0, 1e-38), (1e29, 2.0 ** -133), (3e38, 1e-20)])
def test_small_features_beside_large_ones(kind, large, small):
    """Maxima and minima that are far below the block's unit: the code is 1 or -1, not 0."""
    hkv, d = 2, 64
    ctx = T.context(hkv, hkv, d)
    g = T.gen(70)
    kv, = T.caches(ctx, kind, [256])
    k = T.normal(g, 256, hkv, d)
    k[:, :, 3] *= large
    k[:, :, 7:20] *= small
    k[:, :, 8] = k[:, :, 8].abs()            # above zero only
    k[:, :, 9] = -k[:, :, 9].abs()           # below zero only
    k[64:128, 0, 10], k[64:128, 1, 11] = 0.0, small
    kv.import_(0, k, torch.zeros_like(k))
    codes, units = kv.new_bounds(256)
    ctx.bounds_update(0, [kv])
    x = T.f64(k)
    want_codes, want_units = T.bounds_of(x)
    got_codes, got_units = codes[0].cpu().numpy().astype(np.int64), T.f64(units[0])
    assert np.array_equal(got_units.T, want_units)
    assert np.array_equal(got_codes.transpose(1, 0, 2, 3), want_codes)
    limited = np.clip(x, -T.O.LIMIT, T.O.LIMIT).reshape(4, 64, hkv, d)
    high, low = (got_codes[:, :, i].transpose(1, 0, 2) * got_units.T[..., None] for i in (0, 1))
    assert (limited <= high[:, None]).all() and (limited >= low[:, None]).all()


def test_scores_follow_such_bounds():
    """A query that only such small features tell blocks apart for: the selection is the oracle's."""
    hkv, d, n = 2, 64, 64 * 12
    ctx = T.context(4, hkv, d)
    g = T.gen(71)
    kv, = T.caches(ctx, "contiguous", [n])
    k = T.normal(g, n, hkv, d) * 1e-35
    k[:, :, 3] = 1e30
    k[: 64 * 5, :, 20:] = -k[: 64 * 5, :, 20:].abs()
    v = T.normal(g, n, hkv, d)
    kv.import_(0, k, v)
    kv.new_bounds(n)
    q = T.normal(g, 3, 4 * d).view(3, 4, d).abs()
    q[:, :, 3] = 0.0
    out, chosen = T.run_blocks(ctx, [kv], [3], q.flatten(1), 4, 0, 1)
    codes, units = T.bounds_of(T.f64(k))
    for i in range(3):
        for h in range(hkv):
            bounds = [(codes[b, h, 0], codes[b, h, 1], units[b, h]) for b in range(12)]
            assert chosen[i, h].tolist() == T.O.select_blocks(T.f64(q)[i, 2 * h: 2 * h + 2], bounds, n - 3 + i, 4, 0, 1)
