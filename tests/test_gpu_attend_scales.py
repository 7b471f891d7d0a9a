"""GPU: the smallest scales there are - in 32 bits no longer normal numbers - give the plain average of the values, as 64 bits do."""
import numpy as np
import pytest
import torch

import test_gpu_attend_extremes as E
import test_gpu_cache_operators as T
from oracle import cache_ops as O

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("few", ["0", "1000000"])
@pytest.mark.parametrize("kind", T.KINDS)
@pytest.mark.parametrize("held, rows", [(1, 1), (9000, 1), (400, 100), (3000, 70)])
@pytest.mark.parametrize("scale", [1e-38, 1e-41])
def test_tiny_scales(few, kind, held, rows, scale, monkeypatch):
    monkeypatch.setenv("RS_ATTEND_FEW", few)
    hq, hkv, d = 4, 2, 64
    ctx = T.context(hq, hkv, d)
    g = T.gen(64)
    kv, = T.caches(ctx, kind, [held])
    k, v = T.normal(g, held, hkv, d), T.normal(g, held, hkv, d)
    kv.import_(0, k, v)
    q = T.normal(g, rows, hq, d)
    out = E.run(ctx, [kv], [rows], q, [held], "fp8" in kind, scale=scale)
    ref, mag = O.attend(T.f64(q), T.stored(k, kind, T.K_SCALE), T.stored(v, kind, T.V_SCALE), held - rows, scale=float(np.float32(scale)))
    T.assert_attention(out, ref, mag)
