"""CPU: scales that the kernels could not multiply by are refused, whatever the caches; every other positive one is taken."""
import pytest
import torch

import test_cache_operators_host as H

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="stand-in device pointers: for hosts without a GPU")
ctx = H.ctx


def make(ctx, k_scale):
    import ctypes as C
    h = C.c_void_p()
    H.binding._check(ctx.lib.rs_kv_alloc_fp8(ctx.handle, 1, 256, k_scale, 1.0, 0x7F0000000000, 1 << 30, C.byref(h)))
    return H.KVCache(ctx, h.value, None)


def call(ctx, kv, scale):
    ctx.attend(0, [kv], [0], H.rows(0, H.HQ), H.rows(0, H.HQ), H.workspace(ctx, 1), scale=scale)


def test_scales_beyond_32_bits_are_refused(ctx):
    """scale log2 e, times the keys' scale, overflows or vanishes."""
    H.refused("RS_EINVAL", lambda: call(ctx, H.make(ctx), 3e38), "scale")
    call(ctx, H.make(ctx), 2e38)
    call(ctx, H.make(ctx), 1e-44)
    H.refused("RS_EINVAL", lambda: call(ctx, make(ctx, 2.0 ** -100), 2.0 ** -60), "scale")
    H.refused("RS_EINVAL", lambda: call(ctx, make(ctx, 2.0 ** 100), 2.0 ** 40), "scale")
    call(ctx, make(ctx, 2.0 ** -100), 2.0 ** -20)
    call(ctx, make(ctx, 2.0 ** 100), 2.0 ** 20)
    kv = make(ctx, 2.0 ** -100)
    kv.attach_bounds(torch.zeros((1, H.HKV, 4, 2, H.D), dtype=torch.int8), torch.zeros((1, H.HKV, 4)))
    H.refused("RS_EINVAL", lambda: ctx.attend_blocks(0, [kv], [0], H.rows(0, H.HQ), H.rows(0, H.HQ), H.workspace(ctx, 1, n_blocks=4), 4, scale=2.0 ** -60), "scale")
