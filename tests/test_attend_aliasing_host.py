"""CPU: attention into its own queries is refused where rows of one would lie on other rows of the other."""
import pytest
import torch

import test_cache_operators_host as H

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="stand-in device pointers: for hosts without a GPU")
ctx = H.ctx


@pytest.mark.parametrize("blocks", [False, True])
def test_out_that_is_q_with_another_distance(ctx, blocks):
    kvs = [H.make(ctx), H.make(ctx)]
    for kv in kvs:
        kv.attach_bounds(torch.zeros((1, H.HKV, 4, 2, H.D), dtype=torch.int8), torch.zeros((1, H.HKV, 4)))
    memory = H.rows(4, H.HQ, 64)
    wide, narrow = memory[:3, : H.HQ * H.D], memory.flatten()[: 3 * H.HQ * H.D].view(3, H.HQ * H.D)
    assert wide.data_ptr() == narrow.data_ptr()

    def call(lens, q, out):
        if blocks:
            ctx.attend_blocks(0, kvs, lens, q, out, H.workspace(ctx, 4, 2, n_blocks=4), 4)
        else:
            ctx.attend(0, kvs, lens, q, out, H.workspace(ctx, 4, 2))

    for q, out in ((wide, narrow), (narrow, wide)):
        H.refused("RS_EINVAL", lambda: call([2, 1], q, out), "out is q")
    for q in (wide, narrow):   # (these go on to the next check: nothing is cached here)
        H.refused("RS_EINVAL", lambda: call([2, 1], q, q), "exceeds the 0 cached")
    H.refused("RS_EINVAL", lambda: call([1, 0], wide[:1], narrow[:1]), "exceeds the 0 cached")   # one row has no distance
