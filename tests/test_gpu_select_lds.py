"""GPU: selection for many tokens on caches so long that a workgroup's LDS holds the scores of three, two or one of its four tokens, at the lengths
around which that changes: the blocks are those that a call of one token chooses.

A workgroup has 128 KB, 32768 scores, and a token's scores take a multiple of four: three tokens fit up to 10920 blocks, two up to 16384.
"""
import pytest
import torch

import test_gpu_cache_operators as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("blocks", [8192, 8193, 10920, 10921, 10922, 10923, 16384, 16385])
def test_lengths_at_which_fewer_tokens_fit(blocks):
    hq, hkv, d, rows = 4, 2, 64, 131   # 262 (token, KV head)s: the kernels for many tokens
    n = 64 * (blocks - 1) + 9          # the last block is not finished
    ctx = T.context(hq, hkv, d, max_pos=64 * 16400, max_requests=1, max_tokens_per_call=256)
    g = T.gen(90)
    kv, = T.caches(ctx, "contiguous", [n])
    k = T.normal(g, n, hkv, d)
    kv.import_(0, k, k)
    kv.new_bounds(n)
    q = T.normal(g, rows, hq * d)
    _, many = T.run_blocks(ctx, [kv], [rows], q, 6, 1, 2)
    for i in (130, 129, 128, 64, 3, 2, 1, 0):   # the cache then ends with the token
        kv.truncate(0, n - (rows - 1 - i))
        _, one = T.run_blocks(ctx, [kv], [1], q[i: i + 1], 6, 1, 2)
        assert (one[0] == many[i]).all(), i
