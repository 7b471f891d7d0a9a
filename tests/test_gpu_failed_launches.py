"""GPU: what calls on caches leave behind when a launch reports an error.  The error is one that a call of somebody else's left, a device that is not
there; the kernels run."""
import pytest
import torch

from tests.test_gpu_cache_operators import context, gen, normal

pytestmark = pytest.mark.gpu


def fails(ctx, call):
    """Runs a call that finds an error behind its first launch."""
    from paper_2509_24381_amd.binding import RsError
    assert ctx.lib.hipSetDevice(1 << 20) != 0
    with pytest.raises(RsError) as e:
        call()
    assert e.value.status_name == "RS_EHIP" and "invalid device" in str(e.value)
    ctx.lib.hipGetLastError()
    torch.cuda.synchronize()


@pytest.mark.parametrize("n", [100, 64 * 700])
@pytest.mark.parametrize("kind", ["contiguous", "paged"])
def test_a_fork_whose_copies_fail_leaves_empty_caches(kind, n):
    """Copied destinations; those that share pages are what the call says.  (700 blocks: their numbers are staged.)"""
    from paper_2509_24381_amd.binding import KVPool
    ctx, g = context(4, 2, 64, max_pos=64 * 800), gen(1)
    pool, other = KVPool(ctx, 1500), KVPool(ctx, 1500)
    src, sharer = pool.new_cache(1), pool.new_cache(1)
    dst = other.new_cache(1) if kind == "paged" else ctx.kv_alloc(1, 64 * 800)
    k, v, old = normal(g, n, 2, 64), normal(g, n, 2, 64), normal(g, 300, 2, 64)
    src.import_(0, k, v)
    dst.import_(0, old, old)
    fails(ctx, lambda: ctx.kv_fork([src, src], [dst, sharer]))
    assert dst.length() == 0 and sharer.length() == src.length() == n
    if kind == "paged":
        assert other.free_pages == 1500
    for _ in range(20):
        ctx.kv_fork([src], [dst])
    for kv in (dst, sharer, src):
        got = kv.export(0)
        assert torch.equal(got[0], k) and torch.equal(got[1], v)


@pytest.mark.parametrize("apart", [False, True], ids=["in one launch", "copies apart"])
def test_an_append_that_fails_leaves_what_nobody_had_to_copy(apart):
    """A cache that continues a shared block in a page of its own ends before that block, others where the call began."""
    from paper_2509_24381_amd.binding import KVPool
    ctx, g = context(4, 2, 64), gen(2)
    pool = KVPool(ctx, 40)
    pool.slab.fill_(0xFF)   # (NaN)
    a, alone, flat = pool.new_cache(1), pool.new_cache(1), ctx.kv_alloc(1, 512)
    k, v = normal(g, 100, 2, 64), normal(g, 100, 2, 64)
    for kv in (a, alone, flat):
        kv.import_(0, k, v)
    b, c = a.fork(), a.fork()
    kvs = [b, c, a, alone, flat]
    starts = [100, 100, 70 if apart else 100, 100, 100]   # (what a drops is what the others copy: the last one left does not copy)
    new, free = normal(g, 5 * 3, 2, 64), pool.free_pages
    fails(ctx, lambda: ctx.kv_append(0, kvs, [3] * 5, None, new, new, None, starts=starts))
    assert [kv.length() for kv in kvs] == [64, 64, starts[2], 100, 100]
    assert pool.free_pages == free   # (the last blocks of b and c are gone, a has its page for itself)
    for i, kv in enumerate(kvs):
        n = kv.length()
        got = kv.export(0)
        assert torch.equal(got[0], k[:n]) and torch.equal(got[1], v[:n]), i
    q = normal(g, 5 * 3, 4 * 64)
    ctx.kv_append(0, kvs, [3] * 5, None, new, new, None)
    out = ctx.attend(0, kvs, [3] * 5, q, torch.empty_like(q), ctx.attend_workspace(15, 5))
    fresh = [ctx.kv_alloc(1, 512) for _ in kvs]
    for kv, other, i in zip(kvs, fresh, range(5)):
        n = kv.length() - 3
        other.import_(0, torch.cat((k[:n], new[3 * i: 3 * i + 3])), torch.cat((v[:n], new[3 * i: 3 * i + 3])))
    assert torch.equal(out, ctx.attend(0, fresh, [3] * 5, q, torch.empty_like(q), ctx.attend_workspace(15, 5)))


@pytest.mark.parametrize("kind", ["paged", "paged_fp8"])
def test_a_prefill_that_cannot_copy_a_shared_block_changes_nothing(kind):
    from tests.test_gpu_decode import rows, setup
    from paper_2509_24381_amd import runner
    dec, kvs, _, rng, stack = setup(kind)
    fork = kvs[0].fork()
    x = runner.to_device_bf16(rows(rng, 5, stack.shape.hidden))
    held, shared, free = fork.length(), [fork.shared_pages(layer) for layer in range(2)], fork.pool.free_pages
    assert held % 64 and min(shared) == (held + 63) // 64
    fails(stack.ctx, lambda: stack.prefill_prompt(x, [(0, 5)], fork))
    assert fork.length() == held and [fork.shared_pages(layer) for layer in range(2)] == shared and fork.pool.free_pages == free
    y = stack.prefill_prompt(x, [(0, 5)], fork)
    assert torch.equal(y, stack.prefill_prompt(x, [(0, 5)], kvs[0]))
    assert [fork.shared_pages(layer) for layer in range(2)] == [s - 1 for s in shared]


@pytest.mark.parametrize("kind", ["contiguous", "paged", "paged_fp8"])
@pytest.mark.parametrize("n", [20, 500])
def test_an_import_that_fails_leaves_an_empty_cache(kind, n):
    """Its pages are others than those that hold the tokens it had, or fewer."""
    from paper_2509_24381_amd.binding import KVPool
    ctx, g = context(4, 2, 64), gen(3)
    pool = KVPool(ctx, 40, fp8=kind == "paged_fp8")
    kv = ctx.kv_alloc(1, 512) if kind == "contiguous" else pool.new_cache(1)
    old, new = normal(g, 300, 2, 64), normal(g, n, 2, 64)
    kv.import_(0, old, old)
    sharer = None if kind == "contiguous" else kv.fork()
    fails(ctx, lambda: kv.import_(0, new, new))
    assert kv.length() == 0 and kv.bounded(0) == 0
    kv.import_(0, new, new)
    fresh = ctx.kv_alloc_fp8(1, 512) if kind == "paged_fp8" else ctx.kv_alloc(1, 512)
    for cache, x in ((kv, new), (sharer, old)):
        if cache is None:
            continue
        fresh.import_(0, x, x)
        assert all(torch.equal(*two) for two in zip(cache.export(0), fresh.export(0)))


@pytest.mark.parametrize("blocks", [0, 8])
def test_page_numbers_of_a_call_that_fails_stay_until_they_are_read(blocks):
    """The calls behind it stage theirs elsewhere: the kernel of a call that reports an error reads its own."""
    from paper_2509_24381_amd.binding import KVPool, RsError
    ctx, g = context(4, 2, 64), gen(4)
    pool = KVPool(ctx, 4 * 600)
    kvs = [pool.new_cache(1) for _ in range(4)]
    for kv in kvs:
        k, v = normal(g, 38000, 2, 64), normal(g, 38000, 2, 64)
        kv.import_(0, k, v)
        if blocks:
            kv.new_bounds(38400)
    q = normal(g, 2, 4 * 64)

    def attend(pair, out):
        ws = ctx.attend_workspace(2, 2, n_blocks=blocks)
        return lambda: ctx.attend_blocks(0, pair, [1, 1], q, out, ws, blocks) if blocks else ctx.attend(0, pair, [1, 1], q, out, ws)

    out = [torch.zeros_like(q) for _ in range(20)]
    calls = [attend(kvs[i % 2 * 2: i % 2 * 2 + 2], o) for i, o in enumerate(out)]
    want = []
    for call, o in zip(calls[:2], out):
        call()
        want.append(o.clone())
    torch.cuda.synchronize()
    for _ in range(5):
        for i, call in enumerate(calls):
            out[i].zero_()
            if i % 3 == 0:
                assert ctx.lib.hipSetDevice(1 << 20) != 0
                with pytest.raises(RsError, match="invalid device"):
                    call()
                ctx.lib.hipGetLastError()
            else:
                call()
        torch.cuda.synchronize()
        assert all(torch.equal(o, want[i % 2]) for i, o in enumerate(out) if i % 3 or not blocks)   # (blocks: a launch that follows is left out)
