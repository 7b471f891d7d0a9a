"""CPU: the C ABI of include/rserve_attend.h - symbols, rotary tables against the oracle, every refusal - on host-only contexts.

Calls that pass all checks end in RS_EHIP here, before anything is launched or changed; device pointers are stand-ins.
"""
import ctypes as C
import os
import re
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import cache_ops as O
from paper_2509_24381_amd import binding
from paper_2509_24381_amd.binding import CacheSet, Context, KVCache, LayerConfig, RotaryConfig, RsError

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HQ, HKV, D = 4, 2, 64

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="stand-in device pointers: for hosts without a GPU")


@pytest.fixture(scope="module")
def ctx():
    if not os.path.exists(binding.library_path()):
        from paper_2509_24381_amd.build import build
        build(verbose=False)
    return Context(LayerConfig(hidden=256, n_q_heads=HQ, n_kv_heads=HKV, head_dim=D, mlp_inter=64, max_tokens_per_call=128, max_requests=4, max_pos=512))


def make(ctx, capacity=256, fp8=False, n_layers=1, at=0x7F0000000000):
    h = C.c_void_p()
    if fp8:
        binding._check(ctx.lib.rs_kv_alloc_fp8(ctx.handle, n_layers, capacity, 1.0, 1.0, at, 1 << 30, C.byref(h)))
    else:
        binding._check(ctx.lib.rs_kv_alloc(ctx.handle, n_layers, capacity, at, 1 << 30, C.byref(h)))
    return KVCache(ctx, h.value, None)


def rows(n, heads, extra=0):
    return torch.zeros((n, heads * D + extra), dtype=torch.bfloat16)


def refused(status, call, *words):
    with pytest.raises(RsError) as e:
        call()
    assert e.value.status_name == status, str(e.value)
    assert all(w in str(e.value) for w in words), str(e.value)


def test_header_symbols_are_exported(ctx):
    header = open(os.path.join(ROOT, "include", "rserve_attend.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(rs_[a-z_0-9]+)\s*\(", header))
    assert declared == set(binding.ATTEND_SYMBOLS)
    assert all(hasattr(ctx.lib, name) for name in declared)


@pytest.mark.parametrize("form", [
    dict(rotary_dim=64, theta=1e6), dict(rotary_dim=32, theta=1e4, layout="interleaved"), dict(rotary_dim=64, theta=1e4, scaling="linear", factor=2.5),
    dict(rotary_dim=64, theta=1e6, scaling="ramp", factor=4.0, original_max_pos=4096),
    dict(rotary_dim=48, theta=5e5, scaling="ramp", factor=16.0, original_max_pos=1024, fast_turns=16.0, slow_turns=2.0, magnitude=1.5),
    dict(rotary_dim=64, theta=5e5, scaling="bands", factor=8.0, original_max_pos=8192),
    dict(rotary_dim=16, theta=1e4, scaling="bands", factor=3.0, original_max_pos=300, fast_turns=10.0, slow_turns=0.5),
])
def test_rotary_tables(ctx, form):
    """Every pair at positions up to the table's end, within fp32's rounding of the cosine (2^-24 of the magnitude) and of the angle's own
    64-bit error (position 2^-52 times a few)."""
    cfg = RotaryConfig(max_pos=30000, **form)
    rotary = ctx.rotary(cfg)
    f = O.rotary_frequencies(cfg.rotary_dim, cfg.theta, cfg.scaling, cfg.factor, cfg.original_max_pos, cfg.fast_turns, cfg.slow_turns)
    m = O.rotary_magnitude(cfg.scaling, cfg.factor, cfg.magnitude)
    for pos in (0, 1, 2, 77, 4095, 4096, 29999):
        for j in range(cfg.rotary_dim // 2):
            c, s = rotary.at(pos, j)
            assert abs(c - m * np.cos(pos * f[j])) <= m * 2.0 ** -23 and abs(s - m * np.sin(pos * f[j])) <= m * 2.0 ** -23
    refused("RS_EINVAL", lambda: rotary.at(30000, 0))
    refused("RS_EINVAL", lambda: rotary.at(0, cfg.rotary_dim // 2))


def test_scaled_frequencies_have_the_limits_they_are_defined_by():
    """The forms' meaning, apart from their formulas: the fastest pairs are left as they are, the slowest divided by the factor."""
    plain = O.rotary_frequencies(64, 1e6)
    for scaling in ("ramp", "bands"):
        f = O.rotary_frequencies(64, 1e6, scaling, 8.0, 4096)
        turns = 4096 * plain / (2 * np.pi)
        # (the ramp runs between whole pairs, so a pair's distance from its ends is kept clear of)
        fast, slow = turns > 32 * 1.6, turns < 1 / 1.6
        assert fast.sum() > 3 and slow.sum() > 3
        assert np.allclose(f[fast], plain[fast]) and np.allclose(f[slow], plain[slow] / 8)
        assert (f <= plain * (1 + 1e-12)).all() and (f >= plain / 8 * (1 - 1e-12)).all()


@pytest.mark.parametrize("bad", [
    dict(rotary_dim=0), dict(rotary_dim=24), dict(rotary_dim=80), dict(max_pos=0), dict(theta=1.0), dict(theta=float("inf")), dict(magnitude=-1.0),
    dict(scaling="linear", factor=0.5), dict(scaling="ramp", factor=2.0), dict(scaling="bands", factor=2.0, original_max_pos=100, fast_turns=1.0, slow_turns=2.0),
    dict(scaling="ramp", factor=float("nan"), original_max_pos=100),
    dict(layout="thirds"), dict(scaling="cubic"),
])
def test_rotary_refusals(ctx, bad):
    refused("RS_EINVAL", lambda: ctx.rotary(RotaryConfig(**{**dict(rotary_dim=64, theta=1e4, max_pos=100), **bad})))


def append(ctx, kvs, lens, n=None, **kw):
    n = sum(lens) if n is None else n
    a = dict(q=rows(n, HQ), k=rows(n, HKV), v=rows(n, HKV), q_out=rows(n, HQ))
    a.update({k: kw.pop(k) for k in list(kw) if k in a})
    ctx.kv_append(kw.pop("layer", 0), kvs, lens, a["q"], a["k"], a["v"], a["q_out"], **kw)


def test_append_refusals(ctx):
    kv, other = make(ctx), make(ctx, 64, n_layers=2)
    rot = ctx.rotary(RotaryConfig(rotary_dim=64, theta=1e4, max_pos=100))
    foreign = make(Context(ctx.cfg))
    refused("RS_EHIP", lambda: append(ctx, [kv], [5]))
    refused("RS_EINVAL", lambda: append(ctx, [kv], [-1], n=0), "add up")
    refused("RS_EINVAL", lambda: append(ctx, [kv, other], [-1, 1], n=0), "negative")
    refused("RS_EINVAL", lambda: append(ctx, [kv] * 2, [1, 1]), "twice")
    refused("RS_EINVAL", lambda: append(ctx, [kv], [1], layer=1), "layer")
    refused("RS_EINVAL", lambda: append(ctx, [make(ctx) for _ in range(5)], [1] * 5), "max_requests")
    refused("RS_EINVAL", lambda: append(ctx, [kv], [129]), "max_tokens_per_call")
    refused("RS_ESTATE", lambda: append(ctx, [foreign], [1]), "context")
    refused("RS_EINVAL", lambda: append(ctx, [kv, make(ctx, fp8=True)], [1, 1]), "8-bit")
    refused("RS_ECAPACITY", lambda: append(ctx, [other], [65]), "capacity")
    refused("RS_EINVAL", lambda: append(ctx, [kv], [1], starts=[1]), "starts")
    refused("RS_EINVAL", lambda: append(ctx, [kv], [1], starts=[-1]), "starts")
    refused("RS_ECAPACITY", lambda: append(ctx, [kv], [101], rotary=rot), "rotary")
    refused("RS_ECAPACITY", lambda: append(ctx, [kv], [2], rotary=rot, positions=[3, 100]), "position 100 of row 1")
    refused("RS_ECAPACITY", lambda: append(ctx, [kv], [2], rotary=rot, positions=[-1, 3]))
    refused("RS_EINVAL", lambda: append(ctx, [kv], [2], rotary=rot, positions=[1]), "positions")
    refused("RS_ESTATE", lambda: append(ctx, [kv], [1], rotary=Context(ctx.cfg).rotary(rot.cfg)), "rotary")
    refused("RS_EINVAL", lambda: append(ctx, [kv], [1], q=None), "neither")
    refused("RS_EINVAL", lambda: append(ctx, [kv], [2], k=rows(2, HKV, 4)[:, : HKV * D]), "multiple of 8")
    refused("RS_EINVAL", lambda: append(ctx, [kv], [2], v=rows(2, HKV, 8)[:, 4: 4 + HKV * D]), "aligned")
    refused("RS_EINVAL", lambda: append(ctx, [kv], [2], k=rows(3, HKV)), "lens")
    refused("RS_EINVAL", lambda: append(ctx, [kv], [2], v=rows(2, HKV).float()), "bfloat16")
    refused("RS_EINVAL", lambda: append(ctx, [kv], [2], v=rows(2, 2 * HKV)[:, ::2]), "contiguous")
    assert kv.length(0) == 0 and other.length(1) == 0
    append(ctx, [kv], [0])   # nothing to do


def test_paged_append_refusals_and_bookkeeping(ctx):
    pool = C.c_void_p()
    page = ctx.lib.rs_kv_page_bytes(ctx.handle)
    binding._check(ctx.lib.rs_kv_pool_create(ctx.handle, 0x7F0000000000, 2 * page, C.byref(pool)))
    kvs = []
    for _ in range(2):
        h = C.c_void_p()
        binding._check(ctx.lib.rs_kv_alloc_paged(ctx.handle, pool, 1, C.byref(h)))
        kvs.append(KVCache(ctx, h.value, None))
    refused("RS_ECAPACITY", lambda: append(ctx, kvs, [65, 63]), "3 new KV pages", "2 free")
    refused("RS_EHIP", lambda: append(ctx, kvs, [64, 64]))
    assert ctx.lib.rs_kv_pool_free_pages(pool) == 2 and kvs[0].length(0) == 0
    for kv in kvs:
        ctx.lib.rs_kv_free(kv.handle)
        kv.handle = None
    assert ctx.lib.rs_kv_pool_destroy(pool) == 0


def workspace(ctx, n_rows, requests=1, fp8=0, n_blocks=0):
    n = ctx.lib.rs_attend_workspace_bytes(ctx.handle, n_rows, requests, fp8, n_blocks)
    t = torch.empty(n + 512, dtype=torch.uint8)
    at = (256 - t.data_ptr() % 256) % 256
    return t[at: at + n]


def test_attend_refusals(ctx):
    kv = make(ctx)
    ctx.lib.rs_kv_truncate(kv.handle, 0, 0)
    ws = workspace(ctx, 128, 4, n_blocks=4)
    q = rows(1, HQ)
    refused("RS_EINVAL", lambda: ctx.attend(0, [kv], [1], q, q, ws), "exceeds the 0 cached")
    ctx.attend(0, [kv], [0], rows(0, HQ), rows(0, HQ), ws)   # nothing to do
    for scale in (-1.0, float("inf"), float("nan")):
        refused("RS_EINVAL", lambda: ctx.attend(0, [kv], [0], rows(0, HQ), rows(0, HQ), ws, scale=scale), "scale")
    refused("RS_EINVAL", lambda: ctx.attend(1, [kv], [0], rows(0, HQ), rows(0, HQ), ws), "layer")
    refused("RS_EINVAL", lambda: ctx.attend(0, [kv], [1], rows(2, HQ), rows(2, HQ), ws), "lens")
    assert ctx.lib.rs_attend_workspace_bytes(ctx.handle, 0, 1, 0, 0) == 0 and ctx.lib.rs_attend_workspace_bytes(None, 1, 1, 0, 0) == 0
    small, large = (ctx.lib.rs_attend_workspace_bytes(ctx.handle, n, 1, 0, 0) for n in (1, 128))
    assert 0 < small < large
    assert ctx.lib.rs_attend_workspace_bytes(ctx.handle, 128, 1, 1000, 0) >= large + 4 * HKV * D * 1000


def test_bounds_refusals(ctx):
    kv = make(ctx)
    refused("RS_ESTATE", lambda: ctx.bounds_update(0, [kv]), "attach")
    refused("RS_ESTATE", lambda: ctx.attend_blocks(0, [kv], [0], rows(0, HQ), rows(0, HQ), workspace(ctx, 1, n_blocks=4), 4), "attach")
    codes, units = torch.zeros((1, HKV, 3, 2, D), dtype=torch.int8), torch.zeros((1, HKV, 3))
    refused("RS_EINVAL", lambda: kv.attach_bounds(codes[:, :1], units), "contiguous")
    refused("RS_EINVAL", lambda: kv.attach_bounds(codes.float(), units))
    refused("RS_EINVAL", lambda: kv.attach_bounds(codes, units.double()))
    refused("RS_EINVAL", lambda: binding._check(ctx.lib.rs_kv_attach_bounds(kv.handle, codes.data_ptr(), None, 3)), "both")
    refused("RS_EINVAL", lambda: binding._check(ctx.lib.rs_kv_attach_bounds(kv.handle, codes.data_ptr(), units.data_ptr(), 0)), "positive")
    refused("RS_EINVAL", lambda: binding._check(ctx.lib.rs_kv_attach_bounds(kv.handle, codes.data_ptr() + 4, units.data_ptr(), 3)), "aligned")
    kv.attach_bounds(codes, units)
    assert kv.bounded(0) == 0 and kv.bounded(1) == -1
    ctx.bounds_update(0, [kv])   # nothing finished
    refused("RS_EINVAL", lambda: ctx.bounds_update(0, [kv], firsts=[1]), "firsts")
    ws = workspace(ctx, 1, n_blocks=4)
    for args in ((0, 1, 1), (1025, 1, 1), (4, -1, 1), (4, 1, 0)):
        refused("RS_EINVAL", lambda: ctx.attend_blocks(0, [kv], [0], rows(0, HQ), rows(0, HQ), ws, *args), "n_blocks")
    refused("RS_EINVAL", lambda: ctx.attend_blocks(0, [kv], [0], rows(0, HQ), rows(0, HQ), ws, 4, chosen=torch.zeros((1, HKV, 4), dtype=torch.int32)), "chosen")
    ctx.attend_blocks(0, [kv], [0], rows(0, HQ), rows(0, HQ), ws, 4)
    kv.attach_bounds(None, None)
    refused("RS_ESTATE", lambda: ctx.bounds_update(0, [kv]), "attach")


def test_null_arguments_are_refused(ctx):
    lib = ctx.lib
    assert lib.rs_rotary_create(None, None, None) == -1
    assert lib.rs_kv_append(None, None, 0, None, None, None, 0, None, None, 0, None, 0, None, 0, None, 0, None) == -1
    assert lib.rs_kv_append(ctx.handle, None, 0, None, None, None, 1, None, None, 0, None, 0, None, 0, None, 0, None) == -1
    assert lib.rs_attend(None, 0, None, None, 0, None, 0, None, 0, 0.0, None, 0, None) == -1
    assert lib.rs_kv_bounds_update(None, 0, None, None, 0, None) == -1
    assert lib.rs_kv_attach_bounds(None, None, None, 0) == -1 and lib.rs_kv_bounded(None, 0) == -1
    assert lib.rs_attend_blocks(None, 0, None, None, 0, None, 0, None, 0, 1, 0, 1, 0.0, None, None, 0, None) == -1
    lib.rs_rotary_destroy(None)
    one = (C.c_void_p * 1)(None)
    assert lib.rs_kv_bounds_update(ctx.handle, 0, one, None, 1, None) == -1


def test_prepared_arguments_are_taken_as_they_are(ctx):
    """CacheSet and int_array hold what a call would otherwise convert."""
    kv = make(ctx)
    cs, n = CacheSet([kv]), binding.int_array([3])
    refused("RS_EHIP", lambda: append(ctx, cs, n, n=3))
    assert binding.int_array(n) is n and len(cs) == 1


def test_a_call_without_host_memory_is_refused():
    """Address space is limited, in a process of its own: the table does not fit, and the call says so instead of ending the process."""
    code = """
import resource
from paper_2509_24381_amd.binding import Context, LayerConfig, RotaryConfig, RsError
ctx = Context(LayerConfig(hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=64, mlp_inter=64, max_tokens_per_call=128, max_requests=4, max_pos=512))
held = int(open('/proc/self/statm').read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (held + (2 << 30),) * 2)
try:
    ctx.rotary(RotaryConfig(rotary_dim=64, max_pos=1 << 28, theta=1e4))
except RsError as e:
    print(e.status_name, 'memory' in str(e))
print(ctx.rotary(RotaryConfig(rotary_dim=64, max_pos=512, theta=1e4)).at(0, 0))
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]
    assert r.stdout.splitlines() == ["RS_EHIP True", "(1.0, 0.0)"], r.stdout


def test_the_decode_command_needs_a_gpu():
    from paper_2509_24381_amd import decode
    with pytest.raises(SystemExit, match="GPU"):
        decode.main([])
