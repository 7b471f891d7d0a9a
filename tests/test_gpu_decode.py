"""GPU: generation on prefilled caches (decode.Decoder) - the operators run together - against the 64-bit oracle.

Tolerance: two layers whose intermediate results are rounded to bfloat16 as in the library's own, so the bar of the two-layer parity
tests holds: relative Frobenius error 2e-2 per step (8-bit caches: against an oracle whose cache rounds the same way).
"""
import numpy as np
import pytest
import torch

import synth
from oracle import ChunkedPrefill, LayerParams, rel_fro
from oracle.fp8_kv import ChunkedPrefillFp8KV

pytestmark = pytest.mark.gpu
TOL = 2e-2
N_LAYERS = 2


def setup(kind, *, n=150, room=400, n_blocks=0, requests=2, seed=3):
    from paper_2509_24381_amd import runner
    from paper_2509_24381_amd.decode import Decoder
    shape = synth.TINY
    weights = [synth.layer_weights(shape, seed + l, gains="uniform", std=0.06) for l in range(N_LAYERS)]
    stack = runner.LayerStack(shape, weights, max_tokens=256, max_requests=4, max_pos=512, fp8_visible_tokens=requests * 512)
    if kind.startswith("paged"):
        pool = stack.new_pool(requests * N_LAYERS * 8, fp8=kind == "paged_fp8")
        kvs = [pool.new_cache(N_LAYERS, 0.0625, 0.0625) for _ in range(requests)]
    elif kind == "fp8":
        kvs = [stack.new_cache_fp8(room, 0.0625, 0.0625) for _ in range(requests)]
    else:
        kvs = [stack.new_cache(room) for _ in range(requests)]
    dec = Decoder(stack.ctx, weights, max_rows=256, max_requests=4, n_blocks=n_blocks, fp8_visible_tokens=requests * 512)
    rng = np.random.default_rng(seed)
    prompts = [synth.bf16_round(rng.standard_normal((n + 37 * i, shape.hidden), dtype=np.float32)) for i in range(requests)]
    params = [LayerParams.from_arrays(shape, w) for w in weights]
    states = [[ChunkedPrefillFp8KV(p, 0.0625, 0.0625) if "fp8" in kind else ChunkedPrefill(p) for p in params] for _ in range(requests)]
    for kv, x in zip(kvs, prompts):
        stack.prefill_prompt(runner.to_device_bf16(x), [(0, 100), (100, len(x))], kv)
    for st, x in zip(states, prompts):
        follow(st, x[:100])
        follow(st, x[100:])
    return dec, kvs, states, rng, stack


def follow(layers, x):
    for st in layers:
        x = st.prefill_chunk(x)
    return x


def rows(rng, n, hidden):
    return synth.bf16_round(rng.standard_normal((n, hidden), dtype=np.float32))


@pytest.mark.parametrize("kind", ("contiguous", "paged", "fp8", "paged_fp8"))
@pytest.mark.parametrize("n_blocks", (0, 8))
def test_steps_behind_a_prefilled_prompt(kind, n_blocks):
    """Single tokens, drafts, a request that waits, a piece of a prompt; with n_blocks = 8 every block there is is selected."""
    from paper_2509_24381_amd import runner
    dec, kvs, states, rng, _ = setup(kind, n_blocks=n_blocks)
    if n_blocks:
        dec.prepare_blocks(kvs, 512)
    for lens in ((1, 1), (1, 1), (4, 1), (0, 3), (1, 40), (33, 1)):
        x = rows(rng, sum(lens), synth.TINY.hidden)
        got = runner.to_numpy_f32(dec.step(kvs, lens, runner.to_device_bf16(x)))
        want = np.concatenate([follow(st, part) for st, part in zip(states, np.split(x, [lens[0]])) if len(part)])
        err = rel_fro(got, want)
        assert np.all(np.isfinite(got)) and err <= TOL, f"{lens}: {err:.3e}"
    assert [kv.length(0) for kv in kvs] == [st[0].length for st in states]


def test_dropped_drafts_leave_no_trace():
    from paper_2509_24381_amd import runner
    dec, kvs, states, rng, _ = setup("paged")
    held = [kv.length(0) for kv in kvs]
    dec.step(kvs, (70, 9), runner.to_device_bf16(rows(rng, 79, synth.TINY.hidden)))
    dec.keep(kvs, [held[0] + 2, held[1]])
    dec.keep(kvs, held)
    x = rows(rng, 2, synth.TINY.hidden)
    got = runner.to_numpy_f32(dec.step(kvs, (1, 1), runner.to_device_bf16(x)))
    want = np.concatenate([follow(states[0], x[:1]), follow(states[1], x[1:])])
    assert rel_fro(got, want) <= TOL


def test_a_layer_of_the_library_and_a_step_agree():
    """One token through rs_prefill_model_batch and through Decoder.step, on caches with the same content."""
    from paper_2509_24381_amd import runner
    dec, kvs, states, rng, stack = setup("contiguous", requests=1)
    x = runner.to_device_bf16(rows(rng, 1, synth.TINY.hidden))
    a = dec.step(kvs, [1], x)
    dec.keep(kvs, [kvs[0].length(0) - 1])
    b = torch.empty_like(x)
    stack.ctx.prefill_model_batch(stack.layers, kvs, [1], x, b, stack.ws)
    assert rel_fro(runner.to_numpy_f32(a), runner.to_numpy_f32(b)) <= 2 * TOL


def test_drafted_tokens_are_those_generated_one_at_a_time():
    """A vocabulary in which every token has one successor, far ahead of the others: right, wrong and partly right drafts all end in the
    same tokens, with fewer steps, and in the same cache lengths."""
    from paper_2509_24381_amd import runner
    dec, kvs, states, rng, stack = setup("paged", requests=2, n=100)
    hidden, vocab = synth.TINY.hidden, 32
    emb = runner.to_device_bf16(64.0 * rng.standard_normal((vocab, hidden)).astype(np.float32))
    successor = rng.permutation(vocab)
    w_lm = torch.empty_like(emb)
    w_lm[torch.from_numpy(successor).cuda()] = emb / 64
    gain = torch.ones(hidden, dtype=torch.bfloat16, device="cuda")
    one = runner.to_device_bf16(rows(rng, 1, hidden))
    first = dec.step(kvs, (1, 1), torch.cat([one, one]))
    held = [kv.length(0) for kv in kvs]
    alone = dec.greedy(kvs, first, emb, gain, w_lm, 12)[0].tolist()
    assert all(alone[i + 1] == successor[alone[i]] for i in range(11))
    dec.keep(kvs, held)
    for draft, most in ((lambda t: [successor[t[-1]], successor[successor[t[-1]]], 0], 6), (lambda t: [(successor[t[-1]] + 1) % vocab], 11), (lambda t: [], 11)):
        tokens, steps = dec.greedy_drafted(kvs[0], first[:1], emb, gain, w_lm, 12, draft)
        assert tokens == alone and steps <= most
        assert held[0] + 11 <= kvs[0].length(0) <= held[0] + 14
        dec.keep(kvs[:1], held[:1])
