"""GPU: decode.Decoder behind prompts whose rotary positions are not their cache slots (three-axis positions: an image's tokens share theirs),
against the 64-bit oracle's unchunked layers; and that it does not guess positions.  Tolerances as in test_gpu_decode.py."""
import numpy as np
import pytest
import torch

import synth
from oracle import LayerParams, layer_forward, rel_fro

pytestmark = pytest.mark.gpu
TOL = 2e-2
SECTIONS = (8, 12, 12)
N_LAYERS = 2


def prompt(n_before, grid_h, grid_w, n_after):
    """(kinds of rows, positions [n, 3], the next token's position): text, an image, text."""
    pos = [(i, i, i) for i in range(n_before)]
    pos += [(n_before, n_before + i // grid_w, n_before + i % grid_w) for i in range(grid_h * grid_w)]
    after = n_before + max(grid_h, grid_w)
    pos += [(after + i,) * 3 for i in range(n_after)]
    return [("text", n_before), ("image", grid_h * grid_w), ("text", n_after)], np.asarray(pos, dtype=np.int64), after + n_after


def build(n_blocks=0, sections=SECTIONS, paged=False):
    from paper_2509_24381_amd import runner
    from paper_2509_24381_amd.decode import Decoder
    shape = synth.TINY
    weights = [synth.layer_weights(shape, 40 + l, gains="uniform", std=0.06) for l in range(N_LAYERS)]
    stack = runner.LayerStack(shape, weights, max_tokens=256, max_requests=4, max_pos=512)
    if sections:
        stack.ctx.set_mrope_sections(*sections)
    dec = Decoder(stack.ctx, weights, max_rows=64, max_requests=4, n_blocks=n_blocks)
    pool = stack.new_pool(64) if paged else None
    kvs = [pool.new_cache(N_LAYERS) if paged else stack.new_cache(400) for _ in range(2)]
    if n_blocks:
        dec.prepare_blocks(kvs, 512)
    return stack, weights, dec, kvs


def prefill(stack, kvs, prompts):
    from paper_2509_24381_amd import runner
    x = runner.to_device_bf16(np.concatenate([p[0] for p in prompts]))
    y = torch.empty_like(x)
    stack.ctx.prefill_model_batch_mrope(stack.layers, kvs, [len(p[0]) for p in prompts], np.concatenate([p[1] for p in prompts]), x, y, stack.ws)
    return y


def rows(rng, n):
    return synth.bf16_round(rng.standard_normal((n, synth.TINY.hidden), dtype=np.float32))


@pytest.mark.parametrize("n_blocks, paged", [(0, False), (8, True)])
def test_steps_behind_a_prompt_with_an_image(n_blocks, paged):
    from paper_2509_24381_amd import runner
    stack, weights, dec, kvs = build(n_blocks, paged=paged)
    rng = np.random.default_rng(5)
    prompts = []
    for i, spec in enumerate([(20, 9, 7, 15), (3, 4, 11, 2)]):
        kinds, pos, nxt = prompt(*spec)
        prompts.append((synth.prompt_rows(kinds, synth.TINY.hidden, 50 + i), pos, nxt))
    prefill(stack, kvs, prompts)
    xs, pos, nxt = [p[0] for p in prompts], [p[1] for p in prompts], [p[2] for p in prompts]
    for lens in ((1, 1), (3, 1), (0, 2)):
        new = [rows(rng, n) for n in lens]
        at = [nxt[i] + t for i, n in enumerate(lens) for t in range(n)]
        got = runner.to_numpy_f32(dec.step(kvs, lens, runner.to_device_bf16(np.concatenate(new)), positions=at))
        want = []
        for i, n in enumerate(lens):
            xs[i] = np.concatenate([xs[i], new[i]])
            pos[i] = np.concatenate([pos[i], np.repeat(nxt[i] + np.arange(n), 3).reshape(n, 3)])
            nxt[i] += n
            y = xs[i]
            for w in weights:
                y, k, _ = layer_forward(y, LayerParams.from_arrays(synth.TINY, w), positions3=pos[i], sections=SECTIONS)
            want.append(y[len(y) - n:])
            if n:
                last, _ = kvs[i].export(N_LAYERS - 1)
                assert rel_fro(runner.to_numpy_f32(last), k) <= TOL
        err = rel_fro(got, np.concatenate(want))
        assert np.all(np.isfinite(got)) and err <= TOL, f"{lens}: {err:.3e}"
    # (the slots would have been other angles: the keys of a token there are not the keys that it has)
    slots = pos[0].copy()
    slots[-1] = len(slots) - 1
    _, there, _ = layer_forward(xs[0], LayerParams.from_arrays(synth.TINY, weights[0]), positions3=slots, sections=SECTIONS)
    first, _ = kvs[0].export(0)
    assert rel_fro(runner.to_numpy_f32(first)[-1:], there[-1:]) > 0.05


def test_positions_are_not_guessed():
    """Behind three-axis positions that are not the slots a step without positions is refused, and changes nothing; one with them goes on.
    Requests that wait do not matter; a cache that starts anew is free again."""
    from paper_2509_24381_amd import runner
    from paper_2509_24381_amd.binding import RsError
    stack, weights, dec, kvs = build()
    rng = np.random.default_rng(6)
    kinds, pos, nxt = prompt(5, 6, 6, 4)
    x = synth.prompt_rows(kinds, synth.TINY.hidden, 60)
    prefill(stack, kvs[:1], [(x, pos)])
    text = rows(rng, 30)
    stack.prefill_prompt(runner.to_device_bf16(text), [(0, 30)], kvs[1])
    one = runner.to_device_bf16(rows(rng, 2))
    for lens, n in (((1, 1), 2), ((1, 0), 1)):
        with pytest.raises(RsError, match="positions"):
            dec.step(kvs, lens, one[:n])
    assert [kv.length(l) for kv in kvs for l in range(N_LAYERS)] == [len(x)] * N_LAYERS + [30] * N_LAYERS
    dec.step(kvs, (0, 1), one[:1])
    dec.step(kvs, (1, 1), one, positions=[nxt, 31])
    with pytest.raises(RsError, match="positions"):
        dec.step(kvs, (1, 0), one[:1])
    emb = runner.to_device_bf16(rows(rng, 16))
    gain = torch.ones(synth.TINY.hidden, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(RsError, match="positions"):
        dec.greedy(kvs[:1], one[:1], emb, gain, emb, 2)
    with pytest.raises(RsError, match="position"):
        dec.greedy_drafted(kvs[0], one[:1], emb, gain, emb, 3, lambda t: [])
    kvs[0].reset()
    stack.prefill_prompt(runner.to_device_bf16(text), [(0, 30)], kvs[0])
    dec.step(kvs, (1, 0), one[:1])


def test_three_axis_positions_that_are_the_slots_need_no_others():
    """A text prompt through the three-axis call; and the same bits with the slots given as positions."""
    from paper_2509_24381_amd import runner
    stack, weights, dec, kvs = build()
    rng = np.random.default_rng(7)
    x = rows(rng, 40)
    for kv in kvs:
        prefill(stack, [kv], [(x, np.repeat(np.arange(40), 3).reshape(40, 3))])
    one = runner.to_device_bf16(rows(rng, 3))
    a = dec.step(kvs[:1], [3], one)
    b = dec.step(kvs[1:], [3], one, positions=[40, 41, 42])
    assert torch.equal(a, b)


def test_imported_caches_of_a_context_with_sections():
    """What was imported has positions that only the caller knows; without sections they are the slots, as ever."""
    from paper_2509_24381_amd import runner
    from paper_2509_24381_amd.binding import RsError
    for sections in (SECTIONS, None):
        stack, weights, dec, kvs = build(sections=sections)
        x = runner.to_device_bf16(rows(np.random.default_rng(8), 21))
        stack.prefill_prompt(x[:20], [(0, 20)], kvs[0])
        for l in range(N_LAYERS):
            kvs[1].import_(l, *kvs[0].export(l))
        if sections:
            with pytest.raises(RsError, match="positions"):
                dec.step(kvs[1:], [1], x[20:])
            b = dec.step(kvs[1:], [1], x[20:], positions=[20])
        else:
            b = dec.step(kvs[1:], [1], x[20:])
        assert torch.equal(dec.step(kvs[:1], [1], x[20:]), b)


def test_generation_goes_on_at_the_positions_that_are_given():
    """greedy and greedy_drafted behind an image: the tokens that steps with explicit positions give, one at a time."""
    from paper_2509_24381_amd import runner
    stack, weights, dec, kvs = build()
    rng = np.random.default_rng(9)
    kinds, pos, nxt = prompt(6, 5, 8, 3)
    x = synth.prompt_rows(kinds, synth.TINY.hidden, 61)
    y = prefill(stack, kvs, [(x, pos), (x, pos)])
    emb, gain = runner.to_device_bf16(rows(rng, 40)), torch.ones(synth.TINY.hidden, dtype=torch.bfloat16, device="cuda")
    last = y[[len(x) - 1, 2 * len(x) - 1]]
    row, want = last[:1], []
    for t in range(6):
        want.append(int(dec.ctx.lm_head(gain, emb, row).argmax()))
        row = dec.step(kvs[:1], [1], emb[want[-1:]], positions=[nxt + t])
    dec.keep(kvs[:1], [len(x)])
    got = dec.greedy(kvs, last, emb, gain, emb, 6, positions=[nxt, nxt])
    keys = kvs[0].export(0)[0].clone()
    assert got[0].tolist() == want
    dec.keep(kvs, [len(x)] * 2)
    tokens, _ = dec.greedy_drafted(kvs[0], last[:1], emb, gain, emb, 6, lambda t: [want[len(t)]] if len(t) < 6 else [], position=nxt)
    assert tokens == want
    n = min(kvs[0].length(0), len(x) + 5)
    assert rel_fro(runner.to_numpy_f32(kvs[0].export(0)[0][len(x): n]), runner.to_numpy_f32(keys[len(x): n])) <= 1e-2
