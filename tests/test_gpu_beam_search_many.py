"""GPU: beam searches at the most beams that a call takes, with beams that are out at first (fewer words than beams).  Many paths lie closer than the rounding
of the layers, so that ranks are compared by their scores, within 0.1 a token as in test_gpu_beam_search.py, and every path by its own."""
import numpy as np
import pytest
import torch

import synth
from tests.test_gpu_beam_search import language, reference
from tests.test_gpu_decode import rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("beams, end, power, n_tokens", [(64, None, 0.0, 3), (32, 5, 1.0, 3), (32, None, 0.0, 1), (64, None, 0.5, 2)])
def test_the_most_beams(beams, end, power, n_tokens):
    from paper_2509_24381_amd import runner
    from paper_2509_24381_amd.decode import Decoder
    shape, rng, vocab = synth.TINY, np.random.default_rng(11), 24
    weights = [synth.layer_weights(shape, 3 + l, gains="uniform", std=0.06) for l in range(2)]
    stack = runner.LayerStack(shape, weights, max_tokens=256, max_requests=128, max_pos=512)
    dec = Decoder(stack.ctx, weights, max_rows=128, max_requests=128)
    pool = stack.new_pool(2 * (2 * 3 + 128))
    pool.slab.fill_(0xFF)
    prompts, last = [pool.new_cache(2) for _ in range(2)], []
    for kv, n in zip(prompts, (100, 64)):
        x = runner.to_device_bf16(rows(rng, n, shape.hidden))
        last.append(stack.prefill_prompt(x, [(0, n)], kv)[-1:])
    emb, w_lm, gain = language(rng, vocab, shape.hidden)
    free = pool.free_pages
    got = dec.beam_search(prompts, torch.cat(last), emb, gain, w_lm, n_tokens, beams, end=end, length_power=power)
    assert pool.free_pages == free
    for kv, row, found in zip(prompts, last, got):
        want = reference(dec, kv, row, emb, w_lm, gain, n_tokens, beams, end, power)
        assert len(found) == len(want) == min(beams, vocab ** n_tokens)
        assert len({tuple(t) for t, _ in found}) == len(found)
        assert all(abs(a - b) <= 0.1 * n_tokens for (_, a), (_, b) in zip(found, want))
        scores = {tuple(t): s for t, s in want}
        near = [abs(s - scores[tuple(t)]) for t, s in found if tuple(t) in scores]
        assert len(near) > len(found) // 2 and max(near) <= 0.1 * n_tokens
