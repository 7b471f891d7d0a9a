"""CPU: rs_beam_select refuses results and a workspace that overlap one another, or what is read; ranges that only touch are fine."""
import itertools

import pytest

from tests.test_beams_host import AT, gpu_less, make_context, refused

GROUPS, BEAMS, VOCAB, SELECT = 2, 3, 100, 4
RESULT, LOGITS, SCORES = GROUPS * SELECT * 4, GROUPS * BEAMS * VOCAB * 4, GROUPS * BEAMS * 4


@pytest.fixture(scope="module")
def ctx():
    return make_context()


def call(ctx, **at):
    from paper_2509_24381_amd import binding
    need = ctx.lib.rs_beam_workspace_bytes(ctx.handle, GROUPS, BEAMS, VOCAB)
    a = {**dict(logits=AT, scores=AT + (1 << 20), parents=AT + (2 << 20), tokens=AT + (3 << 20), out_scores=AT + (4 << 20), workspace=AT + (5 << 20)), **at}
    return lambda: binding._check(ctx.lib.rs_beam_select(ctx.handle, a["logits"], 0, VOCAB, VOCAB, GROUPS, BEAMS, a["scores"], SELECT, a["parents"], a["tokens"],
                                                         a["out_scores"], a["workspace"], need, None))


@gpu_less
@pytest.mark.parametrize("one, other", list(itertools.combinations(("parents", "tokens", "out_scores"), 2)))
def test_results_that_overlap(ctx, one, other):
    at = AT + (6 << 20)
    for distance in (0, 4, RESULT - 4):
        refused("RS_EINVAL", call(ctx, **{one: at, other: at + distance}), "one another")
        refused("RS_EINVAL", call(ctx, **{one: at + distance, other: at}), "one another")
    for first, second in ((one, other), (other, one)):
        refused("RS_EHIP", call(ctx, **{first: at, second: at + RESULT}))


@gpu_less
@pytest.mark.parametrize("name, size", [("parents", RESULT), ("tokens", RESULT), ("out_scores", RESULT), ("logits", LOGITS), ("scores", SCORES)])
def test_a_workspace_that_overlaps(ctx, name, size):
    need = ctx.lib.rs_beam_workspace_bytes(ctx.handle, GROUPS, BEAMS, VOCAB)
    at = AT + (6 << 20)
    for offset in (0, 4, need - 4, 4 - size):
        refused("RS_EINVAL", call(ctx, **{"workspace": at, name: at + offset}), "overlap")
    for offset in (need, -size):
        refused("RS_EHIP", call(ctx, **{"workspace": at, name: at + offset}))
