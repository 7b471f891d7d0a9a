"""GPU: attention of many requests on shared pages (rs_attend): calls whose sums just have room, descriptors that are read from device memory, and that pages
are read once at all.  Bounds as in test_gpu_shared_attention.py."""
import pytest
import torch

from tests.test_gpu_cache_operators import normal
from tests.test_gpu_shared_attention import family

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def the_rules_themselves(monkeypatch):
    monkeypatch.delenv("RS_ATTEND_SHARE", raising=False)
    monkeypatch.delenv("RS_ATTEND_TOGETHER", raising=False)


def prompts_with_beams(f, prompts, beams, tokens, new=1):
    who = []
    for i in range(prompts):
        root = f.root(tokens + 5 * i % 64)
        who += [f.fork(root, None, new + (i + b) % 3) for b in range(beams)]
    return who


@pytest.mark.parametrize("hq, hkv, prompts, beams, rows, fp8", [(64, 8, 47, 3, 1, False), (64, 8, 51, 3, 1, False), (64, 8, 51, 3, 1, True), (64, 8, 64, 2, 2, False),
                                                                (28, 4, 102, 3, 1, False)])
def test_sums_that_just_have_room(monkeypatch, hq, hkv, prompts, beams, rows, fp8):
    """17 to 32 stacked rows a prompt, so many that their sums fit the slots only while wavefronts do not share tiles."""
    monkeypatch.setenv("RS_ATTEND_SHARE", "0")
    f = family(hq, hkv, 128, fp8, pages=prompts * (11 + beams), max_requests=320)
    who = prompts_with_beams(f, prompts, beams, 64 * 8, rows)
    f.check(who, [rows] * len(who))


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("together", [False, True], ids=["apart", "together"])
@pytest.mark.parametrize("hq, hkv, d, prompts, beams", [(28, 4, 128, 30, 4), (28, 4, 128, 12, 12), (8, 2, 64, 50, 3)])
def test_descriptors_in_device_memory(monkeypatch, hq, hkv, d, prompts, beams, together, fp8):
    """More than 116 entries, of requests and of what they share: the table is copied to the workspace."""
    monkeypatch.setenv("RS_ATTEND_SHARE", "0")
    if together:
        monkeypatch.setenv("RS_ATTEND_TOGETHER", "0")
    f = family(hq, hkv, d, fp8, pages=prompts * (8 + beams), max_requests=256)
    who = prompts_with_beams(f, prompts, beams, 64 * 4)
    assert prompts + len(who) > 116
    q = normal(f.g, len(who), hq * d)
    first = f.check(who, [1] * len(who), q=q)
    assert torch.equal(first, f.check(who, [1] * len(who), q=q))


@pytest.mark.parametrize("hq, hkv, beams", [(28, 4, 2), (28, 4, 4), (28, 4, 9), (28, 4, 30), (64, 8, 4)])
def test_pages_are_read_once_where_that_pays(monkeypatch, hq, hkv, beams):
    """Reading together adds up in another order than reading alone: on some thousand outputs some bits differ if pages are read once, and none if they are not."""
    def run(prompt, share, check=False):
        if share is None:
            monkeypatch.delenv("RS_ATTEND_SHARE", raising=False)
        else:
            monkeypatch.setenv("RS_ATTEND_SHARE", str(share))
        f = family(hq, hkv, 128, pages=400)
        root = f.root(prompt)
        who = [f.fork(root, None, 2) for _ in range(beams)]
        q = normal(f.g, beams, hq * 128)
        if check:
            return f.check(who, [1] * beams, q=q).clone()
        return f.ctx.attend(0, [f.kvs[i] for i in who], [1] * beams, q, torch.empty_like(q), f.ctx.attend_workspace(beams, beams))

    alone, once = run(5000, 1 << 50, True), run(5000, 0, True)
    assert not torch.equal(alone, once)
    assert torch.equal(alone, run(5000, 1 << 50)) and torch.equal(once, run(5000, 0))
    # the rule: from 60 MB left unread on (a block of all heads: 16 KB a KV head, times keys and values)
    left = (beams - 1) * (5000 // 64) * 64 * 128 * 2 * 2 * hkv
    assert torch.equal(run(5000, None), once if left >= 60 << 20 else alone)
