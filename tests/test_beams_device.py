"""Tensors in host memory are refused where a kernel would follow their addresses: on hosts without a GPU as if there were one, and on a GPU."""
import pytest
import torch

from tests.test_beams_host import Pool, gpu_less, make_context, refused


def calls(ctx, device):
    """beam_select with one tensor in host memory each, by its name."""
    x, scores = torch.zeros((2, 3, 50), device=device), torch.zeros((2, 3), device=device)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=device)
    out = lambda d: [torch.zeros((2, 4), dtype=t, device=d) for t in (torch.int32, torch.int32, torch.float32)]
    host = out("cpu")
    yield "logits", lambda: ctx.beam_select(x.cpu(), scores, 4, ws, out=out(device))
    yield "scores", lambda: ctx.beam_select(x, scores.cpu(), 4, ws, out=out(device))
    yield "workspace", lambda: ctx.beam_select(x, scores, 4, ws.cpu(), out=out(device))
    for i, name in enumerate(("parents", "tokens", "out_scores")):
        yield name, lambda i=i: ctx.beam_select(x, scores, 4, ws, out=[host[j] if i == j else t for j, t in enumerate(out(device))])


class Elsewhere(torch.Tensor):
    """A host tensor that says it is on the GPU (no call with one passes the checks)."""
    is_cuda = True


@gpu_less
def test_host_tensors_are_refused(monkeypatch):
    ctx = make_context()
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    x, scores, ws = (t.as_subclass(Elsewhere) for t in (torch.zeros((2, 3, 50)), torch.zeros((2, 3)), torch.empty(1 << 20, dtype=torch.uint8)))
    out = [torch.zeros((2, 4), dtype=t).as_subclass(Elsewhere) for t in (torch.int32, torch.int32, torch.float32)]
    host = lambda t: t.as_subclass(torch.Tensor)
    refused("RS_EINVAL", lambda: ctx.beam_select(host(x), scores, 4, ws, out=out), "logits", "GPU")
    refused("RS_EINVAL", lambda: ctx.beam_select(x, host(scores), 4, ws, out=out), "scores", "GPU")
    refused("RS_EINVAL", lambda: ctx.beam_select(x, scores, 4, host(ws), out=out), "workspace", "GPU")
    for i, name in enumerate(("parents", "tokens", "out_scores")):
        refused("RS_EINVAL", lambda: ctx.beam_select(x, scores, 4, ws, out=[host(t) if i == j else t for j, t in enumerate(out)]), name, "GPU")
    kv = Pool(ctx).cache()
    refused("RS_EINVAL", lambda: ctx.kv_compact(0, [kv], torch.zeros(5, dtype=torch.int32), [5]), "keep", "GPU")
    ctx.kv_compact(0, [kv], torch.zeros(0, dtype=torch.int32), [0], stream=0)   # (nothing is read)


@pytest.mark.gpu
def test_host_tensors_are_refused_on_a_gpu():
    from tests.test_gpu_cache_operators import context, gen, normal
    from paper_2509_24381_amd.binding import KVPool
    ctx = context(4, 2, 64)
    for name, call in calls(ctx, "cuda"):
        refused("RS_EINVAL", call, name, "GPU")
    kv, k = KVPool(ctx, 8).new_cache(1), normal(gen(1), 100, 2, 64)
    kv.import_(0, k, k)
    keep = torch.arange(50, dtype=torch.int32)
    refused("RS_EINVAL", lambda: ctx.kv_compact(0, [kv], keep, [50]), "keep", "GPU")
    assert kv.length() == 100
    ctx.kv_compact(0, [kv], keep.cuda(), [50])
    assert torch.equal(kv.export(0)[0], k[:50])
