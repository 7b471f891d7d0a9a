"""Generation behind chunked prefill: the operators on KV caches (include/rserve_attend.h) run together, as a serving loop would.

rs_prefill_* fill the caches with the prompt.  From there on `Decoder` runs the layers itself - norms, projections and the MLP
through PyTorch, like any caller-side model - and calls the library for what touches the caches: kv_append rotates and stores the
new tokens, attend reads everything cached, and for requests with long contexts attend_blocks reads the blocks that the bounds
on their keys select.  A step takes any number of new tokens per request: one, a few drafted ones, or a piece of a prompt.

    python -m paper_2509_24381_amd.decode --requests 16 --prompt 4000 --tokens 32 [--paged] [--fp8-kv] [--blocks 32]
"""
from __future__ import annotations

from typing import List, Optional, Sequence

from .binding import CacheSet, Context, KVCache, RotaryConfig, RsError, int_array
from .runner import to_device_bf16


class _Layer:
    """One layer's parameters in torch layout, bf16 on the device."""

    def __init__(self, w):
        import torch
        self.g1, self.g2 = to_device_bf16(w.g1), to_device_bf16(w.g2)
        self.w_qkv = torch.cat([to_device_bf16(m) for m in (w.wq, w.wk, w.wv)])
        self.b_qkv = torch.cat([to_device_bf16(b) for b in (w.bq, w.bk, w.bv)]) if getattr(w, "bq", None) is not None else None
        self.w_o, self.w_down = to_device_bf16(w.wo), to_device_bf16(w.wd)
        self.w_gate_up = torch.cat([to_device_bf16(w.wg), to_device_bf16(w.wu)])


class Decoder:
    """The layers of a model on caches that rs_prefill_* filled, or that its own steps fill.

    layer_weights: as for runner.LayerStack.  rotary: another rotary form than the context's (None: that one).  n_blocks: blocks of 64
    tokens that a token attends to (0: all); caches of fewer blocks are read whole either way.

    New tokens turn by one rotary position each: their cache slot, or what the caller says.  Behind a prompt with three-axis positions
    (rs_prefill_*_mrope: an image's tokens share positions) the next token's position is not its slot; the caches know that
    (KVCache.own_positions), and calls without positions are refused.  A text token there has the same position on all three axes, so that one
    number says it, and the sections do not matter; tokens whose axes differ go through rs_prefill_*_mrope.
    """

    def __init__(self, ctx: Context, layer_weights: Sequence, *, max_rows: int, max_requests: int, rotary: Optional[RotaryConfig] = None,
                 n_blocks: int = 0, n_first: int = 1, n_last: int = 2, fp8_visible_tokens: int = 0):
        cfg = ctx.cfg
        self.ctx, self.layers = ctx, [_Layer(w) for w in layer_weights]
        self.rotary = ctx.rotary(rotary or RotaryConfig(rotary_dim=cfg.head_dim, max_pos=cfg.max_pos, theta=cfg.rope_theta))
        self.blocks = (n_blocks, n_first, n_last)
        self.ws = ctx.attend_workspace(max_rows, max_requests, fp8_visible_tokens, n_blocks)

    def step(self, kvs, lens, x, positions=None):
        """The next lens[i] tokens of every request through all layers: x, and the result, bf16 [sum of lens, H].  positions: every row's
        rotary position, on the host (None: its slot)."""
        import torch
        import torch.nn.functional as F
        ctx, cfg = self.ctx, self.ctx.cfg
        kvs = kvs if isinstance(kvs, CacheSet) else CacheSet(kvs)
        n, (n_blocks, n_first, n_last) = int_array(lens), self.blocks
        if positions is None:
            for i, (kv, new) in enumerate(zip(kvs.caches, n)):
                if new and kv.own_positions:
                    raise RsError(-1, f"kvs[{i}] holds tokens whose rotary positions are not their slots, or that were imported beside three-axis "
                                      "sections: give the new tokens' positions")
        else:
            positions = int_array(positions.tolist() if hasattr(positions, "tolist") else positions)
        q_dim, kv_dim = cfg.n_q_heads * cfg.head_dim, cfg.n_kv_heads * cfg.head_dim
        q = torch.empty((x.shape[0], q_dim), dtype=torch.bfloat16, device=x.device)
        att = torch.empty_like(q)
        for layer, w in enumerate(self.layers):
            qkv = F.linear(F.rms_norm(x, (cfg.hidden,), w.g1, cfg.rms_eps), w.w_qkv, w.b_qkv)
            ctx.kv_append(layer, kvs, n, qkv[:, :q_dim], qkv[:, q_dim:q_dim + kv_dim], qkv[:, q_dim + kv_dim:], q, self.rotary,
                          positions=positions)
            if n_blocks:
                ctx.attend_blocks(layer, kvs, n, q, att, self.ws, n_blocks, n_first, n_last)
            else:
                ctx.attend(layer, kvs, n, q, att, self.ws)
            x = x + F.linear(att, w.w_o)
            gate, up = F.linear(F.rms_norm(x, (cfg.hidden,), w.g2, cfg.rms_eps), w.w_gate_up).chunk(2, dim=1)
            x = x + F.linear(F.silu(gate) * up, w.w_down)
        return x

    def keep(self, kvs, lengths: Sequence[int]):
        """Drops what a step appended behind the first lengths[i] tokens (drafted ones that were not taken)."""
        for kv, n in zip(kvs.caches if isinstance(kvs, CacheSet) else kvs, lengths):
            for layer in range(len(self.layers)):
                kv.truncate(layer, n)

    def prepare_blocks(self, kvs: Sequence[KVCache], capacity_tokens: int):
        """Memory for the bounds that attend_blocks selects by, for caches of up to that many tokens."""
        for kv in kvs:
            kv.new_bounds(capacity_tokens)

    def greedy(self, kvs, last_rows, embedding, final_gain, w_lm, n_tokens: int, positions=None):
        """n_tokens tokens of every request, each the likeliest: last_rows is the last layer's output of the prompts' last tokens.
        embedding [V, H] and w_lm [V, H] bf16.  positions: the rotary position of every request's first new token, the others follow it (None: the
        slots).  Returns int64 [requests, n_tokens]."""
        import torch
        kvs = kvs if isinstance(kvs, CacheSet) else CacheSet(kvs)
        one, out = int_array([1] * len(kvs)), []
        for t in range(n_tokens):
            out.append(self.ctx.lm_head(final_gain, w_lm, last_rows).argmax(dim=1))
            last_rows = self.step(kvs, one, embedding[out[-1]], None if positions is None else [int(p) + t for p in positions])
        return torch.stack(out, dim=1)

    def greedy_drafted(self, kv: KVCache, last_row, embedding, final_gain, w_lm, n_tokens: int, draft, position=None):
        """One request's n_tokens likeliest tokens, several a step: draft(tokens) guesses what follows them, the step checks the guesses
        together, and those after the first wrong one are dropped from the cache.  position: the first new token's rotary position, the others
        follow it (None: the slots).  Returns (tokens, steps)."""
        import torch
        kvs, tokens, steps = CacheSet([kv]), [], 0
        ahead = None if position is None else int(position) - kv.length(0)   # of the slots
        token = int(self.ctx.lm_head(final_gain, w_lm, last_row).argmax())
        while True:
            tokens.append(token)
            if len(tokens) >= n_tokens:
                return tokens[:n_tokens], steps
            guesses: List[int] = [int(t) for t in draft(tokens)]
            held = kv.length(0)
            at = None if ahead is None else range(held + ahead, held + ahead + 1 + len(guesses))
            rows = self.step(kvs, [1 + len(guesses)], embedding[torch.tensor([token] + guesses, device=embedding.device)], at)
            best = self.ctx.lm_head(final_gain, w_lm, rows).argmax(dim=1).tolist()
            steps += 1
            taken = 0
            while taken < len(guesses) and guesses[taken] == best[taken]:
                taken += 1
            self.keep([kv], [held + 1 + taken])
            tokens += guesses[:taken]
            token = best[taken]


def main(argv=None):
    import argparse
    import time

    import torch

    from .runner import LayerStack
    import synth
    p = argparse.ArgumentParser(description="prefill, then generation on the same caches: ms per step")
    p.add_argument("--workload", type=int, default=3, help="the layer shape of this workload (synth.workload)")
    p.add_argument("--layers", type=int, default=2)
    p.add_argument("--requests", type=int, default=16)
    p.add_argument("--prompt", type=int, default=4000)
    p.add_argument("--tokens", type=int, default=32)
    p.add_argument("--drafts", type=int, default=0, help="drafted tokens beside each new one")
    p.add_argument("--blocks", type=int, default=0, help="blocks that a token attends to (0: all)")
    p.add_argument("--paged", action="store_true")
    p.add_argument("--fp8-kv", action="store_true")
    a = p.parse_args(argv)
    if not torch.cuda.is_available():
        raise SystemExit("decode needs a GPU")
    shape, room = synth.workload(a.workload).shape, a.prompt + (a.tokens + 3) * (1 + a.drafts)
    weights = [synth.layer_weights(shape, seed) for seed in range(a.layers)]
    visible = (room + 63) // 64 * 64
    stack = LayerStack(shape, weights, max_tokens=2048, max_requests=max(a.requests, 1), max_pos=room, fp8_visible_tokens=visible if a.fp8_kv else 0)
    if a.paged:
        pool = stack.new_pool(a.requests * a.layers * (visible // 64), fp8=a.fp8_kv)
        kvs = [pool.new_cache(a.layers) for _ in range(a.requests)]
    else:
        kvs = [stack.new_cache_fp8(room) if a.fp8_kv else stack.new_cache(room) for _ in range(a.requests)]
    rows = a.requests * (1 + a.drafts)
    decoder = Decoder(stack.ctx, weights, max_rows=rows, max_requests=a.requests, n_blocks=a.blocks, fp8_visible_tokens=a.requests * visible if a.fp8_kv else 0)
    if a.blocks:
        decoder.prepare_blocks(kvs, room)
    x = torch.randn(a.prompt, shape.hidden, device="cuda").to(torch.bfloat16)
    for kv in kvs:
        stack.prefill_prompt(x, [(i, min(i + 2048, a.prompt)) for i in range(0, a.prompt, 2048)], kv)
    cs, lens, new = CacheSet(kvs), int_array([1 + a.drafts] * a.requests), torch.randn(rows, shape.hidden, device="cuda").to(torch.bfloat16)
    for _ in range(3):
        decoder.step(cs, lens, new)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.tokens):
        decoder.step(cs, lens, new)
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t) / a.tokens * 1e3
    print(f"{shape.name}, {a.layers} layers, {a.requests} requests of {a.prompt} tokens, {1 + a.drafts} new each: {ms:.3f} ms a step, "
          f"{ms / a.layers * 1e3:.0f} us a layer")


if __name__ == "__main__":
    main()
