"""Requests of a hybrid model served from one cache on an MI355X.

One attention layer and one recurrent (gated-delta-rule) layer, as a rank of
such a model holds them, take a prompt, a second prompt that shares a prefix
with it, and several samples of the second one:

1. the prompt runs cold: its keys and values go into cache blocks
   (la_blocks_extend, la_kv_write), its attention runs on what was just
   projected (la_attn_prefill), and the recurrent layer leaves a state in the
   pool at every multiple of the checkpoint interval (la_prefill_paged);
2. the second prompt resumes at the joint boundary of both caches
   (la_hybrid_boundary): it shares the first one's blocks (la_blocks_fork),
   writes its own tokens behind them, attends over the cache
   (la_attn_prefill_paged) and starts the recurrence from a pool page;
3. the samples fork it and take one token a step together (la_attn_decode),
   the prefix they share read once for all of them; half way the first prompt
   is retired (la_blocks_free) and the blocks close up (la_blocks_compact)
   under the running samples.

Projections and sampling are left out: what they would give is drawn at
random, keyed by the position, so that tokens two requests share are the same.

    python examples/hybrid_request.py
"""
from __future__ import annotations

import dataclasses
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_15030_amd import api                     # noqa: E402
from paper_2609_15030_amd import linattn as la           # noqa: E402
from paper_2609_15030_amd import workloads as wl         # noqa: E402


@dataclasses.dataclass
class Sizes:
    q_heads: int = 8
    kv_heads: int = 2
    head_dim: int = 128
    heads: int = 8                 # of the recurrent layer, dk = dv = head_dim
    interval: int = 256            # tokens from one recurrent checkpoint to the next
    block_tokens: int = 64
    prompt: int = 3584
    shared: int = 3000             # tokens of the first prompt that the second begins with
    second: int = 3328
    samples: int = 4
    steps: int = 16


@dataclasses.dataclass
class Tokens:
    """What the projections give for the tokens of one sequence."""
    qkv: torch.Tensor              # [n, q_heads + 2 kv_heads, head_dim]: one projection, read in place
    rec: wl.Inputs                 # the recurrent layer's inputs

    def part(self, a: int, b: int) -> "Tokens":
        return Tokens(self.qkv[a:b], self.rec.tokens(a, b))


def draw_tokens(s: Sizes, seed: int, n: int) -> Tokens:
    gen = torch.Generator().manual_seed(seed)
    qkv = torch.randn((n, s.q_heads + 2 * s.kv_heads, s.head_dim), generator=gen)
    return Tokens(qkv.to(torch.bfloat16).cuda(),
                  wl.random_inputs(seed, [n], s.heads, s.head_dim, s.head_dim, gate_scale=0.01))


def joined(a: Tokens, b: Tokens) -> Tokens:
    x, y = a.rec, b.rec
    both = [np.concatenate([getattr(x, f), getattr(y, f)]) for f in ("q", "k", "v", "g", "beta")]
    n = both[0].shape[0]
    return Tokens(torch.cat([a.qkv, b.qkv]), wl.Inputs(*both, np.array([0, n], np.int32), x.io_dtype))


def _i32(*values) -> torch.Tensor:
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class HybridCache:
    """One block pool for the attention layer's keys and values, one page pool
    for the recurrent layer's states."""

    def __init__(self, s: Sizes, n_rows: int, max_tokens: int):
        self.s = s
        max_blocks = -(-max_tokens // s.block_tokens)
        self.block_bytes = 2 * s.kv_heads * s.block_tokens * s.head_dim * 2
        self.blocks = api.BlockPool.new(n_rows * max_blocks, self.block_bytes, s.block_tokens, n_rows, max_blocks)
        rows = n_rows * (max_tokens // s.interval) * s.heads
        self.states = torch.zeros((rows, s.head_dim * s.head_dim), device="cuda")

    def layer(self, row: int, n: int = 1) -> la.LaKvLayer:
        """The attention layer's cache as sequences [row, row + n) see it."""
        s = self.s
        return la.make_kv_layer(self.blocks.cache, self.blocks.table[row:row + n], s.block_tokens, s.kv_heads,
                                s.head_dim, torch.bfloat16, err_count=self.blocks.err_count)

    def qkv(self, t: torch.Tensor):
        hq, hk = self.s.q_heads, self.s.kv_heads
        return t[:, :hq], t[:, hq:hq + hk], t[:, hq + hk:]

    def prompt(self, row: int, tokens: Tokens):
        """A cold prompt: (attention, recurrent result, its states' pages [checkpoints, heads])."""
        s, n = self.s, tokens.qkv.shape[0]
        q, k, v = self.qkv(tokens.qkv)
        attn = api.AttnPrefill(s.q_heads, s.kv_heads, s.head_dim, [n])
        self.blocks.extend(_i32(row), _i32(n))
        la.la_kv_write(self.layer(row), k, v, attn.cu_dev, _i32(n))
        rec = api.Prefill(api.to_device(tokens.rec), s.interval, emit_ckpt=False)
        pages = torch.arange(rec.n_ckpt_rows * s.heads, dtype=torch.int32, device="cuda")
        return attn.run(q, k, v), rec.run_paged(self.states, ckpt_page_ids=pages), pages.view(-1, s.heads)

    def resume(self, row: int, parent: int, tokens: Tokens, boundary: int, pages: torch.Tensor):
        """A prompt whose first `boundary` tokens the parent row's cache holds: results from there on."""
        s, n = self.s, tokens.qkv.shape[0]
        new = tokens.part(boundary, n)
        q, k, v = self.qkv(new.qkv)
        attn = api.AttnPrefill(s.q_heads, s.kv_heads, s.head_dim, [n - boundary], [n])
        self.blocks.fork(_i32(parent), _i32(row), _i32(boundary))
        self.blocks.extend(_i32(row), _i32(n))
        la.la_kv_write(self.layer(row), k, v, attn.cu_dev, attn.kv_dev)
        o = attn.run_paged(self.layer(row), q)
        if boundary == 0:
            return o, api.Prefill(api.to_device(new.rec), s.interval, emit_ckpt=False).run()
        rec = api.Prefill(api.to_device(new.rec), s.interval, starts=[boundary], emit_ckpt=False)
        return o, rec.run_paged(self.states, state_page_ids=pages[boundary // s.interval - 1].contiguous())

    def sample(self, first: int, parent: int, n_tokens: int, state: torch.Tensor, steps, retire_row: int):
        """Samples in rows [first, first + samples), a token each a step; half
        way row retire_row goes.  steps: Tokens of `samples` tokens, one a step."""
        s, n = self.s, self.s.samples
        rows = torch.arange(first, first + n, dtype=torch.int32, device="cuda")
        self.blocks.fork(_i32(*[parent] * n), rows, _i32(*[n_tokens] * n))
        state = state.expand(n, -1, -1, -1).contiguous()
        shape = la.make_shape(n, s.heads, s.head_dim, s.head_dim, s.interval)
        prefix = n_tokens // s.block_tokens * s.block_tokens           # the blocks that the fork shares
        attn = api.AttnDecode(n, s.q_heads, s.kv_heads, s.head_dim, n_tokens + len(steps), cu_group=_i32(0, n),
                              max_prefix_len=prefix)
        cu, kv_len, shared = torch.arange(n + 1, dtype=torch.int32, device="cuda"), _i32(*[n_tokens] * n), _i32(prefix)
        layer, outs, recs = self.layer(first, n), [], []
        for i, tokens in enumerate(steps):
            if i == len(steps) // 2:
                self.blocks.free(_i32(retire_row))
                self.blocks.compact()
            q, k, v = self.qkv(tokens.qkv)
            kv_len += 1
            self.blocks.extend(rows, kv_len)
            la.la_kv_write(layer, k, v, cu, kv_len)
            outs.append(attn.run(layer, q, kv_len, shared).clone())
            x, o = api.to_device(tokens.rec), torch.empty((n, s.heads, s.head_dim), dtype=torch.bfloat16, device="cuda")
            la.la_decode_step(shape, x.q, x.k, x.v, x.g, x.beta, state, o)
            recs.append(o)
        return torch.stack(outs), torch.stack(recs)


def serve(s: Sizes) -> dict:
    """Runs the three steps; the tokens, the boundary and every layer's outputs."""
    first = draw_tokens(s, 1, s.prompt)
    second = joined(first.part(0, s.shared), draw_tokens(s, 2, s.second - s.shared))
    steps = [draw_tokens(s, 3 + i, s.samples) for i in range(s.steps)]
    cache = HybridCache(s, 2 + s.samples, max(s.prompt, s.second + s.steps))

    attn_first, rec_first, pages = cache.prompt(0, first)
    boundary, _ = la.la_hybrid_boundary(s.second, s.interval, s.block_tokens, s.shared // s.block_tokens * s.block_tokens,
                                        s.shared // s.interval * s.interval)
    attn_second, rec_second = cache.resume(1, 0, second, boundary, pages)
    attn_steps, rec_steps = cache.sample(2, 1, s.second, rec_second.final_state, steps, retire_row=0)
    torch.cuda.synchronize()
    pool = cache.blocks
    return dict(first=first, second=second, steps=steps, boundary=boundary, attn_first=attn_first, rec_first=rec_first.o,
                attn_second=attn_second, rec_second=rec_second.o, attn_steps=attn_steps, rec_steps=rec_steps,
                free=int(pool.free_count), blocks=pool.cache.shape[0], errors=int(pool.err_count))


def main():
    s = Sizes()
    r = serve(s)
    print(f"first prompt: {s.prompt} tokens, cold")
    print(f"second prompt: {s.second} tokens, {s.shared} of them shared; resumed at {r['boundary']}, "
          f"{s.second - r['boundary']} computed")
    print(f"{s.samples} samples of it: {s.steps} tokens each, {s.second // s.block_tokens} blocks shared")
    print(f"blocks in use {r['blocks'] - r['free']} of {r['blocks']}, errors {r['errors']}")


if __name__ == "__main__":
    main()
