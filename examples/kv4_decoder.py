"""One decoder's KV memory at work: the scheduler's local order, block tables, the
4-bit cache and attention over it, step by step on one GPU.

Requests with a prompt and an output length wait in a queue.  Every step the
waiting requests are put in local order (maps_order_local) and admitted while their
prompts and bounds fit the blocks that the admitted ones leave, the first misfit
blocking; blocks are handed out in that order (maps_block_tables), the new tokens'
keys and values go into the cache (maps_kv4_append) and their queries attend over it
(maps_kv4_attention): a chunk of the prompt for a request that is being prefilled, one
token for one that decodes.  A request that has all its tokens gives its blocks
back at the next step.  Keys, values and queries stand in for a model's: they
are drawn at random.

With --sparse N keys and queries are turned by their positions on the way
(maps_kv4_append_rotated), the ranges of the blocks that new tokens went to are kept
(maps_kv4_block_ranges), and the query of a request that decodes attends over the N blocks
alone that score highest for it (maps_kv4_select_blocks, maps_kv4_attention_blocks).  Prompts
attend over all their keys (maps_kv4_attention), as chunks of many queries do sooner.

    python examples/kv4_decoder.py --requests 256 --blocks 8192
    python examples/kv4_decoder.py --requests 256 --blocks 8192 --sparse 32
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_15359_gb300 import maps as M  # noqa: E402


def ok(status: int) -> None:
    if status != M.MAPS_OK:
        raise M.MapsError(status)


class Decoder:
    """State of one decoder: requests, block tables, free blocks and the cache of one layer."""

    def __init__(self, prompt, output, bound, blocks: int, heads=(32, 8), D: int = 128, S: int = 16, chunk: int = 512,
                 max_wait: int = 1000, dtype=torch.bfloat16, seed: int = 0, sparse: int = 0):
        self.R, self.S, self.D, self.chunk, self.max_wait, self.dtype = prompt.numel(), S, D, chunk, max_wait, dtype
        self.Hq, self.H = heads
        self.device = prompt.device
        self.prompt, self.bound, self.total = prompt, bound, prompt + output
        self.gen = torch.Generator(self.device).manual_seed(seed)
        i32 = dict(dtype=torch.int32, device=self.device)
        most = -(-int(self.total.max()) // S)
        self.held = torch.zeros(self.R, **i32)
        self.table = torch.full((self.R, most), -1, **i32)
        self.free = torch.arange(blocks, **i32)
        self.n_free = torch.full((1,), blocks, **i32)
        self.cache = torch.zeros(M.kv4_cache_shape(blocks, self.H, S, D), dtype=torch.uint8, device=self.device)
        self.arrival = torch.arange(self.R, **i32)
        self.admitted = torch.zeros(self.R, dtype=torch.bool, device=self.device)
        self.returned = self.admitted.clone()
        self.wait, self.zero = torch.zeros(self.R, **i32), torch.zeros(self.R, **i32)
        self.order, self.seg = torch.zeros(self.R, **i32), torch.zeros(2, dtype=torch.int64, device=self.device)
        self.ws = M.Workspace(device=self.device)
        self.sparse = sparse
        if sparse:
            self.codes = torch.zeros(M.kv4_range_shape(blocks, self.H, D), dtype=torch.int8, device=self.device)
            self.scale = torch.zeros(blocks, self.H, device=self.device)
            angle = torch.arange(most * S, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))
            self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float().to(self.device)

    def done(self) -> bool:
        return bool((self.held >= self.total).all())

    def attend_lists(self, q, off, n):
        """Attention of each query over the blocks of its own list."""
        lists = torch.empty(len(q), self.H, self.sparse, dtype=torch.int32, device=self.device)
        tokens, out = torch.empty(len(q), self.H, dtype=torch.int32, device=self.device), torch.empty_like(q)
        ok(M.maps_kv4_select_blocks(q, off, n, self.table, self.codes, self.scale, self.S, 1, 2, lists, tokens, ws=self.ws))
        ok(M.maps_kv4_attention_blocks(q, lists, tokens, self.cache, self.S, self.D ** -0.5, out, ws=self.ws))
        return out

    def step(self) -> dict:
        """One step; returns the tokens' queries, keys, values, slots and outputs."""
        S = self.S
        finished = self.held >= self.total
        ok(M.maps_order_local(1, self.zero, self.bound, self.wait, self.arrival, self.max_wait, self.order, self.seg, ws=self.ws))
        # admission: used + prompt + bound <= capacity, in blocks
        need = (self.prompt + torch.maximum(self.bound, self.total - self.prompt) + S - 1) // S
        order = self.order.long()
        waiting = ~self.admitted[order]
        budget = self.free.numel() - need[self.admitted & ~finished].sum()
        self.admitted[order] |= waiting & ((need[order] * waiting).cumsum(0) <= budget)
        live = self.admitted & ~finished
        # the rest of the prompt in chunks, then a token at a time; a finished request wants nothing
        ask = torch.where(self.held < self.prompt, torch.minimum(self.prompt - self.held, torch.full_like(self.held, self.chunk)), 1)
        want = torch.where(live, self.held + ask, 0).int()
        tokens_held = torch.where(finished & self.returned, 0, self.held).int()
        T = int((want - tokens_held).clamp(min=0).sum())
        off = torch.empty(self.R + 1, dtype=torch.int64, device=self.device)
        slots = torch.empty(T, dtype=torch.int64, device=self.device)
        got, n_free = torch.empty_like(self.held), torch.empty_like(self.n_free)
        pos = torch.empty(T, dtype=torch.int32, device=self.device)
        ok(M.maps_block_tables(S, tokens_held, want, self.table, self.free, self.n_free, n_free, got, off, slots,
                               pos_out=pos, order=self.order, ws=self.ws))
        draw = lambda h: torch.randn(T, h, self.D, device=self.device, generator=self.gen).to(self.dtype)  # noqa: E731
        q, k, v = draw(self.Hq), draw(self.H), draw(self.H)
        granted = live & (got == want)  # all that are live: admission leaves blocks for them
        n = torch.where(granted, got, 0)
        out = torch.empty_like(q)
        if self.sparse:
            ok(M.maps_kv4_append_rotated(q, k, v, pos, self.cos_sin, slots, self.cache, S, q, ws=self.ws))
            ok(M.maps_kv4_block_ranges(tokens_held, n, self.table, self.cache, S, self.codes, self.scale, ws=self.ws))
            prompts = self.held < self.prompt
            alone = torch.where(prompts, 0, n)  # requests that decode
            if bool((live & prompts).any()):
                ok(M.maps_kv4_attention(q, off, n - alone, self.table, self.cache, S, self.D ** -0.5, out, ws=self.ws))
                new = off.diff()
                rows = (~prompts).repeat_interleave(new, output_size=T).nonzero()[:, 0]
                ends = torch.where(prompts, 0, new).cumsum(0)
                out[rows] = self.attend_lists(q[rows], torch.cat([ends.new_zeros(1), ends]), alone)
            else:
                out = self.attend_lists(q, off, alone)
        else:
            ok(M.maps_kv4_append(k, v, slots, self.cache, S, ws=self.ws))
            ok(M.maps_kv4_attention(q, off, n, self.table, self.cache, S, self.D ** -0.5, out, ws=self.ws))
        self.wait += 1
        self.wait[granted] = 0
        self.returned |= finished
        self.held = torch.where(finished, self.held, got)
        self.n_free = n_free
        return dict(q=q, k=k, v=v, slots=slots, pos=pos, off=off, n=n, out=out, granted=granted)


def main() -> None:
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=256)
    ap.add_argument("--blocks", type=int, default=8192)
    ap.add_argument("--steps", type=int, default=5000, help="at most so many")
    ap.add_argument("--sparse", type=int, default=0, help="cache blocks that a decoding request's query attends over (3 at least); 0: all")
    a = ap.parse_args()
    g = torch.Generator().manual_seed(1)
    prompt = torch.randint(32, 2049, (a.requests,), generator=g, dtype=torch.int32)
    output = torch.empty(a.requests).log_normal_(5.5, 1.0, generator=g).clamp(1, 1024).int()
    bound = (output.float() * 1.5).int()
    d = Decoder(prompt.cuda(), output.cuda(), bound.cuda(), a.blocks, sparse=a.sparse)
    t0, steps, tokens = time.perf_counter(), 0, 0
    while not d.done() and steps < a.steps:
        r = d.step()
        tokens += int((r["slots"] >= 0).sum())
        steps += 1
    torch.cuda.synchronize()
    ok(M.maps_check(d.ws))
    s = time.perf_counter() - t0
    print(f"{steps} steps, {tokens} tokens placed and attended in {s:.2f} s ({tokens / s:.0f} tokens/s, host-driven); "
          f"{int(d.n_free)} of {a.blocks} blocks free")


if __name__ == "__main__":
    main()
