"""A rollout with a paged KV cache: each step stores a chunk's keys (rotated) and values, and the chunk's
tokens attend to the first frame and a window of recent ones.

    python examples/cache_rollout.py [--bits 8] [--steps 12]

Frames of Hg x Wg tokens have (frame, row, column) positions and see all of their own frame; every third
step a single control token follows its frame, which is the same two calls with one row.  cast_block_step takes
history blocks in the order in which they lie and knows no page table, so the one session's pages are handed
out in order: at the end the anchors of one more chunk are routed over all bf16 pages that are full.  Random data of a small model's shape.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_34144_gb300 import native as cast  # noqa: E402


class Rollout:
    """One session: its pages, its table of them, and what its calls share."""

    def __init__(self, H=4, H_q=8, d=128, grid=(16, 16), page=64, n_pages=128, bits=16, window=1024, seed=0):
        self.H, self.H_q, self.d, self.grid, self.page = H, H_q, d, grid, page
        self.window, self.sinks, self.len, self.frames = window, grid[0] * grid[1], 0, 0
        dtype = torch.bfloat16 if bits == 16 else torch.float8_e4m3fn
        self.k = torch.zeros((n_pages, page, H, d), device="cuda").to(dtype)
        self.v = torch.zeros_like(self.k)
        scales = [None, None] if bits == 16 else [torch.ones((n_pages, H), device="cuda") for _ in range(2)]
        self.cache = cast.kv_cache(self.k, self.v, *scales)
        self.table = torch.arange(n_pages, dtype=torch.int32, device="cuda")[None]   # one session: pages in order
        self.kv_len = torch.zeros(1, dtype=torch.int32, device="cuda")
        # a quarter of the pairs for the frame, the rest for row and column
        self.rotary = cast.rotary_table(d, sections=[d // 2 - 2 * (3 * d // 16), 3 * d // 16, 3 * d // 16])
        self.gen = torch.Generator(device="cuda").manual_seed(seed)

    def positions(self, tokens):
        Hg, Wg = self.grid
        t = torch.arange(tokens, device="cuda")
        return torch.stack([torch.full_like(t, self.frames), t // Wg, t % Wg], 1).int()

    def project(self, tokens):
        """Stands for the layer's q, k and v projections: one fused buffer, heads of q, k, v in a row."""
        qkv = torch.randn((tokens, self.H_q + 2 * self.H, self.d), generator=self.gen, device="cuda").to(torch.bfloat16)
        return qkv[:, :self.H_q], qkv[:, self.H_q:self.H_q + self.H], qkv[:, self.H_q + self.H:]

    def step(self, tokens, causal=False):
        """`tokens` new tokens through the attention site: returns (inputs, rotated queries, output)."""
        q, k, v = self.project(tokens)
        pos = self.positions(tokens)
        self.kv_len += tokens
        self.len += tokens
        turned = cast.cast_cache_append(k, v, self.cache, self.table, self.kv_len, rotary=self.rotary, positions=pos, q=q)
        o = cast.cast_cache_attention(turned, self.cache, self.table, self.kv_len, causal=causal, window=self.window,
                                      sinks=self.sinks)
        self.frames += 1
        return (q, k, v, pos), turned, o

    def routed_chunk(self, n_frames=4, anchors=(0, 3), K=6):
        """A chunk's anchors routed over the session's full pages (bf16 pages are history blocks)."""
        S, used = self.grid[0] * self.grid[1], self.len // self.page
        rows = lambda: torch.randn((n_frames, S, self.H, self.d), generator=self.gen, device="cuda").to(torch.bfloat16)  # noqa: E731
        r = torch.empty((n_frames, S, self.H * self.d), dtype=torch.bfloat16, device="cuda")
        return cast.cast_block_step(rows(), rows(), rows(), list(anchors), self.k[:used], self.v[:used], K, self.grid, r,
                                    refine=cast.REFINE_PAPER)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--bits", type=int, choices=(8, 16), default=16)
    ap.add_argument("--steps", type=int, default=12)
    a = ap.parse_args()
    r = Rollout(bits=a.bits, n_pages=max(16, 6 * a.steps))
    for i in range(a.steps):
        r.step(r.grid[0] * r.grid[1])
        if i % 3 == 2:
            r.step(1, causal=True)
    o = r.step(r.grid[0] * r.grid[1])[2]
    print(f"{a.steps + 1} frames, {r.len} tokens in {a.bits}-bit pages; last frame's output rms {o.float().square().mean().sqrt():.4f}")
    if a.bits == 16:
        print(f"routed chunk over {r.len // r.page} pages: residual rms {r.routed_chunk().float().square().mean().sqrt():.4f}")
    cast.cast_check_device()


if __name__ == "__main__":
    main()
