"""A memory of a video stream: what changed becomes tokens, tokens live in a bounded cache, a query reads it.

    python examples/stream_memory.py [--frames 12] [--budget 512] [--dtype bf16]

Frames of a static camera (a fixed background, moving rectangles, sensor noise below the threshold) go through a small
change-based trunk.  The pixels of its last map that were listed as changed become tokens: their feature vectors are projected to keys
and values, rotated by (time, row, column) and appended to the stream's cache.  One query per frame (a learned vector, here
a random one) attends over everything the cache holds, which adds up how much each token is used; then the cache is
cut back to its budget, the last frames' tokens and the most used ones.  The number of changed pixels stays on the device: no step
waits for the host.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1808_05488_amd as cb  # noqa: E402

TAU = 0.02


class StreamMemory:
    """A change-based trunk and the tokens of what changed in front of it."""

    def __init__(self, height: int, width: int, budget: int, window: int = 2, heads: int = 4, head_dim: int = 64, group: int = 2,
                 dtype=torch.bfloat16, seed: int = 0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rand = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
        channels, layers, pools = [(3, 16), (16, 32), (32, 64)], [], []
        h, w = height, width
        for i, (c, o) in enumerate(channels):
            weight = (rand(o, c, 3, 3) * math.sqrt(2.0 / (9 * c))).to(dtype)
            layers.append(cb.Layer(weight, None, 1, 1, h, w, True))
            pools.append(cb.Pool(layers[-1], 2) if i < 2 else None)
            if i < 2:
                h, w = (h + 1) // 2, (w + 1) // 2
        self.net, self.h, self.w, self.dtype = cb.Network(layers, pools), h, w, dtype
        self.heads, self.head_dim, self.budget, self.window, self.frame = heads, head_dim, budget, window, 0
        self.to_kv = (rand(64, 2 * heads * head_dim) / 8).to(dtype)
        self.query = rand(1, heads * group, head_dim).to(dtype)
        turns = head_dim // 2
        self.rotary = cb.Rotary(head_dim, (turns - 2 * (3 * turns // 8), 3 * turns // 8, 3 * turns // 8))
        # room for the budget and a frame in which every pixel changes
        self.cache = cb.TokenCache.create(1, heads, head_dim, budget + h * w, dtype, page_tokens=64)
        self.offsets = torch.zeros(2, dtype=torch.int32, device="cuda")
        self.now = torch.tensor([[0, h // 2, w // 2]], dtype=torch.int32, device="cuda")      # where the query stands

    def step(self, image: torch.Tensor):
        """One frame: (answer of the query, log of its weights' sum)."""
        features = self.net.forward(image, [TAU] * 3).reshape(64, -1)            # changes in place where something changed
        # rows of all pixels in the order of the list; those behind its end are nobody's (offsets says where it ends)
        self.listed, self.count = self.net.layers[-1].listed()
        pixel = self.listed.long().clamp(0, self.h * self.w - 1)
        tokens = features[:, pixel].t() @ self.to_kv
        k, v = tokens.view(-1, 2, self.heads, self.head_dim).unbind(1)
        time = torch.full_like(pixel, self.frame)
        positions = torch.stack([time, pixel // self.w, pixel % self.w], 1).to(torch.int32)
        self.offsets[1:] = self.count
        self.cache.append(k, v, positions, rotary=self.rotary, offsets=self.offsets)
        self.now[:, 0] = self.frame
        answer, lse = self.cache.attend(self.rotary.rotate(self.query, self.now), accumulate=True, decay=0.95)
        self.cache.evict(self.budget, window=self.window)
        self.frame += 1
        return answer, lse


def video(height: int, width: int, frames: int, dtype, seed: int = 1):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    background = torch.rand((3, height, width), generator=g, device="cuda")
    side = height // 6
    texture = torch.rand((3, side, side), generator=g, device="cuda")
    for t in range(frames):
        image = background + torch.randn(background.shape, generator=g, device="cuda") * 0.003
        x = 4 + 3 * t % (width - side - 8)
        image[:, height // 3:height // 3 + side, x:x + side] = texture
        yield image.to(dtype).contiguous()


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--frames", type=int, default=12)
    ap.add_argument("--height", type=int, default=240)
    ap.add_argument("--width", type=int, default=320)
    ap.add_argument("--budget", type=int, default=512)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    args = ap.parse_args()
    dtype = torch.bfloat16 if args.dtype == "bf16" else torch.float32
    memory = StreamMemory(args.height, args.width, args.budget, dtype=dtype)
    for t, image in enumerate(video(args.height, args.width, args.frames, dtype)):
        answer, lse = memory.step(image)
        print(f"frame {t}: {int(memory.count)} of {memory.h * memory.w} pixels became tokens, {int(memory.cache.lengths[0])} kept; "
              f"|answer| = {answer.float().norm():.4f}, lse = {lse.mean():.4f}")


if __name__ == "__main__":
    main()
