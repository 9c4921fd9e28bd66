"""One sparse-attention layer of a serving loop, from hidden state to attention
output, over a latent cache in 4 bits that is kept within a budget of tokens.

Every decode step of a batch (n_new tokens a sequence, a draft among them):

  pivot_rmsnorm_fp8    hidden + residual, normed, as fp8 rows for the projections;
                       also the indexer's query and key rows with their scales
  pivot_cache4_write   the new tokens' latent and position values into the cache
  pivot_group_index    the new tokens' index sets (PIVOT Refine)
  pivot_cache4_attend  attention over the sets; the weights that tokens get add up
  pivot_evict          once a sequence is over its budget: the first tokens, the
                       latest and the heaviest stay, in cache and indexer keys

Weights are random; the projections are plain products.

    python examples/serve_step.py --batch 8 --prefix 6000 --steps 64
"""
import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_24593_amd as pv  # noqa: E402

HEADS, LATENT, ROPE = 128, pv.PIVOT_CACHE4_LATENT, pv.PIVOT_CACHE4_ROPE
INDEX_HEADS, INDEX_DIM = 64, 128


class Store:
    """A batch's cache and indexer keys, `room` tokens a sequence."""

    def __init__(self, batch, room, device):
        rows, new = batch * room, lambda *s, **k: torch.zeros(s, device=device, **k)
        self.room = room
        self.arrays = (new(rows, LATENT // 2, dtype=torch.uint8), new(rows, LATENT // 32, dtype=torch.uint8),
                       new(rows, ROPE, dtype=torch.bfloat16), new(rows, INDEX_DIM, dtype=torch.uint8), new(rows))
        self.map = pv.make_row_map(seq_stride=room, rows=rows)
        self.cache = pv.make_cache4(*self.arrays[:3], self.map)
        self.keys = self.arrays[3].view(torch.float8_e4m3fn).view(batch, room, INDEX_DIM)
        self.key_scale = self.arrays[4].view(batch, room)


class Layer:
    def __init__(self, batch, dim=512, topk=512, budget=8192, n_new=2, sink=4, recent=256, device="cuda", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.batch, self.n_new, self.topk, self.budget, self.sink, self.recent = batch, n_new, topk, budget, sink, recent

        def weight(out):
            return (torch.randn((dim, out), generator=g, device=device) / math.sqrt(dim)).bfloat16()

        self.to_latent, self.to_rope, self.to_key = weight(LATENT), weight(ROPE), weight(INDEX_DIM)
        self.to_query, self.to_index = weight(HEADS * (LATENT + ROPE)), weight(INDEX_HEADS * INDEX_DIM)
        self.to_gate = weight(INDEX_HEADS)
        one = lambda n: torch.ones(n, dtype=torch.bfloat16, device=device)  # noqa: E731
        self.norm, self.key_norm, self.index_norm = one(dim), one(INDEX_DIM), one(INDEX_HEADS * INDEX_DIM)
        room = budget + 64 * n_new  # evicted only every 64 steps
        self.store, self.spare = Store(batch, room, device), Store(batch, room, device)
        self.acc = torch.zeros((batch, room), device=device)
        self.length = 0

    def rows(self, hidden, residual):
        """The new residual, and the normed hidden rows as the projections' input."""
        codes, scale, residual = pv.pivot_rmsnorm_fp8(hidden, self.norm, residual=residual)
        return residual, (codes.view(torch.float8_e4m3fn).float() * scale).bfloat16()

    def append(self, x):
        """The tokens of x [B, n, dim] into the cache and the indexer's keys."""
        b, n = x.shape[:2]
        pos = self.length
        pv.pivot_cache4_write((x @ self.to_latent).view(b * n, LATENT), (x @ self.to_rope).view(b * n, ROPE),
                              self.store.cache, [pos] * b, n)
        codes, scale, _ = pv.pivot_rmsnorm_fp8(x @ self.to_key, self.key_norm)
        self.store.keys.view(torch.uint8)[:, pos:pos + n] = codes
        self.store.key_scale[:, pos:pos + n] = scale.squeeze(-1)
        self.length += n

    def step(self, hidden, residual):
        """One decode step: (attention output [B, n_new, heads, 512], new residual, index sets)."""
        b, n = hidden.shape[:2]
        if self.length + n > self.store.room:
            self.evict()
        residual, x = self.rows(hidden, residual)
        pos = self.length
        self.append(x)
        codes, scale, _ = pv.pivot_rmsnorm_fp8(x @ self.to_index, self.index_norm)
        q = codes.view(torch.float8_e4m3fn).view(b, n, INDEX_HEADS, INDEX_DIM)
        gate = (x @ self.to_gate).float()
        idx = pv.pivot_group_index(q, scale.view(b, n), gate, self.store.keys, self.store.key_scale, [pos] * b,
                                   [self.length] * b, self.topk, mode=pv.PIVOT_REFINE, g=n, c=2 * self.topk)
        query = (x @ self.to_query).view(b, n, HEADS, LATENT + ROPE)
        out, _ = pv.pivot_cache4_attend(query, self.store.cache, [pos] * b, [self.length] * b,
                                        (LATENT + ROPE) ** -0.5, idx=idx, acc=self.acc)
        return out, residual, idx

    def evict(self):
        """Back to the budget, into the other store.  Returns the kept positions."""
        kept, acc = pv.pivot_evict(self.acc, [self.length] * self.batch, self.budget,
                                   list(zip(self.store.arrays, self.spare.arrays)), self.store.map, self.spare.map,
                                   sink=self.sink, recent=self.recent)
        self.store, self.spare = self.spare, self.store
        self.length = min(self.length, self.budget)
        self.acc.zero_()
        self.acc[:, :self.budget] = acc
        return kept


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--batch", type=int, default=8)
    p.add_argument("--prefix", type=int, default=6000, help="tokens in the cache before the first step")
    p.add_argument("--budget", type=int, default=6016, help="tokens a sequence keeps")
    p.add_argument("--steps", type=int, default=128)
    a = p.parse_args()
    dim = 512
    layer = Layer(a.batch, dim, budget=a.budget)
    if not 0 < a.prefix <= layer.store.room - layer.n_new:
        p.error(f"--prefix must be in [1, {layer.store.room - layer.n_new}]")
    layer.append(layer.rows(torch.randn((a.batch, a.prefix, dim), device="cuda").bfloat16(), None)[1])
    residual = torch.zeros((a.batch, layer.n_new, dim), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(a.steps):
        hidden = torch.randn((a.batch, layer.n_new, dim), device="cuda").bfloat16()
        out, residual, _ = layer.step(hidden, residual)
    torch.cuda.synchronize()
    took = time.perf_counter() - start
    print(f"{a.steps} steps of {a.batch} x {layer.n_new} tokens: {took / a.steps * 1e6:.0f} us a step, "
          f"{layer.length} tokens a sequence at the end, |out| {out.float().abs().mean().item():.4f}")


if __name__ == "__main__":
    main()
