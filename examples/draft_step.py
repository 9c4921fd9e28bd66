"""One attention layer of a serving loop that verifies trees of drafted tokens, for
several samples of one prompt that share its pages.

  pivot_pages_grow, _copy   room for a step's drafts; a sample whose last page others
                            hold too gets its own
  pivot_rmsnorm_fp8         hidden + residual, normed, as fp8 rows
  pivot_linear4             the drafts' latent and position values and their queries,
                            from weights in 4 bits
  pivot_cache4_write        the drafts into the cache, in the order of the tree
  pivot_cache4_attend       every draft over the accepted tokens and its ancestors
  pivot_tree_accept         the accepted path to where the next step expects it
  pivot_pages_free          the pages behind it back to the pool
  pivot_pages_fork          a sample that is given up goes on from another one
  pivot_pages_compact       now and then the pages in use move to the pool's start

Weights are random, and so is what is accepted.

    python examples/draft_step.py --samples 4 --prefix 6000 --steps 64
"""
import argparse
import math
import os
import random
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_24593_amd as pv  # noqa: E402

LATENT, ROPE = pv.PIVOT_CACHE4_LATENT, pv.PIVOT_CACHE4_ROPE


def tree_masks(parents, words, device="cuda"):
    """Parents of a tree's nodes in topological order (-1: the last accepted token) ->
    masks int32 [nodes, words], each node's ancestors and itself."""
    rows, seen = [], []
    for i, p in enumerate(parents):
        seen.append((seen[p] if p >= 0 else 0) | 1 << i)
        rows.append([(seen[i] >> 32 * w & 0xFFFFFFFF) for w in range(words)])
    return torch.tensor([[v - (1 << 32) if v >> 31 else v for v in row] for row in rows], dtype=torch.int32, device=device)


class Layer:
    """The samples' lengths are host numbers; slot s of the table is sample s.  n_pages:
    the pool's pages, fewer than samples times room where samples share a prompt."""

    def __init__(self, samples, room, dim=512, heads=128, page=64, device="cuda", seed=0, n_pages=None):
        g = torch.Generator(device=device).manual_seed(seed)
        self.samples, self.dim, self.heads, self.page = samples, dim, heads, page
        new = lambda *s, **k: torch.zeros(s, device=device, **k)  # noqa: E731
        per = -(-room // page)
        n_pages = samples * per if n_pages is None else n_pages
        self.table = torch.full((samples, per), -1, dtype=torch.int32, device=device)
        self.refs = new(n_pages, dtype=torch.int32)
        self.pages = pv.make_pages(self.table, self.refs, page)
        rows = n_pages * page
        self.arrays = (new(rows, LATENT // 2, dtype=torch.uint8), new(rows, LATENT // 32, dtype=torch.uint8),
                       new(rows, ROPE, dtype=torch.bfloat16))
        self.map = pv.make_row_map(block_table=self.table, page_size=page, rows=rows)
        self.cache = pv.make_cache4(*self.arrays, self.map)

        def weight(out):
            return pv.pivot_linear4_pack((torch.randn((out, dim), generator=g, device=device) / math.sqrt(dim)).bfloat16())

        self.to_row, self.to_query = weight(LATENT + ROPE), weight(heads * (LATENT + ROPE))
        self.norm = torch.ones(dim, dtype=torch.bfloat16, device=device)
        self.length = [0] * samples

    def grow(self, slots, new):
        """Room for new[i] more tokens of slots[i].  Only the device knows whether the pool had
        the pages: this waits for it."""
        now = [self.length[s] for s in slots]
        copies, self.state = pv.pivot_pages_grow(self.pages, slots, now, [n + m for n, m in zip(now, new)])
        if missing := int(self.state[0]):
            raise RuntimeError(f"the pool lacks {missing} pages")
        pv.pivot_pages_copy(self.pages, copies, self.arrays)

    def project(self, hidden, residual, weight, dtype=torch.bfloat16):
        """(rows of weight, residual) of the normed hidden rows [rows, dim]."""
        codes, scale, residual = pv.pivot_rmsnorm_fp8(hidden, self.norm, residual=residual, group=128)
        return [pv.pivot_linear4(codes, *w, x_scale=scale, group=128, dtype=dtype) for w in weight], residual

    def append(self, slot, hidden):
        """Accepted tokens hidden [n, dim] at the end of a slot."""
        n = hidden.shape[0]
        self.grow([slot], [n])
        (row,), _ = self.project(hidden, None, [self.to_row])
        cu = [0] * (slot + 1) + [n] * (self.samples - slot)
        pv.pivot_cache4_write(row[:, :LATENT], row[:, LATENT:], self.cache, self.length, cu=cu)
        self.length[slot] += n

    def step(self, hidden, residual, masks):
        """Drafts hidden [samples, nodes, dim] in the trees' order, masks [samples,
        nodes, words] -> (attention output [samples, nodes, heads, 512], residual, the
        queries)."""
        b, m = hidden.shape[:2]
        self.grow(list(range(b)), [m] * b)
        (row, query), residual = self.project(hidden.view(b * m, self.dim), residual.view(b * m, self.dim),
                                              [self.to_row, self.to_query])
        pv.pivot_cache4_write(row[:, :LATENT], row[:, LATENT:], self.cache, self.length, m)
        query = query.view(b, m, self.heads, LATENT + ROPE)
        out, _ = pv.pivot_cache4_attend(query, self.cache, self.length, [n + m for n in self.length],
                                        (LATENT + ROPE) ** -0.5, tree=masks)
        return out, residual.view(b, m, self.dim), query

    def accept(self, path, counts, nodes):
        """The nodes path[s] (int32 [samples, depth], -1 behind counts[s] of them) stay."""
        pv.pivot_tree_accept(path, self.length, self.arrays, self.map)
        grown = [n + nodes for n in self.length]
        self.length = [n + c for n, c in zip(self.length, counts)]
        pv.pivot_pages_free(self.pages, list(range(self.samples)), grown, self.length)

    def fork(self, src, dst):
        """Sample dst goes on from sample src."""
        pv.pivot_pages_free(self.pages, [dst], [self.length[dst]], [0])
        pv.pivot_pages_fork(self.pages, [src], [dst], [self.length[src]])
        self.length[dst] = self.length[src]

    def compact(self):
        moves, state = pv.pivot_pages_compact(self.pages, self.refs.shape[0] // 2)
        pv.pivot_pages_copy(self.pages, moves, self.arrays)
        return state


def random_tree(rng, nodes):
    return [-1] + [rng.randrange(-1, i) for i in range(1, nodes)]


def random_path(rng, parents, depth):
    """A node's ancestors and itself, ascending, at most depth of them."""
    at, path = rng.randrange(len(parents)), []
    while at >= 0:
        path.append(at)
        at = parents[at]
    return path[::-1][:depth]


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--samples", type=int, default=4)
    p.add_argument("--prefix", type=int, default=6000, help="tokens of the prompt")
    p.add_argument("--nodes", type=int, default=26, help="drafts of a step")
    p.add_argument("--steps", type=int, default=64)
    a = p.parse_args()
    depth, dim, rng = 8, 512, random.Random(0)
    layer = Layer(a.samples, a.prefix + a.steps * depth + a.nodes)
    layer.append(0, torch.randn((a.prefix, dim), device="cuda").bfloat16())
    for s in range(1, a.samples):
        layer.fork(0, s)
    residual = torch.zeros((a.samples, a.nodes, dim), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    start, accepted = time.perf_counter(), 0
    for step in range(a.steps):
        trees = [random_tree(rng, a.nodes) for _ in range(a.samples)]
        masks = torch.stack([tree_masks(t, -(-a.nodes // 32)) for t in trees])
        hidden = torch.randn((a.samples, a.nodes, dim), device="cuda").bfloat16()
        out, _, _ = layer.step(hidden, residual, masks)
        paths = [random_path(rng, t, depth) for t in trees]
        path = torch.tensor([q + [-1] * (depth - len(q)) for q in paths], dtype=torch.int32, device="cuda")
        layer.accept(path, [len(q) for q in paths], a.nodes)
        accepted += sum(len(q) for q in paths)
        if a.samples > 1 and step % 8 == 7:  # one sample is given up
            src, dst = rng.sample(range(a.samples), 2)
            layer.fork(src, dst)
    layer.compact()
    torch.cuda.synchronize()
    took = time.perf_counter() - start
    print(f"{a.steps} steps of {a.samples} trees of {a.nodes} drafts: {took / a.steps * 1e6:.0f} us a step, "
          f"{accepted} tokens accepted, {int((layer.refs > 0).sum())} of {layer.refs.shape[0]} pages in use, "
          f"|out| {out.float().abs().mean().item():.4f}")


if __name__ == "__main__":
    main()
