"""Plain definitions of the operators of a decode step with drafted tokens: 4-bit
products in 64 bits, masks of trees, pages that sequences share.  Nothing here
uses the library."""
import numpy as np

import ops_ref as ref

BLK = ref.BLK


def quantise(x):
    """x [n, k] float64 -> codes uint8 [n, k / 2], scales uint8 [n, k / 32]."""
    n, k = x.shape
    padded = np.zeros((n, -(-k // ref.LATENT) * ref.LATENT))
    padded[:, :k] = x
    codes, scales = ref.quantise(padded.reshape(-1, ref.LATENT))
    return codes.reshape(n, -1)[:, :k // 2].copy(), scales.reshape(n, -1)[:, :k // BLK].copy()


def values(codes, scales):
    """codes [n, k / 2], scales [n, k / 32] -> float64 [n, k]."""
    signed = np.concatenate([ref.GRID, -ref.GRID])
    v = np.stack([signed[codes & 15], signed[codes >> 4]], -1).reshape(codes.shape[0], 2 * codes.shape[1])
    two = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return v * np.repeat(two, BLK, axis=-1)


def linear(x, codes, scales):
    """x [r, k] float64 (scales in it) -> y [r, n] and sum |x w| [r, n]."""
    w = values(codes, scales)
    with np.errstate(invalid="ignore", over="ignore"):
        return x @ w.T, np.abs(x) @ np.abs(w).T


def linear_bound(k, s, y, bf16):
    """Of y = sum x w with s = sum |x w|.  Products are exact; a wave adds at most
    1024 of them, 8 to a step of the matrix instruction at least, each step off by at
    most 2^-23 of the magnitudes; then at most 8 waves, and one part for every 2048
    of k, are added, a scale multiplied, and the result rounded."""
    steps = min(k, 1024) / 8 + 8 + k / 2048 + 4
    return steps * 2.0 ** -23 * s + (2.0 ** -8 if bf16 else 2.0 ** -24) * np.abs(y) + 1e-37


def tree_masks(rng, nodes, words=None, root=0.1):
    """A random tree in topological order: truth values [nodes, nodes] (itself and
    its ancestors) and their words uint32 [nodes, words]."""
    seen = np.zeros((nodes, nodes), dtype=bool)
    for i in range(nodes):
        if i and rng.random() > root:
            seen[i] = seen[int(rng.integers(0, i))]
        seen[i, i] = True
    return seen, pack_bits(seen, words)


def pack_bits(seen, words=None):
    m, n = seen.shape
    words = words or -(-n // 32)
    bits = np.zeros((m, 32 * words), dtype=np.uint64)
    bits[:, :n] = seen
    return (bits.reshape(m, words, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)


class Pool:
    """A table of pages with their counts, one step after the other."""

    def __init__(self, slots, max_pages, page, n_pages):
        self.table = np.full((slots, max_pages), -1, dtype=np.int32)
        self.refs = np.zeros(n_pages, dtype=np.int32)
        self.page = page

    def pages(self, tokens):
        return -(-tokens // self.page)

    def fork(self, src, dst, tokens):
        for s, d, n in zip(src, dst, tokens):
            for i in range(self.pages(n)):
                if 0 <= self.table[s, i] < len(self.refs):
                    self.table[d, i] = self.table[s, i]
                    self.refs[self.table[s, i]] += 1

    def free(self, slots, tokens, keep):
        for s, n, k in zip(slots, tokens, keep):
            for i in range(self.pages(k), self.pages(n)):
                if 0 <= self.table[s, i] < len(self.refs):
                    self.refs[self.table[s, i]] -= 1
                    self.table[s, i] = -1

    def grow(self, slots, tokens, new):
        table, refs = self.table.copy(), self.refs.copy()
        free = [int(i) for i in np.nonzero(refs == 0)[0]][::-1]
        pairs, wanted = [], 0
        for s, a, z in zip(slots, tokens, new):
            pair = (-1, -1)
            if z > a and a % self.page:
                old = table[s, a // self.page]
                if old >= 0 and refs[old] > 1:
                    wanted += 1
                    refs[old] -= 1
                    if free:
                        page = free.pop()
                        table[s, a // self.page], refs[page], pair = page, 1, (int(old), page)
            pairs.append(pair)
            for i in range(self.pages(a), self.pages(z)):
                wanted += 1
                if free:
                    table[s, i] = free.pop()
                    refs[table[s, i]] = 1
        had = int((self.refs == 0).sum())
        if wanted > had:
            return np.full((len(slots), 2), -1, np.int32), (wanted - had, had)
        self.table, self.refs = table, refs
        return np.array(pairs, np.int32).reshape(-1, 2), (0, len(free))

    def compact(self, most):
        live, free = np.nonzero(self.refs > 0)[0][::-1], np.nonzero(self.refs == 0)[0]
        moves = [(int(s), int(d)) for s, d in zip(live, free) if s > d][:most]
        for s, d in moves:
            self.refs[d], self.refs[s] = self.refs[s], 0
            self.table[self.table == s] = d
        out = np.full((most, 2), -1, np.int32)
        if moves:
            out[:len(moves)] = moves
        return out, (len(moves), len(live))
