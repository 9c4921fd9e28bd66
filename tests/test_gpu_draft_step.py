"""The example's steps with drafted tokens against a plain record of every sample's
tokens: the rows that are accepted are the rows the next step attends to, whichever
pages they lie on, after samples were forked, given up and compacted.
"""
import importlib.util
import os
import random

import numpy as np
import pytest
import torch

import draft_ref as plain
import ops_ref as ref
import paper_2607_24593_amd as pv
from ops_edges import out_bound

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("draft_step", os.path.join(ROOT, "examples", "draft_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _rows(layer, slot, n):
    """The cache's values of a slot's first n tokens, float64 [n, 576]."""
    idx = torch.full((layer.samples, n), -1, dtype=torch.int32, device="cuda")
    idx[slot] = torch.arange(n, dtype=torch.int32)
    return pv.pivot_cache4_read(layer.cache, idx)[slot].double().cpu().numpy()


def _values(row):
    """What the cache holds of projected rows [n, 576]."""
    codes, scales = ref.quantise(row[:, :ref.LATENT])
    return np.concatenate([ref.values(codes, scales), row[:, ref.LATENT:]], 1)


def test_draft_steps_run_the_operators_together():
    ex = _example()
    samples, dim, heads, nodes, depth = 3, 256, 24, 37, 6
    layer = ex.Layer(samples, 700, dim=dim, heads=heads, page=16, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    rng = random.Random(5)
    prompt = torch.randn((333, dim), generator=g, device="cuda").bfloat16()
    layer.append(0, prompt)
    (row,), _ = layer.project(prompt, None, [layer.to_row])
    tokens = [_values(row.double().cpu().numpy())] + [None] * (samples - 1)
    for s in range(1, samples):
        layer.fork(0, s)
        tokens[s] = tokens[0]
    pool = plain.Pool(samples, layer.table.shape[1], 16, layer.refs.shape[0])
    pool.grow([0], [0], [333])
    pool.fork([0] * (samples - 1), list(range(1, samples)), [333] * (samples - 1))
    residual = torch.randn((samples, nodes, dim), generator=g, device="cuda").bfloat16()
    slots = list(range(samples))
    for step in range(12):
        print("draft step", step, layer.length, flush=True)
        trees = [ex.random_tree(rng, nodes) for _ in slots]
        masks = torch.stack([ex.tree_masks(t, 2) for t in trees])
        hidden = torch.randn((samples, nodes, dim), generator=g, device="cuda").bfloat16()
        length = list(layer.length)
        codes, scale, _ = pv.pivot_rmsnorm_fp8(hidden.view(-1, dim), layer.norm, residual=residual.view(-1, dim), group=128)
        out, _, query = layer.step(hidden, residual, masks)
        assert layer.state.tolist()[0] == 0
        pool.grow(slots, length, [n + nodes for n in length])
        # the projections
        x = codes.view(torch.float8_e4m3fn).double().cpu().numpy() * np.repeat(scale.double().cpu().numpy(), 128, 1)[:, :dim]
        w = [t.cpu().numpy() for t in layer.to_query]
        y, s = plain.linear(x, *w)
        q = query.double().cpu().numpy()
        assert np.all(np.abs(q.reshape(y.shape) - y) <= plain.linear_bound(dim, s, y, True))
        (row,), _ = layer.project(hidden.view(-1, dim), residual.view(-1, dim), [layer.to_row])
        drafts = _values(row.double().cpu().numpy()).reshape(samples, nodes, -1)
        got = out.double().cpu().numpy()
        for b in slots:
            held = np.concatenate([tokens[b], drafts[b]])
            assert np.array_equal(_rows(layer, b, length[b] + nodes), held), (step, b)
            for i in rng.sample(range(nodes), 6):
                at, seen = i, []
                while at >= 0:
                    seen.append(length[b] + at)
                    at = trees[b][at]
                allowed = np.zeros(len(held), dtype=bool)
                allowed[:length[b]] = True
                allowed[seen] = True
                o, _, _, bound, spread = ref.attend_rows(q[b, i], held[:, :512], held[:, 512:], 576 ** -0.5, allowed)
                assert np.all(np.abs(got[b, i] - o) <= out_bound(o, spread, 2.0 ** -18 * bound, allowed.sum()) + 1e-30), (step, b, i)
        paths = [ex.random_path(rng, t, depth) for t in trees]
        path = torch.tensor([p + [-1] * (depth - len(p)) for p in paths], dtype=torch.int32, device="cuda")
        layer.accept(path, [len(p) for p in paths], nodes)
        pool.free(slots, [n + nodes for n in length], layer.length)
        tokens = [np.concatenate([t, d[p]]) for t, d, p in zip(tokens, drafts, paths)]
        if step % 3 == 2:
            src, dst = rng.sample(slots, 2)
            pool.free([dst], [layer.length[dst]], [0])
            layer.fork(src, dst)
            pool.fork([src], [dst], [layer.length[src]])
            tokens[dst] = tokens[src]
        if step % 5 == 4:
            moves, live = layer.compact().tolist()
            assert (moves, live) == pool.compact(layer.refs.shape[0] // 2)[1]
        assert np.array_equal(layer.table.cpu().numpy(), pool.table) and np.array_equal(layer.refs.cpu().numpy(), pool.refs)
    for b in slots:
        assert layer.length[b] == len(tokens[b])
        assert np.array_equal(_rows(layer, b, layer.length[b]), tokens[b])


def test_masks_of_a_tree():
    ex = _example()
    masks = ex.tree_masks([-1, 0, 0, 2, -1] + [3] * 28 + [32], 2).cpu().numpy().view(np.uint32)
    bits = [{j for j in range(64) if row[j // 32] >> (j % 32) & 1} for row in masks]
    assert bits[0] == {0} and bits[3] == {0, 2, 3} and bits[4] == {4} and bits[31] == {0, 2, 3, 31} and bits[33] == {0, 2, 3, 32, 33}


def test_the_example_runs(capsys):
    ex = _example()
    import sys
    old, sys.argv = sys.argv, ["draft_step.py", "--samples", "2", "--prefix", "500", "--nodes", "12", "--steps", "9"]
    try:
        ex.main()
    finally:
        sys.argv = old
    assert "pages in use" in capsys.readouterr().out
