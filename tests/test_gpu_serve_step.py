"""The example's decode steps against a plain computation in 64 bits.

The sets come from the index calls (their own tests check them); what is checked
here is that the operators fit together: the rows a step writes are the rows it
attends to, weights add up over steps, and eviction keeps both in line.
"""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2607_24593_amd as pv  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("serve_step", os.path.join(ROOT, "examples", "serve_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _host(t):
    return t.detach().cpu().numpy()


def _weights(ex, layer, x, idx, pos):
    """Softmax weights and outputs of one step in 64 bits: ([B, n, heads, k], [B, n, heads, 512])."""
    b, n, k = idx.shape
    got = pv.pivot_cache4_read(layer.store.cache, idx.view(b, n * k))
    key = _host(got.float()).astype(np.float64).reshape(b, n, k, -1)
    q = _host((x @ layer.to_query).float()).astype(np.float64).reshape(b, n, ex.HEADS, -1)
    at = _host(idx)
    z = np.einsum("bnhd,bnkd->bnhk", q, key) * (ex.LATENT + ex.ROPE) ** -0.5
    ok = (at >= 0) & (at <= pos + np.arange(n)[None, :, None])
    z = np.where(ok[:, :, None], z, -np.inf)
    e = np.exp(z - z.max(-1, keepdims=True))
    p = e / e.sum(-1, keepdims=True)
    return p, np.einsum("bnhk,bnkd->bnhd", p, key[..., :ex.LATENT])


def test_serve_step_runs_the_operators_together():
    ex = _example()
    batch, dim, n = 2, 256, 2
    layer = ex.Layer(batch, dim, topk=64, budget=700, n_new=n, recent=32, seed=5)
    g = torch.Generator(device="cuda").manual_seed(6)
    rand = lambda m: torch.randn((batch, m, dim), generator=g, device="cuda").bfloat16()  # noqa: E731
    layer.append(layer.rows(rand(800), None)[1])
    residual = torch.zeros((batch, n, dim), dtype=torch.bfloat16, device="cuda")
    total = np.zeros((batch, layer.store.room))
    evicted = 0
    for step in range(20):
        print("serve step", step, layer.length, flush=True)
        hidden = rand(n)
        if layer.length + n > layer.store.room:
            before = [_host(t.view(torch.uint8)).reshape(batch, layer.store.room, -1).copy()
                      for t in layer.store.arrays]
            length, store = layer.length, layer.store
            kept = _host(layer.evict())
            assert layer.store is not store and length > layer.budget
            after = [_host(t.view(torch.uint8)).reshape(batch, layer.store.room, -1) for t in layer.store.arrays]
            moved = np.zeros_like(total)
            for b in range(batch):
                assert (np.diff(kept[b]) > 0).all()
                assert kept[b, :4].tolist() == [0, 1, 2, 3] and kept[b, -1] == length - 1
                for old, new in zip(before, after):
                    assert np.array_equal(new[b, :layer.budget], old[b, kept[b]])
                moved[b, :layer.budget] = total[b, kept[b]]
            total, evicted = moved, evicted + 1
        want_residual = (hidden.float() + residual.float()).bfloat16()
        _, x = layer.rows(hidden, residual)
        pos = layer.length
        out, residual, idx = layer.step(hidden, residual)
        assert torch.equal(residual, want_residual)
        p, o = _weights(ex, layer, x, idx, pos)
        # weights of 16 bits and an output of 8: 2^-8 of the largest term, doubled
        assert np.abs(_host(out.float()) - o).max() <= 2.0 ** -7 * np.abs(o).max() + 2.0 ** -7
        at = _host(idx)
        for b in range(batch):
            for i in range(n):
                ok = at[b, i] >= 0
                np.add.at(total[b], at[b, i][ok], p[b, i].sum(0)[ok])
        # a step adds n * heads weights of relative error 2^-16 at most
        assert np.abs(_host(layer.acc) - total).max() <= 1e-4 * ex.HEADS * n
    assert evicted >= 1
