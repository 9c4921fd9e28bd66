"""GPU tests of the acceptance that moves the nodes' weights with their rows, alone and
between the attention that adds the weights up and the eviction that ranks by them."""
import numpy as np
import pytest
import torch

import draft_ref as plain
import ops_ref as ref
import paper_2607_24593_amd as pv
from gpu_util import dev, host, say
from test_gpu_operators import Pool, _queries

pytestmark = pytest.mark.gpu


def _accepted(path, nodes, held=lambda node, j: True):
    """The nodes of a path up to where it ends."""
    out = []
    for j, v in enumerate(path):
        if v < j or v >= nodes or (out and v <= out[-1]) or not held(v, j):
            break
        out.append(int(v))
    return out


def _moved(acc, pos, nodes, kept):
    acc = acc.copy()
    acc[pos:pos + nodes] = np.concatenate([acc[pos + np.array(kept, int)], np.zeros(nodes - len(kept), acc.dtype)])
    return acc


@pytest.mark.parametrize("batch,base,nodes,n,page", [(1, 0, 1, 1, 0), (1, 5, 3, 2, 0), (3, 30, 64, 9, 16), (4, 100, 40, 40, 0),
                                                     (2, 15, 1024, 1024, 32), (130, 17, 12, 5, 16), (3, 0, 1000, 7, 64),
                                                     (2, 9, 0, 3, 0), (3, 20, 50, 0, 16)])
def test_weights_move_with_the_rows(batch, base, nodes, n, page):
    rng = np.random.default_rng(batch + nodes)
    pos0 = [base + i % 4 for i in range(batch)]
    trees = [max(0, nodes - i % 3) for i in range(batch)]
    pool = Pool([p + nodes for p in pos0], page, rng)
    path = np.full((batch, n), -1, np.int32)
    for b in range(batch):
        k = int(rng.integers(0, min(n, trees[b]) + 1)) if b != 1 else min(n, trees[b])
        path[b, :k] = np.sort(rng.choice(trees[b], k, replace=False)) if k else path[b, :k]
    x = torch.from_numpy(rng.integers(0, 256, (pool.rows, 20), dtype=np.uint8)).cuda()
    acc0 = rng.random((batch + 1, max(pos0) + nodes + 3)).astype(np.float32)
    acc, want, rows = dev(acc0), acc0.copy(), x.cpu().clone()
    for b in range(batch):
        kept = _accepted(path[b], trees[b])
        want[b] = _moved(acc0[b], pos0[b], trees[b], kept)
        for j, v in enumerate(kept):
            rows[int(pool.row(b, pos0[b] + j))] = rows[int(pool.row(b, pos0[b] + v))].clone()
    say("accept with weights", batch, base, nodes, n, page)
    pv.pivot_tree_accept(dev(path), pos0, [x], pool.map, acc=acc, nodes=trees)
    assert np.array_equal(host(acc), want) and torch.equal(x.cpu(), rows)


def test_weights_and_rows_end_at_one_place():
    """Entries that are no nodes of the tree, that do not go up, or lie where there is no
    page: rows and weights move up to the same one."""
    rng = np.random.default_rng(6)
    page, nodes = 16, 30
    pool = Pool([96] * 6, page, rng)
    path = np.array([[1, 3, 20, 21], [1, 3, 30, 31], [2, 7, 7, 9], [0, 1, 2, 3], [-5, 1, 2, 3], [2**31 - 1, 2, 3, 4]], np.int32)
    pos0 = [14, 14, 30, 16, 0, 5]
    pool.table[0, 2] = -1      # positions 32 .. 47: node 20
    pool.table[3, 1] = pool.rows // page
    pool.upload()
    ok = (pool.table >= 0) & (pool.table < pool.rows // page)
    x = torch.from_numpy(rng.integers(0, 256, (pool.rows, 16), dtype=np.uint8)).cuda()
    acc0 = rng.random((6, 96)).astype(np.float32)
    acc, want, rows = dev(acc0), acc0.copy(), x.cpu().clone()
    lengths = []
    for b in range(6):
        kept = _accepted(path[b], nodes, lambda v, j: ok[b, (pos0[b] + v) // page] and ok[b, (pos0[b] + j) // page])
        lengths.append(len(kept))
        want[b] = _moved(acc0[b], pos0[b], nodes, kept)
        for j, v in enumerate(kept):
            rows[int(pool.row(b, pos0[b] + j))] = rows[int(pool.row(b, pos0[b] + v))].clone()
    assert lengths == [2, 2, 2, 0, 0, 0]
    say("accept with weights, paths that end")
    pv.pivot_tree_accept(dev(path), pos0, [x], pool.map, acc=acc, nodes=[nodes] * 6)
    assert np.array_equal(host(acc), want) and torch.equal(x.cpu(), rows)


def test_accept_with_weights_in_a_graph():
    rng = np.random.default_rng(8)
    pool = Pool([60, 70], 16, rng)
    paths = [np.array([[0, 4, 9], [2, 3, -1]], np.int32), np.array([[-1, -1, -1], [1, 5, 11]], np.int32)]
    acc0 = rng.random((2, 90)).astype(np.float32)
    acc, path = dev(acc0), dev(paths[0])
    x = torch.zeros((pool.rows, 16), dtype=torch.uint8, device="cuda")
    say("accept with weights, graph")
    pv.pivot_tree_accept(path, [40, 50], [x], pool.map, acc=acc, nodes=[20, 12])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pv.pivot_tree_accept(path, [40, 50], [x], pool.map, acc=acc, nodes=[20, 12])
    for i in range(4):
        acc.copy_(dev(acc0))
        path.copy_(dev(paths[i % 2]))
        graph.replay()
        torch.cuda.synchronize()
        want = np.stack([_moved(acc0[b], p, m, _accepted(paths[i % 2][b], m)) for b, (p, m) in enumerate([(40, 20), (50, 12)])])
        assert np.array_equal(host(acc), want)


@pytest.mark.parametrize("heads,page,topk", [(16, 16, 0), (5, 0, 0), (16, 16, 60), (128, 32, 90)])
def test_attention_acceptance_and_eviction(heads, page, topk):
    """Two steps with drafts, the weights added up, the accepted nodes moved, and the
    eviction ranking by what the tokens that stayed were given."""
    rng = np.random.default_rng(heads + topk)
    base, nodes, batch = [70, 33], 21, 2
    room = [n + 2 * nodes + 10 for n in base]
    pool = Pool(room, page, rng)
    acc = torch.zeros((batch, max(room)), device="cuda")
    total, slack = np.zeros((batch, max(room))), np.zeros((batch, max(room)))
    length = list(base)
    for step in range(2):
        trees = [plain.tree_masks(rng, nodes) for _ in base]
        mask = torch.from_numpy(np.stack([t[1] for t in trees]).view(np.int32)).cuda()
        q = _queries((batch * nodes, heads), rng)
        lens = [n + nodes for n in length]
        idx = None
        if topk:
            idx = np.stack([rng.permutation(max(lens))[:topk] for _ in range(batch * nodes)]).astype(np.int32)
        say("attention, acceptance, eviction", heads, page, topk, step)
        pv.pivot_cache4_attend(torch.from_numpy(q).bfloat16().cuda().view(batch, nodes, heads, 576), pool.cache, length, lens,
                               0.04, acc=acc, tree=mask, idx=None if idx is None else dev(idx).view(batch, nodes, topk))
        paths = np.full((batch, 6), -1, np.int32)
        for b in range(batch):
            latent, rope = pool.tokens(b, lens[b])
            for i in range(nodes):
                may = np.concatenate([np.ones(length[b], bool), trees[b][0][i]])
                if idx is not None:
                    s = idx[b * nodes + i]
                    chosen = np.zeros_like(may)
                    chosen[s[s < lens[b]]] = True
                    may &= chosen
                _, _, w, bound, _ = ref.attend_rows(q[b * nodes + i], latent, rope, 0.04, may)
                E = 2.0 ** -18 * bound
                total[b, :lens[b]] += w
                slack[b, :lens[b]] += (2 * E.max() + 2.0 ** -19) * w + 2.0 ** -22 * w
            k = 3 + b
            paths[b, :k] = np.sort(rng.choice(np.arange(1, nodes), k, replace=False))
        pv.pivot_tree_accept(dev(paths), length, pool.parts, pool.map, acc=acc, nodes=[nodes] * batch)
        still = total.copy()
        for b in range(batch):
            kept = _accepted(paths[b], nodes)
            total[b] = _moved(total[b], length[b], nodes, kept)
            slack[b] = _moved(slack[b], length[b], nodes, kept)
        for t, name in zip(pool.parts, ("codes", "scales", "rope")):
            setattr(pool, name, t.double().cpu().numpy() if name == "rope" else host(t).copy())
        length = [n + 3 + b for b, n in enumerate(length)]
        got = host(acc).astype(np.float64)
        tol = slack + 2.0 ** -22 * total + 1e-30
        assert np.all(np.abs(got - total) <= tol)
        # weights left where they were added would lie outside
        assert np.any(np.abs(still - total) > 4 * tol)
        assert not got[0, length[0]:].any() and not got[1, length[1]:].any()
    keep = 40
    say("eviction by weights of drafts")
    kept, out_acc = pv.pivot_evict(acc, length, keep, [], None, None, sink=2, recent=4)
    for b, n in enumerate(length):
        want = ref.evict(got[b].astype(np.float32), n, keep, 2, 4)
        assert host(kept)[b, :len(want)].tolist() == want
        # by the plain sums the tokens that go weigh no more than those that stay, but for the bounds
        gone = np.setdiff1d(np.arange(2, n - 4), want)
        stay = np.setdiff1d(want, np.concatenate([[0, 1], np.arange(n - 4, n)])).astype(int)
        if len(gone) and len(stay):
            assert (total[b, gone] - tol[b, gone]).max() <= (total[b, stay] + tol[b, stay]).min()
