"""GPU tests of attention for trees of drafted tokens, and of the acceptance of one
of their paths, against plain definitions in 64 bits.  Bounds as in
test_gpu_operators.py, the output's as in ops_edges.out_bound."""
import numpy as np
import pytest
import torch

import draft_ref as plain
import ops_ref as ref
import paper_2607_24593_amd as pv
from gpu_util import dev, host, say
from ops_edges import out_bound
from test_gpu_operators import Pool, _queries

pytestmark = pytest.mark.gpu


def _mask(words):
    return torch.from_numpy(np.ascontiguousarray(words).view(np.int32)).cuda()


def _check(pool, q, base, seen, scale, out, lse, idx=None, acc=None, acc0=None, only=None, label=""):
    """seen[b]: truth values [nodes, nodes] of sequence b.  Rows are packed."""
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    out, lse = out.reshape(-1, *out.shape[-2:]), lse.reshape(-1, lse.shape[-1])
    u, r = 2.0 ** -24, 0
    for b, mine in enumerate(seen):
        n = len(mine)
        if n == 0:
            continue
        if only is not None and b not in only:
            r += n
            continue
        size = base[b] + n
        latent, rope = pool.tokens(b, size)
        total, slack = np.zeros(size), np.zeros(size)
        for i in range(n):
            allowed = np.zeros(size, dtype=bool)
            may = np.concatenate([np.ones(base[b], dtype=bool), mine[i]])
            if idx is None:
                allowed = may
            else:
                s = idx[r][(idx[r] >= 0) & (idx[r] < size)]
                allowed[s] = may[s]
            o, l, w, bound, spread = ref.attend_rows(q[r], latent, rope, scale, allowed)
            E = 2.0 ** -18 * bound
            fin = np.isfinite(l)
            assert np.array_equal(np.isnan(out[r]).any(-1), np.isnan(l)), (label, r)
            assert np.array_equal(lse[r][~fin & ~np.isnan(l)], l[~fin & ~np.isnan(l)]), (label, r)
            assert np.all(np.abs(lse[r] - l)[fin] <= (E + 4 * u * (1 + np.abs(l)) + u)[fin]), (label, r)
            tol = out_bound(o, spread, E, allowed.sum()) + 1e-30
            off = np.abs(out[r] - o)
            assert np.all(off[fin] <= tol[fin]), (label, r, (off / tol)[fin].max())
            assert not out[r][~fin & ~np.isnan(l)].any()
            total += w
            slack += (2 * E.max() + 2.0 ** -19) * w
            r += 1
        if acc is not None:
            want, got = total + acc0[b, :size], acc[b, :size].astype(np.float64)
            assert np.array_equal(np.isnan(got), np.isnan(want)), label
            ok = ~np.isnan(want)
            assert np.all(np.abs(got - want)[ok] <= (slack + 2.0 ** -22 * np.abs(want) + 1e-30)[ok]), (label, b)
            assert np.array_equal(acc[b, size:], acc0[b, size:])


PREFIX = [
    # heads, base, nodes, page, words (0: as many as the nodes need)
    (1, [0], 1, 0, 0), (1, [1], 2, 0, 0), (3, [31], 5, 0, 2), (16, [33, 0, 64], 7, 16, 0), (5, [200], 33, 32, 0),
    (40, [130, 65], 3, 16, 1), (128, [300], 1, 0, 0), (128, [520], 26, 64, 0), (64, [1030], 2, 0, 0), (16, [5000, 17], 4, 64, 0),
    (24, [900], 64, 0, 0), (128, [4100], 13, 16, 0), (4, [50] * 66, 9, 16, 0), (1, [70], 300, 0, 0), (2, [0], 1024, 0, 0),
    (16, [95], 1, 0, 32), (32, [0, 1, 2], 2, 16, 0),
]


@pytest.mark.parametrize("heads,base,nodes,page,words", PREFIX)
@pytest.mark.parametrize("with_acc", [False, True])
def test_tree_over_the_prefix(heads, base, nodes, page, words, with_acc):
    rng = np.random.default_rng(heads * 11 + nodes)
    lens = [n + nodes for n in base]
    pool = Pool(lens, page, rng)
    trees = [plain.tree_masks(rng, nodes, words) for _ in base]
    q = _queries((len(lens) * nodes, heads), rng)
    acc0 = rng.random((len(lens), max(lens) + 3)).astype(np.float32)
    acc = dev(acc0) if with_acc else None
    say("tree prefix", heads, base[:3], nodes, page, words, with_acc)
    qd = torch.from_numpy(q).bfloat16().cuda().view(len(lens), nodes, heads, 576)
    out, lse = pv.pivot_cache4_attend(qd, pool.cache, base, lens, 0.04, acc=acc, tree=_mask(np.stack([t[1] for t in trees])))
    _check(pool, q, base, [t[0] for t in trees], 0.04, out, lse, None, host(acc) if with_acc else None, acc0)


SETS = [
    # heads, base, nodes, topk, page
    (1, [0], 1, 1, 0), (3, [40], 4, 1, 0), (16, [40], 7, 31, 16), (17, [100, 33], 5, 32, 0), (32, [300], 40, 33, 64),
    (64, [257], 9, 97, 0), (65, [500], 3, 200, 32), (128, [700, 90], 12, 256, 16), (128, [3000], 3, 2048, 0),
    (16, [2500, 1200], 26, 512, 64), (8, [60] * 66, 4, 20, 16), (2, [10], 200, 100, 0), (100, [0], 30, 30, 0),
]


@pytest.mark.parametrize("heads,base,nodes,topk,page", SETS)
@pytest.mark.parametrize("with_acc", [False, True])
def test_tree_over_index_sets(heads, base, nodes, topk, page, with_acc):
    """Sets that hold prefix positions, ancestors, nodes that the row must not see,
    positions behind the tree, and padding, in any order."""
    rng = np.random.default_rng(heads * 13 + nodes)
    lens = [n + nodes for n in base]
    pool = Pool(lens, page, rng)
    trees = [plain.tree_masks(rng, nodes) for _ in base]
    idx = []
    for n in lens:
        for _ in range(nodes):
            s = np.concatenate([rng.permutation(n + 4), np.full(topk, -1)])[:topk]
            s[rng.random(topk) < 0.1] = -1
            idx.append(rng.permutation(s))
    idx = np.stack(idx).astype(np.int32)
    q = _queries((len(lens) * nodes, heads), rng)
    acc0 = rng.random((len(lens), max(lens) + 3)).astype(np.float32)
    acc = dev(acc0) if with_acc else None
    say("tree sets", heads, base[:3], nodes, topk, page, with_acc)
    qd = torch.from_numpy(q).bfloat16().cuda().view(len(lens), nodes, heads, 576)
    out, lse = pv.pivot_cache4_attend(qd, pool.cache, base, lens, 0.04, acc=acc, idx=dev(idx).view(len(lens), nodes, topk),
                                      tree=_mask(np.stack([t[1] for t in trees])))
    _check(pool, q, base, [t[0] for t in trees], 0.04, out, lse, idx, host(acc) if with_acc else None, acc0)


@pytest.mark.parametrize("sparse", [False, True])
@pytest.mark.parametrize("heads", [3, 24, 128])
def test_any_bits_empty_rows_and_packed_runs(sparse, heads):
    """Masks that are no tree: nothing at all, later nodes, all nodes, bits behind the
    last node; runs of different lengths, an empty one among them; more tokens in the
    cache than the tree's; heads of a wider projection."""
    rng = np.random.default_rng(heads)
    base, cu = [0, 40, 7, 150], [0, 5, 5, 38, 45]
    lens = [20, 60, 41, 157]
    pool = Pool(lens, 16, rng)
    seen, words = [], np.zeros((45, 3), dtype=np.uint32)
    for b in range(4):
        n = cu[b + 1] - cu[b]
        m = rng.random((n, n)) < 0.4
        if n:
            m[0], m[n - 1] = False, True
        seen.append(m)
        if n:
            noise = rng.random((n, 96)) < 0.5
            noise[:, :n] = m
            words[cu[b]:cu[b + 1]] = plain.pack_bits(noise, 3)
    wide = torch.from_numpy(rng.standard_normal((45, heads + 3, 640)) * 2).bfloat16().cuda()
    qd = wide[:, 1:1 + heads, 8:584]
    idx = np.stack([rng.permutation(160)[:48] for _ in range(45)]).astype(np.int32) if sparse else None
    acc0 = np.zeros((4, 157), np.float32)
    acc = dev(acc0)
    say("tree packed", sparse, heads)
    out, lse = pv.pivot_cache4_attend(qd, pool.cache, base, lens, 0.05, cu_q=cu, idx=dev(idx) if sparse else None, acc=acc,
                                      tree=_mask(words))
    _check(pool, qd.double().cpu().numpy(), base, seen, 0.05, out, lse, idx, host(acc), acc0)
    if not sparse:  # row 0 of sequence 0: no prefix, an empty mask
        assert not host(out[0].float()).any() and np.isneginf(host(lse[0])).all()


@pytest.mark.parametrize("heads", [2, 16, 64, 128])
def test_nodes_that_a_row_does_not_see_may_hold_anything(heads):
    rng = np.random.default_rng(17)
    base, nodes = [70], 20
    pool = Pool([90], 0, rng)
    seen, words = plain.tree_masks(rng, nodes)
    bad = [3, 11]
    pool.scales[pool.row(0, 73)] = 255
    pool.rope[pool.row(0, 81), 5] = np.inf
    pool.upload()
    q = _queries((nodes, heads), rng)
    acc0 = np.zeros((1, 90), np.float32)
    acc = dev(acc0)
    say("tree NaN", heads)
    out, lse = pv.pivot_cache4_attend(torch.from_numpy(q).bfloat16().cuda().view(1, nodes, heads, 576), pool.cache, base,
                                      [90], 0.04, acc=acc, tree=_mask(words[None]))
    nan = np.isnan(host(out.float()))[0].any((1, 2))
    clean = ~seen[:, bad].any(1)
    assert clean.sum() > 3 and not nan[clean].any() and nan[seen[:, 3]].all()
    got = out.double().cpu().numpy()[0]
    latent, rope = pool.tokens(0, 90)
    for i in np.nonzero(clean)[0]:
        allowed = np.concatenate([np.ones(70, bool), seen[i]])
        o, l, _, bound, spread = ref.attend_rows(q[i], latent, rope, 0.04, allowed)
        assert np.all(np.abs(got[i] - o) <= out_bound(o, spread, 2.0 ** -18 * bound, allowed.sum()) + 1e-30)
    only_clean = np.array([70 + j for j in range(nodes) if clean[seen[:, j]].all()])
    assert np.isfinite(host(acc)[0][only_clean]).all()


@pytest.mark.parametrize("heads,base,nodes", [(16, 500, 4), (128, 3000, 2), (3, 40, 70), (64, 0, 33)])
@pytest.mark.parametrize("sparse", [False, True])
def test_a_chain_is_the_causal_call(heads, base, nodes, sparse):
    rng = np.random.default_rng(heads + nodes)
    n = base + nodes
    pool = Pool([n], 16, rng)
    words = plain.pack_bits(np.tril(np.ones((nodes, nodes), bool)))
    qd = torch.from_numpy(_queries((1, nodes, heads), rng)).bfloat16().cuda()
    idx = dev(np.stack([rng.permutation(n)[:40] for _ in range(nodes)]).astype(np.int32))[None] if sparse else None
    accs = [torch.zeros((1, n), device="cuda") for _ in range(2)]
    say("tree chain", heads, base, nodes, sparse)
    a = pv.pivot_cache4_attend(qd, pool.cache, [base], [n], 0.04, idx=idx, acc=accs[0])
    b = pv.pivot_cache4_attend(qd, pool.cache, [base], [n], 0.04, idx=idx, acc=accs[1], tree=_mask(words[None]))
    E = 2.0 ** -10  # of two results that round alike but for where sums are cut
    assert torch.allclose(a[0].float(), b[0].float(), rtol=2.0 ** -7, atol=E) and torch.allclose(a[1], b[1], atol=E)
    assert torch.allclose(accs[0], accs[1], rtol=2.0 ** -10, atol=1e-6)


def test_a_sequence_cut_over_two_launches():
    """40 trees of 500 nodes: 20000 rows, the 33rd sequence's in two launches.  Its
    rows still see nodes of either part."""
    rng = np.random.default_rng(41)
    base, nodes = [20 + i % 3 for i in range(40)], 500
    lens = [n + nodes for n in base]
    pool = Pool(lens, 0, rng)
    seen = [rng.random((nodes, nodes)) < 0.3 for _ in base]
    words = np.stack([plain.pack_bits(m) for m in seen])
    q = _queries((40 * nodes, 1), rng)
    acc0 = np.zeros((40, max(lens)), np.float32)
    acc = dev(acc0)
    say("tree cut")
    out, lse = pv.pivot_cache4_attend(torch.from_numpy(q).bfloat16().cuda().view(40, nodes, 1, 576), pool.cache, base, lens,
                                      0.04, acc=acc, tree=_mask(words))
    _check(pool, q, base, seen, 0.04, out, lse, None, host(acc), acc0, only=(0, 31, 32, 33, 39))


def test_tree_in_a_graph():
    rng = np.random.default_rng(43)
    base, nodes, heads = [300, 77], 12, 16
    lens = [n + nodes for n in base]
    pool = Pool(lens, 16, rng)
    trees = [np.stack([plain.tree_masks(rng, nodes)[1] for _ in base]) for _ in range(3)]
    qs = [torch.from_numpy(_queries((2, nodes, heads), rng)).bfloat16().cuda() for _ in range(3)]
    say("tree graph")
    want = [pv.pivot_cache4_attend(q, pool.cache, base, lens, 0.04, tree=_mask(t)) for q, t in zip(qs, trees)]
    q, mask = qs[0].clone(), _mask(trees[0])
    out, lse = torch.empty_like(want[0][0]), torch.empty_like(want[0][1])
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pv.pivot_cache4_attend(q, pool.cache, base, lens, 0.04, tree=mask, out=out, lse=lse, ws=ws)
    for i in (1, 2, 0, 1):
        q.copy_(qs[i])
        mask.copy_(_mask(trees[i]))
        graph.replay()
        eager = pv.pivot_cache4_attend(qs[2 - i], pool.cache, base, lens, 0.04, tree=_mask(trees[2 - i]))
        torch.cuda.synchronize()
        assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1]) and torch.equal(eager[0], want[2 - i][0])


# ------------------------------------------------------------------ acceptance
def _path(rng, n, nodes, length):
    p = np.full(n, -1, dtype=np.int32)
    length = min(length, n, nodes)
    p[:length] = np.sort(rng.choice(nodes, length, replace=False))
    return p


@pytest.mark.parametrize("batch,base,nodes,n,page", [(1, 0, 1, 1, 0), (1, 5, 3, 2, 0), (3, 30, 64, 9, 16), (4, 100, 40, 40, 0),
                                                     (2, 15, 1024, 1024, 32), (130, 17, 12, 5, 16), (2, 60, 300, 17, 64)])
def test_accept(batch, base, nodes, n, page):
    rng = np.random.default_rng(batch * 3 + nodes)
    pos0 = [base + i % 4 for i in range(batch)]
    pool = Pool([p + nodes for p in pos0], page, rng)
    path = np.stack([_path(rng, n, nodes, int(rng.integers(0, n + 1))) for _ in range(batch)])
    if batch > 2:
        path[1] = -1
        k = min(n, nodes)
        path[2, :k] = np.arange(k)
    backing = torch.from_numpy(rng.integers(0, 256, pool.rows * 132 + 4, dtype=np.uint8)).cuda()
    arrays = [torch.from_numpy(rng.integers(0, 256, (pool.rows, w), dtype=np.uint8)).cuda() for w in (256, 16, 128, 4, 20)]
    arrays += [torch.from_numpy(rng.standard_normal((pool.rows, 64))).bfloat16().cuda(),
               torch.from_numpy(rng.standard_normal(pool.rows)).float().cuda(),
               backing[4:].view(pool.rows, 132)]  # 4-byte aligned only
    want = [x.cpu().clone() for x in arrays]
    for b in range(batch):
        for j, v in enumerate(path[b]):
            if v < 0:
                break
            for x in want:
                x[int(pool.row(b, pos0[b] + j))] = x[int(pool.row(b, pos0[b] + v))].clone()
    say("accept", batch, base, nodes, n, page)
    pv.pivot_tree_accept(dev(path), pos0, arrays, pool.map)
    for i, (x, y) in enumerate(zip(arrays, want)):
        assert torch.equal(x.cpu(), y), i


def test_paths_that_are_none():
    """An entry that does not go up, or names a position that the map cannot hold, ends
    the path; the rows before it move."""
    rng = np.random.default_rng(3)
    for page in (0, 16):
        pool = Pool([64] * 5, page, rng)
        cap = pool.table.shape[1] * page if page else pool.stride
        path = np.array([[2, 5, 4, 9], [1, 3, cap, 60], [0, 7, 7, 8], [3, 2**31 - 1, 9, 10], [5, -7, 20, 21]], np.int32)
        lengths = [2, 2, 2, 1, 1]
        pos0 = [10, 20, 30, 1, 40]
        x = torch.from_numpy(rng.integers(0, 256, (pool.rows, 48), dtype=np.uint8)).cuda()
        want = x.cpu().clone()
        for b, k in enumerate(lengths):
            for j in range(k):
                want[int(pool.row(b, pos0[b] + j))] = want[int(pool.row(b, pos0[b] + path[b, j]))].clone()
        say("accept, paths that end", page)
        pv.pivot_tree_accept(dev(path), pos0, [x], pool.map)
        assert torch.equal(x.cpu(), want)


def test_paths_stop_at_pages_that_are_none():
    """A position whose table entry names no page ends the path, read or written: no
    row of another sequence's page changes."""
    rng = np.random.default_rng(5)
    page = 16
    pool = Pool([96] * 5, page, rng)
    n_pages = pool.rows // page
    path = np.array([[1, 3, 20, 21], [1, 3, 20, 21], [2, 7, 8, 9], [0, 1, 2, 3], [1, 30, 50, 51]], np.int32)
    pos0 = [14, 14, 30, 16, 0]
    lengths = [2, 4, 0, 0, 1]
    pool.table[0, 2] = -1  # of positions 32 .. 47: node 20 of the first tree
    pool.table[2, 1] = n_pages  # 16 .. 31: the tree's first position
    pool.table[3, 1] = -2**31
    pool.table[4, 1] = 2**31 - 1  # 16 .. 31: node 30
    pool.upload()
    x = torch.from_numpy(rng.integers(0, 256, (pool.rows, 16), dtype=np.uint8)).cuda()
    want = x.cpu().clone()
    for b, k in enumerate(lengths):
        for j in range(k):
            want[int(pool.row(b, pos0[b] + j))] = want[int(pool.row(b, pos0[b] + path[b, j]))].clone()
    say("accept, pages that are none")
    pv.pivot_tree_accept(dev(path), pos0, [x], pool.map)
    assert torch.equal(x.cpu(), want)
