"""GPU tests that the attention for trees of drafted tokens gives the same bits every
time, whatever its workspace held before and whatever ran in between."""
import numpy as np
import pytest
import torch

import draft_ref as plain
import paper_2607_24593_amd as pv
from gpu_util import dev, say
from test_gpu_operators import Pool, _queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,base,nodes,page,topk", [
    (16, [9000, 300, 4100], 12, 64, 0), (128, [20000], 26, 0, 0), (32, [300 + 40 * i for i in range(32)], 7, 16, 0),
    (128, [6000], 26, 0, 512), (16, [2000, 900], 12, 64, 300), (2, [5], 3, 0, 0), (64, [700, 1500], 40, 16, 0)])
@pytest.mark.parametrize("with_acc", [False, True])
def test_same_bits(heads, base, nodes, page, topk, with_acc):
    rng = np.random.default_rng(heads + nodes + topk)
    lens = [n + nodes for n in base]
    pool = Pool(lens, page, rng)
    mask = torch.from_numpy(np.stack([plain.tree_masks(rng, nodes)[1] for _ in base]).view(np.int32)).cuda()
    q = [torch.from_numpy(_queries((len(lens), nodes, heads), rng)).bfloat16().cuda() for _ in range(2)]
    idx = None
    if topk:
        idx = dev(np.stack([np.stack([rng.permutation(n)[:topk] for _ in range(nodes)]) for n in lens]).astype(np.int32))
    ws = torch.empty(1 << 30, dtype=torch.uint8, device="cuda")

    def run(i, fill):
        ws.view(torch.int32).fill_(fill)
        acc = torch.zeros((len(lens), max(lens)), device="cuda") if with_acc else None
        out, lse = pv.pivot_cache4_attend(q[i], pool.cache, base, lens, 0.04, idx=idx, acc=acc, tree=mask, ws=ws)
        return (out, lse) if acc is None else (out, lse, acc)

    say("tree, same bits", heads, base[:3], nodes, page, topk, with_acc)
    first = run(0, 0)
    assert all(torch.isfinite(t.float()).all() for t in first)
    for fill in (-1, 0x7F800000, 0x3F800000, 0x7149F2CA, 0):   # NaN, infinity, 1, 1e30
        run(1, fill)
        for _ in range(2):
            assert all(torch.equal(a, b) for a, b in zip(run(0, fill), first))
