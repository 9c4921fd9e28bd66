"""GPU tests that copies of pages write nothing beside the pages they name: what lies
before, behind and between stays byte for byte."""
import numpy as np
import pytest
import torch

import paper_2607_24593_amd as pv
from gpu_util import dev, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,width,n_pages", [(16, 12, 5), (16, 4, 9), (32, 132, 7), (64, 16, 40), (4096, 20, 6), (16, 400, 300)])
@pytest.mark.parametrize("at", [4, 8, 16, 1024])
def test_copies_stay_within_their_pages(page, width, n_pages, at):
    """Arrays inside larger ones, from addresses that are multiples of 4 only and of 16."""
    rng = np.random.default_rng(page + width)
    size = n_pages * page * width
    backing = [torch.from_numpy(rng.integers(0, 256, at + size + 64, dtype=np.uint8)).cuda() for _ in range(2)]
    arrays = [t[at:at + size].view(n_pages * page, width) for t in backing]
    place = rng.permutation(n_pages)
    pairs = place[:n_pages // 2 * 2].reshape(-1, 2).astype(np.int32)
    pairs[0] = -1
    want = [t.cpu().clone() for t in backing]
    for w in want:
        rows = w[at:at + size].view(n_pages, page * width)
        for old, new in pairs[1:].tolist():
            rows[new] = rows[old].clone()
    assert len(pairs) > 1 and not all(torch.equal(w, t.cpu()) for w, t in zip(want, backing))
    table, refs = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((1, n_pages), (n_pages,)))
    say("pages, guards", page, width, n_pages, at)
    pv.pivot_pages_copy(pv.make_pages(table, refs, page), dev(pairs), arrays)
    for w, t in zip(want, backing):
        assert torch.equal(t.cpu(), w)
