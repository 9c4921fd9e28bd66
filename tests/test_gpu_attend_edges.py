"""GPU tests of the attention over the 4-bit cache (and of the cache) at the edges
of their inputs, against plain definitions in 64 bits (ops_ref): empty index
sets."""
import numpy as np
import pytest
import torch

import paper_2607_24593_amd as pv
from gpu_util import dev, host, say
from test_gpu_operators import Pool, _queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("with_acc", [False, True])
def test_attend_to_sets_without_entries(packed, with_acc):
    """Index sets of no entries: nothing to attend to, which is not the prefix."""
    rng = np.random.default_rng(71)
    pool = Pool([50, 64], 16, rng)
    q = torch.from_numpy(_queries((2, 3, 16), rng)).bfloat16().cuda()
    idx = torch.empty((2, 3, 0), dtype=torch.int32, device="cuda")
    acc0 = rng.random((2, 64)).astype(np.float32)
    acc = dev(acc0) if with_acc else None
    kw = dict(cu_q=[0, 3, 6]) if packed else {}
    if packed:
        q, idx = q.view(6, 16, 576), idx.view(6, 0)
    say("attend to sets without entries", packed, with_acc)
    out, lse = pv.pivot_cache4_attend(q, pool.cache, [47, 61], [50, 64], 0.04, idx=idx, acc=acc, **kw)
    assert not host(out.float()).any() and np.isneginf(host(lse)).all()
    assert acc is None or np.array_equal(host(acc), acc0)
