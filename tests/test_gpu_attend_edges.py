"""GPU tests of the attention over the 4-bit cache (and of the cache) at the edges
of their inputs, against plain definitions in 64 bits (ops_ref): empty index
sets, rows of NaN."""
import numpy as np
import pytest
import torch

import ops_ref as ref
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


@pytest.mark.parametrize("heads", [3, 16, 64, 128])
def test_attend_weights_of_a_nan_row_end_at_its_position(heads):
    """Over a prefix a row adds to the weights of the tokens up to its own: a row
    of NaN makes those NaN and leaves the later ones as the other rows add them."""
    rng = np.random.default_rng(heads)
    lens, pos0, n = [230, 40], [188, 30], 7
    pool = Pool(lens, 16, rng)
    q = _queries((2 * n, heads), rng)
    q[2, heads - 1, 100] = np.nan
    acc0 = rng.random((2, 233)).astype(np.float32)
    acc = dev(acc0)
    say("attend weights of a NaN row", heads)
    qd = torch.from_numpy(q).bfloat16().cuda().view(2, n, heads, 576)
    pv.pivot_cache4_attend(qd, pool.cache, pos0, lens, 0.04, acc=acc)
    got = host(acc).astype(np.float64)
    for b in range(2):
        size = pos0[b] + n
        latent, rope = pool.tokens(b, size)
        total, slack = np.zeros(size), np.zeros(size)
        for i in range(n):
            if b == 0 and i == 2:
                total[:pos0[0] + 3] = np.nan
                continue
            _, _, w, bound, _ = ref.attend_rows(q[b * n + i], latent, rope, 0.04, np.arange(size) <= pos0[b] + i)
            total += w
            slack += (2.0 ** -17 * bound.max() + 2.0 ** -19) * w
        assert np.array_equal(np.isnan(got[b, :size]), np.isnan(total)), np.flatnonzero(np.isnan(got[b]))
        ok = ~np.isnan(total)
        want = total + acc0[b, :size]
        tol = slack + (n * heads + 8) * 2.0 ** -24 * want
        assert np.all(np.abs(got[b, :size] - want)[ok] <= tol[ok])
        assert np.array_equal(host(acc)[b, size:], acc0[b, size:])
