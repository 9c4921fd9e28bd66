"""GPU tests of the attention over the 4-bit cache: calls that are cut into several
launches, and the precision of its weights, against definitions in 64 bits.  The
outputs' bound is ops_edges.out_bound; a score is off by at most E = 2^-18 * scale *
max_s sum |q k|, lse by E + 4 u (1 + |lse|) + u, u = 2^-24; a token's weight by
2 E + 2^-19 of each weight added to it, and 2^-24 of the sum for each addition."""
import math

import numpy as np
import pytest
import torch

import ops_ref as ref
import paper_2607_24593_amd as pv
from gpu_util import dev, host, say
from ops_edges import cancelling_pairs, out_bound
from test_gpu_operators import Pool

pytestmark = pytest.mark.gpu


def test_attend_prefix_cut_between_launches():
    """Kept scores of 302 rows of 128 heads on 8000 tokens pass 1 GiB, so the call
    is cut inside its second sequence: every row, and the weights of all."""
    rng = np.random.default_rng(101)
    lens, pos0, cu, heads, scale = [40, 8000], [30, 7690], [0, 2, 302], 128, 0.04
    assert 262 * 8000 * heads * 4 < 1 << 30 < 300 * 8000 * heads * 4
    pool = Pool(lens, 16, rng)
    g = torch.Generator(device="cuda").manual_seed(7)
    q = (2 * torch.randn((302, heads, 576), generator=g, device="cuda")).bfloat16()
    acc0 = rng.random((2, 8000)).astype(np.float32)
    acc = dev(acc0)
    say("attend prefix cut between launches")
    out, lse = pv.pivot_cache4_attend(q, pool.cache, pos0, lens, scale, cu_q=cu, acc=acc)
    got = host(acc).astype(np.float64)
    u = 2.0 ** -24
    for b in range(2):
        size = pos0[b] + cu[b + 1] - cu[b]
        latent, rope = pool.tokens(b, size)
        latent = torch.from_numpy(latent).cuda()
        key = torch.cat((latent, torch.from_numpy(rope).cuda()), 1)
        total, slack = (torch.zeros(size, dtype=torch.float64, device="cuda") for _ in range(2))
        for r in range(cu[b], cu[b + 1]):
            n = pos0[b] + r - cu[b] + 1
            qr = q[r].double()
            z = scale * (qr @ key[:n].T)
            E = 2.0 ** -18 * scale * (qr.abs() @ key[:n].abs().T).amax(-1)
            l = torch.logsumexp(z, -1)
            p = torch.exp(z - l[:, None])
            o, spread = p @ latent[:n], p @ latent[:n].abs()
            assert bool(((lse[r].double() - l).abs() <= E + 4 * u * (1 + l.abs()) + u).all()), r
            tol = 2.0 ** -8 * o.abs() + (2.0 ** -16 + (n / 8 + 16) * 2.0 ** -23 + 2 * E + 2.0 ** -21)[:, None] * spread
            assert bool(((out[r].double() - o).abs() <= tol).all()), r
            total[:n] += p.sum(0)
            slack[:n] += (2 * E.max() + 2.0 ** -19) * p.sum(0)
        want = total.cpu().numpy() + acc0[b, :size]
        tol = slack.cpu().numpy() + ((cu[b + 1] - cu[b]) * heads + 8) * u * want
        assert np.all(np.abs(got[b, :size] - want) <= tol), b
        assert np.array_equal(got[b, size:], acc0[b, size:].astype(np.float64))


def test_attend_sets_cut_between_launches():
    """More than 16384 query rows: cut inside the second sequence."""
    rng = np.random.default_rng(102)
    lens, pos0, cu, topk, scale = [70, 16700], [10, 100], [0, 50, 16600], 8, 0.04
    pool = Pool(lens, 0, rng)
    rows = cu[-1]
    at = np.concatenate([pos0[b] + np.arange(cu[b + 1] - cu[b]) for b in range(2)])
    start, step = rng.integers(0, at + 1), rng.integers(1, (at + 1) // topk + 1)
    idx = ((start[:, None] + np.arange(topk) * step[:, None]) % (at + 1)[:, None]).astype(np.int32)
    idx[::7, 3] = -1
    idx[5::11, 2] = at[5::11] + 1  # past the row's own position
    g = torch.Generator(device="cuda").manual_seed(8)
    q = (2 * torch.randn((rows, 1, 576), generator=g, device="cuda")).bfloat16()
    acc0 = rng.random((2, 16700)).astype(np.float32)
    acc = dev(acc0)
    say("attend sets cut between launches")
    out, lse = pv.pivot_cache4_attend(q, pool.cache, pos0, lens, scale, cu_q=cu, idx=dev(idx), acc=acc)
    got = host(acc).astype(np.float64)
    u = 2.0 ** -24
    for b in range(2):
        latent, rope = (torch.from_numpy(t).cuda() for t in pool.tokens(b, lens[b]))
        total, slack = (torch.zeros(lens[b], dtype=torch.float64, device="cuda") for _ in range(2))
        for lo in range(cu[b], cu[b + 1], 4096):
            hi = min(lo + 4096, cu[b + 1])
            s = torch.from_numpy(idx[lo:hi]).cuda().long()
            ok = (s >= 0) & (s <= torch.from_numpy(at[lo:hi]).cuda()[:, None])
            s = s.clamp(0, lens[b] - 1)
            v = latent[s]
            prod = q[lo:hi].double() * torch.cat((v, rope[s]), -1)
            z = (scale * prod.sum(-1)).masked_fill(~ok, -math.inf)
            E = 2.0 ** -18 * scale * prod.abs().sum(-1).amax(-1)
            l = torch.logsumexp(z, -1)
            p = torch.exp(z - l[:, None])
            o, spread = (p[..., None] * v).sum(1), (p[..., None] * v.abs()).sum(1)
            assert bool(((lse[lo:hi, 0].double() - l).abs() <= E + 4 * u * (1 + l.abs()) + u).all()), (b, lo)
            tol = 2.0 ** -8 * o.abs() + (2.0 ** -16 + 18 * 2.0 ** -23 + 2 * E + 2.0 ** -21)[:, None] * spread
            assert bool(((out[lo:hi, 0].double() - o).abs() <= tol).all()), (b, lo)
            total.index_add_(0, s.reshape(-1), p.reshape(-1))
            slack.index_add_(0, s.reshape(-1), ((2 * E + 2.0 ** -19)[:, None] * p).reshape(-1))
        want = total.cpu().numpy() + acc0[b, :lens[b]]
        tol = slack.cpu().numpy() + (cu[b + 1] - cu[b] + 8) * u * want
        assert np.all(np.abs(got[b, :lens[b]] - want) <= tol), b
        assert np.array_equal(got[b, lens[b]:], acc0[b, lens[b]:].astype(np.float64))


@pytest.mark.parametrize("heads", [16, 32, 64, 128])
def test_attend_weights_of_16_bits(heads):
    """Sets of pairs of tokens whose weights stand 3 : 2 and whose values 2 : -3, so
    that the outputs are nearly 0 and nothing hides an error of the weights: 2/3
    in one bf16 would be off by 2^-9.6.  With 40 queries the workgroups have as
    many rows as there are heads."""
    rng = np.random.default_rng(111)
    n_q, topk, size = 40, 512, 760
    pool = Pool([size], 16, rng)
    pool.codes, pool.scales, pool.rope = cancelling_pairs(pool.rows, rng)
    pool.upload()
    q = np.zeros((n_q, heads, 576))
    q[..., 512] = 1
    scale = float(np.float32(math.log(1.5)))
    pos0 = size - n_q
    pairs = np.arange(pos0).reshape(-1, 2)  # pages hold whole pairs
    idx = np.stack([rng.permutation(pairs[rng.permutation(len(pairs))[:topk // 2]].reshape(-1)) for _ in range(n_q)])
    say("attend weights of 16 bits", heads)
    out, lse = pv.pivot_cache4_attend(torch.from_numpy(q).bfloat16().cuda()[None], pool.cache, [pos0], [size], scale,
                                      idx=dev(idx.astype(np.int32))[None])
    out = out[0].double().cpu().numpy()
    latent, rp = pool.tokens(0, size)
    for r in range(n_q):
        allowed = np.zeros(size, bool)
        allowed[idx[r]] = True
        o, l, _, bound, spread = ref.attend_rows(q[r], latent, rp, scale, allowed)
        E = 2.0 ** -18 * bound
        assert np.abs(o).max() < 1e-5 * spread.min()
        assert np.all(np.abs(out[r] - o) <= out_bound(o, spread, E, topk)), (r, (np.abs(out[r] - o) / spread).max())
