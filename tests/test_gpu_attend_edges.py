"""GPU tests of the attention over the 4-bit cache (and of the cache) at the edges
of their inputs, against plain definitions in 64 bits (ops_ref): empty index
sets, rows of NaN, infinities in masked places, the ends of bf16, strides of
single queries."""
import numpy as np
import pytest
import torch

import ops_ref as ref
import paper_2607_24593_amd as pv
from gpu_util import dev, host, say
from ops_edges import out_bound
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


@pytest.mark.parametrize("heads", [8, 32, 64, 128])
def test_attend_infinite_values_reach_only_their_readers(heads):
    """Values that bf16 cannot hold (codes times 2^126 or 2^127 of 2^128 or more)
    in tokens that a row does not attend to, and in token 0, whose row stands in
    for masked keys; the largest values that bf16 holds stay exact."""
    rng = np.random.default_rng(81)
    pool = Pool([200], 16, rng)
    at = pool.row(0, np.arange(200))
    n = 4
    clean = pool.codes.copy(), pool.scales.copy()

    def call(pos0, idx=None, q=None):
        pool.upload()
        q = _queries((n, heads), rng) if q is None else q
        say("attend infinite values", heads, pos0, idx is not None)
        out, lse = pv.pivot_cache4_attend(torch.from_numpy(q).bfloat16().cuda()[None], pool.cache, [pos0], [200], 0.04,
                                          idx=None if idx is None else dev(idx)[None])
        return q, out[0].double().cpu().numpy(), host(lse)[0]

    def check(q, out, lse, r, allowed):
        latent, rope = pool.tokens(0, 200)
        o, l, _, bound, spread = ref.attend_rows(q[r], latent, rope, 0.04, allowed)
        E = 2.0 ** -18 * bound
        assert np.all(np.abs(out[r] - o) <= out_bound(o, spread, E, 200)), r
        assert np.all(np.abs(lse[r] - l) <= E + 2.0 ** -22 * (1 + np.abs(l)) + 2.0 ** -24), r

    def plant(token, byte, code):
        pool.scales[at[token], 2] = byte
        pool.codes[at[token], 32:48] = code * 17

    # later tokens of the same tile; row 0 (position 100) sees none of them
    for token, byte, code in ((101, 254, 7), (102, 253, 6), (103, 254, 4 + 8), (110, 253, 7 + 8)):
        plant(token, byte, code)
    q, out, lse = call(100)
    check(q, out, lse, 0, np.arange(200) <= 100)
    assert np.isnan(out[1:]).all()
    # an infinity in token 0, and sets with padding that do not hold it
    plant(0, 253, 6)
    idx = np.full((n, 40), -1, np.int32)
    for r in range(n):
        idx[r, rng.permutation(40)[:9]] = 1 + rng.permutation(90)[:9]
    idx[3, np.flatnonzero(idx[3] < 0)[0]] = 0
    q, out, lse = call(100, idx)
    for r in range(3):
        allowed = np.zeros(200, bool)
        allowed[idx[r][idx[r] >= 0]] = True
        check(q, out, lse, r, allowed)
    assert np.isnan(out[3]).all()
    # 3 * 2^126 and 1.5 * 2^127 are bf16 values, attended with scores of ordinary size
    pool.codes, pool.scales = clean
    plant(20, 253, 5)
    plant(21, 254, 3 + 8)
    q = _queries((n, heads), rng)
    q[..., 64:96] = 0
    q, out, lse = call(60, q=q)
    for r in range(n):
        check(q, out, lse, r, np.arange(200) <= 60 + r)


def test_cache_values_at_the_ends_of_bf16():
    """Subnormal blocks are read back exactly as quantised; the top half-step of
    the largest values, which bf16 cannot hold once quantised, as infinities."""
    rng = np.random.default_rng(82)
    x = np.zeros((40, 512))
    for r in range(40):  # magnitudes from 2^-133 (the least subnormal) to 2^-124
        x[r] = np.ldexp(rng.integers(-127, 128, 512).astype(float), -133 - int(rng.integers(0, 4)) + r // 8)
    x = ref.bf16(x)
    x[39, :4] = np.ldexp([3.4375, -3.4375, 3.5, -3.96875], 126)
    parts = (torch.zeros((40, 256), dtype=torch.uint8, device="cuda"), torch.zeros((40, 16), dtype=torch.uint8, device="cuda"),
             torch.zeros((40, 64), dtype=torch.bfloat16, device="cuda"))
    c = pv.make_cache4(*parts, pv.make_row_map(seq_stride=40, rows=40))
    say("cache ends of bf16")
    pv.pivot_cache4_write(torch.from_numpy(x).bfloat16().cuda(), torch.zeros((40, 64), dtype=torch.bfloat16, device="cuda"), c,
                          [0], 40)
    codes, scales = ref.quantise(x)
    assert np.array_equal(host(parts[1]), scales)
    want = ref.values(codes, scales)
    assert np.array_equal(ref.values(host(parts[0]), scales), want)
    back = pv.pivot_cache4_read(c, torch.arange(40, dtype=torch.int32, device="cuda")[None]).double().cpu().numpy()[0, :, :512]
    want[39, 2:4] = [np.inf, -np.inf]  # 4 * 2^126
    assert want[39, 0] == 3 * 2.0 ** 126 and np.array_equal(back, want)


@pytest.mark.parametrize("layout", ["slice", "heads first"])
def test_attend_single_queries_of_a_wider_tensor(layout):
    """One query a sequence: its dimension's stride has no meaning."""
    rng = np.random.default_rng(91)
    lens, heads = [70, 33, 50, 64], 16
    pool = Pool(lens, 16, rng)
    if layout == "slice":
        wide = torch.from_numpy(_queries((4, 3, heads), rng)).bfloat16().cuda()
        q = wide[:, 1:2]
    else:
        wide = torch.from_numpy(_queries((4, heads, 1), rng)).bfloat16().cuda()
        q = wide.transpose(1, 2)
    say("attend single queries", layout, tuple(q.stride()))
    want = pv.pivot_cache4_attend(q.contiguous(), pool.cache, [n - 1 for n in lens], lens, 0.04)
    got = pv.pivot_cache4_attend(q, pool.cache, [n - 1 for n in lens], lens, 0.04)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = pv.pivot_cache4_attend(q[1:2], Pool([33], 0, rng).cache, [32], [33], 0.04)  # any row stride, one row
    assert torch.isfinite(got[1]).all()
