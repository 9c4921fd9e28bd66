"""GPU tests of the operators around the index calls against plain definitions
in 64 bits (ops_ref): the norm with fp8 output, writing and reading the 4-bit
cache, attention over it, and eviction.

Bounds, from the arithmetic (u = 2^-24 for fp32, 2^-9 for rounding to bf16):
  norm    sums of at most 32 + 16 terms in a chain: scales and values to 4e-6;
          a code is a nearest one up to that
  cache   exact
  attend  a score is a sum of 576 exact products: off by at most
          E = 2^-18 * scale * max_s sum |q k| (64 u of that sum);  lse: E + 4 u (1 + |lse|) + u;
          out: weights and the result rounded to bf16, each weight off by E:
          2^-9 |out| + (2^-9 + 2 E) sum p |latent|;  acc: (2 E + 2^-19) of each weight
  evict   exact
"""
import numpy as np
import pytest
import torch

import ops_ref as ref
import paper_2607_24593_amd as pv
from gpu_util import dev, host, say

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ norm
def _norm_check(x, r, w, eps, group, codes, scale, h, bf):
    X, R, W = (None if t is None else t.double().cpu().numpy() for t in (x, r, w))
    hh = X if R is None else X + R
    if R is not None:  # one fp32 addition, then the type's rounding
        want = (x.float() + r.float()).to(x.dtype)
        assert torch.equal(h, want)
    hh = hh.astype(np.float32).astype(np.float64)
    y = hh / np.sqrt((hh ** 2).mean(-1, keepdims=True) + eps) * W
    d = y.shape[-1]
    got = ref.e4m3_value(host(codes))
    for g, lo in enumerate(range(0, d, group or d)):
        part = y[:, lo:lo + (group or d)]
        amax = np.abs(part).max(-1)
        s = np.where(amax > 0, amax / 448, 1.0)
        assert np.all(np.abs(host(scale)[:, g] - s) <= 4e-6 * s), (g, lo)
        v = part / s[:, None]
        off = np.abs(got[:, lo:lo + (group or d)] - v)
        assert np.all(off <= ref.e4m3_ulp(v) / 2 + 1e-5 * np.abs(v)), (g, off.max())


@pytest.mark.parametrize("rows,dim", [(1, 1), (1, 7), (3, 8), (2, 63), (5, 127), (4, 128), (3, 129), (2, 511), (2, 2048),
                                      (7, 2049), (1, 4096), (3, 5003), (2, 8192), (2, 8193), (1, 20011), (1, 32768)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("group", [0, 128])
def test_norm(rows, dim, dtype, group):
    g = torch.Generator().manual_seed(rows * 1000 + dim)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.randn((rows, dim), generator=g).to(dt)
    r = (3 * torch.randn((rows, dim), generator=g)).to(dt)
    w = (1 + 0.3 * torch.randn(dim, generator=g)).to(dt)
    say("norm", rows, dim, dtype, group)
    codes, scale, h = pv.pivot_rmsnorm_fp8(x.cuda(), w.cuda(), 1e-5, residual=r.cuda(), group=group)
    _norm_check(x, r, w, 1e-5, group, codes, scale, h.cpu(), dtype == "bf16")
    codes, scale, h = pv.pivot_rmsnorm_fp8(x.cuda(), w.cuda(), 1e-5, group=group)
    assert h is None
    _norm_check(x, None, w, 1e-5, group, codes, scale, None, dtype == "bf16")


def test_norm_strided_in_place_and_zero_rows():
    g = torch.Generator().manual_seed(5)
    big = torch.randn((6, 700), generator=g).bfloat16().cuda()
    x, r = big[:, 3:303], torch.randn((6, 300), generator=g).bfloat16().cuda()
    w = torch.ones(300).bfloat16().cuda()
    r0 = r.clone()
    say("norm strided, residual in place")
    codes, scale, h = pv.pivot_rmsnorm_fp8(x, w, 1e-6, residual=r, residual_out=r)
    assert h is r
    _norm_check(x.cpu(), r0.cpu(), w.cpu(), 1e-6, 0, codes, scale, r.cpu(), True)
    z = torch.zeros((2, 300), dtype=torch.bfloat16, device="cuda")
    say("norm of zeros")
    codes, scale, _ = pv.pivot_rmsnorm_fp8(z, w, 1e-6, group=128)
    assert not host(codes).any() and (host(scale) == 1).all()
    codes, scale, _ = pv.pivot_rmsnorm_fp8(z, w, 0.0)
    assert np.isnan(ref.e4m3_value(host(codes))).all()  # 0 / 0
    bad = torch.ones((3, 300), dtype=torch.bfloat16, device="cuda")
    bad[1, 17] = float("nan")
    say("norm with a NaN row")
    v = ref.e4m3_value(host(pv.pivot_rmsnorm_fp8(bad, w)[0]))
    assert np.isnan(v[1]).all() and np.isfinite(v[0]).all() and np.isfinite(v[2]).all()


# ------------------------------------------------------------------ cache
class Pool:
    """A cache of `lens` tokens, contiguous or on shuffled pages, with its plain values."""

    def __init__(self, lens, page, rng, spare=1, spread=0.5):
        self.lens, self.page, b = lens, page, len(lens)
        per = max(max(lens), 1)
        if page:
            need = -(-per // page)
            n = b * need + spare
            self.table = rng.permutation(n)[:b * need].reshape(b, need).astype(np.int32)
            self.rows, self.stride = n * page, 0
        else:
            self.table, self.stride = None, per + spare
            self.rows = b * self.stride
        self.codes, self.scales, self.rope = ref.random_cache(self.rows, rng, spread)
        self.upload()

    def row(self, b, s):
        s = np.asarray(s)
        return b * self.stride + s if self.table is None else self.table[b][s // self.page] * self.page + s % self.page

    def upload(self):
        self.bt = None if self.table is None else torch.from_numpy(self.table).cuda()
        self.parts = (dev(self.codes), dev(self.scales), torch.from_numpy(self.rope).bfloat16().cuda())
        self.map = pv.make_row_map(seq_stride=self.stride, rows=self.rows, block_table=self.bt, page_size=self.page)
        self.cache = pv.make_cache4(*self.parts, self.map)

    def tokens(self, b, n):
        at = self.row(b, np.arange(n))
        return ref.values(self.codes[at], self.scales[at]), self.rope[at]


@pytest.mark.parametrize("lens,n_new,page", [([1], 1, 0), ([5], 5, 0), ([100, 37, 64], 3, 16), ([300, 40], 33, 32),
                                             ([70] * 67, 2, 16)])
def test_cache_write_and_read(lens, n_new, page):
    rng = np.random.default_rng(7)
    pool = Pool(lens, page, rng)
    before = [t.clone() for t in pool.parts]
    t = len(lens) * n_new
    x = ref.bf16(rng.standard_normal((t, 512)) * np.exp(3 * rng.standard_normal((t, 1))))
    x[:, :64] = ref.bf16(x[:, :64] * 1e-3)
    x[0, 32:64] = 0
    x[-1, 100] = np.inf
    x[t // 2, 511] = np.nan
    rope = ref.bf16(rng.standard_normal((t, 64)))
    pos0 = [n - n_new for n in lens]
    say("cache write", lens[:3], n_new, page)
    pv.pivot_cache4_write(torch.from_numpy(x).bfloat16().cuda(), torch.from_numpy(rope).bfloat16().cuda(), pool.cache, pos0,
                          n_new)
    codes, scales = ref.quantise(x)
    at = np.concatenate([pool.row(b, p + np.arange(n_new)) for b, p in enumerate(pos0)])
    got = [host(t) for t in pool.parts[:2]] + [pool.parts[2].double().cpu().numpy()]
    # a code of a negative value that rounds to 0 may keep its sign
    assert np.array_equal(ref.values(got[0][at], got[1][at]), ref.values(codes, scales), equal_nan=True)
    assert np.array_equal(got[1][at], scales) and np.array_equal(got[2][at], rope)
    rest = np.setdiff1d(np.arange(pool.rows), at)  # nothing else was touched
    for now, old in zip(pool.parts, before):
        assert torch.equal(now[torch.from_numpy(rest).cuda()], old[torch.from_numpy(rest).cuda()])
    cap = pool.table.shape[1] * page if page else pool.stride
    idx = np.stack([np.concatenate([p + np.arange(n_new), [-1, cap, 0]]) for p in pos0]).astype(np.int32)
    say("cache read")
    back = pv.pivot_cache4_read(pool.cache, dev(idx)).double().cpu().numpy()
    for b in range(len(lens)):
        r = pool.row(b, idx[b, :n_new])
        want = np.concatenate([ref.values(got[0][r], got[1][r]), got[2][r]], 1)
        assert np.array_equal(back[b, :n_new], want, equal_nan=True)
        assert not back[b, n_new:n_new + 2].any()


def test_cache_write_packed_and_strided():
    """Runs of different lengths (an empty one among them) out of a wider projection's rows."""
    rng = np.random.default_rng(8)
    pool = Pool([40, 50, 60], 16, rng)
    cu = [0, 4, 4, 11]
    wide = torch.from_numpy(rng.standard_normal((11, 643))).bfloat16().cuda()
    say("cache write packed")
    pv.pivot_cache4_write(wide[:, 1:513], wide[:, 513:577], pool.cache, [3, 9, 20], cu=cu)
    x = wide.double().cpu().numpy()
    for b, p in ((0, 3), (2, 20)):
        n = cu[b + 1] - cu[b]
        codes, scales = ref.quantise(x[cu[b]:cu[b + 1], 1:513])
        at = pool.row(b, p + np.arange(n))
        assert np.array_equal(ref.values(host(pool.parts[0])[at], host(pool.parts[1])[at]), ref.values(codes, scales))
        assert np.array_equal(pool.parts[2].double().cpu().numpy()[at], x[cu[b]:cu[b + 1], 513:577])


def test_cache_extreme_values():
    """Every power of two of bf16 as a block's maximum, with both sides of the scale's step."""
    x = np.zeros((256, 512))
    for e in range(-126, 128):
        for j, m in enumerate((1.0, 1.5, 1.5078125, 1.9921875)):
            x[e + 126, 32 * j] = m * 2.0 ** e
            x[e + 126, 32 * j + 1] = -0.34375 * m * 2.0 ** max(e, -120)
    x = ref.bf16(x)
    parts = (torch.zeros((256, 256), dtype=torch.uint8, device="cuda"), torch.zeros((256, 16), dtype=torch.uint8, device="cuda"),
             torch.zeros((256, 64), dtype=torch.bfloat16, device="cuda"))
    c = pv.make_cache4(*parts, pv.make_row_map(seq_stride=256, rows=256))
    say("cache extremes")
    pv.pivot_cache4_write(torch.from_numpy(x).bfloat16().cuda(), torch.zeros((256, 64), dtype=torch.bfloat16, device="cuda"), c,
                          [0], 256)
    codes, scales = ref.quantise(x)
    assert np.array_equal(host(parts[1]), scales)
    assert np.array_equal(ref.values(host(parts[0]), scales), ref.values(codes, scales))


# ------------------------------------------------------------------ attention
def _queries(shape, rng, std=2.0):
    return ref.bf16(std * rng.standard_normal(shape + (576,)))


def _check(pool, q, pos0, n_rows, scale, out, lse, idx=None, acc=None, acc0=None, rows=None, label=""):
    """Every query row (or `rows`) of packed q [rows, heads, 576] against the definition."""
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    out, lse = out.reshape(-1, *out.shape[-2:]), lse.reshape(-1, lse.shape[-1])
    r = 0
    for b, n in enumerate(n_rows):
        size = pos0[b] + n
        if n == 0:
            continue
        latent, rope = pool.tokens(b, size)
        total, slack = np.zeros(size), np.zeros(size)
        for i in range(n):
            pos = pos0[b] + i
            allowed = np.zeros(size, dtype=bool)
            if idx is None:
                allowed[:pos + 1] = True
            else:
                s = idx[r]
                allowed[s[(s >= 0) & (s <= pos)]] = True
            if rows is None or r in rows or acc is not None:
                o, l, w, bound, spread = ref.attend_rows(q[r], latent, rope, scale, allowed)
                E = 2.0 ** -18 * bound
                fin = np.isfinite(l)
                assert np.array_equal(np.isnan(out[r]).any(-1), np.isnan(l)), (label, r)
                assert np.array_equal(lse[r][~fin & ~np.isnan(l)], l[~fin & ~np.isnan(l)]), (label, r)
                u = 2.0 ** -24
                assert np.all(np.abs(lse[r] - l)[fin] <= (E + 4 * u * (1 + np.abs(l)) + u)[fin]), \
                    (label, r, np.abs(lse[r] - l)[fin].max(), E[fin].max())
                tol = 2.0 ** -9 * np.abs(o) + (2.0 ** -9 + 2 * E)[:, None] * spread + 1e-30
                off = np.abs(out[r] - o)
                assert np.all(off[fin] <= tol[fin]), (label, r, (off / tol)[fin].max())
                assert not out[r][~fin & ~np.isnan(l)].any()
                total += w
                slack += (2 * E.max() + 2.0 ** -19) * w
            r += 1
        if acc is not None:
            want = total + acc0[b, :size]
            got = acc[b, :size].astype(np.float64)
            assert np.array_equal(np.isnan(got), np.isnan(want)), label
            ok = ~np.isnan(want)
            assert np.all(np.abs(got - want)[ok] <= (slack + 2.0 ** -22 * np.abs(want) + 1e-30)[ok]), \
                (label, b, np.abs(got - want)[ok].max())
            assert np.array_equal(acc[b, size:], acc0[b, size:])


def _sets(rng, pos0, n_rows, topk, valid):
    """valid(row, pos) -> positions; padded with -1, in random order, holes anywhere."""
    out = []
    for b, n in enumerate(n_rows):
        for i in range(n):
            s = np.asarray(valid(len(out), pos0[b] + i), dtype=np.int64)[:topk]
            row = np.full(topk, -1, dtype=np.int32)
            row[rng.permutation(topk)[:len(s)]] = s
            out.append(row)
    return np.stack(out) if out else np.zeros((0, topk), np.int32)


def _some(rng, topk):
    return lambda r, pos: rng.permutation(pos + 1)[:topk]


SPARSE = [
    # heads, lens, n_q, topk, page
    (1, [1], 1, 1, 0), (3, [40], 1, 1, 0), (16, [40], 2, 31, 16), (17, [100, 33], 2, 32, 0), (32, [300], 1, 33, 64),
    (33, [300, 64, 5], 3, 64, 16), (64, [257], 2, 97, 0), (65, [500], 1, 200, 32), (100, [400], 2, 129, 0),
    (128, [700, 90], 2, 256, 16), (128, [3000], 2, 2048, 0), (16, [2500, 1200], 1, 2048, 64), (8, [60] * 66, 1, 20, 16),
]


@pytest.mark.parametrize("heads,lens,n_q,topk,page", SPARSE)
@pytest.mark.parametrize("with_acc", [False, True])
def test_attend_sets(heads, lens, n_q, topk, page, with_acc):
    rng = np.random.default_rng(heads * 7 + topk)
    pool = Pool(lens, page, rng)
    n_q = min(n_q, min(lens))
    pos0, n_rows = [n - n_q for n in lens], [n_q] * len(lens)
    q = _queries((len(lens) * n_q, heads), rng)
    idx = _sets(rng, pos0, n_rows, topk, _some(rng, topk))
    acc0 = rng.random((len(lens), max(lens) + 3)).astype(np.float32)
    acc = dev(acc0) if with_acc else None
    say("attend sets", heads, lens[:3], n_q, topk, page, with_acc)
    qd = torch.from_numpy(q).bfloat16().cuda().view(len(lens), n_q, heads, 576)
    out, lse = pv.pivot_cache4_attend(qd, pool.cache, pos0, lens, 0.04, idx=dev(idx).view(len(lens), n_q, topk), acc=acc)
    _check(pool, q, pos0, n_rows, 0.04, out, lse, idx, host(acc) if with_acc else None, acc0)


DENSE = [
    (1, [1], 1, 0), (2, [2], 2, 0), (16, [31], 1, 0), (16, [33, 32, 64], 1, 16), (5, [200], 4, 32), (40, [130, 65], 3, 16),
    (128, [300], 1, 0), (128, [520], 2, 64), (64, [1030], 1, 0), (16, [5000, 17], 1, 64), (24, [900], 5, 0),
    (128, [4100], 1, 16), (4, [50] * 66, 1, 16), (1, [700], 300, 0),
]


@pytest.mark.parametrize("heads,lens,n_q,page", DENSE)
@pytest.mark.parametrize("with_acc", [False, True])
def test_attend_prefix(heads, lens, n_q, page, with_acc):
    rng = np.random.default_rng(heads * 11 + lens[0])
    pool = Pool(lens, page, rng)
    n_q = min(n_q, min(lens))
    pos0, n_rows = [n - n_q for n in lens], [n_q] * len(lens)
    q = _queries((len(lens) * n_q, heads), rng)
    acc0 = rng.random((len(lens), max(lens) + 3)).astype(np.float32)
    acc = dev(acc0) if with_acc else None
    say("attend prefix", heads, lens[:3], n_q, page, with_acc)
    qd = torch.from_numpy(q).bfloat16().cuda().view(len(lens), n_q, heads, 576)
    out, lse = pv.pivot_cache4_attend(qd, pool.cache, pos0, lens, 0.04, acc=acc)
    _check(pool, q, pos0, n_rows, 0.04, out, lse, None, host(acc) if with_acc else None, acc0)


@pytest.mark.parametrize("sparse", [False, True])
def test_attend_packed_strided_and_middle_of_prefix(sparse):
    """Packed runs with empty ones, queries in the middle of what is cached (later
    tokens are there and masked), heads of a wider projection."""
    rng = np.random.default_rng(21)
    lens, pos0, cu = [90, 40, 333, 64], [10, 5, 300, 0], [0, 3, 3, 10, 10]
    pool = Pool(lens, 16, rng)
    wide = torch.from_numpy(rng.standard_normal((10, 20, 640)) * 2).bfloat16().cuda()
    qd = wide[:, 2:14, 8:584]
    q = qd.double().cpu().numpy()
    n_rows = [3, 0, 7, 0]
    idx = _sets(rng, pos0, n_rows, 48, lambda r, pos: rng.permutation(pos + 9)[:48]) if sparse else None
    acc0 = np.zeros((4, 333), np.float32)
    acc = dev(acc0)
    say("attend packed", sparse)
    out, lse = pv.pivot_cache4_attend(qd, pool.cache, pos0, lens, 0.05, cu_q=cu, idx=dev(idx) if sparse else None, acc=acc)
    _check(pool, q, pos0, n_rows, 0.05, out, lse, idx, host(acc), acc0)


@pytest.mark.parametrize("heads", [16, 64])
def test_attend_masked_rows_and_special_values(heads):
    """Empty sets, entries past the row's own position, NaN and infinities in tokens
    that a row does not attend to, and in one that it does."""
    rng = np.random.default_rng(31)
    lens, n_q, topk = [200], 6, 70
    pool = Pool(lens, 16, rng)
    at = pool.row(0, np.arange(200))
    pool.scales[at[50], 3] = 255                       # a NaN block in token 50
    pool.rope[at[60], 5] = np.nan
    pool.rope[at[61], 6] = np.inf
    pool.scales[pool.table.max() * 16 % pool.rows] = 255
    pool.upload()
    pos0 = [150]
    clean = np.setdiff1d(np.arange(150), [50, 60, 61])
    sets = [[], clean[:70], [199, 180, 170], np.append(clean[:20], 50), clean[100:101], np.append(clean[:3], 190)]
    idx = _sets(rng, pos0, [n_q], topk, lambda r, pos: sets[r])
    q = _queries((n_q, heads), rng)
    acc0 = np.zeros((1, 200), np.float32)
    say("attend masked rows", heads)
    out, lse = pv.pivot_cache4_attend(torch.from_numpy(q).bfloat16().cuda()[None], pool.cache, pos0, lens, 0.04,
                                      idx=dev(idx)[None])
    _check(pool, q, pos0, [n_q], 0.04, out, lse, idx)
    o, l = out[0].float().cpu().numpy(), host(lse)[0]
    for r in (0, 2):
        assert not o[r].any() and np.isneginf(l[r]).all()
    assert np.isnan(o[3]).all() and np.isfinite(o[[1, 4, 5]]).all()
    acc = dev(acc0)
    keep = [0, 1, 2, 4, 5]
    out, lse = pv.pivot_cache4_attend(torch.from_numpy(q[keep]).bfloat16().cuda()[None], pool.cache, [151], lens, 0.04,
                                      idx=dev(idx[keep])[None], acc=acc)
    _check(pool, q[keep], [151], [5], 0.04, out, lse, idx[keep], host(acc), acc0)
    # the same NaN tokens behind the prefix of the queries: masked by position
    pool.scales[at[50], 3], pool.rope[at[60], 5], pool.rope[at[61], 6] = 127, 0, 0
    for s in (103, 104, 120):
        pool.scales[at[s]] = 255
    pool.rope[at[110]] = np.nan
    pool.upload()
    q = _queries((4, heads), rng)
    out, lse = pv.pivot_cache4_attend(torch.from_numpy(q).bfloat16().cuda()[None], pool.cache, [100], lens, 0.04)
    _check(pool, q, [100], [4], 0.04, out, lse)
    o = out[0].float().cpu().numpy()
    assert np.isfinite(o[:3]).all() and np.isnan(o[3]).all()  # position 103 is the last row's own
    # a query with a NaN or an infinity
    q = _queries((3, heads), rng)
    q[1, 0, 40], q[1, heads - 1, 570], q[2, 1, 3] = np.nan, np.nan, np.inf
    qd = torch.from_numpy(q).bfloat16().cuda()[None]
    out, lse = pv.pivot_cache4_attend(qd, pool.cache, [60], lens, 0.04)
    o = out[0].float().cpu().numpy()
    assert np.isnan(o[1, [0, heads - 1]]).all() and np.isnan(o[2, 1]).all()
    fine = np.ones((3, heads), bool)
    fine[1, [0, heads - 1]] = fine[2, 1] = False
    assert np.isfinite(o[fine]).all()


@pytest.mark.parametrize("std,scale", [(40.0, 0.3), (1e-3, 1e-3), (2.0, 0.0), (2.0, -0.04), (2e4, 1e-4)])
def test_attend_score_ranges(std, scale):
    """Peaked, flat, constant, negated and wide-ranged scores."""
    rng = np.random.default_rng(41)
    pool = Pool([600], 0, rng, spread=1.5)
    q = _queries((2, 40), rng, std)
    q[0, 1] *= np.exp2(rng.integers(-30, 1, 576))  # a query whose values span many binades
    q = ref.bf16(q)
    say("attend ranges", std, scale)
    out, lse = pv.pivot_cache4_attend(torch.from_numpy(q).bfloat16().cuda()[None], pool.cache, [598], [600], scale)
    _check(pool, q, [598], [2], scale, out, lse)


def test_attend_long_cache_past_32_bit_offsets():
    """Pages at the end of a pool whose codes pass 2^31 bytes, contiguous sequences likewise."""
    rng = np.random.default_rng(51)
    rows = 9 << 20
    small = Pool([70], 16, rng, spare=0)
    codes = torch.zeros((rows, 256), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((rows, 16), dtype=torch.uint8, device="cuda")
    rope = torch.zeros((rows, 64), dtype=torch.bfloat16, device="cuda")
    for t, s in zip((codes, scales, rope), small.parts):
        t[rows - small.rows:] = s
    q = _queries((1, 16), rng)
    table = torch.from_numpy(small.table + (rows - small.rows) // 16).int().cuda()
    c = pv.make_cache4(codes, scales, rope, pv.make_row_map(rows=rows, block_table=table, page_size=16))
    say("attend far pages")
    qd = torch.from_numpy(q).bfloat16().cuda()[None]
    out, lse = pv.pivot_cache4_attend(qd, c, [69], [70], 0.04)
    _check(small, q, [69], [1], 0.04, out, lse)
    back = pv.pivot_cache4_read(c, torch.arange(70, dtype=torch.int32, device="cuda")[None]).double().cpu().numpy()
    v, r = small.tokens(0, 70)
    assert np.array_equal(back[0], np.concatenate([v, r], 1))
    # contiguous: sequence 8 of 9 starts at 2^31 bytes of codes
    at = small.row(0, np.arange(70))
    for t, s in zip((codes, scales, rope), small.parts):
        t[8 << 20:(8 << 20) + 70] = s[torch.from_numpy(at).cuda()]
    c = pv.make_cache4(codes, scales, rope, pv.make_row_map(seq_stride=1 << 20, rows=rows))
    q9 = torch.zeros((9, 1, 16, 576), dtype=torch.bfloat16, device="cuda")
    q9[8] = qd[0]
    say("attend far sequence")
    out, lse = pv.pivot_cache4_attend(q9, c, [69] * 9, [70] * 9, 0.04)
    _check(small, q, [69], [1], 0.04, out[8:], lse[8:])


@pytest.mark.parametrize("topk", [0, 512])
def test_attend_same_bits_streams_and_graph(topk):
    """The same call gives the same bits, on its own stream, on another, and replayed from a graph."""
    rng = np.random.default_rng(61)
    lens = [4000, 1500]
    pool = Pool(lens, 64, rng)
    q = torch.from_numpy(_queries((2, 2, 128), rng)).bfloat16().cuda()
    idx = None
    if topk:
        idx = dev(_sets(rng, [3998, 1498], [2, 2], topk, _some(rng, topk))).view(2, 2, topk)
    acc = torch.zeros((2, 4000), device="cuda")
    out = torch.empty((2, 2, 128, 512), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((2, 2, 128), device="cuda")

    def call(**kw):
        return pv.pivot_cache4_attend(q, pool.cache, [3998, 1498], lens, 0.04, idx=idx, acc=acc, out=out, lse=lse, **kw)

    def bits():
        return [host(t.view(torch.int16) if t.dtype == torch.bfloat16 else t.view(torch.int32)).copy() for t in (out, lse, acc)]

    say("attend repeat", topk)
    call()
    want = bits()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    acc.zero_()
    torch.cuda.synchronize()
    say("attend other stream", topk)
    call(stream=s)
    s.synchronize()
    assert all(np.array_equal(a, b) for a, b in zip(want, bits()))
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    acc.zero_()
    torch.cuda.synchronize()
    say("attend capture", topk)
    with torch.cuda.graph(graph):
        call(ws=ws)
    for rep in range(3):
        out.fill_(0)
        lse.fill_(0)
        acc.zero_()
        pool.parts[0].clone()
        torch.cuda.synchronize()
        say("attend replay", topk, rep)
        graph.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(a, b) for a, b in zip(want, bits())), rep


# ------------------------------------------------------------------ eviction
def _evict_case(lens, keep, sink, recent, page, acc, rng, label):
    pool = Pool(lens, page, rng)
    b = len(lens)
    keys = rng.integers(0, 256, (pool.rows, 128)).astype(np.uint8)
    ks = rng.random(pool.rows).astype(np.float32)
    src = pool.parts + (dev(keys), dev(ks))
    if page:  # to fresh pages of a pool twice as large
        src = tuple(torch.cat([t, torch.zeros_like(t)]) for t in src)
        n = -(-keep // page)
        fresh = (pool.rows // page + rng.permutation(pool.rows // page)[:b * n]).reshape(b, n).astype(np.int32)
        dst, bt = src, torch.from_numpy(fresh).cuda()
        frm = pv.make_row_map(rows=2 * pool.rows, block_table=pool.bt, page_size=page)
        to = pv.make_row_map(rows=2 * pool.rows, block_table=bt, page_size=page)
        place = lambda b, j: fresh[b][j // page] * page + j % page  # noqa: E731
    else:
        dst = tuple(torch.zeros((b * keep,) + t.shape[1:], dtype=t.dtype, device="cuda") for t in src)
        frm, to = pool.map, pv.make_row_map(seq_stride=keep, rows=b * keep)
        place = lambda b, j: b * keep + j  # noqa: E731
    old = [host(t.view(torch.int16) if t.dtype == torch.bfloat16 else t).copy() for t in src]
    say("evict", label, lens[:3], keep, sink, recent, page)
    kept, out_acc = pv.pivot_evict(dev(acc), lens, keep, list(zip(src, dst)), frm, to, sink=sink, recent=recent)
    kept, out_acc = host(kept), host(out_acc)
    new = [host(t.view(torch.int16) if t.dtype == torch.bfloat16 else t) for t in dst]
    for i, n in enumerate(lens):
        want = ref.evict(acc[i], n, keep, sink, recent)
        m = len(want)
        assert m == min(n, keep)
        assert kept[i, :m].tolist() == want, (label, i)
        assert (kept[i, m:] == -1).all() and not out_acc[i, m:].any()
        assert np.array_equal(out_acc[i, :m], acc[i, want], equal_nan=True)
        at, here = pool.row(i, np.array(want, dtype=np.int64)), place(i, np.arange(m))
        for o, t in zip(old, new):
            assert np.array_equal(t[here], o[at]), (label, i)


@pytest.mark.parametrize("lens,keep,sink,recent,page", [
    ([1], 1, 0, 0, 0), ([0, 1, 2], 1, 0, 1, 0), ([2], 1, 1, 0, 0), ([100], 100, 4, 10, 0), ([101], 100, 4, 10, 16),
    ([500, 37, 200], 64, 4, 8, 16), ([500], 64, 32, 32, 0), ([5000, 4096], 1000, 4, 100, 64), ([4097], 4096, 0, 0, 0),
    ([20000], 3333, 4, 64, 0), ([300] * 67, 50, 2, 5, 16), ([131072, 9], 8192, 4, 1024, 64),
])
@pytest.mark.parametrize("kind", ["heavy", "ties"])
def test_evict(lens, keep, sink, recent, page, kind):
    rng = np.random.default_rng(sum(lens) + keep)
    shape = (len(lens), max(lens) + 5)
    acc = np.exp(3 * rng.standard_normal(shape)).astype(np.float32)
    if kind == "ties":
        acc = np.floor(acc * 2).astype(np.float32)  # many equal, zeros among them
    _evict_case(lens, keep, sink, recent, page, acc, rng, kind)


def test_evict_special_values():
    rng = np.random.default_rng(3)
    acc = rng.standard_normal((3, 400)).astype(np.float32)
    acc[0, [5, 300]] = np.nan
    acc[0, [9, 200]] = np.inf
    acc[0, 50:60] = -np.inf
    acc[1] = 0
    acc[1, 100:200] = -0.0
    acc[2] = -np.inf
    _evict_case([400, 400, 399], 37, 3, 7, 0, acc, rng, "special")


def test_evict_without_arrays():
    acc = torch.rand((2, 1000), device="cuda")
    kept, out_acc = pv.pivot_evict(acc, [1000, 900], 100, [], None, None, sink=1, recent=1)
    a = acc.cpu().numpy()
    for b, n in enumerate((1000, 900)):
        assert host(kept)[b].tolist() == ref.evict(a[b], n, 100, 1, 1)


@pytest.mark.parametrize("lens,keep,sink,recent", [
    ([8193, 8192, 100], 500, 1, 1), ([12288, 12289], 9000, 5000, 4000), ([300000, 262145, 5], 4097, 4, 64),
    ([40000], 30000, 9000, 12000), ([40000], 12345, 12000, 300), ([20000, 16385], 20000, 0, 0),
])
def test_evict_long_sequences(lens, keep, sink, recent):
    rng = np.random.default_rng(keep)
    acc = np.floor(4 * rng.standard_normal((len(lens), max(lens) + 3))).astype(np.float32)  # ties over the whole length
    acc[:, rng.integers(0, max(lens), 50)] = np.nan
    acc[:, rng.integers(0, max(lens), 50)] = np.inf
    acc[0, : lens[0] // 3] = np.frombuffer(b"\xff" * 4, dtype=np.float32)[0]  # the lowest key there is
    kept, out_acc = pv.pivot_evict(dev(acc), lens, keep, [], None, None, sink=sink, recent=recent)
    kept, out_acc = host(kept), host(out_acc)
    for b, n in enumerate(lens):
        say("evict long", lens, keep, b)
        want = ref.evict(acc[b], n, keep, sink, recent)
        assert kept[b, : len(want)].tolist() == want and (kept[b, len(want):] == -1).all()
        assert np.array_equal(out_acc[b, : len(want)].view(np.int32), acc[b, want].view(np.int32))


@pytest.mark.parametrize("topk", [130, 2100])
def test_attend_weights_of_many_rows(topk):
    """Weights of many rows on the same tokens, one long run beside a short one,
    added in an order that does not change."""
    rng = np.random.default_rng(topk)
    lens, pos0, cu, heads = [9000, 40], [8880, 33], [0, 120, 127], 2
    pool = Pool(lens, 0, rng)
    n_rows = [120, 7]
    q = _queries((127, heads), rng)
    hot = rng.permutation(8880)[:topk + 20]
    idx = _sets(rng, pos0, n_rows, topk, lambda r, pos: rng.permutation(hot if r < 120 else pos + 1)[:topk])
    acc0 = rng.random((2, 9001)).astype(np.float32)
    qd = torch.from_numpy(q).bfloat16().cuda().view(127, heads, 576)
    got = []
    for _ in range(2):
        acc = dev(acc0)
        say("attend weights of many rows", topk)
        pv.pivot_cache4_attend(qd, pool.cache, pos0, lens, 0.04, cu_q=cu, idx=dev(idx), acc=acc)
        got.append(host(acc))
    assert np.array_equal(got[0], got[1])
    r = 0
    for b, n in enumerate(n_rows):
        size = pos0[b] + n
        latent, rope = pool.tokens(b, size)
        total, slack = np.zeros(size), np.zeros(size)
        for i in range(n):
            allowed = np.zeros(size, dtype=bool)
            s = idx[r]
            allowed[s[(s >= 0) & (s <= pos0[b] + i)]] = True
            _, _, w, bound, _ = ref.attend_rows(q[r], latent, rope, 0.04, allowed)
            total += w
            slack += (2.0 ** -17 * bound.max() + 2.0 ** -19) * w
            r += 1
        # at most rows + heads + 8 additions in fp32, each rounding once
        tol = slack + (n + heads + 8) * 2.0 ** -24 * (total + acc0[b, :size]) + 1e-30
        assert np.all(np.abs(got[0][b, :size].astype(np.float64) - total - acc0[b, :size]) <= tol)
        assert np.array_equal(got[0][b, size:], acc0[b, size:])
