"""GPU tests of operators that write rows through a block table in which entries name
no page of the pool, as a slot's do behind its pages and after a growth for which
pages were missing: nothing is written there, and nothing else changes."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import ops_ref as ref
import paper_2607_24593_amd as pv
from gpu_util import dev, host, say
from test_gpu_operators import Pool

pytestmark = pytest.mark.gpu

NO_PAGE = [-1, -2**31, 2**31 - 1]  # and the number of pages


def _held(pool, b, pos):
    """Whether positions `pos` of sequence b have a page, and their rows (where they have one)."""
    page = pool.table[b][pos // pool.page].astype(np.int64)
    return (page >= 0) & (page < pool.rows // pool.page), page * pool.page + pos % pool.page


def _missing(pool, rng, share):
    """Entries of the table that name no page, of every kind; pages 0 and the last stay held."""
    n = pool.rows // pool.page
    kinds = np.array(NO_PAGE + [n], dtype=np.int64)
    out = rng.random(pool.table.shape) < share
    out &= (pool.table != 0) & (pool.table != n - 1)
    pool.table = np.where(out, rng.choice(kinds, pool.table.shape), pool.table).astype(np.int32)
    pool.upload()


@pytest.mark.parametrize("lens,n_new,page,share", [([96] * 4, 40, 16, 0.4), ([33], 33, 16, 1.0), ([200, 150] * 9, 1, 32, 0.5),
                                                   ([64] * 70, 20, 16, 0.3)])
def test_rows_without_a_page_are_not_written(lens, n_new, page, share):
    rng = np.random.default_rng(len(lens) + n_new)
    pool = Pool(lens, page, rng, spare=0)
    _missing(pool, rng, share)
    t = len(lens) * n_new
    x, rope = ref.bf16(rng.standard_normal((t, 512))), ref.bf16(rng.standard_normal((t, 64)))
    want = [pool.codes.copy(), pool.scales.copy(), pool.rope.copy()]
    codes, scales = ref.quantise(x)
    pos0 = [n - n_new for n in lens]
    written = 0
    for b, p in enumerate(pos0):
        ok, at = _held(pool, b, p + np.arange(n_new))
        mine = np.arange(b * n_new, (b + 1) * n_new)[ok]
        for a, new in zip(want, (codes, scales, rope)):
            a[at[ok]] = new[mine]
        written += ok.sum()
    assert written < t
    say("cache write, pages that are none", lens[:3], n_new, page)
    pv.pivot_cache4_write(torch.from_numpy(x).bfloat16().cuda(), torch.from_numpy(rope).bfloat16().cuda(), pool.cache, pos0,
                          n_new)
    got = [host(t) for t in pool.parts[:2]] + [pool.parts[2].double().cpu().numpy()]
    # a code of a negative value that rounds to 0 may keep its sign
    assert np.array_equal(ref.values(got[0], got[1]), ref.values(want[0], want[1]))
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])


def test_a_growth_without_pages_and_the_write_behind_it():
    """Two sequences share a pool; one grows where no page is left, and its rows come
    all the same.  The other's rows, on page 0 and the last one, stay."""
    rng = np.random.default_rng(7)
    page, n_pages = 16, 6
    table = torch.full((2, 8), -1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    pages = pv.make_pages(table, refs, page)
    codes, scales, rope = ref.random_cache(n_pages * page, rng)
    parts = (dev(codes), dev(scales), torch.from_numpy(rope).bfloat16().cuda())
    cache = pv.make_cache4(*parts, pv.make_row_map(rows=n_pages * page, block_table=table, page_size=page))
    say("a growth without pages")
    assert host(pv.pivot_pages_grow(pages, [0, 1], [0, 0], [64, 20])[1]).tolist() == [0, 0]
    copies, state = pv.pivot_pages_grow(pages, [1], [20], [60])
    assert host(state).tolist() == [2, 0] and host(copies).tolist() == [[-1, -1]]
    before = [t.clone() for t in parts]
    rows = torch.from_numpy(rng.standard_normal((40, 576))).bfloat16().cuda()
    pv.pivot_cache4_write(rows[:, :512], rows[:, 512:], cache, [64, 20], cu=[0, 0, 40])
    own = host(table)[1, 1] * page + np.arange(4, 16)  # positions 20 .. 31 lie on the slot's second page
    rest = torch.from_numpy(np.setdiff1d(np.arange(n_pages * page), own)).cuda()
    for now, old in zip(parts, before):
        assert torch.equal(now[rest], old[rest])
    assert torch.equal(parts[2][torch.from_numpy(own).cuda()], rows[:12, 512:])


@pytest.mark.parametrize("lens,keep,page,share", [([300, 37, 200], 64, 16, 0.5), ([500] * 5, 490, 64, 0.3), ([40] * 70, 33, 16, 0.4)])
def test_kept_rows_without_a_page_are_not_moved(lens, keep, page, share):
    """Rows move to pages of another table; those whose new place has no page are left
    out, the list of the kept positions is whole."""
    rng = np.random.default_rng(keep)
    pool = Pool(lens, page, rng, spare=0)
    b, per = len(lens), -(-keep // page)
    n = pool.rows // page
    fresh = Pool.__new__(Pool)
    fresh.page, fresh.rows = page, 2 * pool.rows
    fresh.table = (n + rng.permutation(n)[:b * per].reshape(b, per)).astype(np.int32)
    fresh.table[rng.random(fresh.table.shape) < share] = -1
    fresh.table[0, 0] = rng.choice([-2**31, 2**31 - 1, 2 * n])
    first = rng.integers(0, 256, (2 * pool.rows, 20), dtype=np.uint8)
    second = rng.standard_normal((2 * pool.rows, 32)).astype(np.float32)
    arrays = [dev(first), dev(second)]
    acc = rng.random((b, max(lens))).astype(np.float32)
    table = dev(fresh.table)
    frm = pv.make_row_map(rows=2 * pool.rows, block_table=pool.bt, page_size=page)
    to = pv.make_row_map(rows=2 * pool.rows, block_table=table, page_size=page)
    say("evict, pages that are none", lens[:3], keep, page)
    kept, _ = pv.pivot_evict(dev(acc), lens, keep, [(x, x) for x in arrays], frm, to, sink=2, recent=3)
    want = [first.copy(), second.copy()]
    left = 0
    for i, m in enumerate(lens):
        mine = np.array(ref.evict(acc[i], m, keep, 2, 3))
        assert host(kept)[i, :len(mine)].tolist() == mine.tolist()
        ok, at = _held(fresh, i, np.arange(len(mine)))
        left += (~ok).sum()
        for w, old in zip(want, (first, second)):
            w[at[ok]] = old[pool.row(i, mine[ok])]
    assert left > 0
    for x, w in zip(arrays, want):
        assert np.array_equal(host(x), w)


def test_the_example_stops_where_pages_are_missing():
    spec = importlib.util.spec_from_file_location(
        "draft_step", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "draft_step.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    layer = ex.Layer(2, 200, dim=128, heads=4, page=16, n_pages=9)
    g = torch.Generator(device="cuda").manual_seed(1)
    layer.append(0, torch.randn((100, 128), generator=g, device="cuda").bfloat16())  # 7 pages
    layer.fork(0, 1)
    before = [t.clone() for t in (layer.table, layer.refs, *layer.arrays)]
    say("a step that lacks pages")
    hidden = torch.randn((2, 20, 128), generator=g, device="cuda").bfloat16()
    masks = torch.stack([ex.tree_masks(list(range(-1, 19)), 1)] * 2)
    with pytest.raises(RuntimeError, match="lacks 1 "):  # 100 + 20 tokens: a copy, and one more each
        layer.step(hidden, torch.zeros_like(hidden), masks)
    assert layer.length == [100, 100]
    for now, old in zip((layer.table, layer.refs, *layer.arrays), before):
        assert torch.equal(now, old)
