"""C ABI of the operators of a decode step with drafted tokens on the CPU: every
argument they refuse, with the documented status and before any launch; tensors in
host memory; the bounds and definitions that the GPU tests compare with."""
import ctypes
import os

import numpy as np
import pytest
import torch

import draft_ref as plain
import paper_2607_24593_amd as pv
from test_abi_operators import attend, ints, row_map

pytestmark = pytest.mark.skipif(not os.path.exists(pv.LIB_PATH), reason="libpivot.so not built")

FAKE = 1 << 40  # a non-null address the library must never dereference before launching
BAD, UNS, WS = pv.PIVOT_ERR_INVALID_ARG, pv.PIVOT_ERR_UNSUPPORTED, pv.PIVOT_ERR_WORKSPACE
FP8, FP32 = pv.PIVOT_DT_FP8_E4M3, pv.PIVOT_DT_FP32


# ------------------------------------------------------------------ products
def linear(**kw):
    a = pv.pivot_linear4_args()
    d = dict(x_dtype=0, out_dtype=0, n_rows=4, n=100, k=512, group=0, x=FAKE, ld_x=512, x_scale=None, codes=FAKE,
             scales=FAKE, out=FAKE, ld_out=100, workspace=None, workspace_bytes=0)
    d.update(kw)
    for name, v in d.items():
        setattr(a, name, v)
    return a


LINEAR = [
    (dict(x_dtype=2), UNS), (dict(x_dtype=-1), UNS), (dict(out_dtype=1), UNS), (dict(n_rows=-1), BAD), (dict(n=-1), BAD),
    (dict(n=(1 << 30) + 1, ld_out=1 << 31), UNS), (dict(k=0), BAD), (dict(k=-32), BAD), (dict(k=48), UNS), (dict(k=(1 << 20) + 32, ld_x=1 << 21), UNS),
    (dict(group=128), UNS), (dict(x_dtype=1, group=64, x_scale=FAKE), UNS), (dict(ld_x=511), BAD), (dict(ld_out=99), BAD),
    (dict(x=None), BAD), (dict(codes=None), BAD), (dict(scales=None), BAD), (dict(out=None), BAD), (dict(x_dtype=1), BAD),
    (dict(codes=FAKE + 8), BAD), (dict(x=FAKE + 1), BAD), (dict(out=FAKE + 1), BAD), (dict(out_dtype=2, out=FAKE + 2), BAD),
    (dict(x_dtype=1, x_scale=FAKE + 2), BAD), (dict(n_rows=64, k=6144, ld_x=6144), WS),
    (dict(n_rows=64, k=6144, ld_x=6144, workspace=FAKE + 64, workspace_bytes=1 << 40), BAD),
]


@pytest.mark.parametrize("kw,status", LINEAR)
def test_linear4_refusals(kw, status):
    assert pv.lib().pivot_linear4(ctypes.byref(linear(**kw))) == status
    assert pv.last_error() != ""


def test_linear4_of_nothing():
    L = pv.lib()
    assert L.pivot_linear4(None) == BAD and L.pivot_linear4_workspace_size(None) == 0
    assert L.pivot_linear4(ctypes.byref(linear(n_rows=0, x=None, out=None))) == pv.PIVOT_OK
    assert L.pivot_linear4(ctypes.byref(linear(n=0, codes=None, ld_out=0))) == pv.PIVOT_OK
    assert L.pivot_linear4_workspace_size(ctypes.byref(linear())) == 0
    assert L.pivot_linear4_workspace_size(ctypes.byref(linear(k=48))) == 0
    assert L.pivot_linear4_workspace_size(ctypes.byref(linear(n_rows=64, k=6144, ld_x=6144))) >= 64 * 100 * 4


@pytest.mark.parametrize("args,status", [
    ((1, 4, 64, FAKE, 64, FAKE, FAKE), UNS), ((0, -1, 64, FAKE, 64, FAKE, FAKE), BAD), ((0, 4, 0, FAKE, 64, FAKE, FAKE), BAD),
    ((0, 4, 40, FAKE, 64, FAKE, FAKE), UNS), ((0, 4, 64, FAKE, 63, FAKE, FAKE), BAD), ((0, 4, 64, None, 64, FAKE, FAKE), BAD),
    ((0, 4, 64, FAKE, 64, None, FAKE), BAD), ((0, 4, 64, FAKE, 64, FAKE, None), BAD), ((2, 4, 64, FAKE + 2, 64, FAKE, FAKE), BAD),
    ((0, 4, 64, FAKE, 64, FAKE + 2, FAKE), BAD), ((0, 0, 64, None, 64, None, None), pv.PIVOT_OK),
])
def test_pack_refusals(args, status):
    assert pv.lib().pivot_linear4_pack(*args, None) == status


# ------------------------------------------------------------------ trees
def tree(mask=FAKE, words=1):
    t = pv.pivot_tree()
    t.mask, t.words = mask, words
    return t


@pytest.mark.parametrize("tw,kw,status", [
    (dict(words=0), {}, UNS), (dict(words=33), {}, UNS), (dict(mask=None), {}, BAD), (dict(mask=FAKE + 2), {}, BAD),
    (dict(), dict(heads=0), UNS), (dict(), dict(q=None), BAD), (dict(), dict(scale=float("nan")), BAD),
])
def test_tree_refusals(tw, kw, status):
    L, a = pv.lib(), attend(**kw)
    assert L.pivot_cache4_attend_tree(ctypes.byref(a), ctypes.byref(tree(**tw))) == status
    assert pv.last_error() != ""


def test_trees_wider_than_their_masks():
    L = pv.lib()
    a = attend(n_q=33, pos=(0, 10), n_k=(100, 100))
    assert L.pivot_cache4_attend_tree(ctypes.byref(a), ctypes.byref(tree(words=1))) == BAD
    assert L.pivot_cache4_attend_tree_workspace_size(ctypes.byref(a), ctypes.byref(tree(words=1))) == 0
    assert L.pivot_cache4_attend_tree(ctypes.byref(a), None) == BAD
    assert L.pivot_cache4_attend_tree(None, ctypes.byref(tree())) == BAD


def accept(batch=2, n=4, path=FAKE, pos0=(3, 5), n_arrays=1, rows=FAKE, row_bytes=16, m=None):
    r = (pv.pivot_rows * 9)()
    for x in r:
        x.rows, x.row_bytes = rows, row_bytes
    m = row_map() if m is None else m
    return pv.lib().pivot_tree_accept(batch, n, path, ints(*pos0), n_arrays, r, ctypes.byref(m), None)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), BAD), (dict(n=-1), BAD), (dict(n=1025), UNS), (dict(path=None), BAD), (dict(path=FAKE + 1), BAD),
    (dict(pos0=(3, -1)), BAD), (dict(pos0=(3, 257)), BAD), (dict(pos0=(0, pv.PIVOT_MAX_KEYS + 1)), UNS),
    (dict(n_arrays=0), BAD), (dict(n_arrays=9), BAD), (dict(rows=None), BAD), (dict(rows=FAKE + 2), BAD),
    (dict(row_bytes=6), BAD), (dict(row_bytes=0), BAD), (dict(m=row_map(rows=0)), BAD), (dict(m=row_map(stride=600)), BAD),
    (dict(n=0, path=None), pv.PIVOT_OK),
])
def test_accept_refusals(kw, status):
    assert accept(**kw) == status


# ------------------------------------------------------------------ pages
def pages(**kw):
    p = pv.pivot_pages()
    d = dict(table=FAKE, slots=8, max_pages=10, page_size=16, refs=FAKE, n_pages=50)
    d.update(kw)
    for name, v in d.items():
        setattr(p, name, v)
    return p


POOLS = [
    (dict(table=None), BAD), (dict(refs=None), BAD), (dict(slots=0), BAD), (dict(max_pages=0), BAD), (dict(page_size=24), BAD),
    (dict(page_size=8), BAD), (dict(page_size=1 << 17), BAD), (dict(n_pages=0), BAD), (dict(n_pages=1 << 27), BAD),
    (dict(slots=1 << 20, max_pages=1 << 12), BAD), (dict(table=FAKE + 2), BAD), (dict(refs=FAKE + 1), BAD),
]


@pytest.mark.parametrize("kw,status", POOLS)
def test_pool_refusals(kw, status):
    L, p = pv.lib(), pages(**kw)
    p = ctypes.byref(p)
    r = (pv.pivot_rows * 1)()
    r[0].rows, r[0].row_bytes = FAKE, 16
    assert L.pivot_pages_fork(p, 1, ints(0), ints(1), ints(5), None) == status
    assert L.pivot_pages_free(p, 1, ints(0), ints(5), ints(1), None) == status
    assert L.pivot_pages_grow(p, 1, ints(0), ints(5), ints(9), FAKE, FAKE, FAKE, 1 << 40, None) == status
    assert L.pivot_pages_compact(p, 5, FAKE, FAKE, FAKE, 1 << 40, None) == status
    if not set(kw) & {"table", "refs"}:
        assert L.pivot_pages_copy(p, 1, FAKE, 1, r, None) == status
        assert L.pivot_pages_compact_workspace_size(p) == 0
        assert L.pivot_pages_grow_workspace_size(p, 1, ints(5), ints(9)) == 0


def test_list_refusals():
    L, p = pv.lib(), ctypes.byref(pages())
    many = ints(*range(257))

    def fork(src, dst, n, count=None):
        return L.pivot_pages_fork(p, len(src) if count is None else count, ints(*src), ints(*dst), ints(*n), None)

    def free(slot, n, keep):
        return L.pivot_pages_free(p, len(slot), ints(*slot), ints(*n), ints(*keep), None)

    def grow(slot, n, new, copies=FAKE, state=FAKE, ws=FAKE, size=1 << 40):
        return L.pivot_pages_grow(p, len(slot), ints(*slot), ints(*n), ints(*new), copies, state, ws, size, None)

    assert fork([0], [1], [5], -1) == BAD and fork([0], [1], [5], 0) == pv.PIVOT_OK
    assert L.pivot_pages_fork(p, 257, many, many, many, None) == UNS
    assert fork([0], [8], [5]) == BAD and fork([-1], [1], [5]) == BAD and fork([0], [1], [161]) == BAD
    assert fork([0], [1], [-1]) == BAD
    assert fork([0, 0], [1, 1], [5, 5]) == BAD and fork([0, 1], [1, 2], [5, 5]) == BAD and fork([3], [3], [5]) == BAD
    assert L.pivot_pages_fork(p, 1, None, ints(1), ints(5), None) == BAD
    assert L.pivot_pages_fork(p, 1, ints(0), ints(1), None, None) == BAD
    long = ctypes.byref(pages(slots=2, max_pages=1 << 24))
    assert L.pivot_pages_fork(long, 1, ints(0), ints(1), ints(pv.PIVOT_MAX_KEYS + 1), None) == UNS
    assert L.pivot_pages_free(long, 1, ints(0), ints(pv.PIVOT_MAX_KEYS + 1), ints(1), None) == UNS
    assert L.pivot_pages_grow(long, 1, ints(0), ints(0), ints(pv.PIVOT_MAX_KEYS + 1), FAKE, FAKE, FAKE, 1 << 40, None) == UNS
    wide = ctypes.byref(pages(slots=200, max_pages=1 << 23))
    most = ints(*[pv.PIVOT_MAX_KEYS] * 200)
    none = ints(*[0] * 200)
    assert L.pivot_pages_grow(wide, 200, ints(*range(200)), none, most, FAKE, FAKE, FAKE, 1 << 40, None) == UNS
    assert L.pivot_pages_grow_workspace_size(wide, 200, none, most) == 0
    assert free([0, 0], [5, 5], [1, 1]) == BAD and free([0], [5], [6]) == BAD and free([0], [5], [-1]) == BAD
    assert free([8], [5], [1]) == BAD and free([0], [161], [1]) == BAD
    assert L.pivot_pages_free(p, 1, ints(0), ints(5), None, None) == BAD
    assert L.pivot_pages_free(p, 0, None, None, None, None) == pv.PIVOT_OK
    assert grow([0, 0], [5, 5], [9, 9]) == BAD and grow([0], [5], [4]) == BAD and grow([0], [5], [161]) == BAD
    assert grow([9], [5], [9]) == BAD and grow([], [], []) == BAD
    assert grow([0], [5], [9], copies=None) == BAD and grow([0], [5], [9], state=None) == BAD
    assert grow([0], [5], [9], state=FAKE + 2) == BAD
    assert grow([0], [5], [9], ws=None) == WS and grow([0], [5], [9], size=8) == WS and grow([0], [5], [9], ws=FAKE + 16) == BAD
    assert L.pivot_pages_grow(p, 1, ints(0), None, ints(9), FAKE, FAKE, FAKE, 1 << 40, None) == BAD
    assert L.pivot_pages_grow(p, 1, ints(0), ints(9), None, FAKE, FAKE, FAKE, 1 << 40, None) == BAD
    assert L.pivot_pages_grow_workspace_size(p, 1, ints(0), ints(160)) > 0
    assert L.pivot_pages_grow_workspace_size(p, 1, None, ints(160)) == 0
    assert L.pivot_pages_compact(p, -1, FAKE, FAKE, FAKE, 1 << 40, None) == BAD
    assert L.pivot_pages_compact(p, 3, None, FAKE, FAKE, 1 << 40, None) == BAD
    assert L.pivot_pages_compact(p, 3, FAKE, None, FAKE, 1 << 40, None) == BAD
    assert L.pivot_pages_compact(p, 3, FAKE, FAKE, None, 1 << 40, None) == WS
    r = (pv.pivot_rows * 1)()
    assert L.pivot_pages_copy(p, 1, FAKE, 1, r, None) == BAD       # no address
    r[0].rows, r[0].row_bytes = FAKE, 10
    assert L.pivot_pages_copy(p, 1, FAKE, 1, r, None) == BAD
    r[0].row_bytes = 12
    assert L.pivot_pages_copy(p, 1, None, 1, r, None) == BAD and L.pivot_pages_copy(p, -1, FAKE, 1, r, None) == BAD
    assert L.pivot_pages_copy(p, 1, FAKE, 0, r, None) == BAD and L.pivot_pages_copy(p, 0, None, 1, r, None) == pv.PIVOT_OK


@pytest.mark.parametrize("slots", [200, 1 << 15, 40000])
def test_slots_that_come_twice(slots):
    """Small tables look them up as bits, large ones sort."""
    L, p = pv.lib(), ctypes.byref(pages(slots=slots))
    for n in (2, 63, 64, 65, 200):
        slot = list(range(slots - n, slots))
        slot[-1] = slot[n // 2 - 1]
        same = ints(*[5] * n)
        assert L.pivot_pages_free(p, n, ints(*slot), same, same, None) == BAD and f"slot {slot[-1]} twice" in pv.last_error()
        assert L.pivot_pages_fork(p, 1, ints(slot[0]), ints(slot[0]), ints(5), None) == BAD
        assert L.pivot_pages_free(pages(slots=slots, refs=None), n, ints(*range(slots - n, slots)), same, same, None) == BAD
        assert "refs" in pv.last_error()   # distinct slots come to the next check


# ------------------------------------------------------------------ the binding
def _pool():
    return pv.make_pages(torch.full((4, 8), -1, dtype=torch.int32), torch.zeros(20, dtype=torch.int32), 16)


HOST_CALLS = [
    lambda: pv.pivot_linear4(torch.zeros((2, 64)).bfloat16(), torch.zeros((5, 32), dtype=torch.uint8),
                             torch.zeros((5, 2), dtype=torch.uint8)),
    lambda: pv.pivot_linear4_pack(torch.zeros((2, 64))),
    lambda: pv.pivot_tree_accept(torch.zeros((2, 3), dtype=torch.int32), [0, 0], [torch.zeros((64, 4))],
                                 pv.make_row_map(seq_stride=32, rows=64)),
    lambda: pv.pivot_pages_fork(_pool(), [0], [1], [5]),
    lambda: pv.pivot_pages_free(_pool(), [0], [5], [1]),
    lambda: pv.pivot_pages_grow(_pool(), [0], [5], [9]),
    lambda: pv.pivot_pages_compact(_pool(), 3),
    lambda: pv.pivot_pages_copy(_pool(), torch.zeros((1, 2), dtype=torch.int32), [torch.zeros((320, 4))]),
]


@pytest.mark.parametrize("call", HOST_CALLS)
def test_host_tensors_are_refused(call):
    with pytest.raises(ValueError, match="GPU"):
        call()


U8, BF = torch.uint8, torch.bfloat16
WRONG = [
    lambda: pv.pivot_linear4(torch.zeros((2, 64)), torch.zeros((5, 32), dtype=U8), torch.zeros((5, 2), dtype=U8)),
    lambda: pv.pivot_linear4(torch.zeros((2, 64), dtype=BF), torch.zeros((5, 31), dtype=U8), torch.zeros((5, 2), dtype=U8)),
    lambda: pv.pivot_linear4(torch.zeros((2, 64), dtype=BF), torch.zeros((5, 32), dtype=U8), torch.zeros((4, 2), dtype=U8)),
    lambda: pv.pivot_linear4(torch.zeros((2, 64), dtype=U8), torch.zeros((5, 32), dtype=U8), torch.zeros((5, 2), dtype=U8)),
    lambda: pv.pivot_linear4(torch.zeros((2, 64), dtype=U8), torch.zeros((5, 32), dtype=U8), torch.zeros((5, 2), dtype=U8),
                             x_scale=torch.zeros((2, 2))),
    lambda: pv.pivot_linear4(torch.zeros((2, 64), dtype=BF), torch.zeros((5, 32), dtype=U8), torch.zeros((5, 2), dtype=U8),
                             dtype=torch.float16),
    lambda: pv.pivot_linear4(torch.zeros((64, 2), dtype=BF).t(), torch.zeros((5, 32), dtype=U8),
                             torch.zeros((5, 2), dtype=U8)),
    lambda: pv.pivot_linear4_pack(torch.zeros((2, 40))),
    lambda: pv.pivot_linear4_pack(torch.zeros(64)),
    lambda: pv.pivot_tree_accept(torch.zeros((2, 3)), [0, 0], [torch.zeros((64, 4))], pv.make_row_map(seq_stride=32, rows=64)),
    lambda: pv.pivot_tree_accept(torch.zeros((2, 3), dtype=torch.int32), [0], [torch.zeros((64, 4))],
                                 pv.make_row_map(seq_stride=32, rows=64)),
    lambda: pv.make_pages(torch.zeros((2, 3)), torch.zeros(4, dtype=torch.int32), 16),
    lambda: pv.make_pages(torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 2), dtype=torch.int32), 16),
    lambda: pv.pivot_pages_fork(_pool(), [0], [1, 2], [5]),
    lambda: pv.pivot_pages_copy(_pool(), torch.zeros((1, 3), dtype=torch.int32), [torch.zeros((320, 4))]),
]


@pytest.mark.parametrize("call", WRONG)
def test_shapes_and_types_are_checked(call):
    with pytest.raises(ValueError):
        call()


# ------------------------------------------------------------------ the definitions
def test_masks_hold_a_node_and_its_ancestors():
    seen, words = plain.tree_masks(np.random.default_rng(0), 70, 3)
    assert words.shape == (70, 3) and seen.diagonal().all() and not np.triu(seen, 1).any()
    for i in range(70):
        bits = {j for j in range(96) if words[i, j // 32] >> (j % 32) & 1}
        assert bits == set(np.nonzero(seen[i])[0])
        parent = max(bits - {i}, default=None)
        assert parent is None or set(np.nonzero(seen[parent])[0]) == bits - {i}


def test_the_pool_keeps_its_counts():
    p = plain.Pool(4, 6, 16, 12)
    assert p.grow([0], [0], [40])[1] == (0, 9)
    p.fork([0], [1], [40])
    pairs, state = p.grow([0, 1], [40, 40], [41, 49])
    assert pairs.tolist() == [[2, 3], [-1, -1]] and state == (0, 7)
    assert p.table[0].tolist() == [0, 1, 3, -1, -1, -1] and p.table[1].tolist() == [0, 1, 2, 4, -1, -1]
    p.free([0], [41], [0])
    assert p.refs[:5].tolist() == [1, 1, 1, 0, 1]
    assert p.compact(4)[0].tolist() == [[4, 3], [-1, -1], [-1, -1], [-1, -1]] and p.table[1, 3] == 3


def test_the_bound_of_a_product_tells_its_rounding():
    """One bf16 step of an output, or a weight off by one code, lies outside the bound."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((4, 512))
    codes, scales = plain.quantise(rng.standard_normal((30, 512)))
    y, s = plain.linear(x, codes, scales)
    assert np.all(plain.linear_bound(512, s, y, False) < 2e-3 * s / np.sqrt(512))
    wrong = codes.copy()
    wrong[:, 7] ^= 1
    assert np.all(np.abs(plain.linear(x, wrong, scales)[0] - y) > plain.linear_bound(512, s, y, False))
