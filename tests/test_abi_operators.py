"""C ABI of the operators around the index calls on the CPU: every argument they
refuse, with the documented status and before any launch, and the definitions
the GPU tests compare with."""
import ctypes
import os

import numpy as np
import pytest
import torch

import ops_ref
import paper_2607_24593_amd as pv

pytestmark = pytest.mark.skipif(not os.path.exists(pv.LIB_PATH), reason="libpivot.so not built")

FAKE = 1 << 40  # a non-null address the library must never dereference before launching
BAD, UNS, WS = pv.PIVOT_ERR_INVALID_ARG, pv.PIVOT_ERR_UNSUPPORTED, pv.PIVOT_ERR_WORKSPACE


def ints(*v):
    return (ctypes.c_int32 * len(v))(*v)


def norm(dtype=0, rows=4, dim=64, x=FAKE, ld=64, res=FAKE, ld_res=64, w=FAKE, eps=1e-6, group=0, out=FAKE, codes=FAKE,
         scale=FAKE):
    return pv.lib().pivot_rmsnorm_fp8(dtype, rows, dim, x, ld, res, ld_res, w, eps, group, out, codes, scale, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=1), UNS), (dict(dtype=7), UNS), (dict(rows=-1), BAD), (dict(dim=0), BAD), (dict(dim=40000, ld=40000), UNS),
    (dict(group=64), UNS), (dict(group=-1), UNS), (dict(eps=-1.0), BAD), (dict(eps=float("nan")), BAD),
    (dict(eps=float("inf")), BAD), (dict(ld=63), BAD), (dict(ld_res=63), BAD), (dict(x=None), BAD), (dict(w=None), BAD),
    (dict(codes=None), BAD), (dict(scale=None), BAD), (dict(x=FAKE + 1), BAD), (dict(scale=FAKE + 2), BAD),
    (dict(dtype=2, w=FAKE + 2), BAD),
])
def test_norm_refusals(kw, status):
    assert norm(**kw) == status
    assert pv.last_error() != ""


def test_norm_of_no_rows():
    assert norm(rows=0, x=None, codes=None) == pv.PIVOT_OK


def row_map(rows=1024, stride=256, table=None, max_pages=0, page=0):
    m = pv.pivot_row_map()
    m.rows, m.seq_stride, m.block_table, m.max_pages, m.page_size = rows, stride, table, max_pages, page
    return m


def cache(codes=FAKE, scales=FAKE, rope=FAKE, **kw):
    c = pv.pivot_cache4()
    c.codes, c.scales, c.rope, c.map = codes, scales, rope, row_map(**kw)
    return c


MAPS = [
    (dict(rows=0), BAD), (dict(rows=1 << 31), BAD), (dict(stride=0), BAD), (dict(stride=4), BAD),
    (dict(stride=600), BAD),                                                 # 2 * 600 rows > 1024
    (dict(table=FAKE, page=24, max_pages=20), BAD), (dict(table=FAKE, page=8, max_pages=50), BAD),
    (dict(table=FAKE, page=16, max_pages=0), BAD), (dict(table=FAKE, page=16, max_pages=3), BAD),   # 48 tokens < 100
    (dict(table=FAKE, page=16, max_pages=50, rows=1000), BAD), (dict(codes=None), BAD), (dict(scales=None), BAD),
    (dict(rope=None), BAD), (dict(codes=FAKE + 8), BAD), (dict(scales=FAKE + 4), BAD), (dict(rope=FAKE + 2), BAD),
]


@pytest.mark.parametrize("kw,status", MAPS)
def test_cache_refusals(kw, status):
    c = cache(**kw)
    assert pv.lib().pivot_cache4_write(ctypes.byref(c), 2, 10, None, ints(0, 90), FAKE, 512, FAKE, 64, None) == status
    assert pv.lib().pivot_cache4_attend(ctypes.byref(attend(cache=c))) == status
    assert pv.last_error() != ""


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), BAD), (dict(n=-1), BAD), (dict(cu=(1, 2, 3)), BAD), (dict(cu=(0, 5, 3)), BAD), (dict(pos=(-1, 0)), BAD),
    (dict(pos=(0, 250)), BAD), (dict(pos=(0, pv.PIVOT_MAX_KEYS)), UNS), (dict(latent=None), BAD), (dict(rope=None), BAD),
    (dict(latent=FAKE + 1), BAD), (dict(ld=511), BAD), (dict(ld_rope=63), BAD), (dict(n=0x7FFFFFFF, pos=(0, 0)), UNS),
])
def test_write_refusals(kw, status):
    a = dict(batch=2, n=10, cu=None, pos=(0, 90), latent=FAKE, ld=512, rope=FAKE, ld_rope=64)
    a.update(kw)
    c = cache()
    assert pv.lib().pivot_cache4_write(ctypes.byref(c), a["batch"], a["n"], None if a["cu"] is None else ints(*a["cu"]),
                                       ints(*a["pos"]), a["latent"], a["ld"], a["rope"], a["ld_rope"], None) == status
    assert pv.last_error() != ""


def test_write_and_read_of_nothing():
    c = cache(codes=None)
    L = pv.lib()
    assert L.pivot_cache4_write(ctypes.byref(c), 2, 0, None, ints(0, 0), None, 0, None, 0, None) == pv.PIVOT_OK
    assert L.pivot_cache4_write(ctypes.byref(c), 2, 9, ints(0, 0, 0), ints(0, 0), None, 0, None, 0, None) == pv.PIVOT_OK
    assert L.pivot_cache4_read(ctypes.byref(c), 2, 0, None, None, None) == pv.PIVOT_OK
    assert L.pivot_cache4_write(None, 2, 0, None, ints(0, 0), None, 0, None, 0, None) == BAD
    assert L.pivot_cache4_read(None, 2, 0, None, None, None) == BAD


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), BAD), (dict(n=-1), BAD), (dict(idx=None), BAD), (dict(out=None), BAD), (dict(out=FAKE + 8), BAD),
    (dict(batch=1 << 20, n=1 << 20), UNS),
])
def test_read_refusals(kw, status):
    a = dict(batch=2, n=10, idx=FAKE, out=FAKE)
    a.update(kw)
    c = cache()
    assert pv.lib().pivot_cache4_read(ctypes.byref(c), a["batch"], a["n"], a["idx"], a["out"], None) == status


def attend(heads=16, batch=2, n_q=2, cu=None, pos=(0, 98), n_k=(50, 100), q=FAKE, row=16 * 576, head=576, cache=cache(),
           idx=None, topk=0, scale=0.04, out=FAKE, acc=None, acc_stride=0, ws=None, ws_bytes=0):
    a = pv.pivot_attend_args()
    a.heads, a.batch, a.n_q, a.topk, a.scale = heads, batch, n_q, topk, scale
    a._k = [ints(*pos) if pos else None, ints(*n_k) if n_k else None, ints(*cu) if cu else None]
    PI = ctypes.POINTER(ctypes.c_int32)
    a.q_pos0 = ctypes.cast(a._k[0], PI) if pos else None
    a.n_k = ctypes.cast(a._k[1], PI) if n_k else None
    a.cu_q = ctypes.cast(a._k[2], PI) if cu else None
    a.q, a.q_row_stride, a.q_head_stride, a.cache, a.idx = q, row, head, cache, idx
    a.out, a.acc, a.acc_stride, a.workspace, a.workspace_bytes = out, acc, acc_stride, ws, ws_bytes
    return a


@pytest.mark.parametrize("kw,status", [
    (dict(heads=0), UNS), (dict(heads=129, row=129 * 576), UNS), (dict(batch=0), BAD), (dict(n_q=-1), BAD),
    (dict(pos=None), BAD), (dict(n_k=None), BAD), (dict(pos=(0, 99)), BAD), (dict(pos=(-1, 0)), BAD),
    (dict(cu=(0, 3, 2)), BAD), (dict(cu=(1, 2, 3)), BAD), (dict(n_k=(50, pv.PIVOT_MAX_KEYS + 1)), UNS),
    (dict(topk=-1), BAD), (dict(scale=float("nan")), BAD), (dict(scale=float("inf")), BAD), (dict(q=None), BAD),
    (dict(out=None), BAD), (dict(q=FAKE + 2), BAD), (dict(out=FAKE + 8), BAD), (dict(head=575), BAD), (dict(head=577), BAD),
    (dict(row=16 * 576 - 8), BAD), (dict(row=16 * 576 + 4), BAD), (dict(acc=FAKE, acc_stride=99), BAD),
    (dict(acc=FAKE, acc_stride=100), WS), (dict(acc=FAKE, acc_stride=100, ws=FAKE, ws_bytes=64), WS),
    (dict(acc=FAKE, acc_stride=100, ws=FAKE + 16, ws_bytes=1 << 30), BAD),
])
def test_attend_refusals(kw, status):
    assert pv.lib().pivot_cache4_attend(ctypes.byref(attend(**kw))) == status
    assert pv.last_error() != ""


def test_attend_of_nothing():
    L = pv.lib()
    assert L.pivot_cache4_attend(ctypes.byref(attend(n_q=0, q=None, out=None))) == pv.PIVOT_OK
    assert L.pivot_cache4_attend(ctypes.byref(attend(cu=(0, 0, 0), q=None))) == pv.PIVOT_OK
    assert L.pivot_cache4_attend(None) == BAD
    assert L.pivot_cache4_attend_workspace_size(None) == 0
    assert L.pivot_cache4_attend_workspace_size(ctypes.byref(attend(heads=0))) == 0
    assert L.pivot_cache4_attend_workspace_size(ctypes.byref(attend(acc=FAKE, acc_stride=100))) > 0


def evict(batch=2, n_k=(100, 50), acc=FAKE, stride=100, keep=20, sink=4, recent=8, out=FAKE, n_arrays=1, src=FAKE,
          dst=2 * FAKE, row_bytes=256, frm=None, to=None):
    a = pv.pivot_evict_args()
    a._k = ints(*n_k) if n_k else None
    a.n_k = ctypes.cast(a._k, ctypes.POINTER(ctypes.c_int32)) if n_k else None
    a.batch, a.acc, a.acc_stride, a.keep, a.sink, a.recent, a.out_keep = batch, acc, stride, keep, sink, recent, out
    a.n_arrays = n_arrays
    a.arrays[0].src, a.arrays[0].dst, a.arrays[0].row_bytes = src, dst, row_bytes
    a.from_, a.to = frm or row_map(), to or row_map()
    return a


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), BAD), (dict(n_k=None), BAD), (dict(n_k=(100, -1)), BAD), (dict(n_k=(100, pv.PIVOT_MAX_KEYS + 1)), UNS),
    (dict(keep=0, sink=0, recent=0), BAD), (dict(keep=11), BAD), (dict(sink=-1), BAD), (dict(recent=-1), BAD),
    (dict(acc=None), BAD), (dict(out=None), BAD), (dict(stride=99), BAD), (dict(n_arrays=9), BAD), (dict(n_arrays=-1), BAD),
    (dict(src=None), BAD), (dict(dst=None), BAD), (dict(row_bytes=6), BAD), (dict(row_bytes=0), BAD),
    (dict(src=FAKE + 2), BAD), (dict(dst=FAKE), BAD), (dict(frm=row_map(stride=99)), BAD), (dict(to=row_map(stride=19)), BAD),
    (dict(to=row_map(table=FAKE, page=16, max_pages=1)), BAD), (dict(frm=row_map(rows=0)), BAD),
    (dict(keep=pv.PIVOT_MAX_KEYS + 1), UNS),
])
def test_evict_refusals(kw, status):
    assert pv.lib().pivot_evict(ctypes.byref(evict(**kw))) == status
    assert pv.last_error() != ""


def test_evict_null():
    assert pv.lib().pivot_evict(None) == BAD
    assert pv.lib().pivot_evict_workspace_size(None) == 0


def test_binding_refusals():
    """The Python binding refuses tensors it cannot describe to the library."""
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    w = torch.ones(64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        pv.pivot_rmsnorm_fp8(x.half(), w.half())
    with pytest.raises(ValueError):
        pv.pivot_rmsnorm_fp8(x.t(), w)
    with pytest.raises(ValueError):
        pv.pivot_rmsnorm_fp8(x, w, residual=x.float())
    with pytest.raises(ValueError):
        pv.pivot_rmsnorm_fp8(x, w.float())
    with pytest.raises(ValueError):
        pv.pivot_rmsnorm_fp8(x, w, residual_out=x)
    parts = (torch.zeros((64, 256), dtype=torch.uint8), torch.zeros((64, 16), dtype=torch.uint8),
             torch.zeros((64, 64), dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        pv.make_cache4(*parts, pv.make_row_map(seq_stride=32, rows=65))
    with pytest.raises(ValueError):
        pv.make_cache4(parts[1], parts[0], parts[2], pv.make_row_map(seq_stride=32, rows=64))
    with pytest.raises(ValueError):
        pv.make_row_map(rows=64, block_table=torch.zeros((2, 2), dtype=torch.int64), page_size=16)
    c = pv.make_cache4(*parts, pv.make_row_map(rows=64, block_table=torch.zeros((1, 2), dtype=torch.int32), page_size=16))
    q = torch.zeros((2, 1, 4, 576), dtype=torch.bfloat16)
    with pytest.raises(ValueError):  # a table of one sequence, a call of two
        pv.pivot_cache4_attend(q, c, [0, 0], [8, 8], 1.0)
    with pytest.raises(ValueError):
        pv.pivot_cache4_attend(q.float(), c, [0], [8], 1.0)
    with pytest.raises(ValueError):
        pv.pivot_cache4_attend(q[:1], c, [0], [8], 1.0, idx=torch.zeros((1, 1, 4), dtype=torch.int64))
    with pytest.raises(ValueError):
        pv.pivot_cache4_write(torch.zeros((3, 512), dtype=torch.bfloat16), torch.zeros((3, 64), dtype=torch.bfloat16), c, [0],
                              n_new=2)
    with pytest.raises(ValueError):
        pv.pivot_cache4_read(c, torch.zeros((2, 2), dtype=torch.int32))
    with pytest.raises(ValueError):
        pv.pivot_evict(torch.zeros((1, 8)), [8], 4, [(parts[0], parts[1])], c.map, c.map)


def test_reference_quantiser():
    """The 64-bit definition itself: its grid, its ties, its scale and its special blocks."""
    x = np.zeros((1, 512))
    x[0, :16] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -6.0]
    x[0, 32:34] = [6.5, -3.0]            # above 6: the scale doubles
    x[0, 64], x[0, 65] = np.inf, 1.0
    x[0, 96] = 2.0 ** -130
    codes, scales = ops_ref.quantise(x)
    v = ops_ref.values(codes, scales)[0]
    assert list(v[:16]) == [0, 1, 1, 2, 2, 4, 4, 6, 0, -1, -1, -2, -2, -4, -4, -6]
    assert list(v[32:34]) == [6.0, -3.0] and scales[0, 1] == 128     # 3.25 -> 3 and 1.5 -> 1.5, times two
    assert scales[0, 2] == 255 and np.isnan(v[64:96]).all()
    assert scales[0, 3] == 0 and v[96] == 0.0 and scales[0, 4] == 0
