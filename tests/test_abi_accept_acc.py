"""C ABI of the acceptance that moves weights too, on the CPU: every argument it
refuses, with the documented status and before any launch."""
import ctypes
import os

import pytest
import torch

import paper_2607_24593_amd as pv
from test_abi_operators import ints, row_map

pytestmark = pytest.mark.skipif(not os.path.exists(pv.LIB_PATH), reason="libpivot.so not built")

FAKE = 1 << 40  # a non-null address the library must never dereference before launching
BAD, UNS = pv.PIVOT_ERR_INVALID_ARG, pv.PIVOT_ERR_UNSUPPORTED


def accept(batch=2, n=4, path=FAKE, pos0=(3, 5), nodes=(7, 9), n_arrays=1, rows=FAKE, acc=FAKE, stride=14, m=None):
    r = (pv.pivot_rows * 9)()
    for x in r:
        x.rows, x.row_bytes = rows, 16
    m = row_map() if m is None else m
    return pv.lib().pivot_tree_accept_acc(batch, n, path, ints(*pos0), None if nodes is None else ints(*nodes), n_arrays, r,
                                          ctypes.byref(m), acc, stride, None)


@pytest.mark.parametrize("kw,status", [
    (dict(acc=None), BAD), (dict(acc=FAKE + 2), BAD), (dict(nodes=None), BAD), (dict(nodes=(7, -1)), BAD),
    (dict(nodes=(7, 1025), stride=5000), UNS), (dict(stride=13), BAD), (dict(stride=-1), BAD),
    (dict(pos0=(3, pv.PIVOT_MAX_KEYS), stride=1 << 31), UNS), (dict(pos0=(250, 0), stride=300), BAD),  # 257 of 256 rows
    (dict(batch=0), BAD), (dict(n=-1), BAD), (dict(n=1025), UNS), (dict(path=None), BAD), (dict(path=FAKE + 1), BAD),
    (dict(n_arrays=0), BAD), (dict(rows=None), BAD), (dict(m=row_map(rows=0)), BAD), (dict(n=0, path=None, stride=13), BAD),
])
def test_refusals(kw, status):
    assert accept(**kw) == status
    assert pv.last_error() != ""


I32 = torch.int32


@pytest.mark.parametrize("kw", [
    dict(acc=torch.zeros((2, 32))), dict(nodes=[3, 3]), dict(acc=torch.zeros((2, 32)), nodes=[3]),
    dict(acc=torch.zeros((1, 32)), nodes=[3, 3]), dict(acc=torch.zeros((2, 32), dtype=torch.float64), nodes=[3, 3]),
    dict(acc=torch.zeros((32, 2)).t(), nodes=[3, 3]), dict(acc=torch.zeros(64), nodes=[3, 3]),
    dict(acc=torch.zeros((2, 32)), nodes=[3, 3]),  # host memory
])
def test_the_binding_checks_them(kw):
    with pytest.raises(ValueError):
        pv.pivot_tree_accept(torch.zeros((2, 3), dtype=I32), [0, 0], [torch.zeros((64, 4))],
                             pv.make_row_map(seq_stride=32, rows=64), **kw)
