"""The binding of the operators around the index calls refuses tensors in host
memory: their addresses would go to kernels as they are."""
import os

import pytest
import torch

import paper_2607_24593_amd as pv

pytestmark = pytest.mark.skipif(not os.path.exists(pv.LIB_PATH), reason="libpivot.so not built")

BF = torch.bfloat16


def _cache(table=False):
    parts = (torch.zeros((64, 256), dtype=torch.uint8), torch.zeros((64, 16), dtype=torch.uint8), torch.zeros((64, 64), dtype=BF))
    bt = torch.zeros((2, 2), dtype=torch.int32) if table else None
    m = pv.make_row_map(seq_stride=32, rows=64, block_table=bt, page_size=16)
    return pv.make_cache4(*parts, m), parts, m


def _norm(group=0):
    x = torch.zeros((4, 64), dtype=BF)
    pv.pivot_rmsnorm_fp8(x, torch.ones(64, dtype=BF), residual=x, group=group)


def _write():
    pv.pivot_cache4_write(torch.zeros((4, 512), dtype=BF), torch.zeros((4, 64), dtype=BF), _cache()[0], [0, 0], 2)


def _read():
    pv.pivot_cache4_read(_cache(table=True)[0], torch.zeros((2, 3), dtype=torch.int32))


def _attend(idx=None, acc=None):
    pv.pivot_cache4_attend(torch.zeros((2, 1, 4, 576), dtype=BF), _cache()[0], [7, 7], [8, 8], 1.0, idx=idx, acc=acc)


def _attend_sets():
    _attend(torch.zeros((2, 1, 4), dtype=torch.int32), torch.zeros((2, 8)))


def _evict():
    pv.pivot_evict(torch.zeros((2, 32)), [32, 32], 4, [], None, None)


def _evict_rows():
    _, parts, m = _cache()
    pv.pivot_evict(torch.zeros((2, 32)), [32, 32], 4, [(parts[0], torch.zeros_like(parts[0]))], m, m)


@pytest.mark.parametrize("call", [_norm, _write, _read, _attend, _attend_sets, _evict, _evict_rows])
def test_host_tensors_are_refused(call):
    with pytest.raises(ValueError, match="GPU"):
        call()
