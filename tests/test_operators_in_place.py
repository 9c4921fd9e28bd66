"""The norm's sums may replace an input only where its rows are not padded."""
import os

import pytest

import paper_2607_24593_amd as pv

pytestmark = pytest.mark.skipif(not os.path.exists(pv.LIB_PATH), reason="libpivot.so not built")

X, RES, W, OTHER = (i << 40 for i in range(1, 5))  # addresses that are not read before a launch


def norm(out, ld_x=64, ld_res=64):
    return pv.lib().pivot_rmsnorm_fp8(0, 4, 64, X, ld_x, RES, ld_res, W, 1e-6, 0, out, OTHER, OTHER, None)


@pytest.mark.parametrize("kw", [dict(out=X, ld_x=80), dict(out=RES, ld_res=65), dict(out=X, ld_x=65, ld_res=70)])
def test_padded_rows_are_not_replaced(kw):
    assert norm(**kw) == pv.PIVOT_ERR_INVALID_ARG
    assert "padded" in pv.last_error()
