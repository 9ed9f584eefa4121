"""Norm rows in a layer's block order: rows too long for LDS or for registers, and many rows at a time."""
import numpy as np
import pytest

from paper_1712_01084_amd import binding as B
import quant_util as U
import test_gpu_norm as N

pytestmark = N.pytestmark
F32, F16, Q8 = B.PIVOT_F32, B.PIVOT_F16, B.PIVOT_Q8


@pytest.mark.parametrize("rows,cols", [(3, 15361), (2, 16384), (3, 16385), (2, 31000), (1, 61441), (2, 65535),      # one, two and more pieces to a thread
                                       (700, 40), (513, 700), (600, 3001), (512, 4096), (520, 5000)])              # few threads to a row
@pytest.mark.parametrize("otype", [F32, F16, Q8])
def test_rows_in_block_order(rows, cols, otype):
    rng = np.random.default_rng(rows + cols)
    L = U.layer(rng, 16, cols, 16, 32, 32, perm=True)
    p = U.plan(L)
    try:
        w = rng.normal(1, 0.3, cols).astype(np.float32)
        for xtype, rtype in ((F16, F16), (F32, F16)):
            x, res = rng.normal(size=(rows, cols)).astype(N.NP[xtype]), rng.normal(size=(rows, cols)).astype(N.NP[rtype])
            N.check(x, res, w, otype, 1e-6, xtype, rtype, order=p, pcol=L["pcol"], in_place=xtype == F32)
    finally:
        B.pivot_qfc_plan_destroy(p)
