"""Every form of the 4-bit layer's product, by the name of the kernel, on inputs whose sums are exact."""
import numpy as np
import pytest
import torch

from oracle import pivot_quant_oracle as Q
from paper_1712_01084_amd import binding as B
import quant_util as U
from test_gpu_qfc import inputs, run

pytestmark = pytest.mark.gpu
FORMS = ({("pivot::qfc_rows_kernel", (rs, fast, "8")) for rs, fast in (("1", "false"), ("1", "true"), ("2", "true"))}
         | {("pivot::qfc_frag_kernel", (nt, rs, "8")) for nt in "124" for rs in "12"})


@pytest.mark.parametrize("group,zeros", [(32, False), (64, True), (128, False)])
@pytest.mark.parametrize("xtype", [B.PIVOT_F16, B.PIVOT_Q8])
def test_all_forms(group, zeros, xtype):
    rng = np.random.default_rng(group)
    seen = set()
    for M, K, bh in ((16384, 608, 32), (4096, 704, 16)):
        L = U.layer(rng, M, K, bh, max(32, group), group, kept=0.9, zeros=zeros, perm=True, whole=True)
        p = U.plan(L)
        try:
            for block in (False, True):
                x, xd, sd = inputs(rng, L, 64, xtype, block)
                want = Q.qfc(L, x)[0].astype(np.float32)
                for batch in (1, 3, 8, 16, 29, 64):
                    name = B.pivot_qfc_run_kernel_name(p, xd.data_ptr(), xtype, K, batch, flags=B.PIVOT_QFC_X_BLOCK_ORDER if block else 0)
                    seen.add((name[:name.index("<")], tuple(name.rstrip(">").split(", ")[3:])))
                    y = run(p, L, xd, sd, batch, xtype, block).cpu().numpy()
                    assert np.array_equal(y, want[:batch]), "%dx%d batch %d: %s" % (M, K, batch, name)
        finally:
            B.pivot_qfc_plan_destroy(p)
    assert seen == FORMS, sorted(FORMS ^ seen)
