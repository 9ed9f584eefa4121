"""The name of the kernel of a 4-bit layer's run follows the run's arguments: order, address and stride of x (no GPU)."""
import numpy as np
import pytest

from paper_1712_01084_amd import binding as B
import quant_util as U


def form(name):
    """(kernel, its arguments without the types)."""
    return name[:name.index("<")], tuple(name.rstrip(">").split(", ")[3:])


@pytest.mark.parametrize("xtype", [B.PIVOT_F16, B.PIVOT_Q8])
def test_names_follow_the_call(xtype):
    rng = np.random.default_rng(1)
    p = U.plan(U.layer(rng, 9000, 512, 32, 32, 32, perm=True), device=-1)
    try:
        rows = "pivot::qfc_rows_kernel"
        name = lambda x=None, ldx=512, flags=0, batch=1: form(B.pivot_qfc_run_kernel_name(p, x, xtype, ldx, batch, flags=flags))  # noqa: E731
        assert name() == form(B.pivot_qfc_kernel_name(p, xtype, 1)) == (rows, ("1", "false", "8"))     # gathers
        block = B.PIVOT_QFC_X_BLOCK_ORDER
        assert name(flags=block) == (rows, ("2", "true", "8"))             # as it lies, two strips to a work item
        assert name(x=4096 + 2, flags=block) == (rows, ("1", "false", "8"))
        assert name(ldx=513, flags=block) == (rows, ("2", "true", "8"))    # a single row has no stride
        assert name(ldx=513, flags=block, batch=2) == (rows, ("1", "false", "8"))
        assert name(flags=block, batch=64)[0] == "pivot::qfc_frag_kernel"
        for code, k in ((B.PIVOT_E_UNSUPPORTED, dict(flags=2)), (B.PIVOT_E_SHAPE, dict(ldx=511)), (B.PIVOT_E_SHAPE, dict(batch=65))):
            with pytest.raises(B.PivotError) as e:
                name(**k)
            assert e.value.code == code
    finally:
        B.pivot_qfc_plan_destroy(p)
    with pytest.raises(B.PivotError) as e:
        B.pivot_qfc_kernel_name(None, xtype, 1)
    assert e.value.code == B.PIVOT_E_NULL
