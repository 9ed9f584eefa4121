"""What the flags of a 4-bit layer's plan are refused for without a device (no GPU)."""
import pytest

from paper_1712_01084_amd import binding as B


@pytest.mark.parametrize("code,k", [(B.PIVOT_E_NO_DEVICE, dict(device=-1)), (B.PIVOT_E_NULL, dict(codes=None)), (B.PIVOT_E_SHAPE, dict(scales=4097)),
                                    (B.PIVOT_E_SHAPE, dict(bias=4098)), (B.PIVOT_E_UNSUPPORTED, dict(flags=3))])
def test_weights_on_the_device(code, k):
    a = dict(dict(codes=4096, scales=4096, bias=4096, device=0, flags=B.PIVOT_QFC_WEIGHTS_ON_DEVICE), **k)
    with pytest.raises(B.PivotError) as e:
        B.pivot_qfc_plan(16, 64, 16, 32, 32, a["codes"], a["scales"], bias=a["bias"], device=a["device"], flags=a["flags"])
    assert e.value.code == code
