"""pivot_norm_run into fp32 and fp16 where weight * h or 1 / rms leave the range of fp32 and the output does not."""
import numpy as np
import pytest

from oracle import pivot_quant_oracle as Q
from paper_1712_01084_amd import binding as B
import test_gpu_norm as N

pytestmark = N.pytestmark
F32, F16 = B.PIVOT_F32, B.PIVOT_F16
# The outputs are rounded once from 64 bits: half a step of their type, and below its normal numbers (beside one of 3e38 the
# others of a row are as small) half the subnormal step, 2^-149 / 2 and 2^-24 / 2.
HALF, SMALLEST = {F32: 2.0 ** -24, F16: 2.0 ** -11}, {F32: 2.0 ** -150, F16: 2.0 ** -25}


def check(x, w, otype, eps):
    out, _, _ = N.run(x, None, w, otype, eps, F32, F32)
    with np.errstate(all="ignore"):
        want = Q.norm(x, None, w, float(np.float32(eps)))[1]
    most = float(np.finfo(np.float16 if otype == F16 else np.float32).max)
    tolerance = HALF[otype] * 1.001 * np.abs(want) + SMALLEST[otype]
    assert np.abs(want).max() < most and (np.abs(out - want) <= tolerance).all()


@pytest.mark.parametrize("cols", [9, 300, 5000, 20000])
@pytest.mark.parametrize("otype", [F32, F16])
def test_large_rows_under_large_weights(cols, otype):
    rng = np.random.default_rng(cols)
    x = rng.normal(size=(3, cols)).astype(np.float32)
    x[0] *= np.float32(1e37)
    x[1, ::3] = 3e38
    w = rng.uniform(2.0, 60.0, cols).astype(np.float32)
    check(x, w, otype, 1e-6)


@pytest.mark.parametrize("cols", [9, 300, 5000, 20000])
def test_rows_whose_sum_is_beyond_fp32(cols):
    """x + res is not rounded before it is normalised; what is left in the residual is, and is infinite there."""
    rng = np.random.default_rng(cols + 1)
    x = (rng.choice([-1, 1], (2, cols)) * rng.uniform(2e38, 3.3e38, (2, cols))).astype(np.float32)
    out, left, _ = N.run(x, x.copy(), None, F32, 1e-6, F32, F32)
    want = Q.norm(x, x, None, 1e-6)[1]
    assert (np.abs(out - want) <= HALF[F32] * 1.001 * np.abs(want)).all()
    assert np.array_equal(np.isinf(left), np.abs(2.0 * x.astype(np.float64)) > np.finfo(np.float32).max)


@pytest.mark.parametrize("cols", [9, 300, 5000, 20000])
@pytest.mark.parametrize("otype", [F32, F16])
def test_small_rows_without_eps(cols, otype):
    """eps = 0: rows of subnormal numbers (1 / rms is beyond fp32), and small weights on small rows."""
    rng = np.random.default_rng(cols + 2)
    x = np.zeros((3, cols), np.float32)
    x[0] = rng.integers(-3, 4, cols) * np.float32(1e-45)
    x[0, 0] = 1e-45
    x[1] = rng.normal(size=cols) * 1e-36
    x[2] = rng.normal(size=cols)
    w = np.full(cols, 1e-6, np.float32) if otype == F32 else None
    check(x, w, otype, 0.0)


@pytest.mark.parametrize("cols", [9, 300, 5000, 20000])
def test_rows_of_fp16_under_large_weights(cols):
    """weight * h is beyond fp32, weight * h / rms is not.  In fp32: h and the products with 1 / rms, itself rounded, and with
    the weight are four roundings."""
    rng = np.random.default_rng(cols + 3)
    x, res = (rng.uniform(20000, 30000, (2, cols)).astype(np.float16) for _ in range(2))
    w = (rng.uniform(0.5, 1.0, cols) * 1e38).astype(np.float32)
    out, left, _ = N.run(x, res, w, F32, 0.0, F16, F16)
    want = Q.norm(x, res, w, 0.0)[1]
    assert np.array_equal(left, (x.astype(np.float64) + res).astype(np.float16))
    assert np.isfinite(want.astype(np.float32)).all() and (np.abs(out - want) <= 4.001 * 2.0 ** -24 * np.abs(want)).all()
