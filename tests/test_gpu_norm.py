"""pivot_norm_run against the float64 oracle.  Tolerances: h and the product with weight and 1 / rms are three roundings
and a correctly rounded factor in fp32 (4 * 2^-24 relative, doubled for what a difference x + res leaves of them), then
half a step of the output's type.  8-bit codes are computed in 64 bits and have to be equal."""
import numpy as np
import pytest
import torch

from oracle import pivot_quant_oracle as Q
from paper_1712_01084_amd import binding as B
import quant_util as U

pytestmark = pytest.mark.gpu
F32, F16, Q8 = B.PIVOT_F32, B.PIVOT_F16, B.PIVOT_Q8
NP = {F32: np.float32, F16: np.float16, Q8: np.int8}
HALF_STEP = {F32: 2.0 ** -24, F16: 2.0 ** -11}


def dev(a, ld=None, off=0):
    """A copy on the device, rows `ld` elements apart, `off` elements into its buffer."""
    ld = a.shape[1] if ld is None else ld
    buf = torch.full((off + a.shape[0] * ld,), 33, dtype=torch.from_numpy(a).dtype, device="cuda")
    v = buf[off:].view(a.shape[0], ld)
    v[:, :a.shape[1]] = torch.from_numpy(a).cuda()
    return v


def run(x, res, weight, otype, eps, xtype, rtype, order=None, in_place=False, ld=None, off=0, keep_res=True):
    rows, cols = x.shape
    xd, rd = dev(x, ld, off), None if res is None else dev(res, ld, off)
    wd = None if weight is None else dev(weight[None], None, off)
    out = dev(np.full((rows, cols), 99).astype(NP[otype]), ld, off)
    ro = None if res is None or not keep_res else (rd if in_place else dev(np.zeros_like(res), ld, off))
    sd = torch.full((rows,), -1.0, device="cuda") if otype == Q8 else None
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    B.pivot_norm_run(ptr(xd), xtype, xd.stride(0), ptr(out), otype, out.stride(0), rows, cols, weight_ptr=ptr(wd), eps=eps, res_ptr=ptr(rd),
                     rtype=rtype, ldr=0 if rd is None else rd.stride(0), res_out_ptr=ptr(ro), ldro=0 if ro is None else ro.stride(0),
                     scale_ptr=ptr(sd), order=order, stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    if ld is not None:
        assert (out[:, cols:] == 33).all() and (ro is None or (ro[:, cols:] == 33).all())      # what lies beside the rows
    host = lambda t: None if t is None else t[:, :cols].cpu().numpy()  # noqa: E731
    return host(out), host(ro), None if sd is None else sd.cpu().numpy()


def check(x, res, weight, otype, eps, xtype, rtype, order=None, pcol=None, **k):
    out, ro, s = run(x, res, weight, otype, eps, xtype, rtype, order=order, **k)
    h, y = Q.norm(x, res, weight, float(np.float32(eps)))
    mag = np.abs(x.astype(np.float64)) + (0 if res is None else np.abs(res.astype(np.float64)))
    if ro is not None:
        assert (np.abs(ro - h) <= HALF_STEP[rtype] * 1.001 * np.abs(h) + 2.0 ** -24 * mag + (2.0 ** -25 if rtype == F16 else 0)).all()
    if otype == Q8:
        codes, scale = Q.norm_codes(x, res, weight, float(np.float32(eps)))
        assert np.array_equal(out, codes if pcol is None else codes[:, pcol])
        assert np.allclose(s, scale, rtol=2.0 ** -22, atol=0)
        return
    want = y if pcol is None else y[:, pcol]
    factor = np.abs(y) / np.maximum(np.abs(h), 1e-300) * mag            # the terms of h, as they reach the output
    factor = factor if pcol is None else factor[:, pcol]
    assert (np.abs(out - want) <= 8 * 2.0 ** -24 * np.maximum(factor, np.abs(want)) + HALF_STEP[otype] * 1.001 * np.abs(want) + (2.0 ** -25 if otype == F16 else 0)).all()


COLS = [1, 7, 8, 64, 65, 500, 512, 513, 1000, 2048, 4096, 4104, 8200, 9203, 16384, 20000, 65535]


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("otype", [F32, F16, Q8])
def test_sizes_and_types(cols, otype):
    rng = np.random.default_rng(cols)
    for i, (xtype, rtype) in enumerate([(F32, None), (F16, None), (F32, F32), (F16, F16), (F32, F16), (F16, F32)]):
        rows = (1, 3, 5, 2, 9, 4)[i]
        x = rng.normal(size=(rows, cols)).astype(NP[xtype])
        res = None if rtype is None else (3 * rng.normal(size=(rows, cols))).astype(NP[rtype])
        w = None if i % 3 == 2 else rng.normal(1, 0.3, cols).astype(np.float32)
        check(x, res, w, otype, 1e-6, xtype, F32 if rtype is None else rtype, in_place=i % 2 == 1, keep_res=i != 4)


@pytest.mark.parametrize("cols", [40, 1024, 5000])
@pytest.mark.parametrize("otype", [F32, F16, Q8])
def test_strides_and_alignment(cols, otype):
    rng = np.random.default_rng(cols)
    x, res = rng.normal(size=(6, cols)).astype(np.float16), rng.normal(size=(6, cols)).astype(np.float32)
    w = rng.normal(1, 0.3, cols).astype(np.float32)
    for ld, off in ((cols + 1, 0), (cols + 8, 0), (cols + 16, 1), (cols + 24, 16)):
        check(x, res, w, otype, 1e-5, F16, F32, ld=ld, off=off)


@pytest.mark.parametrize("cols", [1, 37, 200, 3000, 9203])
@pytest.mark.parametrize("otype", [F32, F16, Q8])
def test_in_the_block_order_of_a_layer(cols, otype):
    rng = np.random.default_rng(cols)
    L = U.layer(rng, 16, cols, 16, 32, 32, perm=True)
    p = U.plan(L)
    try:
        x, res = rng.normal(size=(3, cols)).astype(np.float32), rng.normal(size=(3, cols)).astype(np.float16)
        check(x, res, rng.normal(1, 0.3, cols).astype(np.float32), otype, 1e-6, F32, F16, order=p, pcol=L["pcol"])
        with pytest.raises(B.PivotError) as e:
            run(np.zeros((1, cols + 1), np.float32), None, None, F32, 1e-6, F32, F32, order=p)
        assert e.value.code == B.PIVOT_E_SHAPE
    finally:
        B.pivot_qfc_plan_destroy(p)


def test_many_rows():
    rng = np.random.default_rng(1)
    for rows, cols, otype in ((70001, 24, F16), (5000, 300, Q8), (1000, 4096, Q8)):
        x = rng.normal(size=(rows, cols)).astype(np.float16)
        check(x, x[::-1].copy(), None, otype, 1e-6, F16, F16)


@pytest.mark.parametrize("cols", [16, 700, 5000, 30000])
def test_numbers_at_the_edges(cols):
    """Ties go to the even code; rows of zeros, infinities and NaNs; values near the ends of fp32's range."""
    x = np.zeros((9, cols), np.float32)
    x[0, :16] = [127, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5, -126.5, -127, 0, 1, 2, 3, 4, 5]
    x[2, 3] = np.inf
    x[3, 5] = np.nan
    x[4, 1], x[4, 2] = -np.inf, np.nan
    x[5, :4] = [3e38, -1e38, 1e30, 0]
    x[6, :4] = [1e-38, -3e-39, 1e-45, 0]
    x[7, cols - 1] = 1e-3
    x[8] = 1.0
    codes, scale = Q.norm_codes(x, None, None, float(np.float32(1e-6)))
    out, _, s = run(x, None, None, Q8, 1e-6, F32, F32)
    assert np.array_equal(out, codes) and np.allclose(s, scale, rtol=2.0 ** -22, atol=0, equal_nan=True)
    assert out[0, :16].tolist() == [127, 0, 2, 2, 0, -2, -2, 126, -126, -127, 0, 1, 2, 3, 4, 5]
    assert s[1] == 0 and np.isnan(s[2:5]).all()
    y, _, _ = run(x, None, None, F32, 1e-6, F32, F32)
    assert (y[1] == 0).all() and np.isnan(y[3]).all() and np.allclose(y[8], 1.0, atol=1e-5)
    assert np.allclose(y[5], Q.norm(x[5:6], None, None, 1e-6)[1][0], rtol=1e-6, atol=0)


def test_captured():
    rng = np.random.default_rng(3)
    x = torch.zeros(5, 3000, device="cuda")
    out, s = torch.zeros(5, 3000, dtype=torch.int8, device="cuda"), torch.zeros(5, device="cuda")
    g = torch.cuda.CUDAGraph()

    def go():
        B.pivot_norm_run(x.data_ptr(), F32, 3000, out.data_ptr(), Q8, 3000, 5, 3000, scale_ptr=s.data_ptr(), stream=torch.cuda.current_stream().cuda_stream)

    go()
    with torch.cuda.graph(g):
        go()
    for _ in range(3):
        a = rng.normal(size=(5, 3000)).astype(np.float32)
        x.copy_(torch.from_numpy(a))
        g.replay()
        torch.cuda.synchronize()
        codes, scale = Q.norm_codes(a, None, None, float(np.float32(1e-6)))
        assert np.array_equal(out.cpu().numpy(), codes) and np.allclose(s.cpu().numpy(), scale, rtol=2.0 ** -22, atol=0)
