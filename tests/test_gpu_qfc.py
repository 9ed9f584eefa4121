"""Layers with 4-bit weights on the GPU against the float64 oracle.  Most inputs are small integers with scales that are
powers of two: every sum is then exact in fp32 whatever its order, and the outputs have to be equal."""
import numpy as np
import pytest
import torch

from oracle import pivot_quant_oracle as Q
from paper_1712_01084_amd import binding as B
import gpu_util as G
import quant_util as U

pytestmark = pytest.mark.gpu


def stream():
    return torch.cuda.current_stream().cuda_stream


def inputs(rng, L, batch, xtype, block, whole=True):
    """x in natural coordinates (float64), and what the call gets: device tensor and scales."""
    K = L["K"]
    if xtype == B.PIVOT_Q8:
        q = rng.integers(-9 if whole else -127, 10 if whole else 128, (batch, K)).astype(np.int8)
        s = (2.0 ** rng.integers(-2, 3, batch) if whole else rng.uniform(0.01, 0.03, batch)).astype(np.float32)
        x = q.astype(np.float64) * s[:, None].astype(np.float64)
    else:
        q = (rng.integers(-4, 5, (batch, K)) if whole else rng.normal(size=(batch, K))).astype(np.float16)
        s, x = None, q.astype(np.float64)
    if block and L["pcol"] is not None:
        q = q[:, L["pcol"]]
    return x, torch.from_numpy(np.ascontiguousarray(q)).cuda(), None if s is None else torch.from_numpy(s).cuda()


def run(p, L, xd, sd, batch, xtype, block, ws=None, ldx=None, ldy=None, y=None, y_off=0):
    ws = G.workspace(B.pivot_qfc_workspace_bytes(p, batch)) if ws is None else ws
    ldy = L["M"] if ldy is None else ldy
    y = torch.full((batch, ldy), float("nan"), device="cuda") if y is None else y
    B.pivot_qfc_run(p, xd.data_ptr(), xtype, L["K"] if ldx is None else ldx, None if sd is None else sd.data_ptr(), y.data_ptr() + 4 * y_off,
                    ldy, batch, ws.data_ptr(), ws.numel(), stream(), flags=B.PIVOT_QFC_X_BLOCK_ORDER if block else 0)
    return y


SHAPES = [  # M, K, bh, bw, group, kept
    (1, 1, 16, 32, 32, 1.0), (16, 128, 16, 128, 128, 1.0), (33, 129, 16, 32, 64, 1.0), (100, 333, 32, 64, 32, 0.5),
    (200, 1000, 64, 32, 128, 0.4), (65, 700, 64, 128, 64, 0.6), (500, 260, 16, 64, 64, 0.3), (128, 2000, 32, 128, 32, 0.8),
]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("xtype,block", [(B.PIVOT_F16, False), (B.PIVOT_F16, True), (B.PIVOT_Q8, True), (B.PIVOT_Q8, False)])
def test_exact_sums(shape, zeros, xtype, block):
    M, K, bh, bw, group, kept = shape
    rng = np.random.default_rng(M * K + zeros)
    L = U.layer(rng, M, K, bh, bw, group, kept=kept, zeros=zeros, perm=M % 2 == 0, whole=True, act=M % 3 == 0, empty_row=M == 200)
    p = U.plan(L)
    try:
        for batch in (1, 2, 4, 5, 16, 17, 33, 64):
            x, xd, sd = inputs(rng, L, batch, xtype, block)
            y = run(p, L, xd, sd, batch, xtype, block).cpu().numpy()
            assert np.array_equal(y, Q.qfc(L, x)[0].astype(np.float32)), "batch %d" % batch
    finally:
        B.pivot_qfc_plan_destroy(p)


@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("perm", [False, True])
@pytest.mark.parametrize("xtype", [B.PIVOT_F16, B.PIVOT_Q8])
def test_every_form(group, zeros, perm, xtype):
    """Sizes at which two strips make a work item, x is copied first in either order, or is read as it lies."""
    rng = np.random.default_rng(group + perm)
    seen = set()
    for M, K, bh in ((16384, 600, 32), (8200, 664, 64), (4096, 700, 16)):
        L = U.layer(rng, M, K, bh, max(32, group), group, kept=0.9, zeros=zeros, perm=perm, whole=True, act=1)
        p = U.plan(L)
        try:
            x, xd, sd = inputs(rng, L, 64, xtype, False)
            want = Q.qfc(L, x)[0].astype(np.float32)
            for batch in (1, 4, 7, 16, 24, 64):
                seen.add(B.pivot_qfc_kernel_name(p, xtype, batch))
                y = run(p, L, xd, sd, batch, xtype, False).cpu().numpy()
                assert np.array_equal(y, want[:batch]), "%dx%d batch %d" % (M, K, batch)
        finally:
            B.pivot_qfc_plan_destroy(p)
    forms = {(n[:n.index("<")], tuple(n.rstrip(">").split(", ")[3:])) for n in seen}                     # without the types
    assert len(forms) >= 6, sorted(forms)


def test_the_longest_rows_and_layers_without_tiles():
    rng = np.random.default_rng(65535)
    for M, K, kept in ((40, 65535, 1.0), (100, 300, 0.0)):
        L = U.layer(rng, M, K, 32, 128, 128, kept=kept, zeros=True, perm=True, whole=True)
        L["scales"][:] = 0.5                                   # sums of up to 65535 * 15 * 9 / 2 stay exact
        p = U.plan(L)
        try:
            for batch in (1, 3, 20):
                for xtype in (B.PIVOT_F16, B.PIVOT_Q8):
                    x, xd, sd = inputs(rng, L, batch, xtype, False)
                    y = run(p, L, xd, sd, batch, xtype, False).cpu().numpy()
                    assert np.array_equal(y, Q.qfc(L, x)[0].astype(np.float32))
        finally:
            B.pivot_qfc_plan_destroy(p)


def test_two_streams_at_once():
    rng = np.random.default_rng(12)
    L = U.layer(rng, 1000, 2000, 32, 64, 64, kept=0.8, zeros=True, perm=True, whole=True)
    p = U.plan(L, chunk_blocks=3)
    try:
        jobs = []
        for k in range(2):
            x, xd, sd = inputs(rng, L, 9, B.PIVOT_F16, False)
            jobs.append((torch.cuda.Stream(), xd, Q.qfc(L, x)[0].astype(np.float32), G.workspace(B.pivot_qfc_workspace_bytes(p, 9)),
                         torch.zeros(9, 1000, device="cuda")))
        torch.cuda.synchronize()
        for _ in range(20):
            for s, xd, _, ws, y in jobs:
                with torch.cuda.stream(s):
                    run(p, L, xd, None, 9, B.PIVOT_F16, False, ws=ws, y=y)
        torch.cuda.synchronize()
        for _, _, want, _, y in jobs:
            assert np.array_equal(y.cpu().numpy(), want)
    finally:
        B.pivot_qfc_plan_destroy(p)


@pytest.mark.parametrize("chunk_blocks", [1, 2, 5])
@pytest.mark.parametrize("bh", [16, 64])
def test_block_rows_in_pieces_on_one_workspace(chunk_blocks, bh):
    rng = np.random.default_rng(bh + chunk_blocks)
    L = U.layer(rng, 150, 1700, bh, 64, 64, kept=0.6, zeros=True, perm=True, whole=True, empty_row=True)
    p = U.plan(L, chunk_blocks=chunk_blocks)
    try:
        ws = G.workspace(B.pivot_qfc_workspace_bytes(p, 64))
        for batch in (64, 1, 7, 20, 1, 64):
            for xtype in (B.PIVOT_F16, B.PIVOT_Q8):
                x, xd, sd = inputs(rng, L, batch, xtype, False)
                for _ in range(2):
                    y = run(p, L, xd, sd, batch, xtype, False, ws=ws).cpu().numpy()
                    assert np.array_equal(y, Q.qfc(L, x)[0].astype(np.float32)), "batch %d" % batch
    finally:
        B.pivot_qfc_plan_destroy(p)


@pytest.mark.parametrize("shape", [(700, 3001, 16, 32, 32, 0.5), (1000, 4090, 64, 128, 128, 1.0), (96, 9203, 32, 64, 64, 1.0)])
@pytest.mark.parametrize("xtype", [B.PIVOT_F16, B.PIVOT_Q8])
def test_real_values_within_the_bound(shape, xtype):
    M, K, bh, bw, group, kept = shape
    rng = np.random.default_rng(K)
    L = U.layer(rng, M, K, bh, bw, group, kept=kept, zeros=K % 2 == 1, perm=True)
    p = U.plan(L)
    try:
        for batch in (1, 3, 16, 40):
            x, xd, sd = inputs(rng, L, batch, xtype, False, whole=False)
            y = run(p, L, xd, sd, batch, xtype, False).cpu().numpy()
            again = run(p, L, xd, sd, batch, xtype, False).cpu().numpy()
            assert y.tobytes() == again.tobytes()
            want, bound = Q.qfc(L, x)
            assert (np.abs(y - want) <= bound).all()
            # the order of the sums apart, nothing is rounded: in the mean the error is that of a few fp32 roundings
            assert np.linalg.norm(y - want) <= 16 * 2.0 ** -24 * np.linalg.norm(want)
    finally:
        B.pivot_qfc_plan_destroy(p)


@pytest.mark.parametrize("perm", [False, True])
@pytest.mark.parametrize("xtype", [B.PIVOT_F16, B.PIVOT_Q8])
def test_strides_offsets_and_what_lies_beside(perm, xtype):
    """Rows of x that are no whole 16-byte pieces, x at odd elements, y with gaps: only y's own elements are written."""
    rng = np.random.default_rng(7)
    L = U.layer(rng, 70, 250, 16, 32, 32, perm=perm, whole=True)
    p = U.plan(L)
    try:
        for batch in (1, 6, 20):
            for ldx, off in ((250, 1), (251, 0), (256, 3), (264, 8)):
                x, xd, sd = inputs(rng, L, batch, xtype, False)
                big = torch.full((off + batch * ldx + 16,), float("nan") if xtype == B.PIVOT_F16 else 77, dtype=xd.dtype, device="cuda")
                big[off:off + batch * ldx].view(batch, ldx)[:, :250] = xd
                y = torch.full((batch + 1, 75), -5.0, device="cuda")
                run(p, L, big[off:], sd, batch, xtype, False, ldx=ldx, ldy=75, y=y, y_off=2)
                y = y.cpu().numpy().reshape(-1)
                want = np.full_like(y, -5.0)
                for n in range(batch):
                    want[2 + 75 * n:72 + 75 * n] = Q.qfc(L, x)[0][n]
                assert np.array_equal(y, want)
    finally:
        B.pivot_qfc_plan_destroy(p)


def test_numbers_at_the_edges():
    """Subnormal fp16 inputs count; infinities and NaNs reach the rows that keep their column and no others, and no other
    batch row."""
    rng = np.random.default_rng(8)
    L = U.layer(rng, 64, 128, 16, 32, 32, perm=True, whole=True, bias=False)
    L["mask"] = np.ones((4, 4), np.uint8)
    L["mask"][0, 1] = 0
    L["codes"][:] = 0x99                                       # every code less 8 is 1
    p = U.plan(L)
    try:
        x = np.zeros((3, 128), np.float16)
        x[0] = 2.0 ** -24
        x[1, L["pcol"][40]] = np.inf                           # block column 1, which block row 0 has lost
        x[2, L["pcol"][40]] = np.nan
        y = run(p, L, torch.from_numpy(x).cuda(), None, 3, B.PIVOT_F16, False).cpu().numpy()
        assert np.array_equal(y[0], Q.qfc(L, x[:1].astype(np.float64))[0][0].astype(np.float32)) and (y[0] > 0).all()
        lost = L["prow"][:16]
        assert (y[1:, lost] == 0).all()
        rest = np.setdiff1d(np.arange(64), lost)
        assert np.isposinf(y[1, rest]).all() and np.isnan(y[2, rest]).all()
    finally:
        B.pivot_qfc_plan_destroy(p)
    p = U.plan(dict(L, act=1))
    try:
        x[1] *= -1
        y = run(p, dict(L, act=1), torch.from_numpy(x).cuda(), None, 3, B.PIVOT_F16, False).cpu().numpy()
        assert (y[1] == 0).all() and np.isnan(y[2, rest]).all()              # the activation keeps a NaN
    finally:
        B.pivot_qfc_plan_destroy(p)


@pytest.mark.parametrize("xtype", [B.PIVOT_F16, B.PIVOT_Q8])
def test_captured_and_on_another_stream(xtype):
    rng = np.random.default_rng(9)
    L = U.layer(rng, 300, 1500, 32, 32, 64, kept=0.7, zeros=True, perm=True, whole=True)
    p = U.plan(L, chunk_blocks=4)
    try:
        for batch in (1, 24):
            x, xd, sd = inputs(rng, L, batch, xtype, False)
            want = Q.qfc(L, x)[0].astype(np.float32)
            ws = G.workspace(B.pivot_qfc_workspace_bytes(p, batch))
            y = torch.zeros(batch, 300, device="cuda")
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                run(p, L, xd, sd, batch, xtype, False, ws=ws, y=y)
            side.synchronize()
            assert np.array_equal(y.cpu().numpy(), want)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                run(p, L, xd, sd, batch, xtype, False, ws=ws, y=y)
            for k in range(3):
                y.fill_(float("nan"))
                x, other, s2 = inputs(rng, L, batch, xtype, False)
                xd.copy_(other)
                if sd is not None:
                    sd.copy_(s2)
                g.replay()
                torch.cuda.synchronize()
                assert np.array_equal(y.cpu().numpy(), Q.qfc(L, x)[0].astype(np.float32)), "replay %d" % k
    finally:
        B.pivot_qfc_plan_destroy(p)


def test_run_calls_that_are_refused():
    rng = np.random.default_rng(10)
    L = U.layer(rng, 64, 2000, 64, 32, 32)
    p = U.plan(L, chunk_blocks=2)
    try:
        need = B.pivot_qfc_workspace_bytes(p, 2)
        ws = G.workspace(need)
        x = torch.zeros(2, 2000, dtype=torch.float16, device="cuda")
        s = torch.ones(2, device="cuda")
        y = torch.zeros(2, 64, device="cuda")
        ok = dict(x=x.data_ptr(), t=B.PIVOT_F16, ldx=2000, s=None, y=y.data_ptr(), ldy=64, b=2, ws=ws.data_ptr(), n=need, f=0)

        def call(**k):
            a = dict(ok, **k)
            B.pivot_qfc_run(p, a["x"], a["t"], a["ldx"], a["s"], a["y"], a["ldy"], a["b"], a["ws"], a["n"], stream(), flags=a["f"])

        for code, k in ((B.PIVOT_E_NULL, dict(x=None)), (B.PIVOT_E_NULL, dict(y=None)), (B.PIVOT_E_UNSUPPORTED, dict(t=B.PIVOT_F32)),
                        (B.PIVOT_E_NULL, dict(t=B.PIVOT_Q8)), (B.PIVOT_E_UNSUPPORTED, dict(s=s.data_ptr())), (B.PIVOT_E_SHAPE, dict(ldx=1999)),
                        (B.PIVOT_E_SHAPE, dict(ldy=63)), (B.PIVOT_E_SHAPE, dict(b=0)), (B.PIVOT_E_SHAPE, dict(b=65)),
                        (B.PIVOT_E_WORKSPACE, dict(ws=None)), (B.PIVOT_E_WORKSPACE, dict(n=need - 1)), (B.PIVOT_E_WORKSPACE, dict(ws=ws.data_ptr() + 8)),
                        (B.PIVOT_E_UNSUPPORTED, dict(f=2)), (B.PIVOT_E_SHAPE, dict(x=x.data_ptr() + 1)), (B.PIVOT_E_SHAPE, dict(y=y.data_ptr() + 2))):
            with pytest.raises(B.PivotError) as e:
                call(**k)
            assert e.value.code == code, (k, str(e.value))
        call()
        torch.cuda.synchronize()
    finally:
        B.pivot_qfc_plan_destroy(p)
