"""Plans of 4-bit layers from weights that lie on the device: the same layer as from host memory, and what is refused."""
import numpy as np
import pytest
import torch

from paper_1712_01084_amd import binding as B
import gpu_util as G
import quant_util as U

pytestmark = pytest.mark.gpu
WEIGHTS = ("codes", "scales", "zeros", "bias")


def device_plan(L, offset=0, **k):
    """The plan, and its arrays on the device, `offset` elements into their buffers; these are overwritten once the plan stands."""
    held = {}
    for w in WEIGHTS:
        if L[w] is not None:
            a = torch.from_numpy(np.ascontiguousarray(L[w])).reshape(-1)
            held[w] = torch.empty(offset + a.numel(), dtype=a.dtype, device="cuda")
            held[w][offset:] = a.cuda()
    at = [held[w][offset:].data_ptr() if w in held else None for w in WEIGHTS]
    p = B.pivot_qfc_plan(L["M"], L["K"], L["bh"], L["bw"], L["group"], at[0], at[1], at[2], L["mask"], L["prow"], L["pcol"], at[3],
                         act=L["act"], device=0, flags=B.PIVOT_QFC_WEIGHTS_ON_DEVICE, **k)
    for t in held.values():
        t.fill_(7)
    return p


def outputs(p, L, x):
    out = []
    for xtype in (B.PIVOT_F16, B.PIVOT_Q8):
        xd = torch.from_numpy(x.astype(np.float16 if xtype == B.PIVOT_F16 else np.int8)).cuda()
        s = torch.full((len(x),), 0.5, device="cuda") if xtype == B.PIVOT_Q8 else None
        ws = G.workspace(B.pivot_qfc_workspace_bytes(p, len(x)))
        y = torch.full((len(x), L["M"]), float("nan"), device="cuda")
        B.pivot_qfc_run(p, xd.data_ptr(), xtype, L["K"], None if s is None else s.data_ptr(), y.data_ptr(), L["M"], len(x), ws.data_ptr(),
                        ws.numel(), torch.cuda.current_stream().cuda_stream)
        out.append(y.cpu().numpy())
    return out


@pytest.mark.parametrize("M,K,bh,bw,group,kept", [(1, 1, 16, 32, 32, 1.0), (33, 129, 16, 32, 64, 1.0), (100, 333, 32, 64, 32, 0.5),
                                                  (200, 1001, 64, 32, 128, 0.4), (65, 700, 64, 128, 64, 0.6), (300, 2046, 16, 128, 32, 0.8),
                                                  (48, 130, 16, 32, 32, 0.0)])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("bias", [False, True])
def test_the_same_as_from_host_memory(M, K, bh, bw, group, kept, zeros, bias):
    rng = np.random.default_rng(M + K + zeros)
    L = U.layer(rng, M, K, bh, bw, group, kept=kept, zeros=zeros, perm=M % 2 == 0, bias=bias, act=M % 3 == 0)
    x = rng.integers(-9, 10, (5, K))
    a = U.plan(L)
    try:
        want = outputs(a, L, x)
    finally:
        B.pivot_qfc_plan_destroy(a)
    for offset in (0, 1, 3):                                       # arrays at odd elements
        p = device_plan(L, offset)
        try:
            assert all(np.array_equal(y, w) and not np.isnan(y).any() for y, w in zip(outputs(p, L, x), want))
        finally:
            B.pivot_qfc_plan_destroy(p)


def test_experts_from_device_memory():
    rng = np.random.default_rng(5)
    D, F, E = 96, 70, 3
    up = [U.layer(rng, 2 * F, D, 16, 32, 32, zeros=True) for _ in range(E)]
    down = [U.layer(rng, D, F, 16, 32, 32) for _ in range(E)]
    router = rng.normal(size=(E, D)).astype(np.float16)
    x = torch.from_numpy(rng.normal(size=(4, D)).astype(np.float16)).cuda()
    out = []
    for make in (U.plan, device_plan):
        plans = [[make(L) for L in group] for group in (up, down)]
        m = B.pivot_moe_plan(plans[0], plans[1], 2, router)
        try:
            ws = G.workspace(B.pivot_moe_workspace_bytes(m, 4))
            y = torch.full((4, D), float("nan"), device="cuda")
            B.pivot_moe_run(m, x.data_ptr(), D, y.data_ptr(), D, 4, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
            out.append(y.cpu().numpy())
        finally:
            B.pivot_moe_plan_destroy(m)
            for p in plans[0] + plans[1]:
                B.pivot_qfc_plan_destroy(p)
    assert np.array_equal(out[0], out[1]) and np.isfinite(out[0]).all()


def test_weights_that_are_refused():
    rng = np.random.default_rng(6)
    L = U.layer(rng, 40, 100, 16, 32, 32, zeros=True)
    bad = dict(L, zeros=L["zeros"].copy())
    bad["zeros"][39, 3] = 16
    with pytest.raises(B.PivotError) as e:
        device_plan(bad)
    assert e.value.code == B.PIVOT_E_SHAPE
    there = {w: torch.from_numpy(L[w]).cuda() for w in WEIGHTS}
    for w in WEIGHTS:                                              # host memory where the device's is promised
        at = {k: t.data_ptr() for k, t in there.items()}
        at[w] = L[w].ctypes.data
        with pytest.raises(B.PivotError) as e:
            B.pivot_qfc_plan(40, 100, 16, 32, 32, at["codes"], at["scales"], at["zeros"], bias=at["bias"], device=0, flags=B.PIVOT_QFC_WEIGHTS_ON_DEVICE)
        assert e.value.code == B.PIVOT_E_UNSUPPORTED
