"""The mixture-of-experts layer against the float64 oracle and its error bounds, and a decoder step of norm, layer and experts."""
import numpy as np
import pytest
import torch

from oracle import pivot_quant_oracle as Q
from paper_1712_01084_amd import binding as B
import gpu_util as G
import quant_util as U

pytestmark = pytest.mark.gpu


class Layer:
    """Experts, their plans and the layer's plan."""

    def __init__(self, seed, E, k, D, F, tile=(32, 32, 32), kept=1.0, zeros=False, perm=False, renorm=True, router=np.float16, bias=None, norm=None,
                 down_tile=None):
        rng = self.rng = np.random.default_rng(seed)
        self.E, self.k, self.D, self.F, self.renorm, self.bias = E, k, D, F, renorm, bias
        drow = rng.permutation(D).astype(np.int32) if perm else None
        self.up = [U.layer(rng, 2 * F, D, *tile, kept=kept, zeros=zeros, perm=perm, pairs=True) for _ in range(E)]
        self.down = [U.layer(rng, D, F, *(down_tile or tile), kept=kept, zeros=zeros, perm=perm, prow=drow) for _ in range(E)]
        self.router = (rng.normal(size=(E, D)) / D ** 0.5).astype(router)
        self.norm = norm
        self.plans = [[U.plan(L) for L in group] for group in (self.up, self.down)]
        self.p = B.pivot_moe_plan(self.plans[0], self.plans[1], k, self.router, router_bias=bias, renormalise=renorm, norm_weight=norm, norm_eps=1e-5)

    def close(self):
        B.pivot_moe_plan_destroy(self.p)
        for p in self.plans[0] + self.plans[1]:
            B.pivot_qfc_plan_destroy(p)

    def run(self, xd, tokens, ws=None, ldx=None, ldy=None, xtype=B.PIVOT_F16, res=None, y=None):
        ws = G.workspace(B.pivot_moe_workspace_bytes(self.p, tokens)) if ws is None else ws
        ldy = self.D if ldy is None else ldy
        y = torch.full((tokens, ldy), float("nan"), device="cuda") if y is None else y
        ids = torch.full((tokens, self.k), 77, dtype=torch.int32, device="cuda")
        w = torch.full((tokens, self.k), float("nan"), device="cuda")
        B.pivot_moe_run(self.p, xd.data_ptr(), self.D if ldx is None else ldx, y.data_ptr(), ldy, tokens, ws.data_ptr(), ws.numel(),
                        torch.cuda.current_stream().cuda_stream, xtype=xtype, res_ptr=None if res is None else res.data_ptr(),
                        ids_ptr=ids.data_ptr(), weights_ptr=w.data_ptr())
        return y, ids, w

    def check(self, x, y, ids, w):
        want, bound, wids, ww, dw, _ = Q.moe(x, self.router, self.bias, self.up, self.down, self.k, self.renorm)
        assert np.array_equal(ids.cpu().numpy(), wids)
        assert (np.abs(w.cpu().numpy() - ww) <= dw).all()
        y = y.cpu().numpy()[:, :self.D]
        assert (np.abs(y - want) <= bound).all()
        assert np.linalg.norm(y - want) <= 64 * 2.0 ** -24 * max(np.linalg.norm(want), 1e-30)


CASES = [  # E, k, D, F, tile, kept, zeros, perm, renorm, router
    (1, 1, 32, 16, (16, 32, 32), 1.0, False, False, True, np.float16),
    (2, 2, 130, 77, (16, 32, 32), 1.0, True, True, False, np.float32),
    (8, 2, 256, 300, (64, 128, 128), 1.0, False, False, True, np.float16),
    (64, 6, 200, 90, (32, 64, 64), 1.0, True, True, False, np.float16),
    (256, 8, 96, 40, (16, 32, 64), 0.7, False, True, True, np.float32),
    (5, 3, 1000, 700, (32, 64, 32), 0.4, True, True, True, np.float16),
    (70, 8, 520, 130, (64, 32, 128), 0.5, False, False, False, np.float16),
    (3, 2, 64, 4096, (32, 64, 64), 1.0, True, False, True, np.float16),          # two strips per work item, outputs in parts
    (3, 2, 60, 4100, (64, 32, 32), 0.9, False, True, True, np.float16),          # the same, gathered
    (4, 2, 64, 32, (16, 32, 32), 0.0, False, False, True, np.float16),           # nothing but biases
]


@pytest.mark.parametrize("case", CASES)
def test_against_the_definition(case):
    E, k, D, F, tile, kept, zeros, perm, renorm, router = case
    m = Layer(E + D, E, k, D, F, tile, kept, zeros, perm, renorm, router)
    try:
        ws = G.workspace(B.pivot_moe_workspace_bytes(m.p, 16))
        for tokens in (1, 2, 4, 5, 16, 1):
            x = m.rng.normal(size=(tokens, D)).astype(np.float16)
            xd = torch.from_numpy(x).cuda()
            y, ids, w = m.run(xd, tokens, ws=ws)
            y2, _, _ = m.run(xd, tokens, ws=ws)
            torch.cuda.synchronize()
            assert y.cpu().numpy().tobytes() == y2.cpu().numpy().tobytes()
            m.check(x.astype(np.float64), y, ids, w)
    finally:
        m.close()


def test_tokens_that_all_choose_the_same_experts():
    m = Layer(1, 12, 2, 64, 300, perm=True)
    try:
        for tokens in (7, 8, 16):
            x = np.repeat(m.rng.normal(size=(1, 64)), tokens, 0).astype(np.float16)
            m.check(x.astype(np.float64), *m.run(torch.from_numpy(x).cuda(), tokens))
    finally:
        m.close()


def test_two_streams_at_once():
    m = Layer(12, 16, 2, 128, 200, perm=True)
    try:
        jobs = []
        for k in range(2):
            x = m.rng.normal(size=(5, 128)).astype(np.float16)
            jobs.append((torch.cuda.Stream(), x, torch.from_numpy(x).cuda(), G.workspace(B.pivot_moe_workspace_bytes(m.p, 5))))
        torch.cuda.synchronize()
        outs = [None, None]
        for _ in range(20):
            for k, (s, x, xd, ws) in enumerate(jobs):
                with torch.cuda.stream(s):
                    outs[k] = m.run(xd, 5, ws=ws)
        torch.cuda.synchronize()
        for (s, x, xd, ws), out in zip(jobs, outs):
            m.check(x.astype(np.float64), *out)
    finally:
        m.close()


def test_ties_and_experts_switched_off():
    inf = np.inf
    bias = np.array([0, -inf, 0, 0, -inf, 0], np.float32)
    m = Layer(2, 6, 3, 48, 32, bias=bias)
    try:
        x = m.rng.normal(size=(4, 48)).astype(np.float16)
        x[1] = 0                                              # all logits alike: the lowest indices
        y, ids, w = m.run(torch.from_numpy(x).cuda(), 4)
        m.check(x.astype(np.float64), y, ids, w)
        assert ids[1].tolist() == [0, 2, 3]
    finally:
        m.close()
    for off, want in (([0, 1, 2, 3], -1), ([0, 1, 3], 2)):    # none or one is left, of three asked for
        bias = np.zeros(4, np.float32)
        bias[off] = -inf
        m = Layer(3, 4, 3, 40, 24, bias=bias, perm=True)
        try:
            x = m.rng.normal(size=(2, 40)).astype(np.float16)
            y, ids, w = m.run(torch.from_numpy(x).cuda(), 2)
            assert ids.cpu().tolist() == [[want, -1, -1]] * 2
            assert w.cpu().tolist() == [[0.0 if want < 0 else 1.0, 0.0, 0.0]] * 2
            if want < 0:
                assert (y == 0).all()
            else:
                m.check(x.astype(np.float64), y, ids, w)
        finally:
            m.close()


def test_a_token_of_nans_and_one_of_infinities_leave_the_others_alone():
    m = Layer(4, 8, 2, 100, 60, perm=True)
    try:
        x = m.rng.normal(size=(5, 100)).astype(np.float16)
        bad = x.copy()
        bad[1, 7], bad[3, 8] = np.nan, np.inf
        y, ids, w = m.run(torch.from_numpy(bad).cuda(), 5)
        y = y.cpu().numpy()
        assert np.isnan(y[1]).all() and np.isnan(y[3]).all()
        good = [0, 2, 4]
        want, bound, wids, _, _, _ = Q.moe(x[good].astype(np.float64), m.router, None, m.up, m.down, 2, True)
        assert np.array_equal(ids.cpu().numpy()[good], wids) and (np.abs(y[good] - want) <= bound).all()
    finally:
        m.close()


def test_strides_and_what_lies_beside():
    m = Layer(5, 4, 2, 90, 50, perm=True)
    try:
        for ldx, off in ((91, 0), (96, 3), (104, 8)):
            x = m.rng.normal(size=(3, 90)).astype(np.float16)
            buf = torch.full((off + 3 * ldx,), float("nan"), dtype=torch.float16, device="cuda")
            v = buf[off:].view(3, ldx)
            v[:, :90] = torch.from_numpy(x).cuda()
            y = torch.full((4, 95), -5.0, device="cuda")
            _, ids, w = m.run(v, 3, ldx=ldx, ldy=95, y=y)
            assert (y[3] == -5).all() and (y[:, 90:] == -5).all()
            m.check(x.astype(np.float64), y[:3], ids, w)
    finally:
        m.close()


def test_down_layer_of_other_tiles():
    m = Layer(6, 4, 2, 150, 200, tile=(16, 32, 32), down_tile=(64, 128, 64), kept=0.6, perm=True)
    try:
        x = m.rng.normal(size=(7, 150)).astype(np.float16)
        m.check(x.astype(np.float64), *m.run(torch.from_numpy(x).cuda(), 7))
    finally:
        m.close()


@pytest.mark.parametrize("xtype", [B.PIVOT_F32, B.PIVOT_F16])
def test_with_its_norm(xtype):
    """The norm's output is rounded to fp16 before the experts: what they get is taken from a run of the norm alone."""
    rng = np.random.default_rng(7)
    D = 203
    weight = rng.normal(1, 0.2, D).astype(np.float32)
    m = Layer(7, 6, 2, D, 64, norm=weight, perm=True)
    try:
        td = np.float32 if xtype == B.PIVOT_F32 else np.float16
        x, res = rng.normal(size=(3, D)).astype(td), rng.normal(size=(3, D)).astype(td)
        xd, rd = torch.from_numpy(x).cuda(), torch.from_numpy(res).cuda()
        n, h = torch.zeros(3, D, dtype=torch.float16, device="cuda"), torch.zeros_like(rd)
        wd = torch.from_numpy(weight).cuda()
        B.pivot_norm_run(xd.data_ptr(), xtype, D, n.data_ptr(), B.PIVOT_F16, D, 3, D, weight_ptr=wd.data_ptr(), eps=1e-5, res_ptr=rd.data_ptr(),
                         rtype=xtype, ldr=D, res_out_ptr=h.data_ptr(), ldro=D, stream=torch.cuda.current_stream().cuda_stream)
        _, y = Q.norm(x, res, weight, 1e-5)
        assert np.allclose(n.cpu().numpy(), y, rtol=2.0 ** -10, atol=1e-5)
        y, ids, w = m.run(xd, 3, xtype=xtype, res=rd)
        assert torch.equal(rd, h)
        m.check(n.cpu().numpy().astype(np.float64), y, ids, w)
    finally:
        m.close()


def test_captured():
    m = Layer(8, 16, 4, 128, 96, perm=True, zeros=True)
    try:
        ws = G.workspace(B.pivot_moe_workspace_bytes(m.p, 6))
        x = torch.zeros(6, 128, dtype=torch.float16, device="cuda")
        m.run(x, 6, ws=ws)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = m.run(x, 6, ws=ws)
        for _ in range(3):
            a = m.rng.normal(size=(6, 128)).astype(np.float16)
            x.copy_(torch.from_numpy(a))
            g.replay()
            torch.cuda.synchronize()
            m.check(a.astype(np.float64), *out)
            eager = m.run(x, 6, ws=ws)
            assert all(torch.equal(p, q) for p, q in zip(out, eager))
    finally:
        m.close()


def test_run_calls_that_are_refused():
    m = Layer(9, 4, 2, 64, 32)
    try:
        need = B.pivot_moe_workspace_bytes(m.p, 2)
        ws = G.workspace(need)
        x, y = torch.zeros(2, 64, dtype=torch.float16, device="cuda"), torch.zeros(2, 64, device="cuda")
        ok = dict(x=x.data_ptr(), ldx=64, y=y.data_ptr(), ldy=64, t=2, ws=ws.data_ptr(), n=need)
        for code, k, more in ((B.PIVOT_E_NULL, dict(x=None), {}), (B.PIVOT_E_NULL, dict(y=None), {}), (B.PIVOT_E_SHAPE, dict(ldx=63), {}),
                              (B.PIVOT_E_SHAPE, dict(ldy=63), {}), (B.PIVOT_E_SHAPE, dict(t=0), {}), (B.PIVOT_E_SHAPE, dict(t=17), {}),
                              (B.PIVOT_E_WORKSPACE, dict(ws=None), {}), (B.PIVOT_E_WORKSPACE, dict(n=need - 1), {}),
                              (B.PIVOT_E_UNSUPPORTED, {}, dict(xtype=B.PIVOT_F32)), (B.PIVOT_E_UNSUPPORTED, {}, dict(xtype=B.PIVOT_Q8)),
                              (B.PIVOT_E_UNSUPPORTED, {}, dict(res_ptr=x.data_ptr())), (B.PIVOT_E_SHAPE, dict(x=x.data_ptr() + 1), {}),
                              (B.PIVOT_E_SHAPE, {}, dict(ids_ptr=y.data_ptr() + 2))):
            a = dict(ok, **k)
            with pytest.raises(B.PivotError) as e:
                B.pivot_moe_run(m.p, a["x"], a["ldx"], a["y"], a["ldy"], a["t"], a["ws"], a["n"], **more)
            assert e.value.code == code, (k, more, str(e.value))
    finally:
        m.close()


def test_a_decoder_step():
    """The residual stream through two blocks: norm into 8 bits in the layer's block order, 4-bit layer, then the expert layer
    with its own norm, whose addition takes the first block's output into the stream."""
    rng = np.random.default_rng(10)
    D, T = 160, 5
    weight = rng.normal(1, 0.2, D).astype(np.float32)
    L = U.layer(rng, D, D, 32, 32, 32, kept=0.8, zeros=True, perm=True)
    p = U.plan(L)
    m = Layer(11, 8, 2, D, 100, norm=weight, perm=True)
    try:
        st = torch.cuda.current_stream().cuda_stream
        stream = torch.from_numpy(rng.normal(size=(T, D)).astype(np.float32)).cuda()
        h0 = stream.cpu().numpy().copy()
        wd = torch.from_numpy(weight).cuda()
        q, s = torch.zeros(T, D, dtype=torch.int8, device="cuda"), torch.zeros(T, device="cuda")
        y1 = torch.zeros(T, D, device="cuda")
        ws = G.workspace(B.pivot_qfc_workspace_bytes(p, T))
        B.pivot_norm_run(stream.data_ptr(), B.PIVOT_F32, D, q.data_ptr(), B.PIVOT_Q8, D, T, D, weight_ptr=wd.data_ptr(), eps=1e-5, scale_ptr=s.data_ptr(),
                         order=p, stream=st)
        B.pivot_qfc_run(p, q.data_ptr(), B.PIVOT_Q8, D, s.data_ptr(), y1.data_ptr(), D, T, ws.data_ptr(), ws.numel(), st, flags=B.PIVOT_QFC_X_BLOCK_ORDER)
        y2, ids, w = m.run(y1, T, xtype=B.PIVOT_F32, res=stream)
        codes, scale = Q.norm_codes(h0, None, weight, float(np.float32(1e-5)))
        assert np.array_equal(q.cpu().numpy(), codes[:, L["pcol"]])
        want, bound = Q.qfc(L, codes.astype(np.float64) * scale[:, None])
        y1 = y1.cpu().numpy()
        assert (np.abs(y1 - want) <= bound).all()
        assert np.array_equal(stream.cpu().numpy(), y1 + h0)
        # from here on with the values the device holds: its norm's output is rounded to fp16
        n = torch.zeros(T, D, dtype=torch.float16, device="cuda")
        B.pivot_norm_run(stream.data_ptr(), B.PIVOT_F32, D, n.data_ptr(), B.PIVOT_F16, D, T, D, weight_ptr=wd.data_ptr(), eps=1e-5, stream=st)
        n2 = Q.norm(y1, h0, weight, 1e-5)[1]
        assert np.allclose(n.cpu().numpy(), n2, rtol=2.0 ** -10, atol=1e-5)
        y2 = y2.cpu().numpy()
        ref, ref_bound, wids, _, _, _ = Q.moe(n2, m.router, None, m.up, m.down, 2, True)
        assert np.array_equal(ids.cpu().numpy(), wids)
        # half a step of fp16 in every element of the norm's output, through layers of norm near 1 each
        assert np.linalg.norm(y2 - ref) <= 8 * 2.0 ** -11 * np.linalg.norm(ref)
    finally:
        m.close()
        B.pivot_qfc_plan_destroy(p)
