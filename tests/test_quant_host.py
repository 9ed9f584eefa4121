"""Plans of 4-bit layers and experts on the host: schedules, refusals, and arguments that run calls turn down (no GPU)."""
import numpy as np
import pytest

from paper_1712_01084_amd import binding as B
import quant_util as U


@pytest.mark.parametrize("M,K,bh,bw,group,kept", [(1, 1, 16, 32, 32, 1.0), (100, 203, 16, 32, 64, 0.5), (130, 300, 64, 64, 32, 0.4),
                                                  (64, 257, 32, 128, 128, 0.7), (48, 640, 16, 64, 128, 0.0)])
@pytest.mark.parametrize("chunk_blocks", [0, 1, 3])
def test_schedule(M, K, bh, bw, group, kept, chunk_blocks):
    rng = np.random.default_rng(M + K)
    L = U.layer(rng, M, K, bh, bw, group, kept=kept, perm=True)
    p = U.plan(L, device=-1, chunk_blocks=chunk_blocks)
    try:
        v = B.pivot_qfc_plan_host_view(p)
    finally:
        B.pivot_qfc_plan_destroy(p)
    nbr, nbc, ppb = -(-M // bh), -(-K // bw), 128 // bw
    mask = np.ones((nbr, nbc), bool) if L["mask"] is None else L["mask"].astype(bool)
    assert (v["nbr"], v["nbc"], v["T"], v["groups_per_block"]) == (nbr, nbc, mask.sum(), 128 // min(bw, group))
    seen = {}
    for i in range(nbr):
        cols = np.nonzero(mask[i])[0]
        assert v["col_idx"][v["row_ptr"][i]:v["row_ptr"][i + 1]].tolist() == cols.tolist()
        kb = -(-len(cols) // ppb)
        assert v["block_ptr"][i + 1] - v["block_ptr"][i] == kb
        pieces = v["pieces"][v["block_ptr"][i] * ppb:v["block_ptr"][i + 1] * ppb]
        assert pieces.tolist() == (cols * bw).tolist() + [-1] * (kb * ppb - len(cols))
    lengths = [c[2] - c[1] for c in v["chunks"]]
    assert lengths == sorted(lengths, reverse=True)
    for row, b, e, first, parts, slot, _, _ in v["chunks"].tolist():
        assert e - b <= max(v["chunk_blocks"], 1) and first <= slot < first + parts
        seen.setdefault(row, []).append((slot, b, e))
    assert sorted(s for r in seen.values() for s, _, _ in r) == list(range(v["nchunks"]))
    for i in range(nbr):
        at = v["block_ptr"][i]
        for _, b, e in sorted(seen[i]):
            assert b == at
            at = e
        assert at == v["block_ptr"][i + 1]


def _refused(code, f, *a, **k):
    with pytest.raises(B.PivotError) as e:
        f(*a, **k)
    assert e.value.code == code, str(e.value)


def test_plans_that_are_refused():
    rng = np.random.default_rng(1)
    ok = U.layer(rng, 40, 100, 16, 32, 32, perm=True, zeros=True)
    for change, code in ((dict(bh=8), B.PIVOT_E_UNSUPPORTED), (dict(bh=128), B.PIVOT_E_UNSUPPORTED), (dict(act=7), B.PIVOT_E_UNSUPPORTED),
                         (dict(M=0), B.PIVOT_E_SHAPE), (dict(K=-1), B.PIVOT_E_SHAPE),
                         (dict(prow=np.zeros(40, np.int32)), B.PIVOT_E_NOT_PERMUTATION),
                         (dict(pcol=np.arange(1, 101, dtype=np.int32)), B.PIVOT_E_NOT_PERMUTATION),
                         (dict(zeros=np.full((40, 4), 16, np.uint8)), B.PIVOT_E_SHAPE),
                         (dict(codes=None), B.PIVOT_E_NULL), (dict(scales=None), B.PIVOT_E_NULL),
                         (dict(codes=ok["codes"][:, :-1]), B.PIVOT_E_SHAPE), (dict(scales=ok["scales"][1:]), B.PIVOT_E_SHAPE)):
        L = dict(ok, **change)
        if "bh" in change:
            L["mask"] = None
        _refused(code, U.plan, L, device=-1)
    for bw, group in ((16, 32), (256, 32), (32, 16), (32, 256)):
        L = U.layer(rng, 16, 512, 16, bw, group)
        _refused(B.PIVOT_E_UNSUPPORTED, U.plan, L, device=-1)
    L = U.layer(rng, 16, 65536, 16, 128, 128)
    _refused(B.PIVOT_E_UNSUPPORTED, U.plan, L, device=-1)
    _refused(B.PIVOT_E_SHAPE, U.plan, ok, device=-1, chunk_blocks=-1)


def test_runs_that_are_refused():
    rng = np.random.default_rng(2)
    p = U.plan(U.layer(rng, 40, 100, 16, 32, 32), device=-1)
    try:
        _refused(B.PIVOT_E_NO_DEVICE, B.pivot_qfc_run, p, 1024, B.PIVOT_F16, 100, None, 1024, 40, 1, None, 0)
        _refused(B.PIVOT_E_NULL, B.pivot_qfc_run, None, 1024, B.PIVOT_F16, 100, None, 1024, 40, 1, None, 0)
        _refused(B.PIVOT_E_NO_DEVICE, B.pivot_norm_run, 1024, B.PIVOT_F32, 100, 4096, B.PIVOT_F32, 100, 1, 100, order=p)
        assert B.pivot_qfc_kernel_name(p, B.PIVOT_F16, 1).startswith("pivot::qfc_rows_kernel<false")
        assert B.pivot_qfc_kernel_name(p, B.PIVOT_Q8, 64).startswith("pivot::qfc_frag_kernel<true")
        _refused(B.PIVOT_E_SHAPE, B.pivot_qfc_kernel_name, p, B.PIVOT_F16, 65)
        _refused(B.PIVOT_E_UNSUPPORTED, B.pivot_qfc_kernel_name, p, B.PIVOT_F32, 1)
        assert B.pivot_qfc_workspace_bytes(p, 0) == 0 and B.pivot_qfc_workspace_bytes(None, 1) == 0
    finally:
        B.pivot_qfc_plan_destroy(p)
    n = dict(res_ptr=2048, rtype=B.PIVOT_F16, ldr=8)
    F32, F16, Q8 = B.PIVOT_F32, B.PIVOT_F16, B.PIVOT_Q8
    for code, a, k in ((B.PIVOT_E_NULL, (None, F32, 8, 1024, F32, 8, 1, 8), {}), (B.PIVOT_E_NULL, (1024, F32, 8, None, F32, 8, 1, 8), {}),
                       (B.PIVOT_E_SHAPE, (1024, F32, 8, 4096, F32, 8, 0, 8), {}), (B.PIVOT_E_SHAPE, (1024, F32, 8, 4096, F32, 8, 1, 0), {}),
                       (B.PIVOT_E_SHAPE, (1024, F32, 65536, 4096, F32, 65536, 1, 65536), {}),
                       (B.PIVOT_E_SHAPE, (1024, F32, 7, 4096, F32, 8, 1, 8), {}), (B.PIVOT_E_SHAPE, (1024, F32, 8, 4096, F32, 7, 1, 8), {}),
                       (B.PIVOT_E_UNSUPPORTED, (1024, Q8, 8, 4096, F32, 8, 1, 8), {}), (B.PIVOT_E_UNSUPPORTED, (1024, F32, 8, 4096, 3, 8, 1, 8), {}),
                       (B.PIVOT_E_NULL, (1024, F32, 8, 4096, Q8, 8, 1, 8), {}), (B.PIVOT_E_UNSUPPORTED, (1024, F32, 8, 4096, F32, 8, 1, 8), dict(scale_ptr=64)),
                       (B.PIVOT_E_NULL, (1024, F32, 8, 4096, F32, 8, 1, 8), dict(res_out_ptr=2048, ldro=8)),
                       (B.PIVOT_E_SHAPE, (1024, F32, 8, 4096, F32, 8, 1, 8), dict(n, ldr=4)),
                       (B.PIVOT_E_SHAPE, (1024, F32, 8, 4096, F32, 8, 2, 8), dict(n, res_out_ptr=2048, ldro=9)),
                       (B.PIVOT_E_UNSUPPORTED, (1024, F32, 8, 4096, F32, 8, 1, 8), dict(n, rtype=Q8)),
                       (B.PIVOT_E_SHAPE, (1024, F32, 8, 4096, F32, 8, 1, 8), dict(eps=-1.0)),
                       (B.PIVOT_E_SHAPE, (1024, F32, 8, 4096, F32, 8, 1, 8), dict(eps=float("nan"))),
                       (B.PIVOT_E_UNSUPPORTED, (1024, F32, 8, 1024, F32, 8, 1, 8), {}), (B.PIVOT_E_UNSUPPORTED, (1024, F32, 8, 2048, F32, 8, 1, 8), n),
                       (B.PIVOT_E_UNSUPPORTED, (1024, F32, 8, 4096, F32, 8, 1, 8), dict(n, res_out_ptr=4096, ldro=8)),
                       (B.PIVOT_E_UNSUPPORTED, (1024, F32, 8, 4096, F32, 8, 1, 8), dict(n, res_out_ptr=1024, ldro=8)),
                       (B.PIVOT_E_SHAPE, (1025, F32, 8, 4096, F32, 8, 1, 8), {})):
        _refused(code, B.pivot_norm_run, *a, **k)


def _experts(rng, n, D, F, **k):
    drow = rng.permutation(D).astype(np.int32)
    up = [U.layer(rng, 2 * F, D, 32, 32, 32, perm=True, pairs=True, **k) for _ in range(n)]
    return up, [U.layer(rng, D, F, 16, 64, 64, prow=drow) for _ in range(n)]


def test_experts_that_are_refused():
    rng = np.random.default_rng(4)
    D, F = 70, 50
    up, down = _experts(rng, 3, D, F)
    router = rng.normal(size=(3, D)).astype(np.float32)

    def tried(code, up=up, down=down, top_k=2, **k):
        ps = [[U.plan(L, device=-1) for L in group] for group in (up, down)]
        try:
            _refused(code, B.pivot_moe_plan, ps[0], ps[1], top_k, k.pop("router", router), **k)
        finally:
            for p in ps[0] + ps[1]:
                B.pivot_qfc_plan_destroy(p)

    tried(B.PIVOT_E_NO_DEVICE)                                            # everything else is in order
    tried(B.PIVOT_E_SHAPE, top_k=0)
    tried(B.PIVOT_E_SHAPE, top_k=4)
    tried(B.PIVOT_E_SHAPE, up=up[:2])
    tried(B.PIVOT_E_SHAPE, router=router[:, 1:])
    tried(B.PIVOT_E_UNSUPPORTED, router=router.astype(np.float64))
    tried(B.PIVOT_E_UNSUPPORTED, flags=4)
    tried(B.PIVOT_E_SHAPE, norm_weight=np.ones(D), norm_eps=-1.0)
    tried(B.PIVOT_E_SHAPE, norm_weight=np.ones(D + 1))
    tried(B.PIVOT_E_SHAPE, router_bias=np.ones(2))
    tried(B.PIVOT_E_SHAPE, up=[up[0], up[1], U.layer(rng, 2 * F, D + 1, 32, 32, 32)])
    tried(B.PIVOT_E_SHAPE, down=[down[0], down[1], U.layer(rng, D, F + 1, 16, 64, 64)])
    tried(B.PIVOT_E_UNSUPPORTED, up=[up[0], up[1], U.layer(rng, 2 * F, D, 32, 64, 32)])
    tried(B.PIVOT_E_UNSUPPORTED, up=[up[0], up[1], U.layer(rng, 2 * F, D, 32, 32, 32, zeros=True)])
    tried(B.PIVOT_E_UNSUPPORTED, up=[up[0], up[1], U.layer(rng, 2 * F, D, 32, 32, 32, act=1)])
    tried(B.PIVOT_E_UNSUPPORTED, up=[up[0], up[1], U.layer(rng, 2 * F, D, 32, 32, 32, prow=np.roll(np.arange(2 * F), 1).astype(np.int32))])
    tried(B.PIVOT_E_UNSUPPORTED, down=[down[0], down[1], U.layer(rng, D, F, 16, 64, 64, perm=True)])
    assert B.pivot_moe_workspace_bytes(None, 1) == 0
    _refused(B.PIVOT_E_NULL, B.pivot_moe_run, None, 1024, D, 4096, D, 1, None, 0)
    _refused(B.PIVOT_E_SHAPE, B.pivot_moe_plan, [], [], 1, router)
