"""Several plans of 4-bit layers made in one call (no GPU)."""
import numpy as np
import pytest

from paper_1712_01084_amd import binding as B
import quant_util as U

KEYS = dict(M="M", K="K", bh="bh", bw="bw", group="group", codes="codes", scales="scales", zeros="zeros", mask="tile_mask", prow="prow",
            pcol="pcol", bias="bias", act="act")


def arguments(L):
    return {KEYS[k]: v for k, v in L.items()}


def layers(rng):
    return [U.layer(rng, M, K, bh, bw, group, kept=kept, zeros=zeros, perm=perm, bias=perm)
            for M, K, bh, bw, group, kept, zeros, perm in ((40, 100, 16, 32, 32, 1.0, True, False), (1, 1, 16, 32, 32, 1.0, False, False),
                                                           (130, 300, 64, 64, 32, 0.4, False, True), (48, 640, 16, 64, 128, 0.0, True, True))]


@pytest.mark.parametrize("n", [1, 4])
def test_the_same_schedules(n):
    Ls = layers(np.random.default_rng(1))[:n]
    many = B.pivot_qfc_plan_many([dict(arguments(L), chunk_blocks=1) for L in Ls])
    assert len(many) == n
    for p, L in zip(many, Ls):
        q = U.plan(L, device=-1, chunk_blocks=1)
        a, b = B.pivot_qfc_plan_host_view(p), B.pivot_qfc_plan_host_view(q)
        assert a.keys() == b.keys() and all(np.array_equal(a[k], b[k]) for k in a)
        B.pivot_qfc_plan_destroy(p)
        B.pivot_qfc_plan_destroy(q)


def test_all_or_none():
    Ls = [arguments(L) for L in layers(np.random.default_rng(2))]

    def tried(code, text, changed=Ls, **k):
        with pytest.raises(B.PivotError) as e:
            B.pivot_qfc_plan_many(changed, **k)
        assert e.value.code == code and text in str(e.value)

    tried(B.PIVOT_E_SHAPE, "", [])
    tried(B.PIVOT_E_UNSUPPORTED, "layer 2", Ls[:2] + [dict(Ls[2], act=9)] + Ls[3:])
    tried(B.PIVOT_E_NOT_PERMUTATION, "layer 3", Ls[:3] + [dict(Ls[3], pcol=np.zeros(640, np.int32))])
    tried(B.PIVOT_E_SHAPE, "zero point", [dict(Ls[0], zeros=np.full((40, 4), 16, np.uint8))] + Ls[1:])
    tried(B.PIVOT_E_NULL, "layer 1", [Ls[0], dict(Ls[1], codes=None)])
    tried(B.PIVOT_E_UNSUPPORTED, "flags", Ls, flags=4)
    d = (B.pivot_qfc_desc * 2)(*[B.pivot_qfc_desc(16, 32, 16, 32, 32, 0, 0, device, 0) for device in (-1, 0)])
    a = np.zeros((16, 16), np.uint8)
    two = (B.C.c_void_p * 2)(a.ctypes.data, a.ctypes.data)
    out = (B.C.c_void_p * 2)(1, 1)
    L = B.lib()
    assert L.pivot_qfc_plan_many(2, d, two, two, None, None, None, None, None, out) == B.PIVOT_E_UNSUPPORTED      # two devices
    assert not out[0] and not out[1]
    d[1].device = -1
    assert L.pivot_qfc_plan_many(2, d, two, two, None, None, None, None, None, out) == B.PIVOT_OK and out[0] and out[1]
    for h in out:
        L.pivot_qfc_plan_destroy(h)
    assert L.pivot_qfc_plan_many(2, None, two, two, None, None, None, None, None, out) == B.PIVOT_E_NULL
    assert L.pivot_qfc_plan_many(2, d, None, two, None, None, None, None, None, out) == B.PIVOT_E_NULL
    assert L.pivot_qfc_plan_many(2, d, two, two, None, None, None, None, None, None) == B.PIVOT_E_NULL
