"""Several plans of 4-bit layers made in one call: the same layers as made one by one, from host and from device memory."""
import numpy as np
import pytest
import torch

from paper_1712_01084_amd import binding as B
import quant_util as U
from test_gpu_qfc_plan import WEIGHTS, outputs
from test_quant_plan_many import arguments, layers

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("there", [False, True])
def test_the_same_as_one_by_one(there):
    rng = np.random.default_rng(3)
    Ls = layers(rng) + [U.layer(rng, 3000, 2000, 32, 64, 64, zeros=True)] + layers(rng)
    xs = [rng.integers(-9, 10, (3, L["K"])) for L in Ls]
    want = []
    for L, x in zip(Ls, xs):
        p = U.plan(L)
        want.append(outputs(p, L, x))
        B.pivot_qfc_plan_destroy(p)
    given, held = [arguments(L) for L in Ls], []
    if there:
        for a in given:
            for w in WEIGHTS:
                if a[w] is not None:
                    held.append(torch.from_numpy(np.ascontiguousarray(a[w])).cuda())
                    a[w] = held[-1].data_ptr()
    many = B.pivot_qfc_plan_many(given, device=0, flags=B.PIVOT_QFC_WEIGHTS_ON_DEVICE if there else 0)
    del held
    order = rng.permutation(len(Ls))
    for i in order:                                            # destroyed in another order than made, the rest still run
        got = outputs(many[i], Ls[i], xs[i])
        assert all(np.array_equal(a, b) and not np.isnan(a).any() for a, b in zip(got, want[i])), i
        B.pivot_qfc_plan_destroy(many[i])


def test_memory_is_given_back():
    rng = np.random.default_rng(4)
    L = arguments(U.layer(rng, 4096, 8192, 32, 64, 64))
    free = []
    for _ in range(4):
        many = B.pivot_qfc_plan_many([L] * 8, device=0)
        B.pivot_qfc_plan_destroy(many[0])
        for p in many[1:]:
            B.pivot_qfc_plan_destroy(p)
        torch.cuda.synchronize()
        free.append(torch.cuda.mem_get_info()[0])
    assert free[-1] >= free[0] - (16 << 20)                    # 144 MB a time


def test_a_bad_zero_point_among_many():
    rng = np.random.default_rng(5)
    Ls = layers(rng)
    zeros = [None if L["zeros"] is None else torch.from_numpy(L["zeros"]).cuda() for L in Ls]
    zeros[0][39, 3] = 16
    given = []
    held = []
    for L, z in zip(Ls, zeros):
        a = arguments(L)
        for w in WEIGHTS:
            if a[w] is not None:
                held.append(z if w == "zeros" else torch.from_numpy(np.ascontiguousarray(a[w])).cuda())
                a[w] = held[-1].data_ptr()
        given.append(a)
    with pytest.raises(B.PivotError) as e:
        B.pivot_qfc_plan_many(given, device=0, flags=B.PIVOT_QFC_WEIGHTS_ON_DEVICE)
    assert e.value.code == B.PIVOT_E_SHAPE
