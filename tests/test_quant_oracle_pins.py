"""The oracle of the 4-bit layers, the norm and the mixture of experts against the definitions written out by hand."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import pivot_quant_oracle as Q
import quant_util as U


def test_codes_even_column_in_the_low_half():
    q = np.array([[1, 2, 3, 4, 15], [0, 9, 8, 7, 6]])
    packed = Q.pack_codes(q)
    assert packed.tolist() == [[0x21, 0x43, 0x0f], [0x90, 0x78, 0x06]]
    assert np.array_equal(Q.unpack_codes(packed, 5), q)


@pytest.mark.parametrize("zeros", [False, True])
def test_layer_term_by_term(zeros):
    rng = np.random.default_rng(3)
    L = U.layer(rng, 37, 70, 16, 32, 64, kept=0.6, zeros=zeros, perm=True, whole=True)
    L["mask"][0, 0], L["mask"][1, 1] = 0, 1
    x = rng.integers(-4, 5, (2, 70)).astype(np.float64)
    q = Q.unpack_codes(L["codes"], 70)
    want = [[Fraction(0)] * 37 for _ in range(2)]
    for r in range(37):
        for n in range(2):
            s = Fraction(float(L["bias"][L["prow"][r]]))
            for c in range(70):
                if L["mask"][r // 16, c // 32]:
                    z = int(L["zeros"][r, c // 64]) if zeros else 8
                    s += Fraction(float(L["scales"][r, c // 64])) * (int(q[r, c]) - z) * Fraction(x[n, L["pcol"][c]])
            want[n][L["prow"][r]] = s
    y, bound = Q.qfc(L, x)
    assert [[Fraction(v) for v in row] for row in y.tolist()] == want
    assert (bound >= 0).all()


def test_norm_and_its_codes():
    h, y = Q.norm([[3.0, -4.0]], [[0.0, 8.0]], [2.0, 1.0], 0.0)
    assert h.tolist() == [[3.0, 4.0]] and np.allclose(y, [[6.0, 4.0]] / np.sqrt(12.5), rtol=1e-15)
    codes, scale = Q.norm_codes([[127.0, 0.5, 1.5, -2.5], [0, 0, 0, 0], [1, np.inf, 0, 0], [np.nan, 1, 1, 1]], None, None, 0.0)
    assert codes.tolist() == [[127, 0, 2, -2], [0] * 4, [0] * 4, [0] * 4]
    assert scale[1] == 0 and np.isnan(scale[2:]).all()
    assert np.isclose(scale[0] * 127, 127 / np.sqrt((127.0 ** 2 + 0.25 + 2.25 + 6.25) / 4), rtol=1e-15)


def test_route_ties_and_experts_switched_off():
    inf = np.inf
    ids, w = Q.route(np.array([[1.0, 3.0, 3.0, 2.0], [-inf, 0.0, -inf, -inf], [-inf] * 4]), 2, True)
    assert ids.tolist() == [[1, 2], [1, -1], [-1, -1]]
    assert np.allclose(w, [[0.5, 0.5], [1.0, 0.0], [0.0, 0.0]])
    _, w = Q.route(np.array([[0.0, np.log(3.0)]]), 1, False)
    assert np.isclose(w[0, 0], 0.75)


def test_experts_one_at_a_time():
    rng = np.random.default_rng(5)
    up = [U.layer(rng, 2 * 20, 24, 16, 32, 32, perm=True, pairs=True) for _ in range(3)]
    down = [U.layer(rng, 24, 20, 16, 32, 32) for _ in range(3)]
    x, R = rng.normal(size=(4, 24)), rng.normal(size=(3, 24))
    y, dy, ids, w, _, logits = Q.moe(x, R, None, up, down, 2, False)
    for t in range(4):
        p = np.exp(logits[t]) / np.exp(logits[t]).sum()
        best = np.argsort(-logits[t])[:2]
        assert ids[t].tolist() == best.tolist()
        want = np.zeros(24)
        for e in best:
            z = Q.dense_natural(up[e])[0] @ x[t] + up[e]["bias"]
            h = z[0::2] / (1 + np.exp(-z[0::2])) * z[1::2]
            want += p[e] * (Q.dense_natural(down[e])[0] @ h + down[e]["bias"])
        assert np.allclose(y[t], want, rtol=1e-12)
    assert (dy < 1e-3).all()
