"""The mixture of experts with activations far from 1: beyond the range of fp32 in columns that a block row has lost, beyond
that of fp16, and far below it."""
import numpy as np
import pytest
import torch

from oracle import pivot_quant_oracle as Q
from paper_1712_01084_amd import binding as B
import gpu_util as G
import quant_util as U

pytestmark = pytest.mark.gpu


class Experts:
    def __init__(self, up, down, router, k, bias=None):
        self.up, self.down, self.router, self.k, self.bias = up, down, router, k, bias
        self.D, self.F = up[0]["K"], down[0]["K"]
        self.plans = [[U.plan(L) for L in group] for group in (up, down)]
        self.p = B.pivot_moe_plan(self.plans[0], self.plans[1], k, router, router_bias=bias, renormalise=True)

    def __enter__(self):
        return self

    def __exit__(self, *_):
        B.pivot_moe_plan_destroy(self.p)
        for p in self.plans[0] + self.plans[1]:
            B.pivot_qfc_plan_destroy(p)

    def run(self, x):
        T = len(x)
        xd = torch.from_numpy(x).cuda()
        ws = G.workspace(B.pivot_moe_workspace_bytes(self.p, T))
        y = torch.full((T, self.D), 33.0, device="cuda")
        B.pivot_moe_run(self.p, xd.data_ptr(), self.D, y.data_ptr(), self.D, T, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
        return y.cpu().numpy()

    def expected(self, x):
        return Q.moe(x.astype(np.float64), self.router, self.bias, self.up, self.down, self.k, True)


@pytest.mark.parametrize("F", [89, 92, 95, 121])
@pytest.mark.parametrize("tokens", [1, 7, 16])
def test_an_infinity_reaches_only_the_rows_that_keep_its_column(F, tokens):
    """The last columns of a down layer whose width is no whole tile, infinite for one unit: block rows without that tile have
    lost the column, and the columns that fill up their last block hold nothing of it."""
    rng = np.random.default_rng(F)
    D = 64
    up = [U.layer(rng, 2 * F, D, 16, 32, 32) for _ in range(2)]
    down = [U.layer(rng, D, F, 16, 32, 32) for _ in range(2)]
    for u, d in zip(up, down):
        u["bias"][2 * F - 2:] = 1e30                              # the gate and the up row of the last unit: their product is infinite
        d["mask"] = np.ones((4, -(-F // 32)), np.uint8)
        d["mask"][[0, 2], -1] = 0
    x = rng.normal(size=(tokens, D)).astype(np.float16)
    with Experts(up, down, rng.normal(size=(2, D)).astype(np.float32), 2) as m:
        y = m.run(x)
        want, bound = m.expected(x)[:2]
    lost = np.r_[0:16, 32:48]
    assert np.isfinite(y[:, lost]).all()
    assert (np.abs(y - want)[:, lost] <= bound[:, lost]).all()
    assert not np.isfinite(y[:, 16:32]).any() and not np.isfinite(y[:, 48:]).any()


@pytest.mark.parametrize("power", [-14, -10, -6, 6, 10])
@pytest.mark.parametrize("tokens,perm", [(1, False), (5, True), (16, True)])
def test_small_and_large_activations(power, tokens, perm):
    """x of 2^power: the experts' activations lie near its square, 1e-9 to 1e6, and are held as precisely as those near 1."""
    rng = np.random.default_rng(100 + power)
    E, D, F = 5, 130, 300
    drow = rng.permutation(D).astype(np.int32) if perm else None
    up = [U.layer(rng, 2 * F, D, 32, 32, 32, kept=0.8, perm=perm, pairs=True, bias=False) for _ in range(E)]
    down = [U.layer(rng, D, F, 32, 64, 32, kept=0.8, zeros=False, perm=perm, prow=drow, bias=False) for _ in range(E)]
    x = (2.0 ** power * rng.normal(size=(tokens, D))).astype(np.float16)
    with Experts(up, down, (rng.normal(size=(E, D)) / D ** 0.5).astype(np.float16), 2) as m:
        y = m.run(x)
        want, bound = m.expected(x)[:2]
    assert (np.abs(y - want) <= bound).all()
    assert np.linalg.norm(y - want) <= 64 * 2.0 ** -24 * np.linalg.norm(want)


def test_small_activations_beside_large_ones():
    """Block rows that keep only the columns of small activations, in whole blocks of 128 columns: as precise as alone."""
    rng = np.random.default_rng(7)
    D, F = 64, 512
    up = [U.layer(rng, 2 * F, D, 16, 32, 32)]
    down = [U.layer(rng, D, F, 16, 128, 128, bias=False)]
    up[0]["scales"][:] = 0                                       # the activations are the biases'
    size = np.repeat([1e-9, 1e15, 1.0, 1e-15], 128)               # of the gate and the up rows, by block of columns
    up[0]["bias"] = (np.repeat(size, 2) * rng.uniform(0.5, 1.5, 2 * F)).astype(np.float32)
    down[0]["mask"] = np.eye(4, dtype=np.uint8)
    x = rng.normal(size=(3, D)).astype(np.float16)
    with Experts(up, down, np.ones((1, D), np.float32), 1) as m:
        y = m.run(x)
        want, bound = m.expected(x)[:2]
    for r in range(4):
        rows = slice(16 * r, 16 * r + 16)
        assert np.abs(want[:, rows]).max() > 0
        assert np.linalg.norm((y - want)[:, rows]) <= 64 * 2.0 ** -24 * np.linalg.norm(want[:, rows])
