"""Helpers of the tests of 4-bit layers, the norm and the mixture of experts."""
import numpy as np

from oracle import pivot_quant_oracle as Q
from paper_1712_01084_amd import binding as B


def layer(rng, M, K, bh, bw, group, kept=1.0, zeros=False, perm=False, bias=True, act=0, whole=False, prow=None, pairs=False,
          empty_row=False):
    """A layer as a dict; whole: values whose sums are exact in fp32 (small integers, scales that are powers of two)."""
    nbr, nbc, ng = -(-M // bh), -(-K // bw), -(-K // group)
    L = dict(M=M, K=K, bh=bh, bw=bw, group=group, act=act)
    L["codes"] = Q.pack_codes(rng.integers(0, 16, (M, K)))
    L["scales"] = (2.0 ** rng.integers(-1, 2, (M, ng)) if whole else rng.uniform(0.5, 1.5, (M, ng)) / (5.0 * K ** 0.5)).astype(np.float16)
    L["zeros"] = rng.integers(0, 16, (M, ng)).astype(np.uint8) if zeros else None
    L["mask"] = (rng.random((nbr, nbc)) < kept).astype(np.uint8) if kept < 1.0 else None
    if empty_row:
        L["mask"] = np.ones((nbr, nbc), np.uint8) if L["mask"] is None else L["mask"]
        L["mask"][nbr // 2] = 0
    if prow is not None:
        L["prow"] = prow
    elif pairs and perm:
        p = rng.permutation(M // 2)
        L["prow"] = np.stack([2 * p, 2 * p + 1], 1).reshape(-1).astype(np.int32)
    else:
        L["prow"] = rng.permutation(M).astype(np.int32) if perm else None
    L["pcol"] = rng.permutation(K).astype(np.int32) if perm else None
    L["bias"] = None if not bias else (rng.integers(-8, 9, M) if whole else rng.normal(0, 0.1, M)).astype(np.float32)
    return L


def plan(L, device=0, chunk_blocks=0):
    return B.pivot_qfc_plan(L["M"], L["K"], L["bh"], L["bw"], L["group"], L["codes"], L["scales"], L["zeros"], L["mask"], L["prow"],
                            L["pcol"], L["bias"], act=L["act"], device=device, chunk_blocks=chunk_blocks)
