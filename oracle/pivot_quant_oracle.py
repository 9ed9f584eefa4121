"""CPU oracle of the layers with 4-bit weights, the norm and the mixture of experts.

TEST INFRASTRUCTURE ONLY: shares no code with the HIP path.  Everything is the plain definition in float64, with, beside
each result, how far an fp32 computation of it may be off: every sum of products is bounded by the number of roundings on
the longest path to its result times 2^-23 (one unit in the last place, so that adders that truncate are covered) times
the sum of the products' magnitudes.
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -23


def unpack_codes(codes, K):
    """[M][ceil(K/2)] bytes -> [M][K] integers, the even column in the low half of a byte."""
    codes = np.asarray(codes)
    out = np.empty((codes.shape[0], 2 * codes.shape[1]), dtype=np.int64)
    for r in range(2):
        out[:, r::2] = (codes >> (4 * r)) & 15
    return out[:, :K]


def pack_codes(q):
    """The inverse (an odd last column is filled up with 0)."""
    q = np.asarray(q, dtype=np.uint8)
    if q.shape[1] % 2:
        q = np.concatenate([q, np.zeros((q.shape[0], 1), np.uint8)], axis=1)
    return (q[:, 0::2] | (q[:, 1::2] << 4)).astype(np.uint8)


def dense_natural(L):
    """Natural-coordinate float64 matrix of a layer given as a dict, and the same with every term's magnitude
    (|scale| (|code - 8| + |zero - 8|), what a computation that takes off 8 first adds up)."""
    M, K, G = L["M"], L["K"], L["group"]
    q = unpack_codes(L["codes"], K).astype(np.float64)
    cols = np.arange(K) // G
    s = np.asarray(L["scales"], dtype=np.float64)[:, cols]
    z = np.full((M, K), 8.0) if L["zeros"] is None else np.asarray(L["zeros"], dtype=np.float64)[:, cols]
    keep = np.ones((M, K), bool) if L["mask"] is None else np.asarray(L["mask"]).astype(bool)[np.arange(M) // L["bh"]][:, np.arange(K) // L["bw"]]
    prow = np.arange(M) if L["prow"] is None else np.asarray(L["prow"])
    pcol = np.arange(K) if L["pcol"] is None else np.asarray(L["pcol"])
    W, A = np.zeros((M, K)), np.zeros((M, K))
    W[np.ix_(prow, pcol)] = np.where(keep, s * (q - z), 0.0)
    A[np.ix_(prow, pcol)] = np.where(keep, np.abs(s) * (np.abs(q - 8.0) + np.abs(z - 8.0)), 0.0)
    return W, A


def layer_steps(L):
    """Roundings on the longest path of a row's sum: at most 4 matrix instructions of 33 terms within a group, then one
    addition per group (at least 32 columns each), per wavefront (up to 16) and per piece of the row, bias and scales."""
    nbc = -(-L["K"] // L["bw"])
    groups = nbc * max(1, L["bw"] // min(32, L["group"]))
    return 132 + groups + 16 + 8


def qfc(L, x):
    """y [batch][M] and its bound; x [batch][K] float64 in natural coordinates."""
    W, A = dense_natural(L)
    x = np.asarray(x, dtype=np.float64)
    b = np.zeros(L["M"]) if L["bias"] is None else np.asarray(L["bias"], dtype=np.float64)
    y = x @ W.T + b
    bound = layer_steps(L) * U * (np.abs(x) @ A.T + np.abs(b))
    return (np.maximum(y, 0.0) if L.get("act") else y), bound


def norm(x, res, weight, eps):
    """h = x + res and weight * h / sqrt(mean(h^2) + eps)."""
    h = np.asarray(x, dtype=np.float64)
    if res is not None:
        h = h + np.asarray(res, dtype=np.float64)
    w = np.ones(h.shape[1]) if weight is None else np.asarray(weight, dtype=np.float64)
    with np.errstate(all="ignore"):
        return h, h * w / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps)


def norm_codes(x, res, weight, eps):
    """The same in 8 bits: codes and scale, rounded to nearest, ties to even; a zero row has scale 0, a row that holds
    anything but numbers scale NaN."""
    h, y = norm(x, res, weight, eps)
    w = np.ones(h.shape[1]) if weight is None else np.asarray(weight, dtype=np.float64)
    codes, scale = np.zeros(h.shape, np.int8), np.zeros(h.shape[0])
    for i in range(h.shape[0]):
        with np.errstate(all="ignore"):
            hw = h[i] * w
        if not np.isfinite(hw).all():
            scale[i] = np.nan
        elif np.abs(hw).max() > 0:
            codes[i] = np.rint(hw * (127.0 / np.abs(hw).max()))
            scale[i] = np.abs(hw).max() / np.sqrt((h[i] * h[i]).mean() + eps) / 127.0
    return codes, scale


def route(logits, top_k, renormalise):
    """ids (-1: none) and weights of the experts with the largest logits, ties to the lowest index."""
    T, E = logits.shape
    ids, w = np.full((T, top_k), -1, np.int32), np.zeros((T, top_k))
    for t in range(T):
        order = sorted((e for e in range(E) if logits[t, e] != -np.inf), key=lambda e: (-logits[t, e], e))
        chosen = order[:top_k]
        if not chosen:
            continue
        m = logits[t, chosen[0]]
        among = chosen if renormalise else order
        s = sum(np.exp(logits[t, e] - m) for e in among)
        for j, e in enumerate(chosen):
            ids[t, j], w[t, j] = e, np.exp(logits[t, e] - m) / s
    return ids, w


def moe(x, router, bias, gate_up, down, top_k, renormalise):
    """y, its bound, ids, weights and their bound; x [T][D] float64."""
    x, R = np.asarray(x, dtype=np.float64), np.asarray(router, dtype=np.float64)
    T, D = x.shape
    logits = x @ R.T + (0.0 if bias is None else np.asarray(bias, dtype=np.float64))
    # a lane adds every 64th eight products at most (one wavefront to a token): ceil(D / 512) * 8 roundings; then 6 steps in a
    # wavefront, up to 16 wavefronts, the bias
    dl = (8 * -(-D // 512) + 6 + 16 + 1) * U * (np.abs(x) @ np.abs(R).T + (0.0 if bias is None else np.abs(np.where(np.isinf(bias), 0.0, bias)))).max(axis=1, keepdims=True)
    ids, w = route(logits, top_k, renormalise)
    dw = w * (2 * dl + 80 * U)          # exponentials (2 units each), up to 70 additions, a division
    y, dy = np.zeros((T, D)), np.zeros((T, D))
    for e in sorted(set(ids[ids >= 0].tolist())):
        up, dn = gate_up[e], down[e]
        z, dz = qfc(up, x)
        g, u, dg, du = z[:, 0::2], z[:, 1::2], dz[:, 0::2], dz[:, 1::2]
        silu = g / (1.0 + np.exp(-g))
        h = silu * u
        # the slope of silu is below 1.1; an exponential, a sum, a division and a product, stored in fp32; as value and remainder
        # in fp16 under a power of two by which the largest lies in [2^14, 2^15): of an activation in [2^e, 2^(e+1)) the value
        # leaves at most 2^(e-11), of that the remainder half a step, 2^(e-23), or half its subnormal step, 2^-25 / 2^11 beside 2^14
        dh = (1.1 * dg * np.abs(u) + np.abs(silu) * du + dg * du * 1.1 + np.abs(h) * (8 * U + 2.0 ** -23) + 2.0 ** -149
              + 2.0 ** -50 * np.abs(h).max(axis=1, keepdims=True))
        W, A = dense_natural(dn)
        b = np.zeros(D) if dn["bias"] is None else np.asarray(dn["bias"], dtype=np.float64)
        d = h @ W.T + b
        dd = dh @ np.abs(W).T + (layer_steps(dn) + 4) * U * ((np.abs(h) + dh) @ A.T * 1.001 + np.abs(b))
        for t in range(T):
            for j in range(top_k):
                if ids[t, j] == e:
                    y[t] += w[t, j] * d[t]
                    dy[t] += w[t, j] * dd[t] + dw[t, j] * (np.abs(d[t]) + dd[t]) + (top_k + 40) * U * w[t, j] * np.abs(d[t])
    return y, dy, ids, w, dw, logits
