"""Microscaled 4-bit floats (OCP Microscaling Formats 1.0: MXFP4), the products of such rows and matrices, scored routing with
groups, and the weighted combine - plain numpy in float64, from the definitions.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

BLOCK = 32
VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def pitch(K: int) -> int:
    return 4 * -(-K // 128)


def quantize(x: np.ndarray):
    """x [rows, K] (any float type) -> (codes uint8 [rows, K / 2], scale uint8 [rows, pitch(K)])."""
    x = np.asarray(x, dtype=np.float64)
    rows, K = x.shape
    v = x.reshape(rows, K // BLOCK, BLOCK)
    bad = ~np.isfinite(v).all(-1)
    v = np.where(bad[..., None], 0.0, v)
    top = np.abs(v).max(-1)
    _, e = np.frexp(top)                                   # top = m 2^e with m in [0.5, 1)
    b = np.where(top > 0, np.maximum(e - 1 - 2 + 127, 0), 0)
    a = np.abs(v) / np.exp2(b - 127.0)[..., None]
    d = np.abs(a[..., None] - VALUES)
    near = d.min(-1, keepdims=True)
    hit = d == near                                        # one code, or the two around a tie: the even one of those
    even = np.arange(8) % 2 == 0
    two = hit.sum(-1, keepdims=True) == 2
    code = np.argmax(np.where(two, hit & even, hit), -1).astype(np.uint8)
    code |= (np.signbit(v) << 3).astype(np.uint8)
    code = np.where(bad[..., None], 0, code).reshape(rows, K).astype(np.uint8)
    scale = np.zeros((rows, pitch(K)), np.uint8)
    scale[:, :K // BLOCK] = np.where(bad, 255, b)
    return code[:, 0::2] | (code[:, 1::2] << 4), scale


def dequantize(codes: np.ndarray, scale: np.ndarray) -> np.ndarray:
    rows, half = codes.shape
    n = np.empty((rows, 2 * half), np.uint8)
    n[:, 0::2], n[:, 1::2] = codes & 15, codes >> 4
    v = VALUES[n & 7] * np.where(n & 8, -1.0, 1.0)
    b = scale[:, :half // 16].astype(np.float64)
    s = np.where(b == 255, np.nan, np.exp2(b - 127))
    return (v.reshape(rows, -1, BLOCK) * s[..., None]).reshape(rows, 2 * half)


def silu(v):
    return v / (1.0 + np.exp(-v))


def product(x: np.ndarray, mats, ids: np.ndarray):
    """x float64 [T, K] or [T, k, K]; mats: per expert a matrix [N, K], or a pair of them (gate, up), as values.  Returns (out
    [T, k, N], bound [T, k, N]): NaN where the id names no expert; the sum of the magnitudes that each value is made of, for gated
    ones the error of a result whose two sums are each off by their magnitudes."""
    T, k = ids.shape
    gated = isinstance(mats[0], tuple)
    N = (mats[0][0] if gated else mats[0]).shape[0]
    out, bound = np.full((T, k, N), np.nan), np.full((T, k, N), np.nan)
    for t in range(T):
        for j in range(k):
            e = ids[t, j]
            if not 0 <= e < len(mats):
                continue
            r = x[t, j] if x.ndim == 3 else x[t]
            if gated:
                g, u = mats[e][0] @ r, mats[e][1] @ r
                mg, mu = np.abs(mats[e][0]) @ np.abs(r), np.abs(mats[e][1]) @ np.abs(r)
                out[t, j] = silu(g) * u
                bound[t, j] = 1.1 * np.abs(u) * mg + np.abs(silu(g)) * mu   # |silu'| < 1.1
            else:
                out[t, j] = mats[e] @ r
                bound[t, j] = np.abs(mats[e]) @ np.abs(r)
    return out, bound


def route_scored(logits, k, score="softmax", bias=None, n_group=1, topk_group=1, group_best=1, renorm=False, scale=1.0):
    """(ids int32 [T, k], weights float64 [T, k], the selected scores float64 [T, k])."""
    x = np.asarray(logits, dtype=np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    T, E = x.shape
    with np.errstate(invalid="ignore", over="ignore"):
        if score == "softmax":
            top = x.max(1, keepdims=True)
            s = np.where(x == top, 1.0, np.exp(x - top))
            s = np.where(np.isneginf(top), 0.0, s)
            total = s.sum(1, keepdims=True)
            s = s / np.where(total > 0, total, 1.0)
        else:
            s = 1.0 / (1.0 + np.exp(-x))
        key = s + np.asarray(bias, dtype=np.float64) if bias is not None else s
    key = np.where(np.isnan(key), -np.inf, key)
    order_key = x if bias is None else key
    size = E // n_group
    allowed = np.ones((T, E), bool)
    if n_group > 1:
        of = (x if bias is None and group_best == 1 else key).reshape(T, n_group, size)
        value = np.sort(of, -1)[..., ::-1][..., :group_best].sum(-1)
        rank = np.argsort(np.argsort(-value, 1, kind="stable"), 1, kind="stable")
        allowed = np.repeat(rank < topk_group, size, 1)
    ids = np.empty((T, k), np.int32)
    for t in range(T):
        c = [e for e in range(E) if allowed[t, e]]
        c.sort(key=lambda e: (-order_key[t, e], e))
        ids[t] = c[:k]
    w = np.take_along_axis(s, ids, 1)
    chosen = w.copy()
    if renorm:
        total = w.sum(1, keepdims=True)
        w = np.where(total > 0, w / np.where(total > 0, total, 1.0), 0.0)
    return ids, w * scale, chosen


def combine(rows, weights, ids=None, n_experts=0, base=None):
    T, k, N = rows.shape
    y = np.zeros((T, N)) if base is None else np.asarray(base, np.float64).copy()
    for t in range(T):
        for j in range(k):
            if ids is None or 0 <= ids[t, j] < n_experts:
                y[t] += float(weights[t, j]) * np.asarray(rows[t, j], np.float64)
    return y
