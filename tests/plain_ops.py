"""Plain 64-bit forms of the 8-bit operators and the sampler, and the bounds that their tests hold
the kernels to."""
from __future__ import annotations

import math

import numpy as np
import torch

FP8 = torch.float8_e4m3fn
U32 = 2.0 ** -24  # half a step of fp32, relative


def blocks(n):
    return -(-n // 128)


def e4m3(v: np.ndarray) -> np.ndarray:
    """v rounded to the nearest e4m3 value (ties to even), |v| <= 464."""
    v = np.asarray(v, dtype=np.float64)
    _, exp = np.frexp(v)  # |v| in [2^(exp-1), 2^exp)
    step = np.ldexp(1.0, np.maximum(exp - 1, -6) - 3)  # 3 mantissa bits; subnormals below 2^-6
    return np.round(v / step) * step  # numpy rounds halves to even


def quantize(v: np.ndarray, block_rows: int):
    """(v / scale unrounded, scales) of a float64 matrix with blocks of block_rows x 128."""
    M, K = v.shape
    mb, kb = -(-M // block_rows), blocks(K)
    full = np.zeros((mb * block_rows, kb * 128))
    full[:M, :K] = np.abs(v)
    big = full.reshape(mb, block_rows, kb, 128).max(axis=(1, 3))
    s = np.maximum(big / 448.0, 2.0 ** -126)
    wide = np.repeat(np.repeat(s, block_rows, axis=0)[:M], 128, axis=1)[:, :K]
    return v / wide, s


def check_fp8(q: torch.Tensor, scales: torch.Tensor, v: np.ndarray, block_rows: int, rel: float):
    """q, scales must be the 8-bit form of values that are within a factor 1 +- rel of v: a scale is
    rounded once more, so it is within rel + 2 U32; v / s of such values is within 2 rel + 4 U32 of the
    exact quotient (the value's error, the scale's, and a division with a rounding of its own), so q
    must lie between the roundings of the two ends of that interval."""
    want, s = quantize(v, block_rows)
    got_s = scales.cpu().numpy().astype(np.float64)
    assert got_s.shape == s.shape
    assert np.all(np.abs(got_s - s) <= (rel + 2 * U32) * s), np.max(np.abs(got_s - s) / s)
    got = q.cpu().float().numpy().astype(np.float64)
    d = 2 * rel + 4 * U32
    a, b = e4m3(np.clip(want * (1 - d), -448, 448)), e4m3(np.clip(want * (1 + d), -448, 448))
    lo, hi = np.minimum(a, b), np.maximum(a, b)
    bad = ~((got >= lo) & (got <= hi))
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist())


def norm_rel(D: int, threads: int = 64) -> float:
    """Relative error of a normalised value in fp32.  The squares are added in one chain of at most
    D / threads rounded terms and a tree over the threads (6 levels in a wave, up to 8 waves in a chain), all positive,
    so each rounding moves the sum by at most U32 of it; the square root halves that.  Then come the
    division by D, the addition of eps (halved too), the root, the reciprocal and two products."""
    chain = 8 * math.ceil(D / (8 * threads))
    return ((chain + 6 + 8 + 2) / 2 + 4) * U32


def rmsnorm(h: np.ndarray, g: np.ndarray, eps: float) -> np.ndarray:
    return g * h / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps)


def linear_fp8(xq, xs, wq, ws):
    """(y, bound): float64 product of the 8-bit forms and, per result, the sum of the absolute terms."""
    wide = lambda s, n: np.repeat(s, 128, axis=1)[:, :n]  # noqa: E731
    K, N = xq.shape[1], wq.shape[0]
    x = xq.cpu().float().numpy().astype(np.float64) * wide(xs.cpu().numpy().astype(np.float64), K)
    w = wq.cpu().float().numpy().astype(np.float64) * np.repeat(wide(ws.cpu().numpy().astype(np.float64), K), 128, axis=0)[:N]
    return x @ w.T, np.abs(x) @ np.abs(w).T


def sample_row(z, u, t=None, k=None, p=None, m=None) -> int:
    """The token of one row, from the definition in 64 bits."""
    z = np.asarray(z, dtype=np.float64)
    z = np.where(np.isnan(z), -np.inf, z)
    order = np.lexsort((np.arange(z.size), -z))
    order = order[z[order] > -np.inf]
    if order.size == 0:
        return 0
    t = 1.0 if t is None else float(t)
    if not t > 0:
        return int(order[0])
    top = z[order[0]]
    with np.errstate(invalid="ignore"):
        w = np.where(z == top, 1.0, np.exp((z - top) / t))
    w = np.where(np.isnan(w), 0.0, w)
    n = order.size
    if k is not None and k > 0:
        n = min(n, int(k))
    if p is not None and p < 1:
        c = np.concatenate([[0.0], np.cumsum(w[order[:n]])])
        n = max(1, int(np.sum(c[:-1] < max(float(p), 0.0) * c[-1])))
    kept = order[:n]
    if m is not None and m > 0:
        kept = kept[(w[kept] >= min(float(m), 1.0)) | (np.arange(n) == 0)]
    kept = np.sort(kept)
    c = np.cumsum(w[kept])
    u = float(u)
    target = (u if u > 0 else 0.0) * c[-1]
    above = np.flatnonzero(c > target)
    return int(kept[above[0]]) if above.size else int(kept[w[kept] > 0][-1])
