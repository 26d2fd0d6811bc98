"""Rows between a layer's products, restated plainly: norms, 8-bit rows and their products, sampling.  TEST
INFRASTRUCTURE ONLY; no code is shared with the CUDA path."""
from __future__ import annotations

import math

import numpy as np

F32 = np.float32
TOP, LEAST = 448.0, 2.0 ** -126


def norm_rows(x, residual=None, gain=None, eps: float = 1e-6, norm: bool = True):
    """(sum, values), fp64 [rows, width]."""
    r = np.asarray(x, np.float64)
    if residual is not None:
        r = r + np.asarray(residual, np.float64)
    v = r / np.sqrt((r * r).mean(1, keepdims=True) + eps) if norm else r
    return r, v if gain is None else v * np.asarray(gain, np.float64)


def row_scales(v):
    return np.maximum(np.abs(v).max(1) / TOP, LEAST)


def e4m3_values() -> np.ndarray:
    """The 256 bit patterns' values: sign, 4 bits of exponent (bias 7), 3 of mantissa; 0x7f and 0xff are NaN."""
    out = np.zeros(256)
    for b in range(256):
        e, m = b >> 3 & 15, b & 7
        v = math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)
        out[b] = math.nan if b & 127 == 127 else -v if b >> 7 else v
    return out


def gemm(a, b, a_scale=None, b_scale=None):
    """(result, sum of the terms' sizes), fp64 [N, M]."""
    a, b = np.asarray(a, np.float64), np.asarray(b, np.float64)
    s = np.ones((len(b), len(a)))
    if a_scale is not None:
        s = s * np.asarray(a_scale, np.float64)
    if b_scale is not None:
        s = s * np.asarray(b_scale, np.float64)[:, None]
    return (b @ a.T) * s, (np.abs(b) @ np.abs(a).T) * np.abs(s)


def exp32(d: np.ndarray) -> np.ndarray:
    """exp of fp32 values d <= 0 by the sampler's single steps of fp32 (oracle.sampler.exp32), on arrays."""
    d = np.asarray(d, F32)
    e = np.maximum(d, F32(-100))
    n = np.rint(e * F32(1.4426950408889634))
    r = (e - n * F32(0.693359375)) - n * F32(-2.12194440e-4)
    p = np.full_like(r, F32(1.0 / 5040))
    for k in range(6, -1, -1):
        p = p * r + F32(1.0 / math.factorial(k))
    return np.where(d < F32(-87), 0.0, np.ldexp(p.astype(np.float64), n.astype(int)))


def sample(logits, u: float, temperature: float = 1.0, top_k: int = 0, top_p: float = 1.0, min_p: float = 0.0):
    """(id, W of it, sum of W, how many ids are left), whole numbers; (-1, 0, 1, 0) for a row or setting that does not fit."""
    x = np.asarray(logits, F32)
    bad = np.isnan(x).any() or (x == np.inf).any() or (x == -np.inf).all()
    if bad or not (0 <= temperature < math.inf) or math.isnan(top_p) or math.isnan(min_p) or not 0 <= u < 1:
        return -1, 0, 1, 0
    ranking = np.lexsort((np.arange(x.size), -x))
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        z = x / F32(temperature)
        top = x.max() / F32(temperature)
        if temperature == 0 or not np.isfinite(top) or top_p <= 0:
            return int(ranking[0]), 1, 1, 1
        w = np.floor(exp32(z - top) * 2.0 ** 31).astype(np.int64)
    if 0 < top_k < x.size:
        ranking = ranking[:top_k]
    if top_p < 1:
        sums = np.cumsum(w[ranking])
        need = max(1, math.ceil(float(F32(top_p)) * float(sums[-1])))
        ranking = ranking[:1 + int((sums < need).sum())]
    least = max(1, math.ceil(float(F32(min(min_p, 1.0))) * 2.0 ** 31)) if min_p > 0 else 1
    left = sorted(int(i) for i in ranking if w[i] >= least)
    mass = int(w[left].sum())
    t, run = min(math.floor(u * float(mass)), mass - 1), 0
    for i in left:
        run += int(w[i])
        if run > t:
            return i, int(w[i]), mass, len(left)
    raise AssertionError
