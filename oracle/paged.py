"""fp64 operators of the paged cache.  TEST INFRASTRUCTURE ONLY.

Plain restatements of include/mcd_cache.h on numpy arrays: pools [layers, pages, KV heads, page size, head
dim], page tables with -1 past a sequence's last page.  Loops over sequences, rows and tokens; no
code of the product.
"""
from __future__ import annotations

import math
from typing import List, Optional

import numpy as np


def rotate(x: np.ndarray, pos: int, inv_freq: np.ndarray, interleaved: bool, scale: float = 1.0) -> np.ndarray:
    """Pairs of the last dimension turned by pos * inv_freq; what lies behind them stays."""
    h = len(inv_freq)
    t = float(pos) * inv_freq
    c, s = np.cos(t) * scale, np.sin(t) * scale
    y = np.array(x, dtype=np.float64)
    a, b = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if interleaved else (slice(0, h), slice(h, 2 * h))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def norm(x: np.ndarray, gain: Optional[np.ndarray], eps: float) -> np.ndarray:
    if gain is None:
        return np.array(x, dtype=np.float64)
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain


def rope_row(row: np.ndarray, n_q: int, n_kv: int, pos: int, inv_freq, interleaved, q_norm, k_norm, eps, scale=1.0):
    """(q, k, v) of one packed row [n_q + 2 n_kv, head dim]."""
    q, k, v = row[:n_q], row[n_q:n_q + n_kv], row[n_q + n_kv:]
    return (rotate(norm(q, q_norm, eps), pos, inv_freq, interleaved, scale),
            rotate(norm(k, k_norm, eps), pos, inv_freq, interleaved, scale), np.array(v, dtype=np.float64))


def tokens(pool: np.ndarray, layer: int, table_row, n: int) -> np.ndarray:
    """[n, KV heads, head dim]: a sequence's first n positions."""
    page = pool.shape[3]
    return np.array([pool[layer, table_row[t // page], :, t % page] for t in range(n)], dtype=np.float64).reshape(
        n, pool.shape[2], pool.shape[4])


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, cached: int, scale: float, mask: Optional[np.ndarray] = None):
    """Rows q [n, q heads, D] over k, v [cached + n, KV heads, D]; mask [n, n] among the new rows (None: causal).
    Returns (out, spread, reach): spread = sum of p |v| and reach = the largest scale * sum |q_d k_d| of a
    visible key, what the tolerances of a rounded computation are made of."""
    n, hq, d = q.shape
    group = hq // k.shape[1]
    out, spread, reach = np.zeros((n, hq, d)), np.zeros((n, hq, d)), np.zeros((n, hq, 1))
    for i in range(n):
        see = [True] * cached + [bool(mask[i, j]) if mask is not None else j <= i for j in range(n)]
        see = np.flatnonzero(see)
        if len(see) == 0:
            continue
        for h in range(hq):
            kk, vv = k[see, h // group], v[see, h // group]
            z = scale * (kk @ q[i, h])
            p = np.exp(z - z.max())
            p /= p.sum()
            out[i, h], spread[i, h] = p @ vv, p @ np.abs(vv)
            reach[i, h] = scale * (np.abs(kk) @ np.abs(q[i, h])).max()
    return out, spread, reach


def seen_in_window(n: int, cached: int, window: int, sinks: int, mask: Optional[np.ndarray] = None) -> np.ndarray:
    """[n, cached + n]: which positions each of a sequence's new rows sees."""
    see = np.zeros((n, cached + n), dtype=bool)
    for i in range(n):
        p = cached + i if mask is None else cached + max(1, int(np.asarray(mask[i]).astype(bool).sum())) - 1
        for j in range(cached + n):
            near = p - j < window or j < sinks
            if j < cached:
                see[i, j] = near
            else:
                see[i, j] = bool(mask[i, j - cached]) if mask is not None else j <= p and near
    return see


def attention_seen(q: np.ndarray, k: np.ndarray, v: np.ndarray, see: np.ndarray, scale: float):
    """attention() of rows that see the positions of see [n, keys]; what nobody sees is not looked at."""
    n, hq, d = q.shape
    group = hq // k.shape[1]
    out, spread, reach = np.zeros((n, hq, d)), np.zeros((n, hq, d)), np.zeros((n, hq, 1))
    for i in range(n):
        at = np.flatnonzero(see[i])
        for h in range(hq if len(at) else 0):
            kk, vv = k[at, h // group], v[at, h // group]
            z = scale * (kk @ q[i, h])
            p = np.exp(z - z.max())
            p /= p.sum()
            out[i, h], spread[i, h] = p @ vv, p @ np.abs(vv)
            reach[i, h] = scale * (np.abs(kk) @ np.abs(q[i, h])).max()
    return out, spread, reach


def fork(ref, table, lens, parent, reserve, cols: int, page: int, release: bool):
    """(ref_out, table_out, len_out, copies) or an error's name; copies: (from page, to page, tokens)."""
    ref = list(ref)
    free = [p for p, r in enumerate(ref) if r == 0]
    out_ref, out, out_len, copies, seen = list(ref), [], [], [], set()
    for d, p in enumerate(parent):
        n = lens[p] if p >= 0 else 0
        need, full = -(-(n + (reserve[d] if reserve is not None else 0)) // page), n // page
        if need > cols:
            return "invalid"
        heir = release and p >= 0 and p not in seen
        seen.add(p)
        row = []
        for c in range(need):
            old = table[p][c] if p >= 0 and c < len(table[p]) else -1
            if c < full or (heir and old >= 0 and ref[old] == 1):
                row.append(old)
                continue
            if not free:
                return "oom"
            row.append(free.pop(0))
            if c == full and n % page:
                copies.append((old, row[-1], n % page))
        for c in row:
            out_ref[c] += 1
        out.append(row + [-1] * (cols - need))
        out_len.append(n)
    if release:
        for row in table:
            for c in row:
                if c >= 0:
                    out_ref[c] -= 1
    return out_ref, out, out_len, copies


def compact(pool: np.ndarray, table_in, table_out, start, keep: List[List[int]]) -> np.ndarray:
    """The pool after the moves (all reads before all writes)."""
    page, new = pool.shape[3], pool.copy()
    for s, row in enumerate(keep):
        for i, k in enumerate(row):
            a, b = start[s] + k, start[s] + i
            new[:, table_out[s][b // page], :, b % page] = pool[:, table_in[s][a // page], :, a % page]
    return new


def frequencies(kind: str, rot_dim: int, base: float, factor: float = 1.0, train: int = 0, fast: float = 32.0, slow: float = 1.0):
    w = np.array([base ** (-2.0 * j / rot_dim) for j in range(rot_dim // 2)])
    if kind == "linear":
        return w / factor
    if kind == "base":
        b = base * factor ** (rot_dim / (rot_dim - 2.0))
        return np.array([b ** (-2.0 * j / rot_dim) for j in range(rot_dim // 2)])
    if kind == "parts":
        turns = lambda r: math.log(train / (2 * math.pi * r)) / math.log(base) * rot_dim / 2   # noqa: E731
        lo, hi = turns(fast), turns(slow)
        g = np.clip((np.arange(rot_dim // 2) - lo) / (hi - lo), 0, 1)
        return w * (1 - g) + w / factor * g
    return w
