"""The paged cache's operators on the GPU at head layouts, values and precisions that tests/test_gpu_cache.py does
not reach; tolerances as derived there."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2609_37007_gb300 import mcd
from test_gpu_cache import (DEV, HALF, TYPES, U, Batch, check_attention, check_rope, documents, err_word, nothing_sometimes, np64,
                            pool_pair, tree)

pytestmark = pytest.mark.gpu


# ---- rotary append ---------------------------------------------------------------------------
@pytest.mark.parametrize("inp,cache", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("hq,h", [(1, 1), (2, 1), (4, 1), (16, 1), (3, 3), (5, 5), (20, 5)])
def test_rope_heads_of_a_warp_differ(inp, cache, inter, hq, h):
    """head_dim 64: a warp holds two heads, which may be a query's and a key's, a key's and a value's, or a value's and none."""
    check_rope([3, 1, 0, 18], [0, 15, 3, 200], hq=hq, h=h, d=64, rot=64, inter=inter, inp=inp, cache=cache, seed=hq + 7 * h)


@pytest.mark.parametrize("which", ["q", "k"])
@pytest.mark.parametrize("hq,h", [(1, 1), (2, 1), (3, 3), (4, 2), (16, 1), (21, 3)])
@pytest.mark.parametrize("d,inter", [(64, False), (64, True), (128, False)])
@pytest.mark.parametrize("inp", ["f32", "bf16"])
def test_rope_one_gain_alone(which, hq, h, d, inter, inp):
    """Only the query heads, or only the key heads, are normalised."""
    rows, cached, page = [1, 6, 0, 13], [0, 31, 4, 100], 16
    b = Batch(rows, cached, page, hq)
    r = np.random.RandomState(h)
    k, v = pool_pair((1, b.n_pages, h, page, d), torch.bfloat16, fill=7.0)
    qkv = torch.as_tensor(r.randn(b.n_buf, (hq + 2 * h) * d)).to(DEV, TYPES[inp])
    q = torch.full((b.n_buf, hq * d), 5.0, dtype=torch.bfloat16, device=DEV)
    gain = torch.as_tensor(1 + 0.1 * r.randn(d), dtype=torch.float32).to(DEV)
    w, _ = mcd.mcd_rope_freqs(d, 1e4)
    err = err_word()
    mcd.mcd_rope_append(mcd.paged_kv(k, v), 0, b.ch, hq, qkv, q, mcd.rope(torch.as_tensor(w).to(DEV), d, inter), err,
                        q_norm=gain if which == "q" else None, k_norm=gain if which == "k" else None)
    torch.cuda.synchronize()
    assert err.item() == 0
    x, got, kk, vv = np64(qkv).reshape(b.n_buf, hq + 2 * h, d), np64(q).reshape(b.n_buf, hq, d), np64(k), np64(v)
    g = np64(gain)
    rel = 32 * U + (d + 6) * U                         # (as in check_rope)
    for s in range(len(rows)):
        for i in range(b.rows[s]):
            row, slot = b.start[s] + i, b.cached[s] + i
            rq, rk, rv = paged.rope_row(x[row], hq, h, slot, w, inter, g if which == "q" else None, g if which == "k" else None, 1e-6)
            size = max(np.abs(x[row]).max(), np.abs(rq).max(), np.abs(rk).max()) * 3
            page_at = (0, b.table[s, slot // page], slice(None), slot % page)
            assert (np.abs(got[row] - rq) <= HALF["bf16"] * np.abs(rq) + rel * size).all()
            assert (np.abs(kk[page_at] - rk) <= HALF["bf16"] * np.abs(rk) + rel * size).all()
            assert (np.abs(vv[page_at] - rv) <= HALF["bf16"] * np.abs(rv)).all()
    assert (got[b.n:] == 5.0).all()


# ---- attention: scores of minus infinity ---------------------------------------------------------
def run_attention(b, k, v, q, hq, d, mats=None):
    words = None
    if mats is not None:
        n_words = -(-int(b.rows.max()) // 32)
        bits = np.zeros((b.n_buf, n_words * 32), dtype=np.uint8)
        for s, n in enumerate(b.rows):
            bits[b.start[s]:b.start[s] + n, :n] = mats[s]
        words = torch.as_tensor(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).to(DEV)
    kv, err = mcd.paged_kv(k, v), err_word()
    out = torch.full_like(q, 5.0)
    space = torch.full((mcd.mcd_paged_attention_workspace(kv, b.ch, hq),), 255, dtype=torch.uint8, device=DEV)
    mcd.mcd_paged_attention(kv, 0, b.ch, hq, q, out, d ** -0.5, space, err, mask=words)
    torch.cuda.synchronize()
    assert err.item() == 0
    return np64(out)


def set_keys(b, x, s, positions, value):
    """Component 0 of the keys (or all of the values) of sequence s at these positions."""
    for t in positions:
        x[0, b.table[s, t // b.page], :, t % b.page, :1 if value != np.inf else None] = value


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cached,h", [(1, 37, 2), (4, 700, 2), (3, 9000, 1), (30, 37, 2), (30, 4100, 2), (200, 61, 2)])
@pytest.mark.parametrize("which", ["some", "front", "front and a value", "all"])
def test_scores_of_minus_infinity(cache, rows, cached, h, which):
    """A visible key whose score is -inf has weight zero (times a value that is not finite: NaN); a row that sees no other is
    NaN, unlike one that sees nothing.  With one part of the keys, and with parts, some of them without a finite score."""
    d, hq = 64, 2 * h
    b = Batch([rows, 1], [cached, 5], 16, seed=rows)
    k, v = pool_pair((1, b.n_pages, h, 16, d), TYPES[cache], seed=rows)
    q = torch.randn((b.n_buf, hq * d), generator=torch.Generator(device=DEV).manual_seed(rows), device=DEV).to(TYPES[cache])
    q.view(b.n_buf, hq, d)[:, :, 0] = 1.0
    keys, r = cached + rows, np.random.RandomState(rows)
    low = {"some": np.flatnonzero(r.randint(0, 2, keys)), "all": np.arange(keys)}.get(which, np.arange(cached - 1 - cached // 5))
    set_keys(b, k, 0, low, -np.inf)
    if which == "front and a value":
        set_keys(b, v, 0, [int(low[0])], np.inf)
    got, qq, kk, vv = run_attention(b, k, v, q, hq, d), np64(q), np64(k), np64(v)
    assert (got[b.n:] == 5.0).all()
    for s, n in enumerate(b.rows):
        L, lo = n + b.cached[s], b.start[s]
        x, K = qq[lo:lo + n].reshape(n, hq, d), paged.tokens(kk, 0, b.table[s], L)
        with np.errstate(invalid="ignore"):
            ref, spread, _ = paged.attention(x, K, paged.tokens(vv, 0, b.table[s], L), int(b.cached[s]), d ** -0.5)
        reach = d ** -0.5 * np.abs(x).max(1, keepdims=True) * np.where(np.isinf(K), 0, np.abs(K)).sum(-1).max()     # (of finite scores)
        o = got[lo:lo + n].reshape(n, hq, d)
        assert (np.isnan(o) == np.isnan(ref)).all() and np.isnan(ref).all() == (s == 0 and which in ("all", "front and a value"))
        fine = ~np.isnan(ref)
        tol = HALF[cache] * np.abs(ref) + (2 * ((d + 10) * U * reach + 8 * U) + (2 * L + 4) * U + (2.0 ** -8 if cache == "bf16" else 0.0)) * spread
        assert (np.abs(o - ref)[fine] <= tol[fine]).all()


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [4, 30, 70, 200])
def test_masked_rows_without_a_finite_score(cache, rows):
    """Nothing cached: a row sees nothing (zeros), only a key that scores -inf (NaN), such a key and another (that one's
    value), a key past the first mask word."""
    d, hq, h = 64, 2, 1
    b = Batch([rows, 2], [0, 3], 16, seed=rows)
    k, v = pool_pair((1, b.n_pages, h, 16, d), TYPES[cache], seed=rows)
    q = torch.ones((b.n_buf, hq * d), dtype=TYPES[cache], device=DEV)
    last = rows - 1
    set_keys(b, k, 0, {1, last}, -np.inf)
    m = np.zeros((rows, rows), dtype=np.uint8)
    m[1, 1] = m[2, 1] = m[2, 2] = m[last, last] = 1
    got = run_attention(b, k, v, q, hq, d, [m, np.eye(2, dtype=np.uint8)])
    value = np64(v)[0, b.table[0, 0], 0, 2]
    assert np.isnan(got[[1, last]]).all() and (got[2].reshape(hq, d) == value).all()
    assert (got[[i for i in range(rows) if i not in (1, 2, last)]] == 0).all() and np.isfinite(got[rows:]).all()


# ---- attention: precision and head layouts -------------------------------------------------------
def tolerance(ref, spread, reach, keys, d, p_bits):
    """Of a bf16 result, as in test_gpu_cache.py but for the probabilities: a relative error of 2^-p_bits."""
    return 2.0 ** -8 * np.abs(ref) + (2 * ((d + 10) * U * reach + 8 * U) + (2 * keys + 4) * U + 2.0 ** -p_bits) * spread


@pytest.mark.parametrize("hq,h,d,rows", [(16, 8, 128, [1, 8, 0, 3]), (4, 4, 64, [16, 1, 9, 2]), (7, 1, 128, [1, 2, 2, 1]), (16, 1, 64, [1, 1, 0, 1]),
                                         (6, 2, 128, [5, 1, 4, 2])])
@pytest.mark.parametrize("cached", [[0, 40, 3, 300], [700, 90, 1100, 65], [2500, 2400, 3000, 2600]])
@pytest.mark.parametrize("mask", [None, tree, nothing_sometimes])
def test_few_rows_keep_probabilities_of_16_bits(hq, h, d, rows, cached, mask):
    """Up to 16 query vectors of a KV head multiply probabilities as hi + lo pairs of bf16: hi is off by 2^-8 of a
    probability at most, lo by 2^-8 of that.  (Of one bf16 alone the results would not pass: test_cache_tolerance.py.)"""
    b = Batch(rows, cached, 32, seed=hq)
    k, v = pool_pair((1, b.n_pages, h, 32, d), torch.bfloat16, seed=hq)
    q = (1.5 * torch.randn((b.n_buf, hq * d), generator=torch.Generator(device=DEV).manual_seed(d), device=DEV)).bfloat16()
    r = np.random.RandomState(hq)
    mats = None if mask is None else [mask(r, n) for n in rows]
    got, qq, kk, vv = run_attention(b, k, v, q, hq, d, mats), np64(q), np64(k), np64(v)
    for s, n in enumerate(rows):
        L, lo = n + cached[s], b.start[s]
        ref, spread, reach = paged.attention(qq[lo:lo + n].reshape(n, hq, d), paged.tokens(kk, 0, b.table[s], L), paged.tokens(vv, 0, b.table[s], L),
                                             cached[s], d ** -0.5, None if mats is None else mats[s])
        assert (np.abs(got[lo:lo + n].reshape(n, hq, d) - ref) <= tolerance(ref, spread, reach, L, d, 16)).all()


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("group", [3, 5, 6, 7, 16])
@pytest.mark.parametrize("mask", [None, documents])
def test_attention_chunks_of_wide_groups(cache, group, mask):
    """head_dim 128 and groups that do not divide a tile of 128 vectors, or whose heads fill it with 8 rows."""
    check_attention([40, 6, 0, 1, 130], [20, 0, 4, 60, 129], hq=2 * group, h=2, d=128, cache=cache, mask=mask, seed=group, poison=True)
    check_attention([17, 60], [700, 2500], hq=group, h=1, d=128, cache=cache, mask=mask, seed=group, page=64)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("group,rows", [(1, 17), (1, 127), (1, 128), (1, 129), (1, 130), (2, 64), (2, 65), (3, 43), (16, 8), (16, 9)])
@pytest.mark.parametrize("cached", [0, 100, 2100])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_hidden_infinities_around_a_tile(cache, group, rows, cached, bad):
    """Rows that fill a tile of 128 vectors but for one, exactly, or by one more; new rows whose keys and values are not finite,
    seen by nobody or by themselves alone, beside rows that see nothing at all where nothing is cached."""
    d, h, page = 128, 1, 32
    hq, r = group * h, np.random.RandomState(rows)
    b = Batch([rows, 1], [cached, 3], page, seed=rows)
    k, v = pool_pair((1, b.n_pages, h, page, d), TYPES[cache], seed=rows)
    q = torch.randn((b.n_buf, hq * d), generator=torch.Generator(device=DEV).manual_seed(rows), device=DEV).to(TYPES[cache])
    m = r.randint(0, 2, (rows, rows)).astype(np.uint8)
    odd = [1, rows // 2, rows - 1]
    m[:, odd] = 0
    m[odd[0], odd[0]] = m[odd[2], odd[2]] = 1
    m[2] = 0
    for j in odd:
        t = cached + j
        for x in (k, v):
            x[0, b.table[0, t // page], :, t % page] = bad
    got, qq, kk, vv = run_attention(b, k, v, q, hq, d, [m, np.ones((1, 1), dtype=np.uint8)]), np64(q), np64(k), np64(v)
    for s, n in enumerate(b.rows):
        L, lo = n + b.cached[s], b.start[s]
        with np.errstate(invalid="ignore"):
            ref, spread, reach = paged.attention(qq[lo:lo + n].reshape(n, hq, d), paged.tokens(kk, 0, b.table[s], L),
                                                 paged.tokens(vv, 0, b.table[s], L), int(b.cached[s]), d ** -0.5, m if s == 0 else None)
        o = got[lo:lo + n].reshape(n, hq, d)
        seers = [odd[0], odd[2]] if s == 0 else []
        rest = [i for i in range(n) if i not in seers]
        assert not np.isfinite(o[seers]).any() and np.isfinite(ref[rest]).all()
        p_error = 2.0 ** -8 if cache == "bf16" else 0.0
        tol = HALF[cache] * np.abs(ref) + (2 * ((d + 10) * U * reach + 8 * U) + (2 * L + 4) * U + p_error) * spread
        assert (np.abs(o - ref)[rest] <= tol[rest]).all()


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cached", [([1], [630]), ([3, 1, 2], [70, 900, 5000]), ([1], [9000]), ([65] * 5, [300, 17, 0, 900, 128]), ([40], [4100]),
                                         ([1, 30, 300], [50, 0, 700])])
def test_attention_repeats_itself(cache, rows, cached):
    """No sum depends on which CTA comes first: the same call gives the same bits."""
    d, hq, h = 128, 4, 2
    b = Batch(rows, cached, 64, seed=len(rows))
    k, v = pool_pair((1, b.n_pages, h, 64, d), TYPES[cache], seed=1)
    q = torch.randn((b.n_buf, hq * d), device=DEV).to(TYPES[cache])
    first = run_attention(b, k, v, q, hq, d)
    for _ in range(4):
        assert (run_attention(b, k, v, q, hq, d) == first).all()
