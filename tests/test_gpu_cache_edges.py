"""The paged cache's operators on the GPU at head layouts, values and precisions that tests/test_gpu_cache.py does
not reach; tolerances as derived there."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2609_37007_gb300 import mcd
from test_gpu_cache import DEV, HALF, TYPES, U, Batch, check_rope, err_word, np64, pool_pair

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
