"""mcd_paged_attention_window on the GPU against the fp64 oracle (oracle/paged.py), tolerances as derived in
tests/test_gpu_cache.py.  Pages that nobody can see are given back (-1 in the table); what kept pages hold in places that nobody
sees is NaN and infinity in most tests, and must not touch a result."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2609_37007_gb300 import mcd
from test_gpu_cache import DEV, HALF, TYPES, U, Batch, documents, err_word, i32, nothing_sometimes, np64, pool_pair, tree

pytestmark = pytest.mark.gpu


def words_of(b, mask, seed):
    r = np.random.RandomState(seed + 3)
    n_words = -(-int(b.rows.max()) // 32) + 1
    bits = np.zeros((b.n_buf, n_words * 32), dtype=np.uint8)
    mats = []
    for s, n in enumerate(b.rows):
        mats.append(mask(r, int(n)))
        bits[b.start[s]:b.start[s] + n, :n] = mats[-1]
        bits[b.start[s]:b.start[s] + n, n:] = r.randint(0, 2, (n, n_words * 32 - n))          # bits of no row
    return mats, torch.as_tensor(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).to(DEV)


def check_window(rows, cached, window, sinks, page=16, hq=4, h=2, d=64, cache="bf16", mask=None, order="heads", seed=0, freed=True, poison=True,
                 pad=0, stream=None, loose=0):
    b = Batch(rows, cached, page, seed)
    dt = TYPES[cache]
    k, v = pool_pair((2, b.n_pages, h, page, d), dt, order, seed=seed)
    q = (1.5 * torch.randn((b.n_buf, hq * d + pad), generator=torch.Generator(device=DEV).manual_seed(seed + 7), device=DEV)).to(dt)
    out = torch.full((b.n_buf, hq * d + pad), 5.0, dtype=dt, device=DEV)
    mats, words = words_of(b, mask, seed) if mask else (None, None)
    kk, vv = np64(k), np64(v)
    table, sees = b.table.copy(), []
    for s, n in enumerate(b.rows):
        end = int(n + b.cached[s])
        see = paged.seen_in_window(int(n), int(b.cached[s]), window, sinks, None if mats is None else mats[s])
        sees.append(see)
        some = np.zeros(-(-end // page) * page, dtype=bool)
        some[:end] = see.any(0) if n else False
        if poison:
            for t in np.flatnonzero(~some):
                k[:, b.table[s, t // page], :, t % page] = float("nan")
                v[:, b.table[s, t // page], :, t % page] = float("inf") if t % 3 else float("nan")
        if freed and n:                                # by the rule alone, not by what the mask happens to hide
            for c in range(-(-end // page)):
                if c * page >= sinks and (c + 1) * page - 1 <= b.cached[s] - window:
                    table[s, c] = -1
    ch = mcd.chunks(i32(table), i32(b.cached), i32(b.start), b.n_buf, int(b.rows.max()) + loose, min(int((b.rows + b.cached).max()) + 100 * loose,
                                                                                           table.shape[1] * page))
    kv = mcd.paged_kv(k, v)
    space = torch.full((mcd.mcd_paged_attention_window_workspace(kv, ch, hq, window, sinks),), 255, dtype=torch.uint8, device=DEV)
    err = err_word()
    mcd.mcd_paged_attention_window(kv, 1, ch, hq, q, out, d ** -0.5, window, sinks, space, err, mask=words, stream=stream)
    torch.cuda.synchronize()
    assert err.item() == 0
    got, qq = np64(out), np64(q)
    assert (got[b.n:] == 5.0).all() and (got[:, hq * d:] == 5.0).all()
    for s, n in enumerate(b.rows):
        if not n:
            continue
        L, lo = int(n + b.cached[s]), b.start[s]
        ref, spread, reach = paged.attention_seen(qq[lo:lo + n, :hq * d].reshape(n, hq, d), paged.tokens(kk, 1, b.table[s], L),
                                                  paged.tokens(vv, 1, b.table[s], L), sees[s], d ** -0.5)
        delta = (d + 10) * U * reach + 8 * U
        tol = HALF[cache] * np.abs(ref) + (2 * delta + (2 * L + 4) * U + (2.0 ** -8 if cache == "bf16" else 0.0)) * spread
        far = np.abs(got[lo:lo + n, :hq * d].reshape(n, hq, d) - ref)
        assert np.isfinite(far).all(), s
        assert (far <= tol).all(), (s, float((far / np.maximum(tol, 1e-30)).max()))


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("hq,h,d", [(4, 2, 64), (16, 8, 128), (7, 1, 128), (16, 1, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (37, 4), (64, 64), (100, 0), (128, 1), (500, 70)])
def test_single_rows(cache, hq, h, d, window, sinks):
    check_window([1, 1, 1, 1, 0, 1, 1], [0, 1, 63, 64, 5, 300, 777], window, sinks, hq=hq, h=h, d=d, cache=cache, seed=window)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("hq,h,d", [(4, 2, 64), (16, 8, 128), (6, 2, 128), (5, 1, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 5), (33, 4), (130, 0), (200, 150), (400, 1)])
def test_chunks(cache, hq, h, d, window, sinks):
    check_window([1, 40, 0, 3, 129], [500, 333, 9, 0, 128], window, sinks, hq=hq, h=h, d=d, cache=cache, seed=window + 1)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("order", ["heads", "tokens"])
@pytest.mark.parametrize("freed,poison", [(True, True), (False, True), (True, False)])
def test_pages(cache, page, order, freed, poison):
    check_window([2, 70, 1, 1], [700, 450, 1000, 130], 150, 20, page=page, order=order, cache=cache, freed=freed, poison=poison, seed=page)
    check_window([1, 4, 2], [700, 451, 40], 90, 130, page=page, order=order, cache=cache, freed=freed, poison=poison, pad=8, seed=page + 1)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("mask", [tree, nothing_sometimes, documents])
@pytest.mark.parametrize("rows,cached", [([5, 1, 7, 2], [300, 0, 64, 1]), ([65, 33, 1, 64], [400, 0, 129, 17]), ([200], [300])])
@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 0), (20, 2), (150, 65)])
def test_masks(cache, mask, rows, cached, window, sinks):
    check_window(rows, cached, window, sinks, cache=cache, mask=mask, seed=len(rows) + window)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
def test_around_tiles(cache):
    """Windows and sinks that start and end one before, at and one behind the kernels' tiles of 64 and 128 keys."""
    for edge in (63, 64, 65, 127, 128, 129, 191, 193):
        check_window([1, 1, 9, 30], [edge + 200, 2 * edge, 3 * edge + 1, edge + 129], edge, edge % 67, cache=cache, seed=edge)
        check_window([1, 20], [256 + edge, 511], 128, edge, cache=cache, seed=edge + 1)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 20])
def test_long_caches_in_parts(cache, rows):
    check_window([rows, rows], [20000, 15001], 9000, 4, h=1, hq=2, cache=cache, page=128, seed=3)
    check_window([rows], [9000], 700, 300, h=1, hq=2, cache=cache, page=64, seed=4)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
def test_bounds_may_be_loose(cache):
    check_window([1, 2, 1], [500, 31, 2], 64, 4, cache=cache, loose=3)
    check_window([40, 2, 100], [500, 31, 2], 64, 4, cache=cache, loose=30)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cached", [([1, 3], [90, 40]), ([50, 1], [200, 3])])
def test_a_window_that_hides_nothing_is_none(cache, rows, cached):
    """Bit for bit what mcd_paged_attention gives, up to the largest numbers."""
    b = Batch(rows, cached, 16)
    k, v = pool_pair((1, b.n_pages, 2, 16, 64), TYPES[cache])
    q = torch.randn((b.n_buf, 256), generator=torch.Generator(device=DEV).manual_seed(0), device=DEV).to(TYPES[cache])
    kv, err, outs = mcd.paged_kv(k, v), err_word(), []
    space = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)
    for window, sinks in ((None, 0), (int((b.rows + b.cached).max()), 0), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31 - 1, 0)):
        out = torch.zeros_like(q)
        if window is None:
            mcd.mcd_paged_attention(kv, 0, b.ch, 4, q, out, 0.125, space, err)
        else:
            mcd.mcd_paged_attention_window(kv, 0, b.ch, 4, q, out, 0.125, window, sinks, space, err)
        outs.append(out)
    assert all(torch.equal(o, outs[0]) for o in outs) and err.item() == 0
    # sinks that hold every position
    out = torch.zeros_like(q)
    mcd.mcd_paged_attention_window(kv, 0, b.ch, 4, q, out, 0.125, 1, 2 ** 31 - 1, space, err)
    assert np.abs(np64(out) - np64(outs[0])).max() <= (2.0 ** -6 if cache == "bf16" else 1e-5) and err.item() == 0


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 40])
def test_a_seen_page_that_is_missing_is_reported(cache, rows):
    b = Batch([rows], [300], 16)
    k, v = pool_pair((1, b.n_pages, 2, 16, 64), TYPES[cache])
    q = torch.zeros((b.n_buf, 256), device=DEV).to(TYPES[cache])
    for col, want in ((0, 1), (1, 0), (10, 0), (14, 1), (18, 1)):          # 4 sinks; window 70: from position 231 on
        t = b.table.copy()
        t[0, col] = -1
        ch = mcd.chunks(i32(t), i32(b.cached), i32(b.start), b.n_buf, rows, 300 + rows)
        kv, err = mcd.paged_kv(k, v), err_word()
        space = torch.zeros(mcd.mcd_paged_attention_window_workspace(kv, ch, 4, 70, 4), dtype=torch.uint8, device=DEV)
        mcd.mcd_paged_attention_window(kv, 0, ch, 4, q, torch.zeros_like(q), 0.125, 70, 4, space, err)
        assert err.item() == want, col


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("rows,h", [(1, 2), (30, 2)])
def test_seen_infinities_count(cache, rows, h):
    """A value that is not finite and that a row sees makes the row's result not finite, and only such rows'."""
    b = Batch([rows], [200], 16)
    k, v = pool_pair((1, b.n_pages, h, 16, 64), TYPES[cache])
    t = 205 if rows > 5 else 199
    v[0, b.table[0, t // 16], 1, t % 16, 3] = float("inf")
    q = torch.randn((b.n_buf, 4 * 64), generator=torch.Generator(device=DEV).manual_seed(0), device=DEV).to(TYPES[cache])
    out, kv, err = torch.zeros_like(q), mcd.paged_kv(k, v), err_word()
    space = torch.zeros(mcd.mcd_paged_attention_window_workspace(kv, b.ch, 4, 10, 2), dtype=torch.uint8, device=DEV)
    mcd.mcd_paged_attention_window(kv, 0, b.ch, 4, q, out, 0.125, 10, 2, space, err)
    got = np.isfinite(np64(out)[:rows].reshape(rows, 4, 64))
    see = paged.seen_in_window(rows, 200, 10, 2)[:, t]
    want = np.ones((rows, 4, 64), dtype=bool)
    want[see, 2:, 3] = False
    assert (got == want).all()


@pytest.mark.parametrize("cache,rows,cached,mask", [("bf16", 1, 6, False), ("bf16", 40, 6, False), ("f32", 20, 0, False), ("bf16", 3, 9, True), ("bf16", 40, 9, True)])
def test_rows_whose_every_score_is_minus_infinity(cache, rows, cached, mask):
    """NaN where a row sees keys that all score -inf, zeros where it sees none."""
    b = Batch([rows], [cached], 16)
    k, v = pool_pair((1, b.n_pages, 1, 16, 64), TYPES[cache], fill=1.0)
    k.fill_(-3e38)
    q = torch.full((b.n_buf, 64), 3e38, device=DEV).to(TYPES[cache])
    words = torch.zeros((b.n_buf, 2), dtype=torch.int32, device=DEV) if mask else None
    for window, sinks in ((1, 0), (2, 0), (1, 1)):
        out, kv, err = torch.zeros_like(q), mcd.paged_kv(k, v), err_word()
        space = torch.zeros(mcd.mcd_paged_attention_window_workspace(kv, b.ch, 1, window, sinks), dtype=torch.uint8, device=DEV)
        mcd.mcd_paged_attention_window(kv, 0, b.ch, 1, q, out, 1.0, window, sinks, space, err, mask=words)
        got = np64(out)[:rows]
        # (without new rows in sight, position `cached` with a window of 1 leaves the cached ones out)
        assert (got == 0).all() if mask and window == 1 and sinks == 0 else np.isnan(got).all()


def test_many_sequences_of_both_kinds():
    r = np.random.RandomState(5)
    for cache in ("bf16", "f32"):
        check_window(r.randint(0, 30, 40), r.randint(0, 300, 40), 50, 3, cache=cache, seed=9)
        check_window(np.ones(140, int), r.randint(0, 200, 140), 60, 2, cache=cache, seed=10)


def test_offsets_past_32_bits():
    """Positions past 2^20 with a table of as many columns; a pool of pages beyond 4 GB from its start."""
    page, h, d, cached = 16, 1, 64, (1 << 24) - 3
    n_pages = (9 << 30) // (page * d * 2)
    k = torch.empty((1, n_pages, h, page, d), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    cols = -(-(cached + 1) // page)
    table = torch.full((1, cols), -1, dtype=torch.int32, device=DEV)
    table[0, 0], own = n_pages - 1, {}
    for i, c in enumerate(range((cached - 40) // page, cols)):
        table[0, c] = own[c] = n_pages - 2 - i
    own[0] = n_pages - 1
    g = torch.Generator(device=DEV).manual_seed(1)
    for p in own.values():
        for x in (k, v):
            x[0, p] = torch.randn((h, page, d), generator=g, device=DEV).to(torch.bfloat16)
    q = torch.randn((1, d), generator=g, device=DEV).to(torch.bfloat16)
    out, err = torch.zeros_like(q), err_word()
    kv, ch = mcd.paged_kv(k, v), mcd.chunks(table, i32([cached]), i32([0, 1]), 1, 1, cached + 1)
    space = torch.zeros(mcd.mcd_paged_attention_window_workspace(kv, ch, 1, 30, 5), dtype=torch.uint8, device=DEV)
    mcd.mcd_paged_attention_window(kv, 0, ch, 1, q, out, 0.125, 30, 5, space, err)
    at = list(range(5)) + list(range(cached - 29, cached + 1))
    kk, vv = (np.array([np64(x[0, own[t // page], 0, t % page]) for t in at]) for x in (k, v))
    z = kk @ np64(q)[0] * 0.125
    p = np.exp(z - z.max())
    want = p / p.sum() @ vv
    assert err.item() == 0 and (np.abs(np64(out)[0] - want) <= 2.0 ** -7 * (p / p.sum() @ np.abs(vv))).all()


def test_on_another_stream():
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    check_window([1, 30], [300, 100], 40, 4, stream=side)
