"""The paged cache's operators on the GPU against the fp64 oracle (oracle/paged.py).

Tolerances count the roundings of the arithmetic, from the values themselves.  With u = 2^-24 (fp32):
  a score of D products of exact inputs is off by at most (D + 2) u reach, reach = scale sum |q_d k_d|;
  the exponential's argument adds a few u of its size (below 2 reach) and the exponential 2 ulp, so a
  probability is off by a relative delta = (D + 10) u reach + 8 u, its sum over n keys and the
  division by it by delta + (n + 2) u, and o by (2 delta + (2 n + 4) u) spread, spread = sum p |v|;
  a bf16 result adds 2^-8 |o|, probabilities rounded to bf16 (tensor cores) 2^-8 spread (twice where
  the sum is of unrounded ones: once for the products, nothing for the sum).
"""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2609_37007_gb300 import mcd

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def i32(v):
    return torch.as_tensor(np.ascontiguousarray(v), dtype=torch.int32).to(DEV)


def np64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def err_word():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def pool_pair(shape, dtype, order="heads", seed=0, fill=None):
    """k, v [layers, pages, heads, page, D]; order "tokens": a page holds place after place, all heads of one together."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    L, P, H, T, D = shape
    out = []
    for _ in range(2):
        real = (L, P, T, H, D) if order == "tokens" else shape
        x = torch.empty(real, dtype=dtype, device=DEV)
        x = x.normal_(generator=g) if fill is None else x.fill_(fill)
        out.append(x.transpose(2, 3) if order == "tokens" else x)
    return out


def tables(r, need, n_pages, cols):
    order, t, at = r.permutation(n_pages), np.full((len(need), cols), -1), 0
    for s, n in enumerate(need):
        t[s, :n] = order[at:at + n]
        at += n
    return t


class Batch:
    """Sequences of given new rows and cached lengths with random pages."""

    def __init__(self, rows, cached, page, seed=0, spare_cols=1, spare_rows=2, spare_pages=2):
        r = np.random.RandomState(seed)
        self.rows, self.cached, self.page = np.array(rows), np.array(cached), page
        need = -(-(self.rows + self.cached) // page)
        self.n_pages = int(need.sum()) + spare_pages
        self.table = tables(r, need, self.n_pages, int(need.max()) + spare_cols)
        self.start = np.concatenate([[0], self.rows.cumsum()])
        self.n = int(self.start[-1])
        self.n_buf = self.n + spare_rows
        self.ch = mcd.chunks(i32(self.table), i32(self.cached), i32(self.start), self.n_buf, int(self.rows.max()),
                             int((self.rows + self.cached).max()))


# ---- rotary append ---------------------------------------------------------------------------
def check_rope(rows, cached, page=16, hq=4, h=2, d=64, rot=64, inter=False, with_norm=True, inp="f32", cache="bf16", order="heads",
               positions=False, scale=1.0, seed=0, layer=1, base=1e4, pad=0):
    b = Batch(rows, cached, page, seed)
    r = np.random.RandomState(seed + 1)
    dt = TYPES[cache]
    k, v = pool_pair((2, b.n_pages, h, page, d), dt, order, fill=7.0)
    qkv = torch.randn((b.n_buf, (hq + 2 * h) * d + pad), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(TYPES[inp])
    q = torch.full((b.n_buf, hq * d + pad), 5.0, dtype=dt, device=DEV)
    gains = [torch.as_tensor(1 + 0.1 * r.randn(d), dtype=torch.float32).to(DEV) for _ in range(2)] if with_norm else [None, None]
    w = base ** (-np.arange(rot // 2) / max(rot // 2, 1))
    rope = mcd.rope(torch.as_tensor(w).to(DEV), rot, inter, scale) if rot else mcd.rope()
    pos = i32(r.randint(0, 2 ** 31 - 1, b.n_buf)) if positions == "far" else i32(r.randint(0, 5000, b.n_buf)) if positions else None
    err = err_word()
    mcd.mcd_rope_append(kv := mcd.paged_kv(k, v), layer, b.ch, hq, qkv, q, rope, err, positions=pos, q_norm=gains[0], k_norm=gains[1])
    torch.cuda.synchronize()
    assert err.item() == 0
    want_k, want_v = np.full(k.shape, 7.0), np.full(v.shape, 7.0)
    tol_k = np.zeros(k.shape)
    x = np64(qkv)[:, :(hq + 2 * h) * d].reshape(b.n_buf, hq + 2 * h, d)
    got_q = np64(q)
    gn = [None if g is None else np64(g) for g in gains]
    # one rotation: angle error 2^-31 half turns (cut) + 2^-24 (conversion) + 2 ulp of sincospi, products and sum
    # 3 u of |a| + |b|; the norm (d + 6) u of the value; then one rounding
    rel = 16 * U * max(scale, 1.0) * 2 + (d + 6) * U
    for s in range(len(rows)):
        for i in range(b.rows[s]):
            row, slot = b.start[s] + i, b.cached[s] + i
            p = int(pos[row].item()) if pos is not None else slot
            # (position * inv_freq rounds in fp64: 2^-53 of up to 2^31 radians, below u)
            rq, rk, rv = paged.rope_row(x[row], hq, h, p, w[:rot // 2], inter, gn[0], gn[1], 1e-6, scale)
            size = max(np.abs(x[row]).max(), np.abs(rq).max(), np.abs(rk).max()) * 2 * 1.5
            gq = got_q[row, :hq * d].reshape(hq, d)
            assert (np.abs(gq - rq) <= HALF[cache] * np.abs(rq) + rel * size).all()
            at = (layer, b.table[s, slot // page], slice(None), slot % page)
            want_k[at], want_v[at], tol_k[at] = rk, rv, HALF[cache] * np.abs(rk) + rel * size
    assert (np.abs(np64(k) - want_k) <= tol_k).all()
    got_v = np64(v)
    exact_v = torch.as_tensor(want_v).to(dt).double().numpy() if inp == cache or cache == "f32" else None
    if exact_v is None:
        exact_v = torch.as_tensor(want_v.astype(np.float32)).to(dt).double().numpy()
    assert (got_v == exact_v).all()
    assert (got_q[b.n:] == 5.0).all() and (got_q[:, hq * d:] == 5.0).all()      # rows and columns of nobody
    del kv


@pytest.mark.parametrize("inp,cache", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("d,rot,inter", [(64, 64, False), (128, 128, False), (128, 64, True), (64, 16, False), (128, 96, True), (128, 48, False),
                                         (64, 0, False)])
def test_rope_types_and_layouts(inp, cache, d, rot, inter):
    check_rope([1, 5, 0, 17], [0, 31, 4, 200], d=d, rot=rot, inter=inter, inp=inp, cache=cache, seed=d + rot)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("order", ["heads", "tokens"])
def test_rope_pages_and_strides(page, order):
    check_rope([3, 130, 1], [page - 1, 5, 2 * page], page=page, order=order, pad=8, with_norm=page != 32, seed=page)


@pytest.mark.parametrize("heads", [(1, 1), (16, 8), (5, 1), (3, 3), (32, 2)])
@pytest.mark.parametrize("positions", [False, True, "far"])
def test_rope_heads_and_positions(heads, positions):
    check_rope([2, 9], [1, 100], hq=heads[0], h=heads[1], d=128, rot=128, positions=positions, cache="f32", scale=1.2, seed=heads[0])


def test_rope_single_rows_of_many_sequences():
    check_rope([1] * 70 + [0] * 30 + [1] * 57, list(range(157)), hq=2, h=1, seed=3)


# ---- attention ----------------------------------------------------------------------------------
def check_attention(rows, cached, page=16, hq=4, h=2, d=64, cache="bf16", mask=None, order="heads", seed=0, q_scale=1.5, scale=None,
                    layer=0, layers=1, poison=False, stream=None, spread_bits=None, pad=0):
    b = Batch(rows, cached, page, seed)
    dt = TYPES[cache]
    k, v = pool_pair((layers, b.n_pages, h, page, d), dt, order, seed=seed)
    g = torch.Generator(device=DEV).manual_seed(seed + 7)
    q = (q_scale * torch.randn((b.n_buf, hq * d + pad), generator=g, device=DEV)).to(dt)
    out = torch.full((b.n_buf, hq * d + pad), 5.0, dtype=dt, device=DEV)
    if poison:                                        # what nobody may read into a result
        for s in range(len(rows)):
            end = b.rows[s] + b.cached[s]
            for t in range(end, -(-end // page) * page):
                k[:, b.table[s, t // page], :, t % page] = float("nan")
                v[:, b.table[s, t // page], :, t % page] = float("inf")
    mats, words = None, None
    if mask is not None:
        r = np.random.RandomState(seed + 3)
        n_words = -(-int(b.rows.max()) // 32) + 1
        bits = np.zeros((b.n_buf, n_words * 32), dtype=np.uint8)
        mats = []
        for s, n in enumerate(b.rows):
            m = mask(r, int(n))
            mats.append(m)
            bits[b.start[s]:b.start[s] + n, :n] = m
            bits[b.start[s]:b.start[s] + n, n:] = r.randint(0, 2, (n, n_words * 32 - n))       # bits of no row
        words = torch.as_tensor(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).to(DEV)
    kv = mcd.paged_kv(k, v)
    scale = d ** -0.5 if scale is None else scale
    space = torch.full((mcd.mcd_paged_attention_workspace(kv, b.ch, hq),), 255, dtype=torch.uint8, device=DEV)
    err = err_word()
    mcd.mcd_paged_attention(kv, layer, b.ch, hq, q, out, scale, space, err, mask=words, stream=stream)
    torch.cuda.synchronize()
    assert err.item() == 0
    got, qq, kk, vv = np64(out), np64(q), np64(k), np64(v)
    assert (got[b.n:] == 5.0).all() and (got[:, hq * d:] == 5.0).all()
    worst = 0.0
    for s, n in enumerate(b.rows):
        if not n:
            continue
        L = n + b.cached[s]
        lo = b.start[s]
        ref, spread, reach = paged.attention(qq[lo:lo + n, :hq * d].reshape(n, hq, d), paged.tokens(kk, layer, b.table[s], L),
                                             paged.tokens(vv, layer, b.table[s], L), int(b.cached[s]), scale,
                                             None if mats is None else mats[s])
        delta = (d + 10) * U * reach + 8 * U
        tol = HALF[cache] * np.abs(ref) + (2 * delta + (2 * L + 4) * U + (2.0 ** -8 if cache == "bf16" else 0.0)) * spread
        gap = np.abs(got[lo:lo + n, :hq * d].reshape(n, hq, d) - ref)
        assert np.isfinite(gap).all()
        assert (gap <= tol).all(), (s, float((gap / np.maximum(tol, 1e-30)).max()))
        worst = max(worst, float((gap / np.maximum(tol, 1e-30)).max()))
    return worst


def tree(r, n):
    m = np.eye(n, dtype=np.uint8)
    for i in range(1, n):
        m[i] |= m[r.randint(0, i)]
    return m


def nothing_sometimes(r, n):
    m = r.randint(0, 2, (n, n)).astype(np.uint8)
    m[::3] = 0
    return m


def documents(r, n):
    cut = r.randint(0, n + 1)
    m = np.tril(np.ones((n, n), dtype=np.uint8))
    m[cut:, :cut] = 0
    return m


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("hq,h,d", [(4, 2, 64), (16, 8, 128), (4, 4, 64), (7, 1, 128), (16, 1, 64), (6, 2, 128)])
def test_attention_single_rows(cache, hq, h, d):
    check_attention([1, 1, 0, 1, 1], [0, 1, 9, 63, 300], hq=hq, h=h, d=d, cache=cache, seed=hq)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("hq,h,d", [(4, 2, 64), (16, 8, 128), (4, 4, 128), (5, 1, 64)])
def test_attention_chunks(cache, hq, h, d):
    check_attention([1, 4, 33, 0, 140, 257], [0, 64, 5, 3, 129, 70], hq=hq, h=h, d=d, cache=cache, seed=d)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("order", ["heads", "tokens"])
def test_attention_pages(cache, page, order):
    """Lengths around the ends of pages and of the kernels' key tiles; what lies behind a sequence's end in
    its last page is NaN and infinity."""
    edge = [page - 1, page, page + 1, 127, 128, 129]
    check_attention([1] * 6 + [2] * 6, [e - 1 for e in edge] + [e - 2 for e in edge], page=page, order=order, cache=cache, poison=True, pad=8)
    check_attention([40, 70, page], [edge[0], 127, 0], page=page, order=order, cache=cache, poison=True, layers=3, layer=2, pad=8)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("mask", [tree, nothing_sometimes, documents])
@pytest.mark.parametrize("rows,cached", [([4, 1, 3], [20, 0, 100]), ([65, 17, 33, 0, 64], [0, 130, 64, 5, 700]), ([5, 9], [0, 0]), ([150, 2], [77, 0])])
def test_attention_masks(cache, mask, rows, cached):
    check_attention(rows, cached, cache=cache, mask=mask, hq=4, h=2, d=128, seed=len(rows), poison=True)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("seqs,h", [(1, 1), (1, 8), (3, 2)])
@pytest.mark.parametrize("rows", [1, 3])
def test_attention_long_contexts(cache, seqs, h, rows):
    """Few rows over long caches: the keys are shared out among CTAs and joined."""
    check_attention([rows] * seqs, [5000 + 777 * s for s in range(seqs)], hq=2 * h, h=h, d=128, cache=cache, page=64, seed=seqs)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
def test_attention_chunk_over_a_long_context(cache):
    check_attention([40], [4100], hq=4, h=1, d=128, cache=cache, page=32)
    check_attention([3, 90], [700, 2500], hq=4, h=2, d=64, cache=cache, page=128)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
def test_attention_extreme_scores(cache):
    """Scores far apart: one key takes all; and large equal ones."""
    check_attention([1, 20], [100, 50], cache=cache, q_scale=60.0, seed=5)
    check_attention([1, 20], [100, 50], cache=cache, q_scale=1e-3, scale=1.0, seed=6)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cached,h", [(4, 37, 2), (30, 37, 2), (4, 700, 2), (30, 4100, 2), (3, 9000, 1), (200, 61, 2)])
def test_hidden_rows_do_not_touch_a_row(cache, rows, cached, h):
    """Keys and values of a later new row are NaN or infinite: the rows before it are as without them, it and the
    rows behind it are not finite.  With one part of the keys, and with parts joined by a cluster or in the workspace."""
    d, hq, page = 64, 2 * h, 16
    b = Batch([rows, 1], [cached, 0], page)
    k, v = pool_pair((1, b.n_pages, h, page, d), TYPES[cache])
    q = torch.randn((b.n_buf, hq * d), device=DEV).to(TYPES[cache])
    outs = []
    for bad in (None, float("nan"), float("inf")):
        if bad is not None:
            slot = cached + 2
            for x in (k, v):
                x[0, b.table[0, slot // page], :, slot % page] = bad
        out = torch.zeros_like(q)
        kv, err = mcd.paged_kv(k, v), err_word()
        space = torch.empty(mcd.mcd_paged_attention_workspace(kv, b.ch, hq), dtype=torch.uint8, device=DEV)
        mcd.mcd_paged_attention(kv, 0, b.ch, hq, q, out, d ** -0.5, space, err)
        assert err.item() == 0
        outs.append(np64(out))
    tol = 2.0 ** -6 if cache == "bf16" else 2.0 ** -17       # (another path may compute them: two roundings of values below 4)
    for o in outs[1:]:
        assert np.abs(o[:2] - outs[0][:2]).max() <= tol and np.abs(o[rows] - outs[0][rows]).max() <= tol
        assert not np.isfinite(o[2:rows]).any()


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [[1, 1, 2], [30, 1, 70]])
def test_bounds_may_be_loose(cache, rows):
    """The bounds of the host are bounds only: far larger ones give the same rows (other parts of the keys may)."""
    d, h, hq, page = 64, 2, 4, 16
    b = Batch(rows, [40, 700, 0], page)
    k, v = pool_pair((1, b.n_pages, h, page, d), TYPES[cache])
    q = torch.randn((b.n_buf, hq * d), device=DEV).to(TYPES[cache])
    kv, outs = mcd.paged_kv(k, v), []
    wide = i32(np.concatenate([b.table, np.full((3, 4000), -1)], 1))
    for ch in (b.ch, mcd.chunks(wide, i32(b.cached), i32(b.start), b.n_buf, 2 ** 30, wide.shape[1] * page)):
        out, err = torch.zeros_like(q), err_word()
        space = torch.empty(mcd.mcd_paged_attention_workspace(kv, ch, hq), dtype=torch.uint8, device=DEV)
        mcd.mcd_paged_attention(kv, 0, ch, hq, q, out, d ** -0.5, space, err)
        assert err.item() == 0
        outs.append(np64(out))
    # either side within its tolerance (see above), for |o| and spread below 4, reach below 10 (64 products of normal
    # values at scale 1/8) and 771 keys: bf16 2^-8 (4 + 4), fp32 (2 * 74 * 10 + 2 * 771 + 20) u 4
    assert np.abs(outs[0] - outs[1]).max() <= 2 * (2.0 ** -8 * 8 if cache == "bf16" else 3042 * U * 4)


def test_attention_offsets_past_32_bits():
    """A pool whose pages lie further apart than 2^32 bytes."""
    page, d, h = 16, 128, 2
    apart = (1 << 31) + 8 * 1024                        # elements: 4 GiB and a bit
    rows, cached = [1, 20], [30, 11]
    need = [2, 2]
    flat = [torch.zeros(3 * apart + h * page * d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    k, v = (x.as_strided((1, 4, h, page, d), (4 * apart, apart, page * d, d, 1)) for x in flat)
    for x in (k, v):
        x.normal_()
    table = np.array([[3, 1], [2, 0]])
    ch = mcd.chunks(i32(table), i32(cached), i32([0, 1, 21]), 21, 20, 32)
    q, out, err = torch.randn((21, 4 * d), device=DEV).bfloat16(), torch.zeros((21, 4 * d), dtype=torch.bfloat16, device=DEV), err_word()
    kv = mcd.paged_kv(k, v)
    space = torch.empty(mcd.mcd_paged_attention_workspace(kv, ch, 4), dtype=torch.uint8, device=DEV)
    mcd.mcd_paged_attention(kv, 0, ch, 4, q, out, d ** -0.5, space, err)
    assert err.item() == 0 and need
    lo = 0
    for s, n in enumerate(rows):
        L = n + cached[s]
        t = [(table[s][i // page], i % page) for i in range(L)]
        kk, vv = (np.stack([np64(x[0, p, :, o]) for p, o in t]) for x in (k, v))
        ref, spread, reach = paged.attention(np64(q)[lo:lo + n].reshape(n, 4, d), kk, vv, cached[s], d ** -0.5)
        gap = np.abs(np64(out)[lo:lo + n].reshape(n, 4, d) - ref)
        assert (gap <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2 * (d + 10) * U * reach + 100 * U) * spread).all()
        lo += n
    # and the way in: rows appended to the far page, then moved
    qkv = torch.randn((21, (4 + 2 * h) * d), device=DEV)
    mcd.mcd_rope_append(kv, 0, ch, 4, qkv, q, mcd.rope(), err)
    assert torch.equal(v[0, 1, :, 14], qkv[0].view(4 + 2 * h, d)[4 + h:].bfloat16())
    mcd.mcd_pages_compact(kv, i32(table), i32(table[::-1].copy()), i32([0, 0]), i32([[30], [0]]), i32([1, 0]), None, err)
    assert torch.equal(v[0, 2, :, 0], v[0, 1, :, 14]) and err.item() == 0


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("n", [127, 128, 129])
@pytest.mark.parametrize("kind", ["single", "chunks", "mixed", "alike"])
def test_attention_many_sequences(cache, n, kind):
    """More CTAs than the GPU holds: which sequence a CTA takes depends on the tokens, ties and empty ones among them."""
    r = np.random.RandomState(n)
    rows = {"single": r.randint(0, 2, n), "chunks": r.randint(9, 40, n), "mixed": r.randint(0, 2, n) * r.randint(1, 30, n),
            "alike": np.full(n, 3)}[kind]
    cached = np.full(n, 50) if kind == "alike" else r.randint(0, 8, n) * r.randint(0, 60, n)
    check_attention(rows.tolist(), cached.tolist(), hq=12, h=6, cache=cache, seed=n)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 21])
def test_bad_numbers_among_many_sequences(cache, rows):
    d, h, hq, page, n = 64, 6, 12, 16, 100
    r = np.random.RandomState(rows)
    b = Batch([rows] * n, r.randint(0, 200, n).tolist(), page)
    k, v = pool_pair((1, b.n_pages, h, page, d), TYPES[cache])
    q = torch.randn((b.n_buf, hq * d), device=DEV).to(TYPES[cache])
    kv, outs = mcd.paged_kv(k, v), []
    bad = b.cached.copy()
    bad[[7, 50, 99]] = [-1, 2 ** 31 - 1, b.ch.max_tokens]
    for c in (b.cached, bad):
        ch = mcd.chunks(i32(b.table), i32(c), i32(b.start), b.n_buf, rows, b.ch.max_tokens)
        out, err = torch.full_like(q, 5.0), err_word()
        space = torch.empty(mcd.mcd_paged_attention_workspace(kv, ch, hq), dtype=torch.uint8, device=DEV)
        mcd.mcd_paged_attention(kv, 0, ch, hq, q, out, d ** -0.5, space, err)
        assert err.item() == int(c is bad)                # (1: MCD_ERR_INVALID_ARG)
        outs.append(out)
    for s in range(n):
        at = slice(s * rows, (s + 1) * rows)
        assert torch.equal(outs[1][at], torch.full_like(outs[1][at], 5.0) if s in (7, 50, 99) else outs[0][at])


# ---- numbers that do not fit --------------------------------------------------------------------------
@pytest.mark.parametrize("what", ["cached", "page", "page_minus", "rows", "order", "tokens"])
@pytest.mark.parametrize("n", [1, 30])
def test_bad_numbers_are_reported_and_touch_nothing(what, n):
    """One sequence's numbers do not fit: reported, the other sequences' results stand."""
    d, h, hq, page = 64, 2, 4, 16
    b = Batch([n, n, n], [20, 40, 33], page, spare_rows=0)
    table, cached, start = b.table.copy(), b.cached.copy(), b.start.copy()
    if what == "cached":
        cached[1] = -5
    elif what == "tokens":
        cached[1] = 1 << 30
    elif what == "page":
        table[1, (40 + n - 1) // page] = b.n_pages
    elif what == "page_minus":
        table[1, (40 + n - 1) // page] = -1
    elif what == "rows":
        start[2:] = [b.n_buf + 5, b.n_buf + 5]
    elif what == "order":
        start[1] = -1
    outs, qs = [], []
    k, v = pool_pair((1, b.n_pages, h, page, d), torch.bfloat16)
    qkv = torch.randn((b.n_buf, (hq + 2 * h) * d), device=DEV)
    first = [k.clone(), v.clone()]
    for t, c, s in ((b.table, b.cached, b.start), (table, cached, start)):
        ch = mcd.chunks(i32(t), i32(c), i32(s), b.n_buf, n, b.ch.max_tokens)
        kv, err = mcd.paged_kv(k, v), err_word()
        k.copy_(first[0]), v.copy_(first[1])
        q, out = torch.zeros((b.n_buf, hq * d), dtype=torch.bfloat16, device=DEV), torch.zeros((b.n_buf, hq * d), dtype=torch.bfloat16, device=DEV)
        mcd.mcd_rope_append(kv, 0, ch, hq, qkv, q, mcd.rope(), err)
        codes = [err.item()]
        err.zero_()
        space = torch.empty(mcd.mcd_paged_attention_workspace(kv, ch, hq), dtype=torch.uint8, device=DEV)
        mcd.mcd_paged_attention(kv, 0, ch, hq, q, out, 0.1, space, err)
        codes.append(err.item())
        outs.append(np64(out))
        qs.append(codes)
    assert qs[0] == [0, 0] and qs[1] == [1, 1]
    good = {"order": [], "rows": [0]}.get(what, [0, 2])
    for s in good:
        assert (outs[0][s * n:(s + 1) * n] == outs[1][s * n:(s + 1) * n]).all()


# ---- fork ------------------------------------------------------------------------------------------------
def check_fork(r, lens, parent, reserve, page=16, h=2, d=64, layers=2, cache="bf16", release=True, order="heads", extra=0, spare=3,
               reserved=0, shared=False):
    """reserved: pages that the parents hold behind their tokens; shared: a parent's filled pages are the first one's."""
    lens = np.array(lens)
    have = -(-lens // page) + reserved
    need = -(-(np.array([lens[p] if p >= 0 else 0 for p in parent]) + (0 if reserve is None else np.array(reserve))) // page)
    cols_in, cols = max(1, int(have.max())) + 1, max(1, int(need.max(initial=0))) + 1
    n_pages = int(have.sum() + need.sum()) + spare
    table = tables(r, have, n_pages, cols_in)
    if shared:
        for s in range(1, len(lens)):
            both = min(lens[0], lens[s]) // page
            table[s, :both] = table[0, :both]
    ref = np.zeros(n_pages, dtype=np.int64)
    for row in table:
        for c in row[row >= 0]:
            ref[c] += 1
    ref[np.flatnonzero(ref == 0)[extra::5]] = 2 if extra else 0            # pages of sequences that are not in the call
    k, v = pool_pair((layers, n_pages, h, page, d), TYPES[cache], order, seed=1)
    want = paged.fork(ref.tolist(), table.tolist(), lens.tolist(), parent, reserve, cols, page, release)
    before = [x.clone() for x in (k, v)]
    t_out, l_out = torch.full((len(parent), cols), -7, dtype=torch.int32, device=DEV), torch.full((len(parent),), -7, dtype=torch.int32, device=DEV)
    r_out, err = torch.full((n_pages,), -7, dtype=torch.int32, device=DEV), err_word()
    space = torch.full((mcd.mcd_pages_fork_workspace(len(lens), t_out),), 255, dtype=torch.uint8, device=DEV)
    mcd.mcd_pages_fork(mcd.paged_kv(k, v), i32(ref), r_out, i32(table), i32(lens), i32(parent), t_out, l_out, space, err,
                       reserve=None if reserve is None else i32(reserve), release=release)
    torch.cuda.synchronize()
    if isinstance(want, str):
        assert err.item() == {"oom": 4, "invalid": 1}[want]
        assert (r_out.cpu().numpy() == ref).all() and (t_out == -7).all() and (l_out == -7).all()
        assert torch.equal(k, before[0]) and torch.equal(v, before[1])
        return want
    assert err.item() == 0
    assert t_out.tolist() == want[1] and l_out.tolist() == want[2] and r_out.tolist() == want[0]
    for x, old in zip((k, v), before):
        for a, c, n in want[3]:
            old[:, c, :, :n] = old[:, a, :, :n]
        assert torch.equal(x, old)
    return want


@pytest.mark.parametrize("release", [False, True])
@pytest.mark.parametrize("reserve", [None, 0, 1, 40])
@pytest.mark.parametrize("cache,order", [("bf16", "heads"), ("f32", "tokens")])
def test_fork(release, reserve, cache, order):
    r = np.random.RandomState(3)
    parent = [2, 0, 2, -1, 3, 2, 4, 0, -1]
    res = None if reserve is None else [reserve] * len(parent)
    for reserved, shared in ((0, False), (2, False), (1, True)):
        check_fork(r, [33, 7, 48, 0, 16], parent, res, release=release, cache=cache, order=order, reserved=reserved, shared=shared, extra=1, spare=20)


def test_fork_many():
    r = np.random.RandomState(4)
    lens = r.randint(0, 200, 60)
    check_fork(r, lens, r.randint(-1, 60, 1500).tolist(), r.randint(0, 50, 1500).tolist(), d=64, h=1, layers=1)
    check_fork(r, lens, list(range(60)), [1] * 60, page=32)                 # only room for a token more
    check_fork(r, lens, [], None)                                            # only the ends of the old ones
    check_fork(r, [5000], [0] * 3, [0] * 3, layers=1, h=1)                   # more columns than threads


def test_fork_errors():
    r = np.random.RandomState(5)
    assert check_fork(r, [33, 7], [0, 1, 0, 0], [400] * 4, spare=-60) == "oom"
    page, d = 16, 64
    k, v = pool_pair((1, 12, 1, page, d), torch.bfloat16)
    ref = i32([1, 1, 1, 0, 0, 0, 0, 0, 0, 0, 0, 0])
    good = dict(table=[[0, 1], [2, -1]], lens=[20, 16], parent=[0, 1], reserve=[0, 0], cols=2)
    for bad in (dict(table=[[0, 12], [2, -1]]), dict(table=[[0, -1], [2, -1]]), dict(table=[[0, -2], [2, -1]]), dict(lens=[33, 16]), dict(lens=[-1, 16]),
                dict(parent=[2, 0]), dict(parent=[-2, 0]), dict(reserve=[-1, 0]), dict(reserve=[13, 0])):
        c = dict(good, **bad)
        t_out, l_out = torch.full((2, 2), -7, dtype=torch.int32, device=DEV), torch.full((2,), -7, dtype=torch.int32, device=DEV)
        r_out, err, was = torch.zeros_like(ref), err_word(), k.clone()
        space = torch.empty(mcd.mcd_pages_fork_workspace(2, t_out), dtype=torch.uint8, device=DEV)
        mcd.mcd_pages_fork(mcd.paged_kv(k, v), ref, r_out, i32(c["table"]), i32(c["lens"]), i32(c["parent"]), t_out, l_out, space, err,
                           reserve=i32(c["reserve"]))
        assert err.item() == 1, bad
        assert (t_out == -7).all() and (l_out == -7).all() and torch.equal(r_out, ref) and torch.equal(k, was)


# ---- compact -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("page,cache,order", [(16, "bf16", "heads"), (32, "f32", "tokens"), (128, "bf16", "tokens")])
def test_compact(in_place, page, cache, order):
    r = np.random.RandomState(page)
    h, d, layers, cols = 3, 64, 2, -(-700 // page)
    start, keep = [5, 0, 300, 77, 16], []
    for s, n in enumerate([6, 0, 1, 200, 64]):
        row = r.choice(400, n, replace=False)
        keep.append(sorted(row) if in_place else list(row) if s % 2 else [int(row[0])] * n if n else [])
    n_pages = cols * 10
    order_of = r.permutation(n_pages).reshape(10, cols)
    table, table_out = order_of[:5], order_of[:5] if in_place else order_of[5:]
    k, v = pool_pair((layers, n_pages, h, page, d), TYPES[cache], order)
    want = [paged.compact(np64(x), table, table_out, start, keep) for x in (k, v)]
    most = max(len(x) for x in keep) + 2
    kp = np.full((5, most), -9)
    for s, x in enumerate(keep):
        kp[s, :len(x)] = x
    t = i32(table)
    len_out, err = torch.zeros(5, dtype=torch.int32, device=DEV), err_word()
    mcd.mcd_pages_compact(mcd.paged_kv(k, v), t, t if in_place else i32(table_out), i32(start), i32(kp), i32([len(x) for x in keep]), len_out, err)
    assert err.item() == 0 and len_out.tolist() == [a + len(b) for a, b in zip(start, keep)]
    assert (np64(k) == want[0]).all() and (np64(v) == want[1]).all()


def test_compact_errors():
    page, d, cols = 16, 64, 4
    k, v = pool_pair((1, 20, 1, page, d), torch.bfloat16)
    was = k.clone()
    table = [[0, 1, 2, 3], [4, 5, 6, 7], [8, 9, 10, 11]]
    good = dict(start=[0, 3, 5], keep=[[1, 2], [1, 4], [2, 3]], n=[2, 2, 2], table=table)
    for bad in (dict(start=[0, -1, 5]), dict(keep=[[1, 2], [4, 4], [2, 3]]), dict(keep=[[1, 2], [4, 1], [2, 3]]), dict(keep=[[1, 2], [-1, 1], [2, 3]]),
                dict(keep=[[1, 2], [1, 61], [2, 3]]), dict(n=[2, 3, 2]), dict(n=[2, -1, 2]), dict(start=[0, 63, 5]),
                dict(table=[table[0], [20, 5, 6, 7], table[2]]), dict(table=[table[0], [-1, 5, 6, 7], table[2]])):
        c = dict(good, **bad)
        k.copy_(was)
        t, err, len_out = i32(c["table"]), err_word(), torch.full((3,), -7, dtype=torch.int32, device=DEV)
        mcd.mcd_pages_compact(mcd.paged_kv(k, v), t, t, i32(c["start"]), i32(c["keep"]), i32(c["n"]), len_out, err)
        assert err.item() == 1, bad
        assert torch.equal(k[0, 4:8], was[0, 4:8]) and len_out.tolist() == [2, -7, 7]
        assert torch.equal(k[0, 0, :, 0], was[0, 0, :, 1]) and torch.equal(k[0, 8, :, 5], was[0, 8, :, 7])


# ---- together: as a serving program uses them ------------------------------------------------------------------
@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("captured", [False, True])
def test_serving_loop(cache, captured):
    """Two layers of attention for several utterances on one pool: prompts in two chunks, two of the utterances forked, single
    rows, a drafted tree of which a path is kept, single rows again; every row's output against the oracle on the
    utterance's own contiguous history.  On a side stream; optionally every step captured into a graph and replayed."""
    layers, hq, h, d, page, n_pages, cols = 2, 4, 2, 64, 16, 96, 12
    dt, r = TYPES[cache], np.random.RandomState(0)
    stream = torch.cuda.Stream()
    k, v = pool_pair((layers, n_pages, h, page, d), dt, fill=float("nan"))
    kv, err = mcd.paged_kv(k, v), err_word()
    w, _ = mcd.mcd_rope_freqs(d, 1e4)
    rope = mcd.rope(torch.as_tensor(w).to(DEV), d)
    state = dict(table=torch.full((4, cols), -1, dtype=torch.int32, device=DEV), len=torch.zeros(4, dtype=torch.int32, device=DEV),
                 ref=torch.zeros(n_pages, dtype=torch.int32, device=DEV))
    history = [[np.zeros((0, 2, h, d)) for _ in range(layers)] for _ in range(4)]   # [tokens, k / v, heads, d] as stored
    torch.cuda.synchronize()

    def go(fn):
        if not captured:
            with torch.cuda.stream(stream):
                fn(stream)
            stream.synchronize()
            return
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            fn(torch.cuda.current_stream())
        g.replay()
        torch.cuda.synchronize()

    def fork(parent, reserve, release=True):
        t, n = torch.empty((len(parent), cols), dtype=torch.int32, device=DEV), torch.empty(len(parent), dtype=torch.int32, device=DEV)
        ref, pa, re = torch.empty_like(state["ref"]), i32(parent), i32(reserve)
        space = torch.empty(mcd.mcd_pages_fork_workspace(len(state["len"]), t), dtype=torch.uint8, device=DEV)
        go(lambda s: mcd.mcd_pages_fork(kv, state["ref"], ref, state["table"], state["len"], pa, t, n, space, err, reserve=re,
                                        release=release, stream=s))
        state.update(table=t, len=n, ref=ref)
        history[:] = [[x.copy() for x in history[p]] for p in parent]

    def rows(counts, mask=None, depth=None):
        """New rows of every utterance through both layers; returns nothing, checks the outputs."""
        counts = np.array(counts)
        start = np.concatenate([[0], counts.cumsum()])
        n, cached = int(start[-1]), state["len"].cpu().numpy()
        ch = mcd.chunks(state["table"], state["len"], i32(start), n, int(counts.max()), cols * page)
        words, pos = None, None
        if mask is not None:
            bits = np.zeros((n, 32), dtype=np.uint8)
            for s, c in enumerate(counts):
                bits[start[s]:start[s] + c, :c] = mask
            words = torch.as_tensor(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).to(DEV)
            pos = i32(np.concatenate([cached[s] + depth for s in range(len(counts))]))
        for layer in range(layers):
            qkv = torch.randn((n, (hq + 2 * h) * d), device=DEV)
            q, out = torch.empty((n, hq * d), dtype=dt, device=DEV), torch.empty((n, hq * d), dtype=dt, device=DEV)
            space = torch.empty(mcd.mcd_paged_attention_workspace(kv, ch, hq), dtype=torch.uint8, device=DEV)
            torch.cuda.synchronize()

            def step(s):
                mcd.mcd_rope_append(kv, layer, ch, hq, qkv, q, rope, err, positions=pos, stream=s)
                mcd.mcd_paged_attention(kv, layer, ch, hq, q, out, d ** -0.5, space, err, mask=words, stream=s)
            go(step)
            assert err.item() == 0
            x, qq, got = np64(qkv).reshape(n, hq + 2 * h, d), np64(q).reshape(n, hq, d), np64(out).reshape(n, hq, d)
            for s, c in enumerate(counts):
                lo = start[s]
                new = np.zeros((c, 2, h, d))
                for i in range(c):
                    p = cached[s] + (depth[i] if depth is not None else i)
                    rq, rk, rv = paged.rope_row(x[lo + i], hq, h, p, w, False, None, None, 0)
                    # (v |x| <= 6: half a step of the type, and 64 u of the rotation)
                    assert (np.abs(qq[lo + i] - rq) <= HALF[cache] * np.abs(rq) + 64 * U * 12).all()
                    new[i] = np.stack([rk, rv])
                new = np64(torch.as_tensor(new).to(torch.float32).to(dt))
                full = np.concatenate([history[s][layer], new])
                ref, spread, reach = paged.attention(qq[lo:lo + c], full[:, 0], full[:, 1], int(cached[s]), d ** -0.5, mask)
                # keys near a rounding border may be stored a step apart: 2^-7 of a score's reach
                gap = HALF[cache] * 2 * reach + 64 * U * 12 * np.abs(qq[lo:lo + c]).sum(-1, keepdims=True) * d ** -0.5
                tol = HALF[cache] * np.abs(ref) + (2 * gap + 3 * HALF[cache] + 200 * U) * spread
                assert (np.abs(got[lo:lo + c] - ref) <= tol).all()
                # later steps see what is stored
                slots = [(int(state["table"][s, t // page]), t % page) for t in range(cached[s], cached[s] + c)]
                stored = np.array([[np64(y[layer, p, :, o]) for y in (k, v)] for p, o in slots]).reshape(c, 2, h, d)
                assert (np.abs(stored - new) <= 2 * HALF[cache] * np.abs(new) + 64 * U * 12).all()
                history[s][layer] = np.concatenate([history[s][layer], stored])
        state["len"] = state["len"] + i32(counts)

    fork([-1, -1, -1], [40, 40, 40], release=True)
    rows([37, 5, 20])
    fork([0, 1, 2], [40, 3, 1])
    rows([40, 3, 1])
    fork([2, 0, 0, 1, 0], [1] * 5)
    rows([1] * 5)
    assert int((state["ref"] < 0).sum()) == 0
    fork(list(range(5)), [6] * 5)
    mask = np.array([[1, 0, 0, 0, 0, 0], [1, 1, 0, 0, 0, 0], [1, 0, 1, 0, 0, 0], [1, 1, 0, 1, 0, 0], [1, 0, 1, 0, 1, 0], [1, 0, 1, 0, 1, 1]])
    before = state["len"].clone()
    rows([6] * 5, mask, np.array([0, 1, 1, 2, 2, 3]))
    keep, n_keep, length = i32([[0, 2, 4, 5]] * 5), i32([4, 3, 1, 2, 4]), torch.empty(5, dtype=torch.int32, device=DEV)
    go(lambda s: mcd.mcd_pages_compact(kv, state["table"], state["table"], before, keep, n_keep, length, err, stream=s))
    state["len"] = length
    for s, c in enumerate([4, 3, 1, 2, 4]):
        for layer in range(layers):
            x = history[s][layer]
            base = len(x) - 6
            history[s][layer] = np.concatenate([x[:base], x[base + np.array([0, 2, 4, 5])][:c]])
    assert length.tolist() == [len(x[0]) for x in history]
    fork([4, 3, 2, 1, 0], [1] * 5)
    rows([1] * 5)
    held = {int(c) for row in state["table"].cpu().numpy() for c in row if c >= 0}
    assert held == set(torch.nonzero(state["ref"])[:, 0].tolist()) and err.item() == 0


def test_two_graphs_share_a_workspace():
    """Two captured calls with one workspace, replayed one after the other, any number of times."""
    page, d, h, hq = 64, 128, 1, 2
    b = Batch([1], [6000], page)
    k, v = pool_pair((1, b.n_pages, h, page, d), torch.bfloat16)
    kv, err = mcd.paged_kv(k, v), err_word()
    space = torch.empty(max(16, mcd.mcd_paged_attention_workspace(kv, b.ch, hq)), dtype=torch.uint8, device=DEV)
    qs = [torch.randn((b.n_buf, hq * d), device=DEV).bfloat16() for _ in range(2)]
    outs = [torch.zeros((b.n_buf, hq * d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    want, graphs = [], []
    for q, o in zip(qs, outs):
        mcd.mcd_paged_attention(kv, 0, b.ch, hq, q, o, 0.1, space, err)
        torch.cuda.synchronize()
        want.append(o.clone())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            mcd.mcd_paged_attention(kv, 0, b.ch, hq, q, o, 0.1, space, err, stream=torch.cuda.current_stream())
        graphs.append(g)
    for o in outs:
        o.zero_()
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1]) and err.item() == 0
