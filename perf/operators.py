"""The paged cache's operators, case by case: what they are measured on.

Four operators of a program that serves many utterances from one cache of pages:

  rope      packed q | k | v rows of new tokens: per-head RMSNorm, rotary positions, q out, K and V
            into the sequences' pages (mcd_rope_append);
  attn      attention of every sequence's new rows over its pages, causal or with a mask among
            the new rows (mcd_paged_attention);
  fork      children of sequences: full pages shared, part-filled ones copied, fresh ones reserved,
            the parents released (mcd_pages_fork);
  compact   kept tokens of every sequence moved together in all layers (mcd_pages_compact).

The CodeDecoder's shape (16 query heads on 8 KV heads of 128, 28 layers, bf16 cache) and the small
fp32 model's (4 heads of 64) stand in most cases.  A pool is [layers, pages, KV heads, page
size, head dim]; a sequence's row of the table names its pages in order, -1 past the last.
Lengths are a function of the case, values of the seed.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-6
BASE = 1e4


# ---- the cases ---------------------------------------------------------------------------
def listed():
    rope = dict(kind="rope", q_heads=16, kv_heads=8, dim=128, rot=128, interleaved=False, norm=True, inp="f32",
                cache="bf16", page=16, tree=False, stretch=1.0, lens=1)
    attn = dict(kind="attn", q_heads=16, kv_heads=8, dim=128, cache="bf16", page=16, tree=False, lens=1)
    fork = dict(kind="fork", kv_heads=8, dim=128, cache="bf16", page=16, release=True, lens=1)
    comp = dict(kind="compact", kv_heads=8, dim=128, cache="bf16", page=16, in_place=False, lens=1)
    return [
        # one utterance's next row, the fp32 output of the QKV product: all latency
        dict(rope, name="rope_1", seqs=1, rows_min=1, rows_max=1, cached_max=630),
        # prompts and text chunks of many utterances at once, bf16 rows
        dict(rope, name="rope_prompts", seqs=24, rows_min=101, rows_max=1021, cached_max=2000, inp="bf16", page=64),
        # one utterance's next row over the cache of 30 s of audio: all latency
        dict(attn, name="attn_1", seqs=1, rows_min=1, rows_max=1, cached_min=629, cached_max=629),
        # the next row of 128 utterances, each at its own place
        dict(attn, name="attn_128", seqs=128, rows_min=1, rows_max=1, cached_min=17, cached_max=1023),
        # a few drafted rows each over very long caches
        dict(attn, name="attn_long", seqs=4, rows_min=2, rows_max=4, cached_min=70000, cached_max=120000, page=64),
        # tree drafts of 64 nodes, verified together: 65 rows that see their ancestors
        dict(attn, name="attn_tree", seqs=32, rows_min=65, rows_max=65, cached_min=200, cached_max=1500, tree=True),
        # long prompts, part of them in the cache already
        dict(attn, name="attn_prompt", seqs=2, rows_min=5003, rows_max=6001, cached_min=0, cached_max=2500, page=64),
        # the small fp32 model: prompts and single rows side by side
        dict(attn, name="attn_f32", seqs=24, rows_min=1, rows_max=200, cached_min=0, cached_max=600, q_heads=4,
             kv_heads=4, dim=64, cache="f32"),
        # a beam step of one utterance: 8 beams reordered, room for the next token
        dict(fork, name="fork_8", src=8, dst=8, len_min=600, len_max=631, reserve=1, layers=28),
        # variants of 16 prompts: 128 utterances that share them
        dict(fork, name="fork_128", src=16, dst=128, len_min=257, len_max=511, reserve=32, layers=28),
        # accepted nodes of 32 drafted trees move to their places
        dict(comp, name="commit_32", seqs=32, start_min=200, start_max=700, span=64, keep_min=1, keep_max=7, layers=28,
             in_place=True),
        # half of long caches is dropped, the rest moved into fresh pages
        dict(comp, name="evict_8", seqs=8, start_min=4, start_max=64, span=4000, keep_min=1500, keep_max=2500, layers=5),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(("rope", "attn", "attn", "attn", "fork", "compact"))
    dim = rng.choice((64, 128))
    kv = rng.choice((1, 2, 4, 8))
    page = rng.choice((16, 32, 64, 128))
    cache = rng.choice(("bf16", "bf16", "f32"))
    base = dict(kind=kind, dim=dim, kv_heads=kv, page=page, cache=cache, lens=rng.randrange(1 << 20))
    if kind == "rope":
        rows = _log(rng, 1, 700)
        return dict(base, seqs=_log(rng, 1, 24), rows_min=rng.randint(1, rows), rows_max=rows, cached_max=_log(rng, 1, 100000),
                    q_heads=kv * rng.randint(1, 16 // kv), rot=rng.choice([r for r in (16, 32, 64, 96, 128) if r <= dim]),
                    interleaved=rng.random() < 0.5, norm=rng.random() < 0.5, inp="f32" if cache == "f32" else rng.choice(("f32", "bf16")),
                    tree=rng.random() < 0.3, stretch=rng.choice((1.0, 4.0)))
    if kind == "attn":
        group = rng.randint(1, min(8, 16 // kv))
        what = rng.choice(("step", "tree", "chunk"))
        if what == "step":
            seqs = _log(rng, 1, 128)
            rows, cached, tree = rng.randint(1, 4), _log(rng, 1, min(100000, 400000 // seqs)), False
        elif what == "tree":
            seqs = _log(rng, 1, 32)
            rows, cached, tree = rng.randint(2, 65), _log(rng, 1, 1500), True
        else:
            seqs = _log(rng, 1, 16)
            rows, cached, tree = _log(rng, 5, 2000 // seqs), _log(rng, 1, 2000), False
        return dict(base, seqs=seqs, rows_min=rng.randint(1, rows), rows_max=rows, cached_min=rng.randint(0, cached),
                    cached_max=cached, q_heads=kv * group, tree=tree)
    if kind == "fork":
        return dict(base, src=_log(rng, 1, 16), dst=_log(rng, 1, 64), len_min=rng.randint(0, 100), len_max=rng.randint(100, 600),
                    reserve=rng.randint(0, 40), layers=rng.randint(1, 12), release=rng.random() < 0.7)
    span = _log(rng, 16, 2000)
    keep = rng.randint(1, span // 2)
    return dict(base, seqs=_log(rng, 1, 16), start_min=0, start_max=rng.randint(0, 500), span=span, keep_min=rng.randint(0, keep),
                keep_max=keep, layers=rng.randint(1, 6), in_place=rng.random() < 0.5)


# ---- lengths: of the case alone ------------------------------------------------------------
def _spread(case, lo, hi, n, salt):
    v = np.random.RandomState((case["lens"] * 31 + salt) % (1 << 31)).randint(lo, hi + 1, n)
    v[0] = hi  # the bound is met
    return v.astype(np.int64)


def _rows(case):
    return _spread(case, case["rows_min"], case["rows_max"], case["seqs"], 1)


def _cached(case):
    return _spread(case, case.get("cached_min", 0), case["cached_max"], case["seqs"], 2)


def _fork_shape(case):
    lens = _spread(case, case["len_min"], case["len_max"], case["src"], 3)
    r = np.random.RandomState(case["lens"])
    parent = r.randint(0, case["src"], case["dst"])
    need = -(-(lens[parent] + case["reserve"]) // case["page"])
    cols = int(max(need.max(), (-(-lens // case["page"])).max(), 1)) + 1
    return lens, parent, need, cols


def _keep_shape(case):
    start = _spread(case, case["start_min"], case["start_max"], case["seqs"], 4)
    n = _spread(case, case["keep_min"], case["keep_max"], case["seqs"], 5)
    return start, n


def _cdiv(a, b):
    return -(-a // b)


# ---- work ------------------------------------------------------------------------------------
def work(case):
    e, d, h = SIZE[case["cache"]], case["dim"], case["kv_heads"]
    if case["kind"] == "rope":
        n, w = int(_rows(case).sum()), (case["q_heads"] + 2 * h) * d
        return {"bytes": n * w * (SIZE[case["inp"]] + e), "flops": n * (case["q_heads"] + h) * (4 * d * case["norm"] + 3 * case["rot"])}
    if case["kind"] == "attn":
        rows, cached = _rows(case), _cached(case)
        keys = int((cached + rows).sum())
        if case["tree"]:
            pairs = sum(int(c) * int(r) + int(_ancestors(int(r), case["lens"] + s).sum()) for s, (r, c) in enumerate(zip(rows, cached)))
        else:
            pairs = int((rows * cached + rows * (rows + 1) // 2).sum())
        words = _cdiv(case["rows_max"], 32) * case["tree"]
        return {"bytes": 2 * keys * h * d * e + int(rows.sum()) * (2 * case["q_heads"] * d * e + 4 * words), "flops": 4 * pairs * case["q_heads"] * d}
    if case["kind"] == "fork":
        lens, parent, need, cols = _fork_shape(case)
        first = np.zeros(case["dst"], dtype=bool)
        first[np.unique(parent, return_index=True)[1]] = case["release"]
        tokens = int(np.where(first, 0, lens[parent] % case["page"]).sum())
        return {"bytes": 2 * tokens * case["layers"] * 2 * h * d * e + 4 * (2 * _fork_pages(case) + (case["src"] + case["dst"]) * (cols + 2)), "flops": 0}
    start, n = _keep_shape(case)
    return {"bytes": int(n.sum()) * (4 + 2 * case["layers"] * 2 * h * d * e), "flops": 0}


# ---- inputs ------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(g, shape, dtype, scale=1.0):
    x = torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=g)
    return x if scale == 1.0 else x.mul_(scale)


def _dev(v, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(v)).to(device=DEV, dtype=dtype)


def _table(g, need, n_pages, cols, first=0):
    """Rows of a table: need[s] pages each, in a random order of the pool's pages from `first` on."""
    order = torch.randperm(n_pages - first, generator=g, device=DEV).to(torch.int32) + first
    col, need = torch.arange(cols, device=DEV), _dev(need, torch.int64)
    at = (need.cumsum(0) - need)[:, None] + col
    return torch.where(col < need[:, None], order[at.clamp(max=n_pages - first - 1)], -1).to(torch.int32)


def _ancestors(n, salt):
    """Ancestor-or-self matrix of a random tree of n rows: row 0 is the root, each other row's parent an earlier row."""
    r = np.random.RandomState(salt % (1 << 31))
    m = np.eye(n, dtype=bool)
    for i in range(1, n):
        m[i] |= m[r.randint(0, i) if r.rand() < 0.7 else max(0, i - 1)]
    return m


def _mask_words(case, rows):
    words = _cdiv(case["rows_max"], 32)
    parts = []
    for s, n in enumerate(rows):
        m = np.zeros((n, words * 32), dtype=np.uint8)
        m[:, :n] = _ancestors(int(n), case["lens"] + s)
        parts.append(np.packbits(m, axis=1, bitorder="little").view(np.int32))
    return _dev(np.concatenate(parts))


def _fork_pages(case):
    lens, parent, need, cols = _fork_shape(case)
    return int(_cdiv(lens, case["page"]).sum() + need.sum()) + 7


def prepare(case, seed):
    g = _generator(seed)
    kv = TYPES[case["cache"]]
    page, d, h = case["page"], case["dim"], case["kv_heads"]
    st = {"case": case}
    if case["kind"] in ("rope", "attn"):
        rows, cached = _rows(case), _cached(case)
        need = _cdiv(rows + cached, page)
        cols, n_pages, n = int(need.max()), int(need.sum()) + 3, int(rows.sum())
        st.update(n=n, max_rows=int(rows.max()), max_tokens=int((rows + cached).max()), rows=_dev(rows), cached=_dev(cached),
                  row_start=_dev(np.concatenate([[0], rows.cumsum()])), table=_table(g, need, n_pages, cols))
        pool = (1, n_pages, h, page, d)
        if case["kind"] == "rope":
            half = case["rot"] // 2
            st.update(k=torch.zeros(pool, dtype=kv, device=DEV), v=torch.zeros(pool, dtype=kv, device=DEV),
                      qkv=_normal(g, (n, (case["q_heads"] + 2 * h) * d), TYPES[case["inp"]]),
                      q=torch.zeros((n, case["q_heads"], d), dtype=kv, device=DEV),
                      inv_freq=(BASE ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)) / case["stretch"],
                      q_norm=1 + _normal(g, (d,), torch.float32, 0.1) if case["norm"] else None,
                      k_norm=1 + _normal(g, (d,), torch.float32, 0.1) if case["norm"] else None, positions=None)
            if case["tree"]:  # a row's position is its depth's, not its slot's
                r = np.random.RandomState(case["lens"])
                st["positions"] = _dev(np.concatenate([c + r.randint(0, 4, n) for c, n in zip(cached, rows)]))
        else:
            st.update(k=_normal(g, pool, kv), v=_normal(g, pool, kv), q=_normal(g, (n, case["q_heads"], d), kv, 1.5),
                      o=torch.zeros((n, case["q_heads"], d), dtype=kv, device=DEV),
                      mask=_mask_words(case, rows) if case["tree"] else None)
    elif case["kind"] == "fork":
        lens, parent, need, cols = _fork_shape(case)
        n_pages = _fork_pages(case)
        table = _table(g, _cdiv(lens, page), n_pages, cols)
        ref = torch.zeros(n_pages + 1, dtype=torch.int32, device=DEV)
        ref[table.flatten().long()] = 1  # (-1: the element past the pages)
        pool = (case["layers"], n_pages, h, page, d)
        st.update(k=_normal(g, pool, kv), v=_normal(g, pool, kv), table=table, len=_dev(lens), parent=_dev(parent), ref=ref[:-1].clone(),
                  reserve=_dev(np.full(case["dst"], case["reserve"])), ref_out=torch.zeros(n_pages, dtype=torch.int32, device=DEV),
                  table_out=torch.zeros((case["dst"], cols), dtype=torch.int32, device=DEV),
                  len_out=torch.zeros(case["dst"], dtype=torch.int32, device=DEV))
    else:
        start, n = _keep_shape(case)
        most, span, seqs = max(1, case["keep_max"]), case["span"], case["seqs"]
        have, want = _cdiv(start + span, page), _cdiv(start + n, page)
        both = int(have.sum()) + (0 if case["in_place"] else int(want.sum())) + 2
        cols = int(have.max())
        # kept offsets, ascending; in place they come from behind all the places they move to
        low = most if case["in_place"] else 0
        pick = torch.rand((seqs, span - low), generator=g, device=DEV).argsort(1)[:, :most] + low
        nk = _dev(n)
        keep = torch.where(torch.arange(most, device=DEV) < nk[:, None], pick, 1 << 20).sort(1).values.to(torch.int32)
        if case["in_place"]:
            table = _table(g, have, both, cols)
            table_out = table
        else:
            every = _table(g, np.concatenate([have, want]), both, cols)
            table, table_out = every[:seqs].contiguous(), every[seqs:].contiguous()
        pool = (case["layers"], both, h, page, d)
        st.update(k=_normal(g, pool, kv), v=_normal(g, pool, kv), table=table, table_out=table_out, start=_dev(start), keep=keep,
                  n_keep=nk, len_out=torch.zeros(seqs, dtype=torch.int32, device=DEV))
    return st


# ---- plain forms ----------------------------------------------------------------------------------
def _row_places(st):
    """Sequence of every row and its place in the chunk."""
    row = torch.arange(st["n"], device=DEV)
    seq = torch.searchsorted(st["row_start"][1:].long(), row, right=True)
    return seq, row - st["row_start"].long()[seq]


def _plain_rope(st):
    c = st["case"]
    hq, h, d, half, page = c["q_heads"], c["kv_heads"], c["dim"], c["rot"] // 2, c["page"]
    seq, i = _row_places(st)
    slot = st["cached"].long()[seq] + i
    pos = slot if st["positions"] is None else st["positions"].long()
    x = st["qkv"].view(st["n"], hq + 2 * h, d).float()
    qk, v = x[:, :hq + h], x[:, hq + h:]
    if c["norm"]:
        gain = torch.cat([st["q_norm"].expand(hq, d), st["k_norm"].expand(h, d)])
        qk = qk * torch.rsqrt(qk.square().mean(-1, keepdim=True) + EPS) * gain
    angle = pos.double()[:, None] * st["inv_freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    r = qk[..., :2 * half]
    a, b = (r[..., 0::2], r[..., 1::2]) if c["interleaved"] else (r[..., :half], r[..., half:])
    a, b = a * cos - b * sin, a * sin + b * cos
    r = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    qk = torch.cat([r, qk[..., 2 * half:]], -1)
    st["q"].copy_(qk[:, :hq])
    at, off = st["table"].long()[seq, slot // page], slot % page
    st["k"][0].transpose(1, 2)[at, off] = qk[:, hq:].to(st["k"].dtype)
    st["v"][0].transpose(1, 2)[at, off] = v.to(st["v"].dtype)
    return {"q": st["q"], "k": st["k"], "v": st["v"]}


def _plain_attn(st):
    c = st["case"]
    h, group, d = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"]
    seqs, n, keys = c["seqs"], st["max_rows"], st["max_tokens"]
    cached, rows = st["cached"].long(), st["rows"].long()
    i, j = torch.arange(n, device=DEV), torch.arange(keys, device=DEV)
    own_j = j - cached[:, None]                                              # [seqs, keys]: row of the chunk
    old = own_j < 0
    row = (st["row_start"].long()[:-1, None] + i).clamp(max=st["n"] - 1)      # [seqs, n]
    if st["mask"] is None:
        see = own_j[:, None] <= i[:, None]
    else:
        at = own_j.clamp(0, n - 1)[:, None].expand(seqs, n, keys)
        words = st["mask"][row].long()                                       # [seqs, n, words]
        see = old[:, None] | ((words.gather(2, at // 32) >> (at % 32)) & 1).bool()
    see = see & (own_j < rows[:, None])[:, None]                              # [seqs, n, keys]
    table = st["table"].long().clamp(min=0)
    k = st["k"][0][table].transpose(1, 2).reshape(seqs, h, -1, d)[:, :, :keys].float()
    v = st["v"][0][table].transpose(1, 2).reshape(seqs, h, -1, d)[:, :, :keys].float()
    q = st["q"][row].float().view(seqs, n, h, group, d).permute(0, 2, 3, 1, 4).reshape(seqs, h, group * n, d)
    s = (q @ k.transpose(-1, -2)).view(seqs, h, group, n, keys).mul_(d ** -0.5)
    s.masked_fill_(~see[:, None, None], -math.inf)
    s = s.sub_(s.amax(-1, keepdim=True)).exp_()
    total = s.sum(-1)
    o = (s.view(seqs, h, group * n, keys) @ v).view(seqs, h, group, n, d) / total[..., None]
    seq, place = _row_places(st)
    st["o"].copy_(o.permute(0, 3, 1, 2, 4)[seq, place].reshape(st["n"], h * group, d))
    return st["o"]


def _plain_fork(st):
    c = st["case"]
    page, release = c["page"], c["release"]
    table, ref, parent = st["table"].long(), st["ref"].long(), st["parent"].long()
    dst, cols = st["table_out"].shape
    n_pages = ref.numel()
    d, col = torch.arange(dst, device=DEV), torch.arange(cols, device=DEV)
    length = st["len"].long()[parent]
    need, full = (length + st["reserve"].long() + page - 1) // page, length // page
    eldest = torch.full((table.shape[0],), dst, device=DEV).scatter_reduce(0, parent, d, "amin")
    heir = (eldest[parent] == d) & release
    src = table[parent]
    alone = ref[src.clamp(min=0)] == 1
    kept = (col < full[:, None]) | (heir[:, None] & alone & (src >= 0) & (col < need[:, None]))
    fresh = (col < need[:, None]) & ~kept
    order = fresh.flatten().long().cumsum(0).view(dst, cols) - 1
    free = torch.argsort((ref != 0).long(), stable=True)
    out = torch.where(kept, src, torch.where(fresh, free[order.clamp(min=0, max=n_pages - 1)], -1))
    count = torch.zeros(n_pages + 1, dtype=torch.int64, device=DEV)
    count[:-1] = ref
    ones = torch.ones((), dtype=torch.int64, device=DEV)
    count.index_add_(0, torch.where(out >= 0, out, n_pages).flatten(), ones.expand(out.numel()))
    if release:
        count.index_add_(0, torch.where(table >= 0, table, n_pages).flatten(), -ones.expand(table.numel()))
    last = full.clamp(max=cols - 1)[:, None]
    copy = ((length % page > 0) & fresh.gather(1, last)[:, 0]).nonzero()[:, 0]
    come, go = src.gather(1, last)[copy, 0], out.gather(1, last)[copy, 0]
    part = (torch.arange(page, device=DEV) < (length % page)[copy, None])[None, :, None, :, None]
    for pool in (st["k"], st["v"]):
        pool[:, go] = torch.where(part, pool[:, come], pool[:, go])
    st["table_out"].copy_(out)
    st["len_out"].copy_(length)
    st["ref_out"].copy_(count[:-1])
    return {key: st[key] for key in ("table_out", "len_out", "ref_out", "k", "v")}


def _plain_compact(st):
    page = st["case"]["page"]
    seq, i = (torch.arange(st["keep"].shape[1], device=DEV) < st["n_keep"][:, None]).nonzero(as_tuple=True)
    start = st["start"].long()[seq]
    come, go = start + st["keep"].long()[seq, i], start + i
    a, b = st["table"].long()[seq, come // page], st["table_out"].long()[seq, go // page]
    for pool in (st["k"], st["v"]):
        pool.transpose(2, 3)[:, b, go % page] = pool.transpose(2, 3)[:, a, come % page]
    st["len_out"].copy_(st["start"] + st["n_keep"])
    return {"k": st["k"], "v": st["v"], "len_out": st["len_out"]}


# ---- the framework's calls --------------------------------------------------------------------------
def _own_calls(st):
    """What a program builds once for buffers that it keeps: descriptors, the workspace, the error word."""
    from paper_2609_37007_gb300 import mcd
    c = st["case"]
    kv = mcd.paged_kv(st["k"], st["v"])
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    if c["kind"] in ("rope", "attn"):
        chunks = mcd.chunks(st["table"], st["cached"], st["row_start"], n_rows=st["n"], max_rows=st["max_rows"], max_tokens=st["max_tokens"])
    if c["kind"] == "rope":
        rope = mcd.rope(st["inv_freq"], rot_dim=c["rot"], interleaved=c["interleaved"])
        return lambda: mcd.mcd_rope_append(kv, 0, chunks, c["q_heads"], st["qkv"], st["q"], rope, err, positions=st["positions"],
                                           q_norm=st["q_norm"], k_norm=st["k_norm"], eps=EPS)
    if c["kind"] == "attn":
        space = torch.empty(mcd.mcd_paged_attention_workspace(kv, chunks, c["q_heads"]), dtype=torch.uint8, device=DEV)
        return lambda: mcd.mcd_paged_attention(kv, 0, chunks, c["q_heads"], st["q"], st["o"], c["dim"] ** -0.5, space, err, mask=st["mask"])
    if c["kind"] == "fork":
        space = torch.empty(mcd.mcd_pages_fork_workspace(c["src"], st["table_out"]), dtype=torch.uint8, device=DEV)
        return lambda: mcd.mcd_pages_fork(kv, st["ref"], st["ref_out"], st["table"], st["len"], st["parent"], st["table_out"], st["len_out"],
                                          space, err, reserve=st["reserve"], release=c["release"])
    return lambda: mcd.mcd_pages_compact(kv, st["table"], st["table_out"], st["start"], st["keep"], st["n_keep"], st["len_out"], err)


OUTPUTS = {"rope": ("q", "k", "v"), "fork": ("table_out", "len_out", "ref_out", "k", "v"), "compact": ("k", "v", "len_out")}


def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"rope": _plain_rope, "attn": _plain_attn, "fork": _plain_fork, "compact": _plain_compact}[kind](st)
    if "call" not in st:
        st["call"] = _own_calls(st)
    st["call"]()
    return st["o"] if kind == "attn" else {key: st[key] for key in OUTPUTS[kind]}


# ---- from the definition, in 64 bits ------------------------------------------------------------------
def _tokens(pool, table, page, upto):
    """[H, upto, D] of one sequence, one layer: its pages in order."""
    pages = table[:_cdiv(upto, page)].tolist()
    return torch.cat([pool[p] for p in pages], 1)[:, :upto].double() if pages else pool[0][:, :0].double()


def exact(case, seed):
    st = prepare(case, seed)
    page, h = case["page"], case["kv_heads"]
    if case["kind"] == "attn":
        out = torch.zeros(st["o"].shape, dtype=torch.float64, device=DEV)
        at, group = 0, case["q_heads"] // h
        for s, (n, c) in enumerate(zip(_rows(case).tolist(), _cached(case).tolist())):
            k, v = (_tokens(st[x][0], st["table"][s], page, n + c) for x in "kv")
            if st["mask"] is None:
                see = torch.ones((n, n), dtype=torch.bool, device=DEV).tril()
            else:
                see = _dev(_ancestors(n, case["lens"] + s), torch.bool)
            hide = torch.cat([torch.zeros((n, c), dtype=torch.bool, device=DEV), ~see], 1)
            for head in range(case["q_heads"]):
                z = st["q"][at:at + n, head].double() @ k[head // group].T / math.sqrt(case["dim"])
                z[hide] = -math.inf
                out[at:at + n, head] = torch.softmax(z, -1) @ v[head // group]
            at += n
        return out
    if case["kind"] == "rope":
        x = st["qkv"].double().view(st["n"], -1, case["dim"]).clone()
        hq, half = case["q_heads"], case["rot"] // 2
        for lo, hi, gain in ((0, hq, st["q_norm"]), (hq, hq + h, st["k_norm"])):
            if gain is not None:
                part = x[:, lo:hi]
                x[:, lo:hi] = part / torch.sqrt((part * part).sum(-1, keepdim=True) / case["dim"] + EPS) * gain.double()
        slot = torch.cat([torch.arange(c, c + n, device=DEV) for n, c in zip(_rows(case).tolist(), _cached(case).tolist())])
        pos = slot if st["positions"] is None else st["positions"]
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), pos.double()[:, None] * st["inv_freq"])[:, None]
        first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["interleaved"] else (slice(0, half), slice(half, 2 * half))
        z = torch.complex(x[:, :hq + h, first], x[:, :hq + h, second]) * turn
        x[:, :hq + h, first], x[:, :hq + h, second] = z.real, z.imag
        k, v, at = st["k"].double(), st["v"].double(), 0
        for s, (n, c) in enumerate(zip(_rows(case).tolist(), _cached(case).tolist())):
            pages = st["table"][s].long()
            p = torch.arange(c, c + n, device=DEV)
            k[0].transpose(1, 2)[pages[p // page], p % page] = x[at:at + n, hq:hq + h]
            v[0].transpose(1, 2)[pages[p // page], p % page] = x[at:at + n, hq + h:]
            at += n
        return {"q": x[:, :hq].contiguous(), "k": k, "v": v}
    k, v = st["k"].double(), st["v"].double()
    table = st["table"].cpu().numpy()
    if case["kind"] == "compact":
        start, n = _keep_shape(case)
        to = st["table_out"].cpu().numpy()
        for s in range(case["seqs"]):
            come = start[s] + st["keep"][s, :n[s]].cpu().numpy()
            go = start[s] + np.arange(n[s])
            a, b = _dev(table[s][come // page], torch.int64), _dev(to[s][go // page], torch.int64)
            for pool, old in ((k, st["k"]), (v, st["v"])):
                pool.transpose(2, 3)[:, b, _dev(go % page, torch.int64)] = old.transpose(2, 3)[:, a, _dev(come % page, torch.int64)].double()
        return {"k": k, "v": v, "len_out": None}
    lens, parent, need, cols = _fork_shape(case)
    ref = st["ref"].cpu().numpy()
    free, taken = iter(np.flatnonzero(ref == 0)), set()
    for child in range(case["dst"]):
        p, full = parent[child], lens[parent[child]] // page
        heir = case["release"] and p not in taken
        taken.add(p)
        for c in range(full, need[child]):
            if heir and table[p][c] >= 0 and ref[table[p][c]] == 1:
                continue
            new = next(free)
            if c == full and lens[p] % page:
                for pool, old in ((k, st["k"]), (v, st["v"])):
                    pool[:, new, :, :lens[p] % page] = old[:, table[p][c], :, :lens[p] % page].double()
    return {"k": k, "v": v, "table_out": None, "len_out": None, "ref_out": None}
