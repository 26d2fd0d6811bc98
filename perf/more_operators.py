"""Operators around the paged cache and the products, case by case: what they are measured on.

Four operators that a program which serves many utterances runs in every step, between the ones of `operators.py`:

  norm      rows x + residual, RMSNorm with a gain, rounded to the next product's type: fp32, bf16 or
            8 bits (e4m3) with a scale per row; the sum goes back as the new residual (mcd_norm_rows);
  gemm      the product of 8-bit rows with 8-bit weights, scales applied (mcd_tc_gemm_e4m3);
  window    attention of new rows over a paged cache with a sliding window and a few first
            positions that stay visible (mcd_paged_attention_window);
  sample    one token of every row of logits: temperature, top-k, top-p and min-p per row, from given
            uniform numbers (mcd_sample_rows).

The shapes are the CodeDecoder's (hidden 1024, QKV rows of 4096, gate/up rows of 6144, 16 query heads on 8 KV
heads of 128, 2048 codes) and larger ones of the same kind.  A page that no row of a call can see may
have been given back: its entry of the table is -1.  Lengths are a function of the case, values of the
seed.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
SIZE = {"f32": 4, "bf16": 2, "e4m3": 1}
EPS = 1e-6
TOP = 448.0            # the largest e4m3 value
TINY = 2.0 ** -126     # the least scale of a row


# ---- the cases ---------------------------------------------------------------------------
def listed():
    norm = dict(kind="norm", width=1024, inp="f32", res="f32", out="e4m3", gain=True, norm=True)
    gemm = dict(kind="gemm", m=4096, k=1024, out="f32", scales=True)
    win = dict(kind="window", q_heads=16, kv_heads=8, dim=128, cache="bf16", page=16, tree=False, freed=True, sinks=4, lens=1)
    samp = dict(kind="sample", inp="f32", vocab=2048, mixed=False, spread=2.5)
    return [
        # one utterance's next row between two products: all latency
        dict(norm, name="norm_1", rows=1),
        # rows of many prompts in a wider model, bf16 throughout but for the 8-bit result
        dict(norm, name="norm_prompts", rows=30011, width=4096, inp="bf16", res="bf16"),
        # the QKV product of one utterance's next row and its three drafts: a stream of weights
        dict(gemm, name="gemm_step", n=4),
        # the gate/up product of 128 utterances' next rows
        dict(gemm, name="gemm_128", n=128, m=6144, out="bf16"),
        # prompts and text chunks of many utterances through a wide layer
        dict(gemm, name="gemm_prompts", n=8191, m=6144, k=4096, out="bf16"),
        # one utterance's next row long after its start: all latency
        dict(win, name="win_1", seqs=1, rows_min=1, rows_max=1, cached_min=9001, cached_max=9001, window=1024),
        # the next row of 128 utterances, young and old ones
        dict(win, name="win_128", seqs=128, rows_min=1, rows_max=1, cached_min=200, cached_max=60000, window=4096, page=64),
        # tree drafts of 64 nodes, verified together
        dict(win, name="win_tree", seqs=32, rows_min=65, rows_max=65, cached_min=200, cached_max=6000, window=1000, sinks=3, tree=True),
        # long prompts, part of them in the cache already
        dict(win, name="win_prompt", seqs=2, rows_min=8003, rows_max=9001, cached_min=0, cached_max=2500, window=2048, page=64),
        # one row of a code's logits: the smallest call
        dict(samp, name="sample_1", rows=1),
        # the next codes of 128 utterances, each with settings of its own
        dict(samp, name="sample_codes", rows=128, mixed=True),
        # text tokens of 96 sequences, bf16 logits of a large vocabulary
        dict(samp, name="sample_text", rows=96, vocab=131072, inp="bf16", mixed=True, spread=3.0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(("norm", "gemm", "gemm", "window", "window", "sample"))
    if kind == "norm":
        width = _log(rng, 1, 8200)
        return dict(kind=kind, rows=_log(rng, 1, min(30000, 100_000_000 // width)), width=width, inp=rng.choice(("f32", "bf16")),
                    res=rng.choice(("f32", "bf16", "none")), out=rng.choice(("e4m3", "e4m3", "bf16", "f32")), gain=rng.random() < 0.8,
                    norm=rng.random() < 0.8)
    if kind == "gemm":
        m, k = _log(rng, 1, 8000), _log(rng, 1, 5000)
        return dict(kind=kind, n=_log(rng, 1, min(8191, 200_000_000_000 // (m * k))), m=m, k=k, out=rng.choice(("f32", "bf16")),
                    scales=rng.random() < 0.8)
    if kind == "sample":
        vocab = _log(rng, 2, 200000)
        return dict(kind=kind, rows=_log(rng, 1, min(300, 12_000_000 // vocab)), vocab=vocab, inp=rng.choice(("f32", "bf16")),
                    mixed=rng.random() < 0.8, spread=rng.choice((0.5, 2.5, 6.0)))
    kv = rng.choice((1, 2, 4, 8))
    base = dict(kind=kind, dim=rng.choice((64, 128)), kv_heads=kv, q_heads=kv * rng.randint(1, min(8, 16 // kv)), page=rng.choice((16, 32, 64, 128)),
                cache=rng.choice(("bf16", "bf16", "f32")), lens=rng.randrange(1 << 20), window=_log(rng, 1, 4096),
                sinks=rng.choice((0, 1, 4, rng.randint(5, 200))), freed=rng.random() < 0.6)
    what = rng.choice(("step", "tree", "chunk"))
    if what == "step":
        seqs, rows, cached, tree = _log(rng, 1, 128), rng.randint(1, 4), _log(rng, 1, 60000), False
    elif what == "tree":
        seqs, rows, cached, tree = _log(rng, 1, 32), rng.randint(2, 65), _log(rng, 1, 6000), True
    else:
        seqs = _log(rng, 1, 16)
        rows, cached, tree = _log(rng, 5, 3000 // seqs), _log(rng, 1, 4000), False
    if not base["freed"]:
        cached = min(cached, 200000 // seqs)
    return dict(base, seqs=seqs, rows_min=rng.randint(1, rows), rows_max=rows, cached_min=rng.randint(0, cached), cached_max=cached, tree=tree)


# ---- lengths: of the case alone ------------------------------------------------------------
def _spread(case, lo, hi, n, salt):
    v = np.random.RandomState((case["lens"] * 31 + salt) % (1 << 31)).randint(lo, hi + 1, n)
    v[0] = hi  # the bound is met
    return v.astype(np.int64)


def _rows(case):
    return _spread(case, case["rows_min"], case["rows_max"], case["seqs"], 1)


def _cached(case):
    return _spread(case, case["cached_min"], case["cached_max"], case["seqs"], 2)


def _cdiv(a, b):
    return -(-a // b)


def _ancestors(n, salt):
    """Ancestor-or-self matrix of a random tree of n rows: row 0 is the root, each other row's parent an earlier row."""
    r = np.random.RandomState(salt % (1 << 31))
    m = np.eye(n, dtype=bool)
    for i in range(1, n):
        m[i] |= m[r.randint(0, i) if r.rand() < 0.7 else max(0, i - 1)]
    return m


# ---- work ------------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "norm":
        per = SIZE[case["inp"]] + SIZE[case["out"]] + (0 if case["res"] == "none" else 2 * SIZE[case["res"]])
        return {"bytes": case["rows"] * (case["width"] * per + 4 * (case["out"] == "e4m3")) + 4 * case["width"] * case["gain"],
                "flops": case["rows"] * case["width"] * 6}
    if kind == "gemm":
        n, m, k = case["n"], case["m"], case["k"]
        return {"bytes": n * k + m * k + n * m * SIZE[case["out"]] + 4 * (n + m) * case["scales"], "flops": 2 * n * m * k}
    if kind == "sample":
        return {"bytes": case["rows"] * (case["vocab"] * SIZE[case["inp"]] + 36), "flops": 0}
    e, d, h, w, sinks = SIZE[case["cache"]], case["dim"], case["kv_heads"], case["window"], case["sinks"]
    rows, cached = _rows(case), _cached(case)
    keys = int(sum(n + c - max(0, c - w + 1) + min(sinks, max(0, c - w + 1)) for n, c in zip(rows.tolist(), cached.tolist())))
    pairs = 0
    for s, (n, c) in enumerate(zip(rows.tolist(), cached.tolist())):
        own_rows = _ancestors(n, case["lens"] + s).sum(1) if case["tree"] else np.minimum(np.arange(n) + 1, w)
        pos = c + own_rows - 1 if case["tree"] else c + np.arange(n)
        low = np.maximum(pos - w + 1, 0)
        pairs += int((own_rows + np.maximum(c - low, 0) + np.minimum(np.minimum(sinks, low), c if case["tree"] else 1 << 40)).sum())
    words = _cdiv(case["rows_max"], 32) * case["tree"]
    return {"bytes": 2 * keys * h * d * e + int(rows.sum()) * (2 * case["q_heads"] * d * e + 4 * words), "flops": 4 * pairs * case["q_heads"] * d}


# ---- inputs ------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(g, shape, dtype, scale=1.0):
    x = torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=g)
    return x if scale == 1.0 else x.mul_(scale)


def _uniform(g, shape, lo, hi):
    return torch.empty(shape, dtype=torch.float32, device=DEV).uniform_(lo, hi, generator=g)


def _dev(v, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(v)).to(device=DEV, dtype=dtype)


def _even(n, size):
    """A row's stride: n elements of `size` bytes, up to the next 16 bytes."""
    per = 16 // size
    return _cdiv(n, per) * per


def _padded(x):
    """x's rows at a stride of whole 16 bytes."""
    n, w = x.shape
    y = torch.zeros((n, _even(w, x.element_size())), dtype=x.dtype, device=DEV)
    y[:, :w] = x
    return y[:, :w]


def _eight_bits(g, rows, k):
    """Rows of a model as 8-bit values with a scale each."""
    x = _normal(g, (rows, k), torch.float32) * _uniform(g, (rows, 1), 0.5, 2.0)
    s = x.abs().amax(1).clamp(min=1e-20) / TOP
    return _padded((x / s[:, None]).to(torch.float8_e4m3fn).view(torch.uint8)).view(torch.float8_e4m3fn), s


def _mask_words(case, rows):
    words = _cdiv(case["rows_max"], 32)
    parts = []
    for s, n in enumerate(rows):
        m = np.zeros((n, words * 32), dtype=np.uint8)
        m[:, :n] = _ancestors(int(n), case["lens"] + s)
        parts.append(np.packbits(m, axis=1, bitorder="little").view(np.int32))
    return _dev(np.concatenate(parts))


def prepare(case, seed):
    g = _generator(seed)
    kind = case["kind"]
    st = {"case": case}
    if kind == "norm":
        n, w = case["rows"], case["width"]
        st.update(x=_padded(_normal(g, (n, w), TYPES[case["inp"]])), gain=1 + _normal(g, (w,), torch.float32, 0.1) if case["gain"] else None)
        if case["res"] != "none":
            st.update(res=_padded(_normal(g, (n, w), TYPES[case["res"]], 3.0)), sum=_padded(torch.zeros((n, w), dtype=TYPES[case["res"]], device=DEV)))
        st["y"] = _padded(torch.zeros((n, w), dtype=torch.uint8 if case["out"] == "e4m3" else TYPES[case["out"]], device=DEV))
        if case["out"] == "e4m3":
            st.update(y=st["y"].view(torch.float8_e4m3fn), scale=torch.zeros(n, device=DEV))
    elif kind == "gemm":
        st["a"], a_scale = _eight_bits(g, case["m"], case["k"])
        st["b"], b_scale = _eight_bits(g, case["n"], case["k"])
        if case["scales"]:
            st.update(a_scale=a_scale, b_scale=b_scale)
        st["y"] = _padded(torch.zeros((case["n"], case["m"]), dtype=TYPES[case["out"]], device=DEV))
    elif kind == "sample":
        n, v = case["rows"], case["vocab"]
        st.update(logits=_padded(_normal(g, (n, v), TYPES[case["inp"]], case["spread"])),
                  u=torch.rand(n, dtype=torch.float64, device=DEV, generator=g))
        pick = torch.rand((4, n), device=DEV, generator=g)
        off = pick < 0.3  # of every setting some rows go without
        if case["mixed"]:
            st.update(temperature=torch.where(pick[0] < 0.1, 0.0, _uniform(g, (n,), 0.5, 1.3)),
                      top_k=torch.where(off[1], 0, _uniform(g, (n,), 1.0, 101.0).int()).int(),
                      top_p=torch.where(off[2], 1.0, _uniform(g, (n,), 0.5, 1.0)),
                      min_p=torch.where(off[3], 0.0, _uniform(g, (n,), 0.0, 0.1)))
        else:
            st.update(temperature=torch.full((n,), 0.9, device=DEV), top_k=torch.full((n,), 50, dtype=torch.int32, device=DEV), top_p=None, min_p=None)
        st.update(ids=torch.zeros(n, dtype=torch.int32, device=DEV), probs=torch.zeros(n, device=DEV), kept=torch.zeros(n, dtype=torch.int32, device=DEV))
    else:
        page, d, h, w, sinks = case["page"], case["dim"], case["kv_heads"], case["window"], case["sinks"]
        rows, cached = _rows(case), _cached(case)
        need = _cdiv(rows + cached, page)
        cols, n = int(need.max()), int(rows.sum())
        # pages in use: not those past the end, nor (given back) those whose positions nobody can see any more
        col = np.arange(cols)
        used = col < need[:, None]
        if case["freed"]:
            used &= ~((col * page >= sinks) & ((col + 1) * page - 1 <= (cached - w)[:, None]))
        n_pages = int(used.sum()) + 3
        order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        at = _dev(np.where(used, used.reshape(-1).cumsum().reshape(used.shape) - 1, 0), torch.int64)
        pool = (1, n_pages, h, page, d)
        kv = TYPES[case["cache"]]
        st.update(n=n, max_rows=int(rows.max()), max_tokens=int((rows + cached).max()), rows=_dev(rows), cached=_dev(cached),
                  row_start=_dev(np.concatenate([[0], rows.cumsum()])), table=torch.where(_dev(used, torch.bool), order[at], -1).to(torch.int32),
                  k=_normal(g, pool, kv), v=_normal(g, pool, kv), q=_normal(g, (n, case["q_heads"], d), kv, 1.5),
                  o=torch.zeros((n, case["q_heads"], d), dtype=kv, device=DEV), mask=_mask_words(case, rows) if case["tree"] else None)
    return st


# ---- plain forms ----------------------------------------------------------------------------------
def _plain_norm(st):
    c = st["case"]
    x = st["x"].float()
    out = {}
    if c["res"] != "none":
        x = x + st["res"].float()
        st["sum"].copy_(x)
        out["sum"] = st["sum"]
    if c["norm"]:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    if c["gain"]:
        x = x * st["gain"]
    if c["out"] == "e4m3":
        torch.clamp(x.abs().amax(-1) / TOP, min=TINY, out=st["scale"])
        out["scale"] = st["scale"]
        x = x / st["scale"][:, None]
    st["y"].copy_(x)
    out["y"] = st["y"]
    return out


def _plain_gemm(st):
    y = st["b"].float() @ st["a"].float().T
    if st["case"]["scales"]:
        y = y * st["b_scale"][:, None] * st["a_scale"]
    return st["y"].copy_(y)


def _exp32(d):
    """e^d for d <= 0 in single steps of fp32: what the weights of the sampler are defined with."""
    n = torch.round(d.clamp(min=-87.0) * 1.4426950408889634)
    r = (d.clamp(min=-87.0) - n * 0.693359375) - n * -2.12194440e-4
    p = torch.full_like(r, 1 / 5040)
    p = p * r + 1 / 720
    p = p * r + 1 / 120
    p = p * r + 1 / 24
    p = p * r + 1 / 6
    p = p * r + 0.5
    p = p * r + 1.0
    p = p * r + 1.0
    p = p * ((n.int() + 127) << 23).view(torch.float32)
    return torch.where(d < -87.0, 0.0, p)


def _plain_sample(st):
    x = st["logits"].float()
    n, v = x.shape
    greedy = st["temperature"] == 0
    z = x / torch.where(greedy, 1.0, st["temperature"])[:, None]
    w = (_exp32(z - z.amax(1, keepdim=True)) * 2.0 ** 31).floor().to(torch.int64)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    ranked = w.gather(1, order)
    k = torch.where((st["top_k"] <= 0) | (st["top_k"] > v), v, st["top_k"])
    k = torch.where(greedy, 1, k)
    ranked = torch.where(torch.arange(v, device=DEV) < k[:, None], ranked, 0)
    if st["top_p"] is not None:
        above = ranked.cumsum(1) - ranked
        need = torch.ceil(st["top_p"].double() * (above[:, -1] + ranked[:, -1]).double()).long()
        ranked = torch.where((above < need[:, None]) | (st["top_p"] >= 1)[:, None], ranked, 0)
    if st["min_p"] is not None:
        least = torch.ceil(st["min_p"].double() * 2.0 ** 31).long()
        ranked = torch.where(ranked >= least[:, None], ranked, 0)
    w = torch.zeros_like(w).scatter_(1, order, ranked)
    total = w.cumsum(1)
    mass = total[:, -1]
    t = torch.minimum((st["u"] * mass.double()).floor().long(), mass - 1)
    at = torch.searchsorted(total, t[:, None], right=True)
    st["ids"].copy_(at[:, 0])
    st["probs"].copy_(w.gather(1, at)[:, 0].double() / mass.double())
    st["kept"].copy_((w > 0).sum(1))
    return {"ids": st["ids"], "probs": st["probs"], "kept": st["kept"]}


def _plain_window(st):
    c = st["case"]
    h, group, d, win, sinks, page = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"], c["window"], c["sinks"], c["page"]
    seqs, n = c["seqs"], st["max_rows"]
    cached, rows = st["cached"].long(), st["rows"].long()
    low = (cached - win + 1).clamp(min=0)                                     # the first position that row 0's window holds
    first = low.clamp(max=sinks)                                             # sinks in front of it
    # key w of a sequence: a sink, or a position from `low` on
    keys = st["max_tokens"] if win + sinks + n >= st["max_tokens"] else win - 1 + sinks + n
    w = torch.arange(keys, device=DEV)
    pos = torch.where(w < first[:, None], w, w - first[:, None] + low[:, None])      # [seqs, keys]
    own_j = pos - cached[:, None]                                            # row of the chunk
    i = torch.arange(n, device=DEV)
    row = (st["row_start"].long()[:-1, None] + i).clamp(max=st["n"] - 1)      # [seqs, n]
    if st["mask"] is None:
        at = cached[:, None] + i                                             # a row's position
        see = (own_j[:, None] <= i[:, None]) & ((pos[:, None] > at[..., None] - win) | (pos[:, None] < sinks))
    else:
        bits = (st["mask"][row].long()[..., None] >> torch.arange(32, device=DEV)) & 1
        bits = bits.flatten(2)[..., :n] * (i < rows[:, None])[:, None]         # [seqs, n, n]
        at = cached[:, None] + bits.sum(-1).clamp(min=1) - 1
        mine = bits.bool().gather(2, own_j.clamp(0, n - 1)[:, None].expand(seqs, n, keys))
        see = torch.where((own_j >= 0)[:, None], mine, (pos[:, None] > at[..., None] - win) | (pos[:, None] < sinks))
    see = see & (own_j < rows[:, None])[:, None]                              # [seqs, n, keys]
    col = (pos // page).clamp(max=st["table"].shape[1] - 1)
    place = st["table"].long().gather(1, col).clamp(min=0) * page + pos % page
    k = st["k"][0].transpose(1, 2).reshape(-1, h, d)[place].transpose(1, 2).float()  # [seqs, h, keys, d]
    v = st["v"][0].transpose(1, 2).reshape(-1, h, d)[place].transpose(1, 2).float()
    q = st["q"][row].float().view(seqs, n, h, group, d).permute(0, 2, 3, 1, 4).reshape(seqs, h, group * n, d)
    s = (q @ k.transpose(-1, -2)).view(seqs, h, group, n, keys).mul_(d ** -0.5)
    s.masked_fill_(~see[:, None, None], -math.inf)
    s = s.sub_(s.amax(-1, keepdim=True)).exp_()
    total = s.sum(-1)
    o = (s.view(seqs, h, group * n, keys) @ v).view(seqs, h, group, n, d) / total[..., None]
    all_rows = torch.arange(st["n"], device=DEV)
    seq = torch.searchsorted(st["row_start"][1:].long(), all_rows, right=True)
    st["o"].copy_(o.permute(0, 3, 1, 2, 4)[seq, all_rows - st["row_start"].long()[seq]].reshape(st["n"], h * group, d))
    return st["o"]


# ---- the framework's calls --------------------------------------------------------------------------
def _own_calls(st):
    """What a program builds once for buffers that it keeps: descriptors, the workspace, the error word."""
    from paper_2609_37007_gb300 import mcd
    c = st["case"]
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    if c["kind"] == "norm":
        return lambda: mcd.mcd_norm_rows(st["x"], st["y"], residual=st.get("res"), sum_out=st.get("sum"), norm=c["norm"], gain=st["gain"], eps=EPS,
                                         y_scale=st.get("scale"))
    if c["kind"] == "gemm":
        return lambda: mcd.mcd_tc_gemm_e4m3(st["a"], st["b"], st["y"], err, a_scale=st.get("a_scale"), b_scale=st.get("b_scale"))
    if c["kind"] == "sample":
        return lambda: mcd.mcd_sample_rows(st["logits"], st["u"], st["ids"], err, temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"],
                                           min_p=st["min_p"], probs=st["probs"], kept=st["kept"])
    kv = mcd.paged_kv(st["k"], st["v"])
    chunks = mcd.chunks(st["table"], st["cached"], st["row_start"], n_rows=st["n"], max_rows=st["max_rows"], max_tokens=st["max_tokens"])
    space = torch.empty(mcd.mcd_paged_attention_window_workspace(kv, chunks, c["q_heads"], c["window"], c["sinks"]), dtype=torch.uint8, device=DEV)
    return lambda: mcd.mcd_paged_attention_window(kv, 0, chunks, c["q_heads"], st["q"], st["o"], c["dim"] ** -0.5, c["window"], c["sinks"], space, err,
                                                  mask=st["mask"])


OUTPUTS = {"norm": ("sum", "scale", "y"), "sample": ("ids", "probs", "kept")}


def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"norm": _plain_norm, "gemm": _plain_gemm, "window": _plain_window, "sample": _plain_sample}[kind](st)
    if "call" not in st:
        st["call"] = _own_calls(st)
    st["call"]()
    return st["y"] if kind == "gemm" else st["o"] if kind == "window" else {key: st[key] for key in OUTPUTS[kind] if key in st}


# ---- from the definition, in 64 bits ------------------------------------------------------------------
def _exact_sample(st):
    """Row by row in whole numbers, from the weights' definition in single precision."""
    f = np.float32
    probs = np.zeros(st["case"]["rows"])
    settings = [None if st[key] is None else st[key].cpu().numpy() for key in ("temperature", "top_k", "top_p", "min_p")]
    u = st["u"].cpu().numpy()
    terms = [f(1.0 / math.factorial(i)) for i in range(7, -1, -1)]
    for r, x in enumerate(st["logits"].float().cpu().numpy()):
        t, k, p, least = (None if s is None else s[r] for s in settings)
        best = np.lexsort((np.arange(x.size), -x))
        if t == 0:
            probs[r] = 1.0
            continue
        z = x / f(t)
        d = np.maximum(z - z.max(), f(-100))
        turns = np.rint(d * f(1.4426950408889634))
        rest = (d - turns * f(0.693359375)) - turns * f(-2.12194440e-4)
        e = np.full_like(rest, terms[0])
        for term in terms[1:]:
            e = e * rest + term
        w = np.where(d < f(-87), 0, np.floor(np.ldexp(e.astype(np.float64), turns.astype(int) + 31))).astype(np.int64)
        if 0 < k < x.size:
            best = best[:k]
        if p is not None and p < 1:
            sums = w[best].cumsum()
            best = best[:1 + np.count_nonzero(sums < math.ceil(float(p) * float(sums[-1])))]
        if least is not None:
            best = best[w[best] >= float(least) * 2.0 ** 31]
        best = np.sort(best[w[best] > 0])
        sums = w[best].cumsum()
        at = np.count_nonzero(sums <= min(math.floor(u[r] * float(sums[-1])), sums[-1] - 1))
        probs[r] = float(w[best[at]]) / float(sums[-1])
    return {"ids": None, "kept": None, "probs": torch.from_numpy(probs)}


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "sample":
        return _exact_sample(st)
    if case["kind"] == "gemm":
        y = torch.empty((case["n"], case["m"]), dtype=torch.float64, device=DEV)
        a = st["a"].to(torch.float64)
        for lo in range(0, case["n"], 1024):
            part = torch.einsum("mk,nk->nm", a, st["b"][lo:lo + 1024].to(torch.float64))
            y[lo:lo + 1024] = torch.einsum("nm,n,m->nm", part, st["b_scale"][lo:lo + 1024].double(), st["a_scale"].double()) if case["scales"] else part
        return y
    if case["kind"] == "norm":
        x = st["x"].double()
        out = {}
        if case["res"] != "none":
            out["sum"] = x = x.add_(st["res"].double())
        if case["norm"]:
            x = x / torch.sqrt((x * x).sum(1) / case["width"] + EPS)[:, None]
        if case["gain"]:
            x = torch.einsum("nw,w->nw", x, st["gain"].double())
        if case["out"] == "e4m3":
            out["scale"] = torch.maximum(torch.linalg.vector_norm(x, math.inf, dim=1) / TOP, torch.tensor(TINY, dtype=torch.float64, device=DEV))
            x = x / out["scale"][:, None]
        out["y"] = x
        return out
    page, h, group, win, sinks = case["page"], case["kv_heads"], case["q_heads"] // case["kv_heads"], case["window"], case["sinks"]
    out = torch.zeros(st["o"].shape, dtype=torch.float64, device=DEV)
    at = 0
    for s, (n, c) in enumerate(zip(_rows(case).tolist(), _cached(case).tolist())):
        start = max(0, c - win + 1)
        where = np.concatenate([np.arange(min(sinks, start)), np.arange(start, c + n)])
        below = np.tril(np.ones((n, n), dtype=bool)) if not case["tree"] else _ancestors(n, case["lens"] + s)
        place = c + below.sum(1) - 1
        near = (where[None] > place[:, None] - win) | (where[None] < sinks)
        new = where.size - n
        hide = np.concatenate([~near[:, :new], ~(below if case["tree"] else below & near[:, new:])], 1)
        hide, where = _dev(hide, torch.bool), _dev(where, torch.int64)
        pages = st["table"][s].long()[where // page]
        for head in range(h):
            k, v = (st[x][0][pages, head, where % page].double() for x in "kv")
            for qh in range(head * group, (head + 1) * group):
                z = st["q"][at:at + n, qh].double() @ k.T / math.sqrt(case["dim"])
                out[at:at + n, qh] = torch.softmax(z.masked_fill_(hide, -math.inf), -1) @ v
        at += n
    return out
