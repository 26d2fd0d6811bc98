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
