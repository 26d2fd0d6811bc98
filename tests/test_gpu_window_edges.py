"""mcd_paged_attention_window where new rows are sinks too: what a row does not see, by causality or by the mask, does not touch it,
whatever it holds."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2609_37007_gb300 import mcd
from test_gpu_cache import DEV, HALF, TYPES, U, Batch, documents, err_word, np64, pool_pair, tree
from test_gpu_window import words_of

pytestmark = pytest.mark.gpu


def check_bad_token(rows, cached, window, sinks, at, group=2, d=64, cache="bf16", mask=None, what="v", bad=float("inf"), seed=0):
    """Token `at` holds a value (what "v": in dimension 3 of KV head 1) or a key ("k") that is not finite: the rows that see it have
    none in that dimension (in all), every other result is right."""
    b, h = Batch([rows], [cached], 16, seed), 2
    k, v = pool_pair((1, b.n_pages, h, 16, d), TYPES[cache], seed=seed)
    kk, vv = np64(k), np64(v)
    if what == "v":
        v[0, b.table[0, at // 16], 1, at % 16, 3] = bad
    else:
        k[0, b.table[0, at // 16], 1, at % 16] = bad
    hq = h * group
    q = (1.5 * torch.randn((b.n_buf, hq * d), generator=torch.Generator(device=DEV).manual_seed(seed + 1), device=DEV)).to(TYPES[cache])
    mats, words = words_of(b, mask, seed) if mask else (None, None)
    out, kv, err = torch.zeros_like(q), mcd.paged_kv(k, v), err_word()
    space = torch.zeros(mcd.mcd_paged_attention_window_workspace(kv, b.ch, hq, window, sinks), dtype=torch.uint8, device=DEV)
    mcd.mcd_paged_attention_window(kv, 0, b.ch, hq, q, out, d ** -0.5, window, sinks, space, err, mask=words)
    torch.cuda.synchronize()
    assert err.item() == 0
    n, L = rows, rows + cached
    got = np64(out)[:n].reshape(n, hq, d)
    see = paged.seen_in_window(n, cached, window, sinks, None if mats is None else mats[0])
    touched = np.zeros((n, hq, d), dtype=bool)
    touched[see[:, at], group:, 3 if what == "v" else slice(None)] = True
    assert touched.any() and not touched.all()
    assert (np.isfinite(got) == ~touched).all(), int((np.isfinite(got) != ~touched).any((1, 2)).sum())
    ref, spread, reach = paged.attention_seen(np64(q)[:n].reshape(n, hq, d), paged.tokens(kk, 0, b.table[0], L), paged.tokens(vv, 0, b.table[0], L),
                                              see, d ** -0.5)
    # tolerances as derived in tests/test_gpu_cache.py
    delta = (d + 10) * U * reach + 8 * U
    tol = HALF[cache] * np.abs(ref) + (2 * delta + (2 * L + 4) * U + (2.0 ** -8 if cache == "bf16" else 0.0)) * spread
    assert (np.abs(got - ref) <= tol)[~touched].all()


@pytest.mark.parametrize("cache", ["bf16", "f32"])
@pytest.mark.parametrize("group,d", [(1, 64), (2, 128), (4, 64)])
@pytest.mark.parametrize("rows,cached,window,sinks,at", [(300, 0, 64, 4, 3), (300, 0, 64, 4, 1), (200, 100, 64, 130, 101), (200, 100, 64, 130, 129), (400, 50, 10, 300, 299),
                                                         (40, 0, 8, 4, 2), (3, 1, 1, 4, 2)])
def test_a_bad_value_of_a_new_row_among_the_sinks(cache, group, d, rows, cached, window, sinks, at):
    check_bad_token(rows, cached, window, sinks, at, group, d, cache)
    check_bad_token(rows, cached, window, sinks, at, group, d, cache, what="k", bad=float("nan"), seed=1)


@pytest.mark.parametrize("cache", ["bf16", "f32"])
@pytest.mark.parametrize("mask", [tree, documents])
@pytest.mark.parametrize("rows,cached,window,sinks,at", [(100, 10, 20, 64, 40), (65, 0, 3, 30, 5), (200, 100, 50, 150, 120), (6, 2, 2, 8, 4)])
def test_a_bad_value_of_a_masked_row_among_the_sinks(cache, mask, rows, cached, window, sinks, at):
    check_bad_token(rows, cached, window, sinks, at, cache=cache, mask=mask)
    check_bad_token(rows, cached, window, sinks, at, cache=cache, mask=mask, what="k", bad=float("nan"), seed=1)


@pytest.mark.parametrize("rows,cached,window", [(300, 0, 64), (130, 500, 300), (1, 700, 256)])
@pytest.mark.parametrize("cache", ["bf16", "f32"])
def test_a_window_gives_the_same_bits_every_time(rows, cached, window, cache):
    b = Batch([rows, rows, 1], [cached, cached // 2, cached], 16)
    k, v = pool_pair((1, b.n_pages, 2, 16, 64), TYPES[cache])
    q = torch.randn((b.n_buf, 256), generator=torch.Generator(device=DEV).manual_seed(0), device=DEV).to(TYPES[cache])
    kv, err, outs = mcd.paged_kv(k, v), err_word(), []
    space = torch.zeros(mcd.mcd_paged_attention_window_workspace(kv, b.ch, 4, window, 5), dtype=torch.uint8, device=DEV)
    for _ in range(20):
        outs.append(torch.zeros_like(q))
        mcd.mcd_paged_attention_window(kv, 0, b.ch, 4, q, outs[-1], 0.125, window, 5, space, err)
    torch.cuda.synchronize()
    assert err.item() == 0 and all(torch.equal(o, outs[0]) for o in outs)
