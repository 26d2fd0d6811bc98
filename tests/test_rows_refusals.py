"""The rows' operators without a GPU: what they refuse before anything is launched (pointers are made up and never
read), and the plain forms that the GPU tests go by."""
import math

import numpy as np
import pytest

from oracle import paged, rows, sampler

OK, INVALID, UNSUPPORTED = 0, 1, 7
P = 1 << 20            # a 16-byte aligned address
Q = 1 << 30


@pytest.fixture(scope="module")
def lib():
    from paper_2609_37007_gb300 import build, mcd
    build.build()
    return mcd.load_library()


def norm_call(lib, n=3, w=64, x=P, xs=64, xd=1, res=None, rs=64, sum_out=None, ss=64, rd=1, norm=1, gain=None, eps=1e-6, y=Q, ys=64, yd=1, scale=None):
    return lib.mcd_norm_rows(n, w, x, xs, xd, res, rs, sum_out, ss, rd, norm, gain, eps, y, ys, yd, scale, None)


@pytest.mark.parametrize("bad,want", [
    (dict(n=-1), INVALID), (dict(w=0), INVALID), (dict(w=-5), INVALID), (dict(x=None), INVALID), (dict(y=None), INVALID),
    (dict(xs=63), INVALID), (dict(ys=63), INVALID), (dict(res=2 * Q, rs=63), INVALID), (dict(sum_out=2 * Q, ss=60), INVALID),
    (dict(eps=-1e-6), INVALID), (dict(eps=math.nan), INVALID), (dict(eps=math.inf), INVALID), (dict(yd=3, ys=64, scale=None), INVALID),
    (dict(xd=2), UNSUPPORTED), (dict(xd=3), UNSUPPORTED), (dict(yd=2), UNSUPPORTED), (dict(yd=4), UNSUPPORTED), (dict(res=2 * Q, rd=3), UNSUPPORTED),
    (dict(w=16385, xs=16392, ys=16392), UNSUPPORTED), (dict(x=P + 2), UNSUPPORTED), (dict(xs=65), UNSUPPORTED), (dict(y=Q + 8), UNSUPPORTED),
    (dict(xs=1 << 62), UNSUPPORTED), (dict(yd=3, ys=72, scale=2 * Q), UNSUPPORTED), (dict(gain=2 * Q + 4), UNSUPPORTED), (dict(yd=3, scale=2 * Q + 2), UNSUPPORTED),
    # outputs over inputs and each other
    (dict(y=P + 16), INVALID), (dict(y=P, ys=72), INVALID), (dict(y=P, yd=0), INVALID), (dict(y=P + 64), INVALID), (dict(sum_out=Q, y=Q), INVALID),
    (dict(sum_out=Q, y=Q + 128), INVALID), (dict(yd=3, y=Q, scale=Q + 64), INVALID), (dict(yd=3, scale=P + 8), INVALID),
    (dict(gain=Q), INVALID), (dict(yd=3, gain=2 * Q, scale=2 * Q + 16), INVALID), (dict(res=2 * Q, sum_out=2 * Q + 16), INVALID)])
def test_norm_rows_refuses(lib, bad, want):
    assert norm_call(lib, **bad) == want


def test_nothing_to_do_is_done(lib):
    assert norm_call(lib, n=0, x=None, y=None) == OK
    assert sample_call(lib, n=0, x=None, u=None, ids=None) == OK
    assert gemm_call(lib, n=0, b=None) == OK and gemm_call(lib, m=0, a=None) == OK


def sample_call(lib, n=3, v=64, x=P, xs=64, xd=0, u=Q, ids=2 * Q, err=3 * Q, temp=None, k=None, p=None, m=None, probs=None, kept=None):
    return lib.mcd_sample_rows(n, v, x, xs, xd, temp, k, p, m, u, ids, probs, kept, err, None)


@pytest.mark.parametrize("bad,want", [
    (dict(n=-1), INVALID), (dict(v=0), INVALID), (dict(x=None), INVALID), (dict(u=None), INVALID), (dict(ids=None), INVALID), (dict(err=None), INVALID),
    (dict(xs=63), INVALID), (dict(xd=2), UNSUPPORTED), (dict(xd=3), UNSUPPORTED), (dict(v=262145, xs=262152), UNSUPPORTED), (dict(x=P + 4), UNSUPPORTED),
    (dict(xs=66), UNSUPPORTED), (dict(xs=68, xd=1), UNSUPPORTED), (dict(n=(1 << 27) + 1), UNSUPPORTED), (dict(xs=1 << 60), UNSUPPORTED),
    (dict(u=Q + 4), UNSUPPORTED), (dict(ids=2 * Q + 2), UNSUPPORTED), (dict(temp=5 * Q + 1), UNSUPPORTED), (dict(kept=5 * Q + 2), UNSUPPORTED),
    (dict(ids=P + 256), INVALID), (dict(probs=2 * Q + 8), INVALID), (dict(kept=Q), INVALID), (dict(probs=5 * Q, kept=5 * Q), INVALID),
    (dict(k=2 * Q), INVALID), (dict(temp=5 * Q, probs=5 * Q), INVALID), (dict(ids=3 * Q), INVALID), (dict(err=P + 4), INVALID)])
def test_sample_rows_refuses(lib, bad, want):
    assert sample_call(lib, **bad) == want


def gemm_call(lib, m=128, n=16, k=64, a=P, lda=64, sa=None, b=Q, ldb=64, sb=None, y=2 * Q, ldy=128, yd=0, err=3 * Q):
    return lib.mcd_tc_gemm_e4m3(m, n, k, a, lda, sa, b, ldb, sb, y, ldy, yd, err, None)


@pytest.mark.parametrize("bad,want", [
    (dict(m=-1), INVALID), (dict(n=-1), INVALID), (dict(k=-1), INVALID), (dict(k=0), INVALID), (dict(a=None), INVALID), (dict(b=None), INVALID),
    (dict(y=None), INVALID), (dict(err=None), INVALID), (dict(lda=63), INVALID), (dict(ldb=48), INVALID), (dict(ldy=127), INVALID), (dict(y=P), INVALID),
    (dict(y=Q + 512), INVALID), (dict(sa=2 * Q), INVALID), (dict(sb=2 * Q + 1024), INVALID), (dict(yd=2), UNSUPPORTED), (dict(yd=3), UNSUPPORTED),
    (dict(a=P + 8), UNSUPPORTED), (dict(b=Q + 1), UNSUPPORTED), (dict(lda=72), UNSUPPORTED), (dict(ldb=72), UNSUPPORTED), (dict(ldy=130), UNSUPPORTED),
    (dict(m=(1 << 24) + 1, ldy=1 << 25), UNSUPPORTED), (dict(n=(1 << 24) + 1), UNSUPPORTED), (dict(lda=1 << 40), UNSUPPORTED),
    (dict(ldy=1 << 36), UNSUPPORTED), (dict(sa=5 * Q + 2), UNSUPPORTED), (dict(sb=5 * Q + 1), UNSUPPORTED)])
def test_gemm_refuses(lib, bad, want):
    assert gemm_call(lib, **bad) == want


# ---- the plain forms -------------------------------------------------------------------------------
def test_exp_is_the_samplers():
    d = -np.abs(np.random.RandomState(0).randn(500).astype(np.float32)) * np.float32(20)
    d[:4] = 0, -87, np.float32(-87.00001), -1e30
    assert all(float(a) == float(sampler.exp32(b)) for a, b in zip(rows.exp32(d), d))


def test_e4m3_values():
    v = rows.e4m3_values()
    assert v[0x7e] == 448 and v[0x08] == 2.0 ** -6 and v[1] == 2.0 ** -9 and math.isnan(v[0x7f]) and (v[128:255] == -v[:127]).all()
    import torch
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.nan_to_num(t, nan=1e9), np.nan_to_num(v, nan=1e9))


def test_sampling_law():
    """Drawn over a fine grid of u, ids come as often as their weights say, and filters leave what they name."""
    x = np.array([1.0, 3.0, 2.0, 3.0, -np.inf, 0.5], np.float32)
    p = np.exp(x.astype(float) / 0.7)
    p /= p.sum()
    n = 4000
    ids = [rows.sample(x, (i + 0.5) / n, 0.7)[0] for i in range(n)]
    assert np.abs(np.bincount(ids, minlength=6) / n - p).max() <= 1.5 / n
    assert rows.sample(x, 0.999, 0.7, top_k=3) == (3, 2 ** 31, 2 * 2 ** 31 + rows.sample(x, 0.5, 0.7, top_k=3)[2] - 2 ** 32, 3)
    assert rows.sample(x, 0.0, 0.7, top_k=1)[0] == 1 and rows.sample(x, 0.9, 0.0)[0] == 1
    assert rows.sample(x, 0.9, 0.7, top_p=p[1] * 0.99)[3] == 1 and rows.sample(x, 0.9, 0.7, top_p=p[1] * 1.01)[3] == 2
    assert rows.sample(x, 0.9, 0.7, min_p=1.0)[3] == 2 and rows.sample(x, 0.9, 0.7)[3] == 5


# ---- windowed attention --------------------------------------------------------------------------------
def window_call(m, window=10, sinks=2, **k):
    import ctypes
    from test_cache_refusals import ch, kv
    d, c = kv(m, **{x: k[x] for x in k if x in ("dtype", "k")}), ch(m)
    return m.load_library().mcd_paged_attention_window(ctypes.addressof(d), 0, ctypes.addressof(c), k.get("n_q", 16), P, 2048, k.get("out", 2 * P), 2048, 0.1,
                                                       window, sinks, k.get("mask"), k.get("words", 0), P, 1 << 40, k.get("err", P), None)


@pytest.mark.parametrize("bad,want", [
    (dict(window=0), INVALID), (dict(window=-5), INVALID), (dict(sinks=-1), INVALID), (dict(n_q=15), INVALID), (dict(err=None), INVALID),
    (dict(mask=P, words=0), INVALID), (dict(out=P), INVALID), (dict(k=None), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(n_q=136), UNSUPPORTED)])
def test_window_refuses(lib, bad, want):
    from paper_2609_37007_gb300 import mcd
    assert window_call(mcd, **bad) == want


def test_what_a_window_sees():
    see = paged.seen_in_window(3, 6, 4, 1)
    assert see.tolist() == [[True, False, False, True, True, True, True, False, False], [True, False, False, False, True, True, True, True, False],
                            [True, False, False, False, False, True, True, True, True]]
    assert (paged.seen_in_window(3, 6, 100, 0) == np.tril(np.ones((3, 9), bool), 6)).all()
    tree = np.array([[1, 0, 0], [1, 1, 0], [1, 0, 1]])
    see = paged.seen_in_window(3, 6, 4, 0, tree)
    assert see[1, :6].tolist() == see[2, :6].tolist() == [False, False, False, False, True, True] and (see[:, 6:] == tree).all()
    nothing = paged.seen_in_window(1, 6, 2, 0, np.array([[0]]))
    assert nothing.tolist() == [[False] * 5 + [True, False]]
