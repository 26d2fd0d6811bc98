"""The paged cache's entry points without a GPU: what they refuse before anything is launched (pointers
are made up and never read), the frequencies of the rotation, and the descriptors' layout."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from conftest import ROOT
from oracle import paged

OK, INVALID, UNSUPPORTED = 0, 1, 7
P = 1 << 20            # a 16-byte aligned address


@pytest.fixture(scope="module")
def mcd():
    from paper_2609_37007_gb300 import build, mcd
    build.build()
    mcd.load_library()
    return mcd


def kv(mcd, **k):
    d = dict(k=P, v=P, layer_stride=10 * 8 * 16 * 128, page_stride=8 * 16 * 128, head_stride=16 * 128, token_stride=128,
             n_layers=2, n_pages=10, n_kv_heads=8, page_size=16, head_dim=128, dtype=1)
    d.update(k)
    return mcd.McdPagedKV(**d)


def ch(mcd, **k):
    d = dict(table=P, cached=P, row_start=P, n_seqs=3, table_stride=4, n_rows=9, max_rows=5, max_tokens=64)
    d.update(k)
    return mcd.McdChunks(**d)


def addr(x):
    return ctypes.addressof(x) if x is not None else None


BAD_KV = [(dict(k=None), INVALID), (dict(v=None), INVALID), (dict(n_layers=0), INVALID), (dict(n_pages=0), INVALID),
          (dict(n_kv_heads=0), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED),
          (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(page_size=256), UNSUPPORTED),
          (dict(k=P + 8), UNSUPPORTED), (dict(token_stride=132), UNSUPPORTED), (dict(token_stride=64), UNSUPPORTED),
          (dict(page_stride=-16384), UNSUPPORTED), (dict(layer_stride=0), UNSUPPORTED), (dict(n_kv_heads=2000), UNSUPPORTED)]
BAD_CH = [(dict(n_seqs=-1), INVALID), (dict(n_rows=-1), INVALID), (dict(max_rows=-2), INVALID), (dict(max_tokens=-1), INVALID),
          (dict(table=None), INVALID), (dict(cached=None), INVALID), (dict(row_start=None), INVALID),
          (dict(max_tokens=65), INVALID), (dict(n_seqs=70000), UNSUPPORTED), (dict(n_rows=1 << 27), UNSUPPORTED)]


def rope_call(mcd, k=None, c=None, layer=0, n_q=16, qkv=P, qkv_stride=32 * 128, dtype=1, q=P, q_stride=16 * 128, rope="", pos=None, qn=None,
              kn=None, eps=1e-6, err=P):
    k, c = k or kv(mcd), c or ch(mcd)
    rope = mcd.McdRope(P, 1.0, 128, 0) if rope == "" else rope
    return mcd.load_library().mcd_rope_append(addr(k), layer, addr(c), n_q, qkv, qkv_stride, dtype, q, q_stride, addr(rope), pos,
                                              qn, kn, eps, err, None)


def attn_call(mcd, k=None, c=None, layer=0, n_q=16, q=P, q_stride=2048, out=2 * P, out_stride=2048, scale=0.1, mask=None, words=0, err=P):
    k, c = k or kv(mcd), c or ch(mcd)
    return mcd.load_library().mcd_paged_attention(addr(k), layer, addr(c), n_q, q, q_stride, out, out_stride, scale, mask, words, P,
                                                  1 << 40, err, None)


def fork_call(mcd, k=None, ref=P, ref_out=2 * P, n_src=3, table=P, src_cols=4, lens=P, n_dst=5, parent=P, reserve=None, out=2 * P,
              dst_cols=4, len_out=2 * P, ws=P, ws_bytes=1 << 30, err=P):
    k = k or kv(mcd)
    return mcd.load_library().mcd_pages_fork(addr(k), ref, ref_out, n_src, table, src_cols, lens, n_dst, parent, reserve, out, dst_cols,
                                             len_out, 1, ws, ws_bytes, err, None)


def compact_call(mcd, k=None, n=3, table=P, out=2 * P, cols=4, start=P, keep=P, max_keep=5, n_keep=P, err=P):
    k = k or kv(mcd)
    return mcd.load_library().mcd_pages_compact(addr(k), n, table, out, cols, start, keep, max_keep, n_keep, None, err, None)


@pytest.mark.parametrize("bad,want", BAD_KV)
def test_pool_descriptors(mcd, bad, want):
    for call in (rope_call, attn_call, fork_call, compact_call):
        assert call(mcd, k=kv(mcd, **bad)) == want, call.__name__


@pytest.mark.parametrize("bad,want", BAD_CH)
def test_row_descriptors(mcd, bad, want):
    for call in (rope_call, attn_call):
        assert call(mcd, c=ch(mcd, **bad)) == want, call.__name__


def test_nothing_to_do(mcd):
    for empty in (dict(n_seqs=0), dict(n_rows=0), dict(max_rows=0), dict(n_seqs=0, table=None, cached=None, row_start=None)):
        assert rope_call(mcd, c=ch(mcd, **empty)) == OK
        assert attn_call(mcd, c=ch(mcd, **empty)) == OK
    assert compact_call(mcd, n=0) == OK


@pytest.mark.parametrize("bad,want", [
    (dict(layer=2), INVALID), (dict(layer=-1), INVALID), (dict(n_q=0), INVALID), (dict(qkv=None), INVALID), (dict(q=None), INVALID),
    (dict(err=None), INVALID), (dict(rope=None), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=-1.0), INVALID),
    (dict(qkv_stride=4095), INVALID), (dict(q_stride=2040), INVALID), (dict(qkv_stride=4100), UNSUPPORTED),
    (dict(qkv=P + 2), UNSUPPORTED), (dict(q=P + 8), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(qn=P + 4), UNSUPPORTED)])
def test_rope_refusals(mcd, bad, want):
    assert rope_call(mcd, **bad) == want


@pytest.mark.parametrize("rope,want", [((P, 1.0, 136, 0), INVALID), ((P, 1.0, -16, 0), INVALID), ((None, 1.0, 64, 0), INVALID),
                                       ((P, float("inf"), 64, 0), INVALID), ((P, 1.0, 24, 0), UNSUPPORTED)])
def test_rotations(mcd, rope, want):
    assert rope_call(mcd, rope=mcd.McdRope(*rope)) == want


def test_bf16_rows_need_a_bf16_cache(mcd):
    assert rope_call(mcd, k=kv(mcd, dtype=0), dtype=1) == UNSUPPORTED


@pytest.mark.parametrize("bad,want", [
    (dict(layer=2), INVALID), (dict(n_q=12), INVALID), (dict(n_q=8 * 17), UNSUPPORTED), (dict(q=None), INVALID), (dict(out=None), INVALID),
    (dict(out=P), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=3e38), INVALID), (dict(q_stride=2047), INVALID), (dict(out_stride=2052), UNSUPPORTED), (dict(q=P + 8), UNSUPPORTED),
    (dict(err=None), INVALID), (dict(mask=P, words=0), INVALID)])
def test_attention_refusals(mcd, bad, want):
    if bad.get("n_q") == 8 * 17:
        bad = dict(bad, q_stride=17 * 1024, out_stride=17 * 1024)
    assert attn_call(mcd, **bad) == want


@pytest.mark.parametrize("bad,want", [
    (dict(ref=None), INVALID), (dict(ref_out=None), INVALID), (dict(ref_out=P), INVALID), (dict(n_src=-1), INVALID),
    (dict(n_dst=-1), INVALID), (dict(table=None), INVALID), (dict(lens=None), INVALID), (dict(parent=None), INVALID),
    (dict(out=None), INVALID), (dict(out=P), INVALID), (dict(len_out=P), INVALID), (dict(ws=None), INVALID), (dict(ws=P + 4), INVALID),
    (dict(ws_bytes=16), INVALID), (dict(err=None), INVALID), (dict(n_src=5000), UNSUPPORTED), (dict(n_dst=5000), UNSUPPORTED)])
def test_fork_refusals(mcd, bad, want):
    assert fork_call(mcd, **bad) == want


@pytest.mark.parametrize("bad,want", [
    (dict(n=-1), INVALID), (dict(table=None), INVALID), (dict(out=None), INVALID), (dict(start=None), INVALID), (dict(keep=None), INVALID),
    (dict(n_keep=None), INVALID), (dict(max_keep=-1), INVALID), (dict(err=None), INVALID), (dict(n=70000), UNSUPPORTED)])
def test_compact_refusals(mcd, bad, want):
    assert compact_call(mcd, **bad) == want


@pytest.mark.parametrize("rot", [2, 16, 64, 96, 128])
def test_frequencies(mcd, rot):
    w, scale = mcd.mcd_rope_freqs(rot, 1e4)
    assert np.allclose(w, paged.frequencies("plain", rot, 1e4), rtol=1e-13) and scale == 1.0
    w, scale = mcd.mcd_rope_freqs(rot, 1e4, mcd.ROPE_LINEAR, 4.0)
    assert np.allclose(w, paged.frequencies("linear", rot, 1e4, 4.0), rtol=1e-13) and scale == 1.0
    w, scale = mcd.mcd_rope_freqs(rot, 1e6, mcd.ROPE_BY_PARTS, 8.0, 4096)
    assert np.allclose(w, paged.frequencies("parts", rot, 1e6, 8.0, 4096), rtol=1e-12)
    assert scale == np.float32(0.1 * np.log(8.0) + 1.0)
    plain = paged.frequencies("plain", rot, 1e6)
    assert (w <= plain * (1 + 1e-12)).all() and (w >= plain / 8.0 * (1 - 1e-12)).all()
    if rot > 2:
        w, _ = mcd.mcd_rope_freqs(rot, 1e4, mcd.ROPE_BASE, 4.0)
        assert np.allclose(w, paged.frequencies("base", rot, 1e4, 4.0), rtol=1e-12)
        assert w[0] == 1.0 and abs(w[-1] * 4.0 / paged.frequencies("plain", rot, 1e4)[-1] - 1) < 1e-12


def test_frequency_refusals(mcd):
    f = mcd.load_library().mcd_rope_freqs
    buf = np.zeros(64)
    good = [0, 64, 1e4, 1.0, 0, 32.0, 1.0, buf.ctypes.data, None]
    assert f(*good) == OK
    for i, v in ((0, 4), (0, -1), (1, 0), (1, 63), (2, 1.0), (2, float("nan")), (3, 0.5), (3, 2.0), (7, None)):
        assert f(*(good[:i] + [v] + good[i + 1:])) == INVALID, (i, v)
    parts = [3, 64, 1e4, 2.0, 4096, 32.0, 1.0, buf.ctypes.data, None]
    assert f(*parts) == OK
    for i, v in ((4, 0), (5, 1.0), (5, float("inf")), (6, 0.0), (6, 40.0)):
        assert f(*(parts[:i] + [v] + parts[i + 1:])) == INVALID, (i, v)
    assert f(2, 2, 1e4, 2.0, 0, 32.0, 1.0, buf.ctypes.data, None) == INVALID


def test_descriptor_layouts(mcd, tmp_path):
    src = tmp_path / "sz.c"
    src.write_text('#include "mcd_cache.h"\n#include <stdio.h>\n#include <stddef.h>\n'
                   'int main(void){printf("%zu %zu %zu %zu %zu %zu", sizeof(mcd_paged_kv), sizeof(mcd_chunks), sizeof(mcd_rope),'
                   ' offsetof(mcd_paged_kv, dtype), offsetof(mcd_chunks, max_tokens), offsetof(mcd_rope, interleaved));return 0;}\n')
    exe = tmp_path / "sz"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert out == [ctypes.sizeof(mcd.McdPagedKV), ctypes.sizeof(mcd.McdChunks), ctypes.sizeof(mcd.McdRope),
                   mcd.McdPagedKV.dtype.offset, mcd.McdChunks.max_tokens.offset, mcd.McdRope.interleaved.offset]


def test_oracle_rotation_and_attention():
    """The plain forms themselves: a rotation keeps lengths and turns by differences of positions; attention of one
    visible key is its value, of equal keys the mean."""
    r = np.random.RandomState(0)
    w = paged.frequencies("plain", 32, 1e4)
    x, y = r.randn(64), r.randn(64)
    for inter in (False, True):
        a, b = paged.rotate(x, 7, w, inter), paged.rotate(y, 4, w, inter)
        c, d = paged.rotate(x, 1003, w, inter), paged.rotate(y, 1000, w, inter)
        assert abs(a @ b - c @ d) < 1e-9 and abs(a @ a - x @ x) < 1e-9 and (a[32:] == x[32:]).all()
    q, k, v = r.randn(2, 2, 8), np.ones((5, 1, 8)), r.randn(5, 1, 8)
    out, _, _ = paged.attention(q, k, v, 3, 0.3)
    assert np.allclose(out[0], v[:4, 0].mean(0)) and np.allclose(out[1], v[:, 0].mean(0))
    out, _, _ = paged.attention(q, k[:2], v[:2], 0, 0.3, np.array([[0, 0], [1, 0]]))
    assert (out[0] == 0).all() and np.allclose(out[1], v[0, 0])
