"""A layer's step of a serving program, its operators one after another as such a program calls them: row norm to 8 bits, 8-bit
QKV product, rotary append, windowed attention, 8-bit rows of its result, output product, residual sum and norm, head product,
sampling.  Pages that a sequence's window has left behind go to whoever needs one next.  Every operator's result is compared
with the 64-bit oracle on the operator's own inputs, so that a misplaced buffer, row or page shows where it happens."""
import numpy as np
import pytest
import torch

from oracle import paged, rows
from paper_2609_37007_gb300 import mcd
from test_gpu_cache import DEV, HALF, TYPES, U, err_word, i32, np64
from test_gpu_rows import dev

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
HID, HQ, HKV, D, VOCAB, PAGE, WINDOW, SINKS = 256, 4, 2, 64, 1000, 16, 24, 3


class Model:
    """Random 8-bit weights, laid out once by mcd_norm_rows without its norm."""

    def __init__(self, seed=0):
        r = np.random.RandomState(seed)
        self.w, self.s = {}, {}
        for name, (m, k) in {"qkv": ((HQ + 2 * HKV) * D, HID), "o": (HID, HQ * D), "head": (VOCAB, HID)}.items():
            x = dev(r.randn(m, k) / np.sqrt(k), torch.float32)
            self.w[name], self.s[name] = torch.zeros((m, k), dtype=E4M3, device=DEV), torch.zeros(m, device=DEV)
            mcd.mcd_norm_rows(x, self.w[name], norm=False, y_scale=self.s[name])
        self.gain = [dev(1 + 0.1 * r.randn(HID), torch.float32) for _ in range(2)]
        self.rope = mcd.rope(dev(1e4 ** (-np.arange(D // 2) / (D // 2)), torch.float64), D)


class Buffers:
    def __init__(self, n, cache):
        z = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device=DEV)      # noqa: E731
        self.x, self.res, self.sum = z(n, HID), z(n, HID), z(n, HID)
        self.n8, self.ns = z(n, HID, dtype=E4M3), z(n)
        self.qkv, self.q, self.a = z(n, (HQ + 2 * HKV) * D), z(n, HQ * D, dtype=cache), z(n, HQ * D, dtype=cache)
        self.a8, self.as_ = z(n, HQ * D, dtype=E4M3), z(n)
        self.o, self.f8, self.fs = z(n, HID), z(n, HID, dtype=E4M3), z(n)
        self.logits, self.ids, self.probs = z(n, VOCAB), z(n, dtype=torch.int32), z(n)
        self.u = torch.rand(n, dtype=torch.float64, device=DEV)
        self.temp, self.top_p = torch.full((n,), 0.8, device=DEV), torch.full((n,), 0.95, device=DEV)


def run_step(m, b, kv, ch, space, err, stream=None):
    mcd.mcd_norm_rows(b.x, b.n8, residual=b.res, sum_out=b.sum, gain=m.gain[0], y_scale=b.ns, stream=stream)
    mcd.mcd_tc_gemm_e4m3(m.w["qkv"], b.n8, b.qkv, err, a_scale=m.s["qkv"], b_scale=b.ns, stream=stream)
    mcd.mcd_rope_append(kv, 0, ch, HQ, b.qkv, b.q, m.rope, err, stream=stream)
    mcd.mcd_paged_attention_window(kv, 0, ch, HQ, b.q, b.a, D ** -0.5, WINDOW, SINKS, space, err, stream=stream)
    mcd.mcd_norm_rows(b.a, b.a8, norm=False, y_scale=b.as_, stream=stream)
    mcd.mcd_tc_gemm_e4m3(m.w["o"], b.a8, b.o, err, a_scale=m.s["o"], b_scale=b.as_, stream=stream)
    mcd.mcd_norm_rows(b.o, b.f8, residual=b.sum, sum_out=b.sum, gain=m.gain[1], y_scale=b.fs, stream=stream)
    mcd.mcd_tc_gemm_e4m3(m.w["head"], b.f8, b.logits, err, a_scale=m.s["head"], b_scale=b.fs, stream=stream)
    mcd.mcd_sample_rows(b.logits, b.u, b.ids, err, temperature=b.temp, top_p=b.top_p, probs=b.probs, stream=stream)


def near8(got, scale, want):
    """8-bit rows against the values they stand for (tolerances of tests/test_gpu_rows.py)."""
    q = want / np64(scale)[:, None]
    assert (np.abs(np64(got) - q) <= np.maximum(2.0 ** -4 * np.abs(q), 2.0 ** -10) + 90 * U * np.abs(q)).all()


def product(m, name, x8, xs, y):
    want, size = rows.gemm(np64(m.w[name]), np64(x8), np64(m.s[name]), np64(xs))
    assert (np.abs(np64(y) - want) <= HALF["f32"] * np.abs(want) + (2 * x8.shape[1] + 3) * U * size).all()


@pytest.mark.parametrize("cache", ["bf16", "f32"])
@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("chunk", [1, 9])
def test_steps_of_a_layer(cache, captured, chunk):
    n_seqs, steps = 3, 24 // chunk + 14
    dt, n, cols = TYPES[cache], n_seqs * chunk, -(-(steps * chunk + 40) // PAGE)
    r = np.random.RandomState(chunk)
    m, b, err = Model(), Buffers(n, dt), err_word()
    # as many pages as windows, sinks and new rows can be in, and no more
    n_pages = n_seqs * (1 + -(-(WINDOW + chunk) // PAGE) + 1)
    k, v = (torch.full((1, n_pages, HKV, PAGE, D), float("nan"), dtype=dt, device=DEV) for _ in range(2))
    kv = mcd.paged_kv(k, v)
    table, cached, free = np.full((n_seqs, cols), -1), np.array([0, 0, 0]), list(range(n_pages))
    d_table, d_cached, start = i32(table), i32(cached), i32(np.arange(n_seqs + 1) * chunk)
    ch = mcd.chunks(d_table, d_cached, start, n, chunk, cols * PAGE)
    space = torch.zeros(mcd.mcd_paged_attention_window_workspace(kv, ch, HQ, WINDOW, SINKS), dtype=torch.uint8, device=DEV)
    past = [[np.zeros((0, HKV, D)), np.zeros((0, HKV, D))] for _ in range(n_seqs)]
    side, graph = torch.cuda.Stream(), None
    for step in range(steps):
        for s in range(n_seqs):                        # pages behind the window are given back, the new rows' taken
            for c in range(cols):
                if table[s, c] >= 0 and c * PAGE >= SINKS and (c + 1) * PAGE - 1 <= cached[s] - WINDOW:
                    free.append(table[s, c])
                    table[s, c] = -1
        for s in range(n_seqs):
            for c in range(cached[s] // PAGE, (cached[s] + chunk - 1) // PAGE + 1):
                if table[s, c] < 0:
                    table[s, c] = free.pop(r.randint(len(free)))
        d_table.copy_(i32(table)), d_cached.copy_(i32(cached))
        b.x.copy_(dev(r.randn(n, HID), torch.float32)), b.res.copy_(dev(r.randn(n, HID), torch.float32))
        b.u.copy_(dev(r.rand(n), torch.float64))
        torch.cuda.synchronize()
        if not captured:
            run_step(m, b, kv, ch, space, err)
        elif graph is None:                            # (the first step runs as it is, so that nothing is set up while captured)
            run_step(m, b, kv, ch, space, err, side)
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            x, res = b.x.clone(), b.res.clone()
            with torch.cuda.graph(graph, stream=side):
                run_step(m, b, kv, ch, space, err, side)
            assert torch.equal(b.x, x) and torch.equal(b.res, res)
        else:
            graph.replay()
        torch.cuda.synchronize()
        assert err.item() == 0
        # ---- every operator on its own inputs
        total, normed = rows.norm_rows(np64(b.x), np64(b.res), np64(m.gain[0]))
        near8(b.n8, b.ns, normed)
        product(m, "qkv", b.n8, b.ns, b.qkv)
        x = np64(b.qkv).reshape(n, HQ + 2 * HKV, D)
        got_q, kk, vv = np64(b.q).reshape(n, HQ, D), np64(k), np64(v)
        freq = np64(m.rope.kept)
        for s in range(n_seqs):
            new_k, new_v = np.zeros((chunk, HKV, D)), np.zeros((chunk, HKV, D))
            for i in range(chunk):
                row, slot = s * chunk + i, cached[s] + i
                rq, rk, rv = paged.rope_row(x[row], HQ, HKV, slot, freq, False, None, None, 1e-6)
                at = (0, table[s, slot // PAGE], slice(None), slot % PAGE)
                size = np.abs(x[row]).max() * 3
                for got, want in ((got_q[row], rq), (kk[at], rk), (vv[at], rv)):
                    assert (np.abs(got - want) <= HALF[cache] * np.abs(want) + 32 * U * size).all()
                new_k[i], new_v[i] = kk[at], vv[at]
            past[s][0], past[s][1] = np.concatenate([past[s][0], new_k]), np.concatenate([past[s][1], new_v])
            see = paged.seen_in_window(chunk, int(cached[s]), WINDOW, SINKS)
            ref, spread, reach = paged.attention_seen(got_q[s * chunk:(s + 1) * chunk], past[s][0], past[s][1], see, D ** -0.5)
            delta = (D + 10) * U * reach + 8 * U
            tol = HALF[cache] * np.abs(ref) + (2 * delta + (2 * see.shape[1] + 4) * U + (2.0 ** -8 if cache == "bf16" else 0.0)) * spread
            assert (np.abs(np64(b.a).reshape(n, HQ, D)[s * chunk:(s + 1) * chunk] - ref) <= tol).all()
        near8(b.a8, b.as_, np64(b.a))
        product(m, "o", b.a8, b.as_, b.o)
        want_sum, normed = rows.norm_rows(np64(b.o), total, np64(m.gain[1]))
        # (b.sum has been rounded to fp32 on its way: 2^-24 of it, and again)
        assert (np.abs(np64(b.sum) - want_sum) <= 4 * U * (np.abs(want_sum) + np.abs(total))).all()
        # (two roundings of the sum, each u of it, reach the norm's result divided by the row's root mean square)
        q, fs = normed / np64(b.fs)[:, None], np64(b.fs)[:, None]
        rms = np.sqrt((want_sum ** 2).mean(1, keepdims=True) + 1e-6)
        extra = 2 * U * (np.abs(total) + np.abs(want_sum)) * np.abs(np64(m.gain[1])) / rms / fs
        # (and move the mean square by as much: 4 u of what the sums' sizes are to it, on every value)
        extra += np.abs(q) * 4 * U * ((np.abs(total) + np.abs(want_sum)) * np.abs(want_sum)).mean(1, keepdims=True) / rms ** 2
        assert (np.abs(np64(b.f8) - q) <= np.maximum(2.0 ** -4 * np.abs(q), 2.0 ** -10) + 90 * U * np.abs(q) + extra).all()
        product(m, "head", b.f8, b.fs, b.logits)
        logits, u = b.logits.cpu().numpy(), b.u.cpu().numpy()
        want = [rows.sample(logits[i], float(u[i]), float(np.float32(0.8)), 0, float(np.float32(0.95))) for i in range(n)]
        assert b.ids.cpu().tolist() == [w[0] for w in want]
        assert np.array_equal(b.probs.cpu().numpy(), np.array([w[1] / w[2] for w in want], np.float32))
        cached += chunk


def test_calls_on_two_streams_at_once():
    """The operators need no workspace (the attention: one each): two programs' calls may run side by side."""
    g = torch.Generator(device=DEV).manual_seed(3)
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    x = [torch.randn((700, 2048), generator=g, device=DEV) for _ in range(2)]
    w = torch.randn((1024, 2048), generator=g, device=DEV).to(E4M3)
    u = torch.rand(700, dtype=torch.float64, generator=g, device=DEV)
    k = torch.full((700,), 40, dtype=torch.int32, device=DEV)

    def go(i, stream):
        y, s, z = torch.zeros((700, 2048), dtype=E4M3, device=DEV), torch.zeros(700, device=DEV), torch.zeros((700, 1024), device=DEV)
        ids, err = torch.zeros(700, dtype=torch.int32, device=DEV), err_word()
        torch.cuda.synchronize() if stream is None else stream.wait_stream(torch.cuda.current_stream())
        for _ in range(5):
            mcd.mcd_norm_rows(x[i], y, y_scale=s, stream=stream)
            mcd.mcd_tc_gemm_e4m3(w, y, z, err, b_scale=s, stream=stream)
            mcd.mcd_sample_rows(z, u, ids, err, top_k=k, stream=stream)
        return y, s, z, ids, err

    for i in range(2):
        outs.append(go(i, streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        want = go(i, None)
        torch.cuda.synchronize()
        assert all(torch.equal(p.view(torch.uint8) if p.dtype is E4M3 else p, q.view(torch.uint8) if q.dtype is E4M3 else q)
                   for p, q in zip(outs[i], want))
        assert outs[i][4].item() == 0
