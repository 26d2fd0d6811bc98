"""The rows' operators on the GPU against oracle/rows.py in 64 bits.

Tolerances count the roundings, u = 2^-24 (fp32):
  norm: the sum r is off by u; its squares are summed 16 at a time in a thread, then in at most 5 + 32 joins, so the mean is off
  by 60 u relative (all terms have one sign) and 1 / sqrt by 30 u + 2 u; with the products by the gain and by it, v is off by
  40 u |v|, a scale by 44 u, and the quotient of both by 90 u; then one rounding to the result's type: half a step;
  8-bit products: every term is exact (4 bits times 4 bits); their sum in fp32, in whatever order and cut off instead of
  rounded at worst, by 2 K u sum |a b|, the scales by 3 u, then one rounding.
Samples are whole numbers and equal; a probability is one division, rounded to fp32.
"""
import numpy as np
import pytest
import torch

from oracle import rows
from paper_2609_37007_gb300 import mcd

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def np64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def dev(v, dtype):
    return torch.as_tensor(np.ascontiguousarray(v)).to(device=DEV, dtype=dtype)


def strided(n, w, dtype, pad, fill=0.0):
    """(whole buffer, its first w columns): rows at a stride of whole 16 bytes and `pad` more pieces of 16 bytes, one row behind."""
    size = torch.empty(0, dtype=dtype).element_size()
    per = 16 // size
    whole = torch.full((n + 1, (-(-w // per) + pad) * per), fill, device=DEV).to(dtype)
    return whole, whole[:n, :w]


def untouched(whole, part, fill):
    n, w = part.shape
    x = np64(whole)
    return (x[n:] == fill).all() and (x[:n, w:] == fill).all()


# ---- norm ------------------------------------------------------------------------------------
def check_norm(n, w, inp="bf16", res="f32", out="e4m3", gain=True, norm=True, pad=0, seed=0, scale=1.0, eps=1e-6, store=True):
    r = np.random.RandomState(seed)
    x = strided(n, w, TYPES[inp], pad)[1]
    x.copy_(dev(r.randn(n, w) * scale, torch.float32))
    residual = whole_sum = total = None
    if res:
        residual = strided(n, w, TYPES[res], pad)[1]
        residual.copy_(dev(3 * r.randn(n, w) * scale, torch.float32))
        if store:
            whole_sum, total = strided(n, w, TYPES[res], pad, 5.0)
    g = dev(1 + 0.1 * r.randn(w), torch.float32) if gain else None
    whole, y = strided(n, w, TYPES[out], pad, 5.0)
    s = torch.full((n + 1,), 5.0, device=DEV)
    mcd.mcd_norm_rows(x, y, residual=residual, sum_out=total, gain=g, eps=eps, norm=norm, y_scale=s[:n] if out == "e4m3" else None)
    torch.cuda.synchronize()
    want_sum, want = rows.norm_rows(np64(x), None if residual is None else np64(residual), None if g is None else np64(g), eps, norm)
    off = 0.0 if residual is None else U * np.abs(want_sum)
    if total is not None:
        assert (np.abs(np64(total) - want_sum) <= HALF[res] * np.abs(want_sum) + off).all()
        assert untouched(whole_sum, total, 5.0)
    got = np64(y)
    assert untouched(whole, y, 5.0)
    if out != "e4m3":
        assert (np.abs(got - want) <= HALF[out] * np.abs(want) + 40 * U * np.abs(want)).all()
        return
    scales = rows.row_scales(want)
    assert (np.abs(np64(s)[:n] - scales) <= 44 * U * scales).all() and s[n].item() == 5.0
    q = want / scales[:, None]
    assert (np.abs(got - q) <= np.maximum(2.0 ** -4 * np.abs(q), 2.0 ** -10) + 90 * U * np.abs(q)).all()
    assert (np.abs(got).max(1) == 448).all() or (want == 0).any()


@pytest.mark.parametrize("inp", ["f32", "bf16"])
@pytest.mark.parametrize("res", ["f32", "bf16", None])
@pytest.mark.parametrize("out", ["f32", "bf16", "e4m3"])
def test_norm_types(inp, res, out):
    check_norm(5, 1024, inp, res, out)
    check_norm(3, 1000, inp, res, out, gain=False, pad=1, seed=1)
    check_norm(3, 77, inp, res, out, norm=False, pad=2, seed=2)


@pytest.mark.parametrize("w", [1, 7, 8, 9, 255, 256, 257, 1016, 1025, 2048, 2049, 4095, 4097, 8192, 8193, 12345, 16383, 16384])
@pytest.mark.parametrize("out", ["bf16", "e4m3"])
def test_norm_widths(w, out):
    check_norm(3, w, out=out, seed=w)
    check_norm(6, w, "f32", "bf16", out, pad=1, seed=w + 1, store=False)


@pytest.mark.parametrize("n", [1, 2, 4, 5, 127, 1001])
def test_norm_rows_of_a_block(n):
    check_norm(n, 64, seed=n)
    check_norm(n, 512, "f32", None, "bf16", seed=n)


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e12, 1e17])
def test_norm_sizes(scale):
    check_norm(4, 640, "f32", "f32", "e4m3", scale=scale, norm=False)
    check_norm(4, 640, "f32", "f32", "f32", scale=scale, eps=0.0 if scale > 1e-20 else 1e-6)


def test_norm_tiny_rows_have_the_least_scale():
    x = torch.full((2, 64), 1e-40, device=DEV)
    x[1] = 0
    y, s = torch.zeros((2, 64), dtype=torch.float8_e4m3fn, device=DEV), torch.zeros(2, device=DEV)
    mcd.mcd_norm_rows(x, y, norm=False, y_scale=s)
    want = np.array([[np.float64(np.float32(1e-40)) * 2.0 ** 126], [0.0]]) * np.ones((1, 64))
    assert (np64(s) == 2.0 ** -126).all() and (np.abs(np64(y) - want) <= 2.0 ** -10).all()


def test_norm_a_row_that_is_not_finite_stays_alone():
    for bad in (float("nan"), float("inf"), -float("inf")):
        for norm in (True, False):
            x = torch.randn((5, 300), generator=torch.Generator(device=DEV).manual_seed(0), device=DEV)
            x = torch.nn.functional.pad(x, (0, 4))[:, :300]
            x[2, 17] = bad
            y, s = strided(5, 300, torch.float8_e4m3fn, 0)[1], torch.zeros(5, device=DEV)
            mcd.mcd_norm_rows(x, y, norm=norm, y_scale=s)
            with np.errstate(invalid="ignore"):
                back = np64(y) * np64(s)[:, None]
            assert not np.isfinite(back[2]).any() and np.isfinite(back[[0, 1, 3, 4]]).all()
            z = strided(5, 300, torch.float32, 0)[1]
            mcd.mcd_norm_rows(x, z, norm=norm)
            assert np.isfinite(np64(z)[[0, 1, 3, 4]]).all() and not np.isfinite(np64(z)[2, 17])
            assert not norm or not np.isfinite(np64(z)[2]).any()


def test_norm_in_place():
    g = torch.Generator(device=DEV).manual_seed(3)
    x, res = torch.randn((9, 1024), generator=g, device=DEV), torch.randn((9, 1024), generator=g, device=DEV)
    want_sum, want = rows.norm_rows(np64(x), np64(res))
    mcd.mcd_norm_rows(x, x, residual=res, sum_out=res)
    assert (np.abs(np64(res) - want_sum) <= U * np.abs(want_sum)).all() and (np.abs(np64(x) - want) <= 41 * U * np.abs(want)).all()


# ---- 8-bit products ----------------------------------------------------------------------------
def bytes8(r, n, k, pad=0, ints=None):
    whole, x = strided(n, k, torch.float8_e4m3fn, pad)
    whole.view(torch.uint8).fill_(0x7f)                     # NaN around the rows
    v = r.randint(-ints, ints + 1, (n, k)) if ints else r.randn(n, k) * 2
    x.copy_(dev(v, torch.float32).to(torch.float8_e4m3fn))
    return x


def check_gemm(m, n, k, out="f32", scales=True, pad=0, seed=0, ints=None):
    r = np.random.RandomState(seed)
    a, b = bytes8(r, m, k, pad, ints), bytes8(r, n, k, pad, ints)
    sa, sb = (dev(0.5 + r.rand(x), torch.float32) for x in (m, n)) if scales else (None, None)
    whole, y = strided(n, m, TYPES[out], pad, 5.0)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    mcd.mcd_tc_gemm_e4m3(a, b, y, err, a_scale=sa, b_scale=sb)
    torch.cuda.synchronize()
    assert err.item() == 0 and untouched(whole, y, 5.0)
    want, size = rows.gemm(np64(a), np64(b), None if sa is None else np64(sa), None if sb is None else np64(sb))
    got = np64(y)
    if ints and not scales:
        assert (got == want).all()
        return
    assert (np.abs(got - want) <= HALF[out] * np.abs(want) + (2 * k + 3) * U * size).all()


@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 1, 5000), (128, 1, 128), (129, 17, 129), (1024, 4, 1024), (200, 33, 300), (77, 128, 1000), (300, 129, 64),
                                   (256, 255, 640), (512, 257, 500), (130, 600, 1024), (1000, 1023, 200), (2048, 300, 17)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_gemm_sizes(m, n, k, out):
    check_gemm(m, n, k, out, seed=m + n + k)
    check_gemm(m, n, k, out, scales=False, pad=1, seed=m * n + k)


@pytest.mark.parametrize("m,n,k", [(128, 16, 128), (256, 40, 1024), (4096, 3, 1024), (384, 200, 2048), (640, 1000, 256), (1111, 333, 555), (2500, 2222, 1000)])
def test_gemm_exact_on_integers(m, n, k):
    check_gemm(m, n, k, scales=False, ints=8, seed=k)


def test_gemm_many_rows():
    check_gemm(1030, 8191, 272, "bf16", seed=5)
    check_gemm(6144, 700, 1024, "bf16", seed=6)


def test_gemm_a_value_that_is_not_a_number_stays_in_its_row():
    r = np.random.RandomState(1)
    a, b = bytes8(r, 256, 512), bytes8(r, 40, 512)
    b[7, 100] = float("nan")
    y, err = torch.zeros((40, 256), device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    mcd.mcd_tc_gemm_e4m3(a, b, y, err)
    got = np.isnan(np64(y))
    assert got[7].all() and not np.delete(got, 7, 0).any()


def test_gemm_gives_the_same_bits_every_time():
    r = np.random.RandomState(2)
    a, b, err = bytes8(r, 4096, 1024), bytes8(r, 4, 1024), torch.zeros(1, dtype=torch.int32, device=DEV)
    ys = [torch.zeros((4, 4096), device=DEV) for _ in range(5)]
    for y in ys:
        mcd.mcd_tc_gemm_e4m3(a, b, y, err)
    assert all(torch.equal(y, ys[0]) for y in ys)


# ---- sampling ------------------------------------------------------------------------------------
def check_sample(x, u, temperature=None, top_k=None, top_p=None, min_p=None, dtype="f32", pad=0):
    """x fp32 [rows, vocab] (rounded to the type first); settings per row."""
    n, v = x.shape
    logits = strided(n, v, TYPES[dtype], pad, 1e4)[1]
    logits.copy_(dev(x, torch.float32))
    settings = {"temperature": (temperature, torch.float32), "top_k": (top_k, torch.int32), "top_p": (top_p, torch.float32), "min_p": (min_p, torch.float32)}
    given = {k: dev(val, t) for k, (val, t) in settings.items() if val is not None}
    out = torch.full((3, n + 2), 7, dtype=torch.int32, device=DEV)
    probs, err = torch.full((n + 2,), 7.0, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    mcd.mcd_sample_rows(logits, dev(u, torch.float64), out[0, :n], err, probs=probs[:n], kept=out[1, :n], **given)
    mcd.mcd_sample_rows(logits, dev(u, torch.float64), out[2, :n], err, **given)
    torch.cuda.synchronize()
    rounded = logits.float().cpu().numpy()
    at = {k: given[k].cpu().numpy().tolist() for k in given}
    want = [rows.sample(rounded[i], float(u[i]), **{k: at[k][i] for k in at}) for i in range(n)]
    got = out.cpu().numpy()
    assert got[0, :n].tolist() == [w[0] for w in want] and got[1, :n].tolist() == [w[3] for w in want]
    assert (got[2] == got[0]).all() and (got[:, n:] == 7).all() and (probs[n:] == 7).all()
    assert np.array_equal(probs[:n].cpu().numpy(), np.array([w[1] / w[2] for w in want], np.float32))
    assert err.item() == (1 if any(w[0] < 0 for w in want) else 0)


def settings(r, n):
    pick = r.rand(4, n)
    return dict(temperature=np.where(pick[0] < 0.15, 0, r.choice([0.01, 0.3, 0.7, 1.0, 1.3, 20.0], n)), top_k=np.where(pick[1] < 0.4, r.choice([0, -3, 1 << 30], n), r.randint(1, 200, n)),
                top_p=np.where(pick[2] < 0.4, r.choice([1.0, 2.0], n), r.choice([0.0, -1.0, 1e-6, 0.1, 0.5, 0.9, 0.999, 1 - 2.0 ** -24], n)),
                min_p=np.where(pick[3] < 0.4, r.choice([0.0, -2.0], n), r.choice([1e-9, 1e-4, 0.05, 0.5, 1.0, 3.0], n)))


@pytest.mark.parametrize("v", [1, 2, 3, 8, 63, 500, 2048, 4099, 8192, 8193, 20001, 50000, 70001, 151000, 262144])
@pytest.mark.parametrize("dtype,spread", [("f32", 2.5), ("bf16", 0.4), ("bf16", 6.0), ("f32", 0.01)])
def test_sample_settings(v, dtype, spread):
    n = 40 if v <= 8193 else 10
    r = np.random.RandomState(v + int(10 * spread))
    check_sample((spread * r.randn(n, v)).astype(np.float32), r.rand(n), dtype=dtype, pad=v % 2, **settings(r, n))


@pytest.mark.parametrize("v", [5, 300, 3585, 9000, 40000])
def test_sample_ties(v):
    """Few values, many ids of each: cuts fall between equal logits, where the lowest ids stay."""
    r = np.random.RandomState(v)
    x = r.randint(0, 4, (24, v)).astype(np.float32) * np.float32(0.7)
    x[:4] = 1.5
    x[4:8] = np.where(r.rand(4, v) < 0.5, 0.0, -0.0)
    check_sample(x, r.rand(24), **settings(r, 24))


@pytest.mark.parametrize("v", [7, 2048, 30000])
def test_sample_hidden_ids(v):
    r = np.random.RandomState(v)
    x = (2 * r.randn(20, v)).astype(np.float32)
    x[r.rand(20, v) < 0.5] = -np.inf
    x[3] = -np.inf
    x[3, v - 2] = -5.0                                     # one id is left
    x[4, 1:] = -np.inf
    x[:, 0] = np.where(np.isinf(x[:, 0]), 0.1, x[:, 0])
    check_sample(x, r.rand(20), **settings(r, 20))


@pytest.mark.parametrize("v", [2048, 30000])
def test_sample_ends_of_u(v):
    r = np.random.RandomState(v)
    x = (2 * r.randn(6, v)).astype(np.float32)
    for u in (0.0, 2.0 ** -60, 0.5, 1 - 2.0 ** -53):
        check_sample(x, np.full(6, u))
        check_sample(x, np.full(6, u), top_k=np.full(6, 20), top_p=np.full(6, 0.8))


@pytest.mark.parametrize("v", [100, 30000])
def test_sample_rows_that_do_not_fit(v):
    """Each gives id -1 and an error, its neighbours what they give alone."""
    r = np.random.RandomState(v)
    x = (2 * r.randn(16, v)).astype(np.float32)
    u, t, p, m = r.rand(16), np.full(16, 0.8), np.full(16, 0.9), np.full(16, 0.01)
    x[1, v - 1], x[3, 5], x[5] = np.nan, np.inf, -np.inf
    u[7], u[8], u[9] = 1.0, -1e-9, np.nan
    t[10], t[11], t[12], p[13], m[14] = -1.0, np.nan, np.inf, np.nan, np.nan
    check_sample(x, u, temperature=t, top_p=p, min_p=m)


@pytest.mark.parametrize("v", [5000, 50000])
def test_sample_ids_without_weight_beside_the_cut(v):
    """200 ids of weight 1 (2^31 e^-21.484 = 1.0036) and thousands of weight 0 (e^-21.5) in one step of the histogram; top_p = 1 - 2^-24
    cuts between the 200."""
    r = np.random.RandomState(v)
    x = np.full((4, v), -21.5, np.float32)
    for i in range(4):
        x[i, r.permutation(v)[:201]] = -21.484
        x[i, r.randint(v)] = 0.0
    check_sample(x, np.array([0.2, 1 - 2.0 ** -40, 0.999999999, 0.5]), top_p=np.full(4, 1 - 2.0 ** -24))
    check_sample(x, np.array([0.2, 1 - 2.0 ** -40, 0.999999999, 0.5]), top_k=np.full(4, 150), top_p=np.full(4, 1 - 2.0 ** -24))


@pytest.mark.parametrize("n,v,dtype", [(233, 9001, "f32"), (515, 8193, "f32"), (58, 70001, "f32"), (90, 70001, "bf16"), (200, 20001, "bf16"), (60, 20001, "f32")])
def test_sample_more_rows_than_run_together(n, v, dtype):
    """Rows of several CTAs that wait for SMs are taken in an order by their settings, 256 at a time: each one once."""
    r = np.random.RandomState(n)
    given = settings(r, n)
    given["temperature"][:3] = 0.0
    check_sample((2.5 * r.randn(n, v)).astype(np.float32), r.rand(n), dtype=dtype, **given)
    check_sample((2.5 * r.randn(n, v)).astype(np.float32), r.rand(n), dtype=dtype, top_p=given["top_p"])


@pytest.mark.parametrize("v", [300, 2048, 8192, 8193, 16385, 40000, 140000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sample_min_p_beside_top_p(v, dtype):
    """min_p that leaves less than the cut, more, and as much, with sets from one id to all."""
    r = np.random.RandomState(v)
    n = 24
    p, m = np.repeat([0.05, 0.5, 0.9, 0.999], 6), np.tile([0.0, 1e-9, 1e-4, 0.02, 0.3, 1.0], 4)
    for spread, t in ((0.3, 1.0), (3.0, 0.9), (3.0, 8.0)):
        x = (spread * r.randn(n, v)).astype(np.float32)
        check_sample(x, r.rand(n), dtype=dtype, temperature=np.full(n, t), top_p=p, min_p=m)
        check_sample(x, r.rand(n), dtype=dtype, temperature=np.full(n, t), top_k=np.tile([129, 5000, 0], 8), top_p=p, min_p=m)


def test_sample_extreme_logits():
    """Temperatures and logits at the ends of fp32: a quotient that overflows means the first of the ranking."""
    x = np.array([[3e38, 1e38, -3e38, 3e38], [1e-40, 0, 2e-40, -1e-40], [-3e38, -3.1e38, -2.9e38, -np.inf], [5, 4, 3, 5]], np.float32)
    for t in (1e-30, 1e-3, 1.0, 1e30, 3e38):
        for k in (0, 2):
            check_sample(x, np.array([0.1, 0.6, 0.9, 0.99]), temperature=np.full(4, t), top_k=np.full(4, k), top_p=np.full(4, 0.95))


def test_sample_law_on_the_gpu():
    """20,000 rows of one distribution: ids as often as the filtered weights say (chi-square, 99.9 %)."""
    r = np.random.RandomState(11)
    x = np.tile((2 * r.randn(64)).astype(np.float32), (20000, 1))
    n = len(x)
    ids, err = torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    mcd.mcd_sample_rows(dev(x, torch.float32), torch.rand(n, dtype=torch.float64, generator=torch.Generator(device=DEV).manual_seed(5), device=DEV), ids, err,
                        temperature=dev(np.full(n, 0.9), torch.float32), top_k=dev(np.full(n, 12), torch.int32))
    order = np.lexsort((np.arange(64), -x[0]))[:12]
    p = np.zeros(64)
    p[order] = np.exp((x[0, order] - x[0].max()) / 0.9)
    p /= p.sum()
    got = np.bincount(ids.cpu().numpy(), minlength=64)
    assert got[p == 0].sum() == 0
    assert ((got[order] - n * p[order]) ** 2 / (n * p[order])).sum() <= 31.3      # 11 degrees of freedom


# ---- together, on streams and in graphs ------------------------------------------------------------
def test_rows_on_another_stream_and_replayed():
    """norm -> product -> sample, captured on a side stream; a replay with new inputs gives what the calls give."""
    g = torch.Generator(device=DEV).manual_seed(0)
    w, n, v = 512, 7, 1000
    x, y, s = torch.randn((n, w), generator=g, device=DEV), torch.zeros((n, w), dtype=torch.float8_e4m3fn, device=DEV), torch.zeros(n, device=DEV)
    head, hs = torch.zeros((v, w), dtype=torch.float8_e4m3fn, device=DEV), torch.zeros(v, device=DEV)
    mcd.mcd_norm_rows(torch.randn((v, w), generator=g, device=DEV), head, norm=False, y_scale=hs)
    z, u = torch.zeros((n, v), device=DEV), torch.rand(n, dtype=torch.float64, generator=g, device=DEV)
    ids, err = torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)

    def step(stream):
        mcd.mcd_norm_rows(x, y, y_scale=s, stream=stream)
        mcd.mcd_tc_gemm_e4m3(head, y, z, err, a_scale=hs, b_scale=s, stream=stream)
        mcd.mcd_sample_rows(z, u, ids, err, stream=stream)

    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    step(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(side)
    for seed in range(3):
        x.copy_(torch.randn((n, w), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV))
        ids.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want_z, size = rows.gemm(np64(head), np64(y), np64(hs), np64(s))
        assert (np.abs(np64(z) - want_z) <= 2.0 ** -24 * np.abs(want_z) + (2 * w + 3) * U * size).all()
        logits, uu = z.cpu().numpy(), u.cpu().numpy()
        assert ids.cpu().tolist() == [rows.sample(logits[i], float(uu[i]))[0] for i in range(n)]
    assert err.item() == 0
