"""mcd_norm_rows where r * gain leaves fp32's range and v does not; tolerances as derived in tests/test_gpu_rows.py."""
import numpy as np
import pytest
import torch

from oracle import rows
from paper_2609_37007_gb300 import mcd
from test_gpu_rows import HALF, TYPES, U, dev, np64, strided

pytestmark = pytest.mark.gpu


def check(x, gain, out, eps, res=False):
    n, w = x.shape
    xs = strided(n, w, torch.float32, 0)[1]
    xs.copy_(dev(x, torch.float32))
    g, s, y = dev(gain, torch.float32), torch.zeros(n, device="cuda"), strided(n, w, TYPES[out], 0)[1]
    half = strided(n, w, torch.float32, 0)[1]
    half.copy_(xs * 0.5)                                     # (exact: r = x again)
    if res:
        mcd.mcd_norm_rows(half, y, residual=half, gain=g, eps=eps, y_scale=s if out == "e4m3" else None)
    else:
        mcd.mcd_norm_rows(xs, y, gain=g, eps=eps, y_scale=s if out == "e4m3" else None)
    torch.cuda.synchronize()
    want = rows.norm_rows(np64(xs), None, np64(g), eps)[1]
    got = np64(y)
    if out != "e4m3":
        assert (np.abs(got - want) <= HALF[out] * np.abs(want) + 40 * U * np.abs(want)).all()
        return
    scales = rows.row_scales(want)
    assert (np.abs(np64(s) - scales) <= 44 * U * scales).all()
    q = want / scales[:, None]
    assert (np.abs(got - q) <= np.maximum(2.0 ** -4 * np.abs(q), 2.0 ** -10) + 90 * U * np.abs(q)).all()
    assert (np.abs(got).max(1) == 448).all()


@pytest.mark.parametrize("out", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("w", [1, 64, 300, 1000, 2000, 4096, 8000, 16384])
def test_gain_times_row_out_of_range(out, w):
    r = np.random.RandomState(w)
    x = np.where(r.rand(5, w) < 0.5, -1, 1) * (0.1 + r.rand(5, w))      # (r / rms well within fp32's normal range)
    gain = np.where(r.rand(w) < 0.5, -1, 1) * (0.5 + r.rand(w))
    check(x * 1e16, gain * 1e25, out, 1e-6)                  # 1e41; the row's squares sum to 1e36 at most
    check(x * 1e16, gain * 1e25, out, 1e-6, res=True)
    check(x * 1e-15, gain * 1e-28, out, 0.0)                 # 1e-43
    check(x * 1e-10, gain * 1e-32, out, 0.0)
    mixed = x * 10.0 ** r.randint(-14, 16, (5, 1))           # rows of every size, one gain
    check(mixed, gain * 1e24, out, 0.0)
    check(mixed, gain * 1e-25, out, 0.0)


@pytest.mark.parametrize("out", ["f32", "bf16", "e4m3"])
def test_gains_far_apart(out):
    r = np.random.RandomState(2)
    x = np.where(r.rand(4, 500) < 0.5, -1, 1) * (0.1 + r.rand(4, 500))
    gain = 10.0 ** r.randint(-30, 31, 500)
    for size in (1e15, 1.0, 1e-12):
        check(x * size, gain, out, 0.0)


def test_one_value():
    for out in ("f32", "bf16", "e4m3"):
        check(np.array([[1e19]]), np.array([1e20]), out, 1e-6)
        check(np.array([[-2e-18]]), np.array([3e-30]), out, 0.0)
