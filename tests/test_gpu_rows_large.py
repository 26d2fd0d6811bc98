"""The rows' operators on arrays of more than 2^31 elements: the last rows are right, as the first are."""
import numpy as np
import pytest
import torch

from oracle import rows
from paper_2609_37007_gb300 import mcd
from test_gpu_rows import DEV, HALF, U, np64

pytestmark = pytest.mark.gpu
BF16, F8 = torch.bfloat16, torch.float8_e4m3fn


def noise(n, w, dtype, seed):
    """n x w values, made of one block so that making them is quick, with first and last rows of their own."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.empty((n, w), dtype=dtype, device=DEV)
    block = torch.randn((1000, w), generator=g, device=DEV).to(dtype)
    for lo in range(0, n, 1000):
        x[lo:lo + 1000] = block[:min(1000, n - lo)]
    x[:2], x[-2:] = (torch.randn((2, w), generator=g, device=DEV).to(dtype) for _ in range(2))
    return x


def ends(t):
    return np64(torch.cat([t[:2].float(), t[-2:].float()]))


def test_norm():
    n, w = 140001, 16384
    x, y, s = noise(n, w, BF16, 0), torch.zeros((n, w), dtype=F8, device=DEV), torch.zeros(n, device=DEV)
    assert n * w > 2 ** 31
    mcd.mcd_norm_rows(x, y, residual=x, sum_out=x, y_scale=s)
    half = ends(x)                                           # 2 x, exact
    want = rows.norm_rows(half)[1]
    scale = np64(torch.cat([s[:2], s[-2:]]))
    q = want / scale[:, None]
    assert (np.abs(scale - rows.row_scales(want)) <= 44 * U * scale).all()
    assert (np.abs(ends(y) - q) <= np.maximum(2.0 ** -4 * np.abs(q), 2.0 ** -10) + 90 * U * np.abs(q)).all()


@pytest.mark.parametrize("m,n", [(16384, 140001), (140001, 16384)])
def test_gemm(m, n):
    k = 48
    a, b = noise(m, k, BF16, 1).to(F8), noise(n, k, BF16, 2).to(F8)
    ld = -(-m // 8) * 8
    y, err = torch.zeros((n, ld), dtype=BF16, device=DEV)[:, :m], torch.zeros(1, dtype=torch.int32, device=DEV)
    mcd.mcd_tc_gemm_e4m3(a, b, y, err)
    want, size = rows.gemm(np64(a), ends(b))
    assert err.item() == 0 and (np.abs(ends(y) - want) <= HALF["bf16"] * np.abs(want) + (2 * k + 3) * U * size).all()


def test_sample():
    n, v = 8300, 262144
    x = noise(n, v, BF16, 3)
    u = torch.rand(n, dtype=torch.float64, generator=torch.Generator(device=DEV).manual_seed(4), device=DEV)
    ids, err, p = torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV), torch.full((n,), 0.9, device=DEV)
    mcd.mcd_sample_rows(x, u, ids, err, top_p=p)
    got, uu, z = ids.cpu().tolist(), u.cpu().tolist(), ends(x).astype(np.float32)
    assert err.item() == 0
    for i, r in enumerate((0, 1, n - 2, n - 1)):
        assert got[r] == rows.sample(z[i], uu[r], top_p=float(np.float32(0.9)))[0]
