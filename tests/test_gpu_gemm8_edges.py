"""mcd_tc_gemm_e4m3 with scales at the ends of fp32: the result goes by the formula, whichever kernel the sizes choose."""
import numpy as np
import pytest
import torch

from oracle import rows
from paper_2609_37007_gb300 import mcd
from test_gpu_rows import TYPES, bytes8, dev, np64, strided

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", [(1024, 4, 1024), (4096, 1, 512), (256, 40, 2048), (200, 300, 640), (2500, 2222, 128)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_scales_whose_product_leaves_the_range(m, n, k, out):
    """Whole numbers and powers of two, so that every step is exact: the scales' product is infinite beside sums of 0, or 0 beside
    sums that bring the result back into fp32's range (sums are multiples of 2^8, results of 2^-144)."""
    r = np.random.RandomState(k)
    a, b = ((16 * bytes8(r, x, k, ints=2).float()).to(torch.float8_e4m3fn) for x in (m, n))
    b[0] = 0
    b[:, 8:] = 0
    sums = rows.gemm(np64(a), np64(b))[0]
    assert (sums == 0).any() and (n == 1 or (sums != 0).any())
    for power in (66, -76):
        sa, sb = (dev(np.full(x, 2.0 ** power), torch.float32) for x in (m, n))
        y, err = strided(n, m, TYPES[out], 0, 5.0)[1], torch.zeros(1, dtype=torch.int32, device="cuda")
        mcd.mcd_tc_gemm_e4m3(a, b, y, err, a_scale=sa, b_scale=sb)
        with np.errstate(invalid="ignore"):
            want = np.where(sums == 0, 0.0, np.sign(sums) * np.inf) if power > 0 else sums * 2.0 ** (2 * power)
        if out == "bf16" and power < 0:
            want = np.zeros_like(sums)                       # (below half of its least step, 2^-133)
        assert err.item() == 0 and np.array_equal(np64(y), want)


@pytest.mark.parametrize("n", [1, 4, 16, 64, 65])
def test_many_rows_of_a_for_few_of_b(n):
    """More tiles of A than SMs, few rows of B: either side of the rule that chooses the kernel."""
    m, k = 20000, 272
    r = np.random.RandomState(n)
    a, b = bytes8(r, m, k, ints=8), bytes8(r, n, k, ints=8)
    for out in ("f32", "bf16"):
        whole, y = strided(n, m, TYPES[out], 1, 5.0)
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        mcd.mcd_tc_gemm_e4m3(a, b, y, err)
        want = dev(rows.gemm(np64(a), np64(b))[0], torch.float32).to(TYPES[out])
        assert err.item() == 0 and torch.equal(y, want) and (np64(whole)[n:] == 5.0).all()
