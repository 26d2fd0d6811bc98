"""mcd_sample_rows at the ends of its settings against oracle/rows.py, whole numbers throughout: temperatures whose multiples leave
fp32's range, up or down, beside many hidden ids or many ids without weight."""
import numpy as np
import pytest

from test_gpu_rows import check_sample

pytestmark = pytest.mark.gpu


def rows_of_few(r, v, finite, lo, hi, rest):
    """Eight rows of `finite` logits from lo to hi, the others `rest`."""
    x = np.full((8, v), rest, np.float32)
    for i in range(8):
        x[i, r.permutation(v)[:finite]] = r.uniform(lo, hi, finite).astype(np.float32)
    return x


@pytest.mark.parametrize("v", [5000, 8192, 20001, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t", [1e37, 1.6e37, 2e37, 1e38, 3e38])
def test_large_temperatures_beside_hidden_ids(v, dtype, t):
    """22 T above fp32's range: all finite ids lie in the histogram's first step, hidden ones in none."""
    r = np.random.RandomState(v)
    given = dict(temperature=np.full(8, t), dtype=dtype)
    for finite in (1, 100, 3300, v - 1):
        x = rows_of_few(r, v, finite, 0.0, 1.0, -np.inf)
        check_sample(x, r.rand(8), top_p=np.full(8, 0.9), **given)
        check_sample(x, r.rand(8), top_k=np.tile([50, 129, 500, 4000], 2), **given)
        check_sample(x, r.rand(8), top_k=np.tile([50, 129, 500, 4000], 2), top_p=np.full(8, 0.7), min_p=np.repeat([0.5, 1.0], 4), **given)
    # logits as far apart as fp32 has them
    x = rows_of_few(r, v, v // 2, -3.3e38, 3.3e38, -np.inf)
    check_sample(x, r.rand(8), top_p=np.repeat([0.3, 0.999], 4), min_p=np.tile([0.0, 1e-6, 0.2, 0.9], 2), **given)
    check_sample(x, r.rand(8), top_k=np.tile([129, 3000], 4), **given)


@pytest.mark.parametrize("v", [5000, 8192, 40000])
@pytest.mark.parametrize("t", [1e-36, 3e-38, 1e-40, 1e-43])
def test_tiny_temperatures_beside_ids_without_weight(v, t):
    """255 / (22 T) above fp32's range: one step of the histogram holds ids with weight and thousands without."""
    r = np.random.RandomState(v)
    given = dict(temperature=np.full(8, t))
    step = np.float32(t)
    for finite in (2, 100, v // 2):
        x = rows_of_few(r, v, finite, -3 * step, 4 * step, -600 * step)      # (e^-600: no weight)
        check_sample(x, r.rand(8), top_p=np.repeat([0.4, 0.95], 4), **given)
        check_sample(x, r.rand(8), top_k=np.tile([20, 129, 500, 4000], 2), top_p=np.tile([1.0, 0.8], 4), **given)
        check_sample(x, r.rand(8), top_p=np.full(8, 0.9), min_p=np.tile([0.0, 1e-3, 0.3, 1.0], 2), **given)
