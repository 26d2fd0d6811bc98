"""The tolerances of the paged cache's GPU tests tell the precisions apart that they are there for (no GPU: mistakes
planted in the oracle)."""
import numpy as np
import pytest
import torch

from oracle import paged
from test_gpu_cache_edges import tolerance


def rounded(x):
    return torch.as_tensor(x).to(torch.bfloat16).double().numpy()


@pytest.mark.parametrize("terms,p_bits,passes", [(1, 8, True), (1, 16, False), (2, 16, True)])
def test_probabilities_of_one_or_two_bf16(terms, p_bits, passes):
    """Attention of 3 rows whose probabilities are one bf16, or a hi + lo pair, against the oracle."""
    r, n, d, keys = np.random.RandomState(0), 3, 128, 303
    q, k, v = (rounded(r.randn(*shape)) for shape in ((n, 2, d), (keys, 1, d), (keys, 1, d)))
    ref, spread, reach = paged.attention(1.5 * q, k, v, keys - n, d ** -0.5)
    got = np.zeros_like(ref)
    for i in range(n):
        see = keys - n + i + 1
        z = 1.5 * q[i] @ k[:see, 0].T * d ** -0.5
        p = np.exp(z - z.max(-1, keepdims=True))
        hi = rounded(p)
        lo = rounded(p - hi) if terms == 2 else 0.0
        got[i] = (hi + lo) @ v[:see, 0] / p.sum(-1, keepdims=True)
    assert (np.abs(rounded(got) - ref) <= tolerance(ref, spread, reach, keys, d, p_bits)).all() == passes
