"""Weights at the ends of fp32's range in the distillation loss: the gradient holds only their shares of the sum, which
are ordinary numbers.  Tolerances as in test_gpu_distill."""
import numpy as np
import pytest

from test_gpu_distill import check, dev, eng, make  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("n", [6, 1500])
def test_weights_whose_sum_is_below_the_normal_numbers(eng, n):  # noqa: F811
    """1e-41 and its like: erase gates are products of probabilities.  scale / W alone is beyond fp32."""
    rows, ids, logp, tail, w = make(n, 90, torch.float32, 21)
    w = (w * np.float32(1e-40) / n).astype(np.float32)
    w[:2] = np.float32(1e-44), np.float32(3e-42)
    got = check(eng, rows, ids, logp, tail, w)
    assert bool(torch.isfinite(got[2]).all()) and bool((got[2][1] != 0).any())
