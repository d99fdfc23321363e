"""Ends of the sampler's limits that test_gpu_sample does not reach: min_p at temperatures at which every weight is
near 1, where its cut lies at the lowest float or at the largest logit itself."""
import numpy as np
import pytest

from test_gpu_sample import check, draw, eng, rows_of  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("V", [48, 5000])
def test_min_p_keeps_the_lowest_floats_where_their_weight_suffices(eng, V):  # noqa: F811
    """At temperature 1e38 the lowest float weighs e^-3.4 = 0.033."""
    n, rng = 32, np.random.default_rng(V)
    z = rng.standard_normal((n, V))
    z[:, rng.random(V) < 0.8] = float(torch.finfo(torch.float32).min)
    lim = dict(temperature=np.full(n, 1e38, np.float32), min_p=np.resize([1e-30, 1e-4, 0.03, 0.04], n).astype(np.float32))
    check(eng, rows_of(z, torch.float32), rng.random(n, np.float32), **lim)


@pytest.mark.parametrize("V", [48, 5000])
def test_min_p_of_one_keeps_the_largest_logits_alone(eng, V):  # noqa: F811
    """A weight is 1 at the largest logit only, however near 1 the others' round at a high temperature."""
    n, rng = 32, np.random.default_rng(V)
    z = np.float32(1) - rng.integers(1, 60, (n, V)).astype(np.float32) * np.float32(2.0 ** -24)
    top = rng.integers(0, V, n)
    z[np.arange(n), top] = 1
    got, lp = draw(eng, rows_of(z, torch.float32), rng.random(n, np.float32),
                   temperature=np.full(n, 1e30, np.float32), min_p=np.resize([1.0, 7.0], n).astype(np.float32))
    assert (got == top).all() and (lp == 0).all()
