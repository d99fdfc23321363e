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


def test_weights_whose_sum_is_beyond_fp32(eng):  # noqa: F811
    """W is returned as inf where it is, but the loss and the gradient are those of the sum in 64 bits, at any number of rows."""
    for n in (8, 1500):
        rows, ids, logp, tail, w = make(n, 90, torch.float32, 22)
        with np.errstate(over="ignore"):
            got = check(eng, rows, ids, logp, tail, (w * np.float32(3e38)).astype(np.float32))
        # 0.52 * 3e38 = 1.6e38 for the eight rows (their first three have weight 0), 181 * 3e38 for the others
        assert np.isinf(float(got[0][1])) == (n > 8) and bool((got[2] != 0).any())


@pytest.mark.parametrize("V", [90, 700])
def test_the_sum_of_weights_is_not_rounded_at_any_number_of_rows(eng, V):  # noqa: F811
    """Rows of weight 0 behind the others leave their gradients as they are, bit for bit, wherever the sum is formed.
    The weights are such that 1.5 / W and 1.5 / fp32(W) differ in fp32."""
    rows, ids, logp, tail, _ = make(1030, V, torch.float32, 23)
    tried = 0
    for seed in range(40):
        w = np.random.default_rng(seed).random(1030).astype(np.float32)
        w[1024:] = 0
        W = float(np.sum(w.astype(np.float64)))
        if np.float32(1.5 / W) == np.float32(1.5 / float(np.float32(W))):
            continue
        tried += 1
        few = eng.distill_loss(rows[:1024], *dev(ids[:1024], logp[:1024], tail[:1024], w[:1024]), scale=1.5)
        many = eng.distill_loss(rows, *dev(ids, logp, tail, w), scale=1.5)
        torch.cuda.synchronize()
        assert torch.equal(few[1], many[1][:1024]) and torch.equal(few[0], many[0])
        assert torch.equal(few[2], many[2][:1024]) and not bool(many[2][1024:].any())
    assert tried >= 5
