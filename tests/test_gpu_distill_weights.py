"""Weights at the ends of fp32's range in the distillation loss: the gradient holds only their shares of the sum, which
are ordinary numbers.  Tolerances as in test_gpu_distill."""
import math

import numpy as np
import pytest

from op_util import distill_ref
from test_gpu_distill import H, check, dev, eng, make  # noqa: F401

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
    """W is returned as inf where it is, but the loss and the gradient are those of the sum in 64 bits."""
    for n in (8, 1500):
        rows, ids, logp, tail, w = make(n, 90, torch.float32, 22)
        w = (w * np.float32(3e38)).astype(np.float32)
        z = rows.double().cpu().numpy()
        loss, W, row, grad = distill_ref(z, ids, logp, tail, w, 1.013441, 0.75)
        got = eng.distill_loss(rows, *dev(ids, logp, tail, w), scale=1.013441,
                               grad_out=torch.tensor([0.75], device="cuda"))
        torch.cuda.synchronize()
        # 0.52 * 3e38 = 1.6e38 for the eight rows (their first three have weight 0), 181 * 3e38 for the others
        assert np.isinf(float(got[0][1])) == (n > 8)
        E, size = (math.ceil(90 / 64) + 64) * H, np.abs(z - z.max(1)[:, None]).max(1) + math.log(90) + 1
        tol = 2 * E * 1.1 + 4 * H * (size + np.abs(row))
        assert abs(float(got[0][0]) - loss) <= 1.013441 * tol.max() + 2 * H * abs(loss)
        # the sizes of a gradient's terms, in 64 bits: a share of W is no fp32 quotient here
        q = np.exp(z - z.max(1)[:, None])
        outside = np.ones_like(q)
        np.put_along_axis(outside, ids, 0, 1)
        tails = q * outside / (q * outside).sum(1, keepdims=True)
        q /= q.sum(1, keepdims=True)
        pi = np.exp(logp.astype(np.float64))
        terms = (pi.sum(1) + tail)[:, None] * q + tail[:, None] * tails
        np.put_along_axis(terms, ids, np.take_along_axis(terms, ids, 1) + pi, 1)
        terms *= 0.75 * 1.013441 * (w.astype(np.float64) / W)[:, None]
        err = np.abs(got[2].double().cpu().numpy() - grad)
        assert (err <= (2 * E + 8 * H + 6 * H * size[:, None]) * terms + H * np.abs(grad) + 1e-37).all()
        assert bool((got[2] != 0).any())


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
