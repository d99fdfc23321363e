"""The operators on the caller's tensors without a GPU: null contexts, and the oracle's q/k norms."""
import dataclasses

import numpy as np
import pytest

import oracle as O
from op_util import sample_ref
from oracle import reference as R
from paper_2609_38795_amd import binding, workloads as W


def test_null_context_is_refused():
    import os

    if not os.path.exists(binding.LIB_PATH):
        from paper_2609_38795_amd import build
        build.build()
    lib = binding.load_library()
    assert lib.alr_sample(None, 1, 1, None, 0, 1, None, None, None, None, None) == 1
    assert lib.alr_rollout_sampled(None, 1, None, None, 1, None, *([None] * 10)) == 1
    assert lib.alr_distill_loss(None, 1, 1, None, 0, 1, None, None, None, None, 1.0, None, None, None, None, 1,
                                None) == 1
    assert lib.alr_qk_norm_rope(None, 1, 1, 1, None, None, 1, None, 1, None, None, None, 1, None, 1, None) == 1
    assert lib.alr_qk_norm_rope_backward(None, 1, 1, 1, None, None, 1, None, 1, None, None, None, 1, None, 1, None,
                                         1, None, 1, None, None, None) == 1
    assert lib.alr_set_qk_norm(None, None, None, None) == 1


def _normed(gain=None):
    w = W.get("tiny_fp32")
    shape = dataclasses.replace(w.shape, n_layers=2, vocab=64, d_ffn=64)
    wt = W.random_weights(shape, 3, scale=0.1, norm_gain="random")
    if gain is not None:
        for ld in wt["layers"]:
            ld["q_norm"] = gain[0]
            ld["k_norm"] = gain[1]
    return shape, wt


def test_oracle_head_norm_by_hand():
    class P:
        w = {"layers": [{"q_norm": np.array([2.0, 1.0], np.float32)}]}

        @staticmethod
        def get(name, layer):
            return P.w["layers"][layer][name].astype(np.float64)

    x = np.array([[[3.0, 4.0], [0.0, 1.0]]])
    y = R.head_norm(P, "q_norm", 0, x, 0.0, lambda v: v)
    # mean squares 12.5 and 0.5
    np.testing.assert_allclose(y, [[[6 / 12.5 ** 0.5, 4 / 12.5 ** 0.5], [0.0, 1 / 0.5 ** 0.5]]], rtol=1e-15)
    assert R.head_norm(P, "k_norm", 0, x, 0.0, None) is x  # no such gains: nothing changes


def test_oracle_forms_agree_with_head_norms():
    rng = np.random.default_rng(0)
    shape, wt = _normed((1 + 0.3 * rng.standard_normal((2, 32))).astype(np.float32))
    P = O.Params(wt)
    toks = rng.integers(0, 64, (1, 12))
    a_s, a_p = np.array([0, 0]), np.array([3, 9])
    naive = O.rollout_naive(P, shape, toks, a_s, a_p, 3)
    shared = O.rollout_kv_shared(P, shape, toks, a_s, a_p, 3)
    np.testing.assert_allclose(naive[1], shared[1], atol=1e-11)
    plain = O.rollout_naive(O.Params(_normed()[1]), shape, toks, a_s, a_p, 3)
    assert np.abs(naive[1] - plain[1]).max() > 1e-3
    # scores of normed heads do not depend on the scale of the projections
    for ld in wt["layers"]:
        ld["wq"] = ld["wq"] * np.float32(1024)
        ld["wk"] = ld["wk"] * np.float32(512)
    scaled = O.rollout_naive(O.Params(wt), dataclasses.replace(shape, rms_eps=0.0), toks, a_s, a_p, 3)
    again = O.rollout_naive(P, dataclasses.replace(shape, rms_eps=0.0), toks, a_s, a_p, 3)
    np.testing.assert_allclose(scaled[1], again[1], atol=1e-9)


@pytest.mark.parametrize("u,kw,tok", [
    (0.0, {}, 0), (0.24, {}, 0), (0.26, {}, 1), (0.99, {}, 2), (0.5, dict(temperature=0.0), 1),
    (0.0, dict(top_k=1), 1), (0.1, dict(top_k=2), 0), (0.34, dict(top_k=2), 1), (0.9, dict(top_p=0.5), 1),
    (0.0, dict(top_p=0.51), 0), (0.9, dict(min_p=0.6), 1), (0.2, dict(min_p=0.4), 0)])
def test_sampling_reference_by_hand(u, kw, tok):
    """Probabilities 1/4, 1/2, 1/4 (the first and the last tie, the first ranks before it)."""
    assert sample_ref(np.log([1.0, 2.0, 1.0]), u, **kw)[0] == tok
