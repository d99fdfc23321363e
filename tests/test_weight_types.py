"""Weights handed to a context whose dtype they are not of: the library copies head_dim (and so on) values of the
context's dtype from the addresses it is given, so a narrower array would be read past its end.  No GPU: the
library is a stand-in that takes down what it is called with."""
import dataclasses

import numpy as np
import pytest

from paper_2609_38795_amd import binding, workloads as W

torch = pytest.importorskip("torch")


class Library:
    def __init__(self):
        self.calls = []

    def alr_set_qk_norm(self, *args):
        self.calls.append(args)
        return 0


class Stream:
    cuda_stream = 0

    def synchronize(self):
        pass


def context(dtype):
    eng = binding.Engine.__new__(binding.Engine)
    eng.torch, eng.lib, eng.ctx, eng.stream, eng.device = torch, Library(), None, Stream(), torch.device("cpu")
    eng.shape = dataclasses.replace(W.get("tiny_fp32").shape, n_layers=2, dtype=dtype)
    return eng


def gains(eng, kind):
    hd = eng.shape.head_dim
    return [np.ones(hd, kind) for _ in range(eng.shape.n_layers)]


@pytest.mark.parametrize("dtype,kind", [("bf16", np.float32), ("bf16", np.float64), ("bf16", np.int16),
                                        ("f32", np.uint16)])
def test_gains_of_another_type_are_refused(dtype, kind):
    eng = context(dtype)
    right = gains(eng, np.uint16 if dtype == "bf16" else np.float32)
    for q, k in ((gains(eng, kind), right), (right, gains(eng, kind)), (right, right[:1] + gains(eng, kind)[:1])):
        with pytest.raises(ValueError, match="dtype"):
            eng.set_qk_norm(q, k)
    assert not eng.lib.calls


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_so_are_other_weights(dtype):
    eng = context(dtype)
    wrong = np.zeros((64, 64), np.float32 if dtype == "bf16" else np.uint16)
    with pytest.raises(ValueError, match="dtype"):
        eng._upload_weights({"tok_embed": wrong, "lm_head": wrong, "final_norm": wrong[0], "layers": []})


@pytest.mark.parametrize("dtype,kind", [("bf16", np.uint16), ("f32", np.float32), ("f32", np.float64),
                                        ("f32", np.float16)])
def test_gains_of_the_contexts_type_are_taken(dtype, kind):
    eng = context(dtype)
    eng.set_qk_norm(gains(eng, kind), gains(eng, kind))
    assert len(eng.lib.calls) == 1


@pytest.mark.parametrize("case", ["no k", "no q", "one layer's missing", "fewer layers", "another length"])
def test_incomplete_gains_are_refused(case):
    eng = context("f32")
    g = gains(eng, np.float32)
    q, k = {"no k": (g, None), "no q": (None, g), "one layer's missing": (g, [g[0], None]),
            "fewer layers": (g[:1], g), "another length": (g, [g[0], g[1][:-1]])}[case]
    with pytest.raises(ValueError, match="gains"):
        eng.set_qk_norm(q, k)
    assert not eng.lib.calls
