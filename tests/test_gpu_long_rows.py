"""The operators at the ends of their index ranges: vocabularies of which a place no longer fits 32 bits are
refused, and rows whose offsets do not fit 32 bits are found."""
import numpy as np
import pytest

from op_util import distill_ref, engine, qk_ref, sample_ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

STRIDE = 2 ** 30 + 8  # elements: the third row starts beyond 2^31 of them, 2^32 bytes in bf16


@pytest.fixture(scope="module")
def eng():
    e = engine("bf16", 32, 32, 64, 64)
    yield e
    e.close()


@pytest.mark.parametrize("vocab", [2147483633, 2147483647])
def test_vocabularies_beyond_the_largest_are_refused(eng, vocab):
    z = torch.zeros(64, device="cuda")
    ids = torch.full((1, 8), -1, dtype=torch.int32, device="cuda")
    a = z.data_ptr()
    st = eng.lib.alr_distill_loss(eng.ctx, 1, vocab, a, 0, 2 ** 31, ids.data_ptr(), a, a, None, 1.0, None, a, a, None,
                                  1, eng._sp())
    assert st == 5 and b"vocab" in eng.lib.alr_last_error(eng.ctx)


def test_rows_beyond_32_bit_offsets(eng):
    n, V, rng = 3, 1001, np.random.default_rng(1)
    buf = torch.empty((n - 1) * STRIDE + 2048, dtype=torch.bfloat16, device="cuda")
    rows = buf.as_strided((n, V), (STRIDE, 1))
    rows.copy_(torch.from_numpy(rng.standard_normal((n, V)).astype(np.float32) * 2))
    z = rows.double().cpu().numpy()
    u = rng.random(n, np.float32)
    p = np.array([0.9, 0.5, 1.0], np.float32)
    tok, _ = eng.sample(rows, torch.from_numpy(u).cuda(), top_p=torch.from_numpy(p).cuda())
    assert tok.tolist() == [sample_ref(z[r], u[r], top_p=p[r])[0] for r in range(n)]
    ids = np.argsort(-z, axis=1)[:, :8].astype(np.int32)
    logp = (np.take_along_axis(z, ids, 1) - np.log(np.exp(z).sum(1))[:, None]).astype(np.float32) - np.float32(0.5)
    tail = (1 - np.exp(logp.astype(np.float64)).sum(1)).astype(np.float32)
    loss, _, row, grad = distill_ref(z, ids, logp, tail, np.ones(n, np.float32), 1.0)
    got = eng.distill_loss(rows, *(torch.from_numpy(t).cuda() for t in (ids, logp, tail)),
                           out=(torch.empty(2, device="cuda"), torch.empty(n, device="cuda"), rows))
    torch.cuda.synchronize()
    # losses below 10 of sums of 16 terms a lane and a tree: 2^-18 is 64 half steps of 1; the gradient to half a bf16 step
    assert np.abs(got[1].double().cpu().numpy() - row).max() <= 10 * 2.0 ** -18
    assert (np.abs(got[2].double().cpu().numpy() - grad) <= 2.0 ** -8 * np.abs(grad) + 2.0 ** -18).all()
    x = buf.as_strided((n, 128), (STRIDE, 1))
    x.copy_(torch.from_numpy(rng.standard_normal((n, 128)).astype(np.float32)))
    g = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda")[:, None].expand(n, 3).contiguous()
    ref = qk_ref(x.double().cpu().numpy().reshape(n, 2, 64), np.ones(64), pos.cpu().numpy(), (0, 0, 0))
    eng.qk_norm_rope(x, None, g, None, positions=pos, out=(x, None))
    torch.cuda.synchronize()
    y = x.double().cpu().numpy().reshape(n, 2, 64)
    # values below 8 of both halves: 26 half steps of 16 at most (as in test_gpu_qk_norm), and half a bf16 step
    assert (np.abs(y - ref) <= 26 * 2.0 ** -24 * 16 + 2.0 ** -8 * np.abs(ref)).all()
