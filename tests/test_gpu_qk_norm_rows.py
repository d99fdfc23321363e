"""The q/k norms' gradients where a workgroup's lanes or its loop over the rows run past the heads or come round:
eps = 0 with head counts that leave lanes without a head, and more rows than the grid has waves.

Tolerances as in test_gpu_qk_norm, but for the gains' sums.  The grid has at most 4096 waves, so a lane adds up at most
(ceil(n / 4096) + 1) * heads terms in turn, whether a wave takes whole rows, parts of rows or single heads; then
come at most 5 levels over the lanes, 4 waves, 16 partial sums of workgroups in turn and 6 levels: 32.
"""
import numpy as np
import pytest

import op_util
from op_util import engine, qk_back_ref, qk_ref
from test_gpu_qk_norm import DT, H_, close, f64, make, sections

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def check(n, H, G, hd, dtype, offset, mrope, seed):
    sec, max_pos = sections(hd, mrope), 4097
    eng = engine(dtype, 32, 32, hd, max_pos, sec)
    q, k, gq, gk, pos, rng = make(n, H, G, hd, dtype, seed, max_pos, 0, offset)
    p = torch.from_numpy(pos).cuda()
    dq, dk = (torch.from_numpy(rng.standard_normal(tuple(t.shape)).astype(np.float32)).to(DT[dtype]).cuda()
              for t in (q, k))
    fwd = eng.qk_norm_rope(q, k, gq, gk, positions=p)
    back = eng.qk_norm_rope_backward(q, k, gq, gk, dq, dk, positions=p)
    torch.cuda.synchronize()
    half, step = hd // 2, torch.finfo(DT[dtype]).eps / 2
    for x, g, y, dy, dx, dg in ((q, gq, fwd[0], dq, back[0], back[2]), (k, gk, fwd[1], dk, back[1], back[3])):
        x, dy, g = f64(x, n, hd), f64(dy, n, hd), g.double().cpu().numpy()
        ref = qk_ref(x, g, pos, sec)
        r = 1 / np.sqrt(np.mean(x * x, 2, keepdims=True) + op_util.EPS)
        a, ad = np.abs(x * r * g), np.abs(dy)
        close(f64(y, n, hd), ref, 26 * H_ * np.tile(a[..., :half] + a[..., half:], 2) + step * np.abs(ref) + 1e-30)
        rx, rg, _ = qk_back_ref(x, g, pos, sec, dy)
        d = np.tile(ad[..., :half] + ad[..., half:], 2)
        t = r * (np.abs(g) * d + np.abs(x * r) * np.mean(np.abs(g) * d * np.abs(x * r), 2, keepdims=True))
        close(f64(dx, n, hd), rx, 64 * H_ * t + step * np.abs(rx) + 1e-30)
        depth = (-(-n // 4096) + 1) * x.shape[1] + 32
        close(dg.double().cpu().numpy(), rg, (26 + depth) * H_ * np.sum(d * np.abs(x * r), (0, 1)) + 1e-30)
    eng.close()


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("n,H,G,hd,dtype", [
    (5, 28, 4, 128, "bf16"), (9, 5, 3, 64, "f32"), (7, 3, 1, 96, "bf16"), (300, 28, 4, 128, "bf16"),
    (6, 3, 5, 256, "f32"), (2, 1, 1, 16, "bf16")])
def test_no_eps_and_head_counts_that_leave_lanes_idle(n, H, G, hd, dtype, offset, monkeypatch):
    """A lane without a head has x = 0, whose 1 / sqrt(mean + 0) is infinite."""
    monkeypatch.setattr(op_util, "EPS", 0.0)
    check(n, H, G, hd, dtype, offset, False, 17 * n + H + hd)


@pytest.mark.parametrize("n,H,G,hd,dtype,offset,mrope", [
    (8195, 2, 1, 64, "f32", 0, True), (12289, 4, 1, 128, "bf16", 0, True), (8195, 2, 1, 64, "f32", 1, True),
    (12289, 4, 1, 128, "bf16", 3, False), (4097, 3, 2, 36, "bf16", 0, True)])
def test_more_rows_than_the_grid_has_waves(n, H, G, hd, dtype, offset, mrope):
    """A wave takes a second and a third row: its sums of the gains' gradients go on, its factors are read anew."""
    check(n, H, G, hd, dtype, offset, mrope, n + hd + offset)


def test_a_lost_term_would_show():
    """The bound on the gains' sums is narrower than one row of one head in at least some columns."""
    n, H, hd = 12289, 5, 128
    rng = np.random.default_rng(1)
    x, dy = rng.standard_normal((2, 64, H, hd))
    pos = rng.integers(0, 4097, (64, 3))
    _, _, size = qk_back_ref(x, np.ones(hd), pos, (0, 0, 0), dy)
    d = np.abs(dy)
    d = np.tile(d[..., :hd // 2] + d[..., hd // 2:], 2)
    r = 1 / np.sqrt(np.mean(x * x, 2, keepdims=True) + op_util.EPS)
    tol = (26 + (-(-n // 4096) + 1) * H + 32) * H_ * np.sum(d * np.abs(x * r), (0, 1)) * n / 64
    one = [np.abs(qk_back_ref(x[i:i + 1, :1], np.ones(hd), pos[i:i + 1], (0, 0, 0), dy[i:i + 1, :1])[1])
           for i in range(64)]
    assert all((t > tol).any() for t in one) and (size > 0).all()
