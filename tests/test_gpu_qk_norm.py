"""Per-head q/k norms with the rotation in the same pass, and their gradients, against float64.

Tolerances in half steps H = 2^-24 of fp32.  A head's mean square is a sum of at most hd positive terms (at most
16 in turn in one lane, then a tree of 6 levels), a division and a root: the normed value is off by (16 + 6 + 8) / 2
+ 3 < 20 H, the table's cos and sin by H each, a turned value by 4 H more: 26 H of |lo| + |hi|, plus half a step
of the output type.  A gradient of x adds a mean over hd terms of both signs (26 H of the mean of their sizes) and four
operations: 64 H of r (|g d| + |xh| mean |g d xh|).  A gain's gradient sums n * heads terms, each off by 26 H:
at most ceil(n heads / (16 lanes' groups)) of them in turn bounds any split, and is taken here as n * heads.
"""
import numpy as np
import pytest

from op_util import angles, engine, qk_back_ref, qk_ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
H_ = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def sections(hd, mrope):
    half = hd // 2
    return (half - 2 * (half // 3), half // 3, half // 3) if mrope else (0, 0, 0)


def make(n, H, G, hd, dtype, seed, max_pos, pad=0, offset=0):
    """q and k as column ranges of one buffer of rows."""
    rng = np.random.default_rng(seed)
    width = (H + G) * hd + pad
    buf = torch.zeros(n * width + offset, dtype=DT[dtype], device="cuda")
    rows = buf[offset:].view(n, width)
    rows.copy_(torch.from_numpy(rng.standard_normal((n, width)).astype(np.float32)))
    q = rows[:, :H * hd] if H else None
    k = rows[:, H * hd:(H + G) * hd] if G else None
    g = [torch.from_numpy((1 + 0.3 * rng.standard_normal(hd)).astype(np.float32)).to(DT[dtype]).cuda()
         for _ in range(2)]
    pos = rng.integers(0, max_pos, (n, 3)).astype(np.int32)
    return q, k, g[0], g[1], pos, rng


def f64(t, n, hd):
    return t.double().cpu().numpy().reshape(n, -1, hd)


def close(got, ref, tol):
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= tol).all(), (np.abs(got - ref) - tol).max()


CASES = [  # n, q heads, k heads, head size, padding of a row, elements before the first
    (1, 1, 1, 2, 0, 0), (1, 32, 8, 128, 0, 0), (7, 32, 8, 128, 1024, 0), (3, 28, 4, 128, 0, 0),
    (5, 16, 4, 64, 0, 8), (33, 4, 4, 32, 64, 0), (9, 3, 1, 36, 0, 0), (6, 2, 1, 50, 4, 0),
    (4, 5, 3, 80, 0, 0), (4, 5, 3, 96, 16, 0), (6, 3, 2, 256, 0, 0), (2, 1, 1, 250, 0, 0),
    (11, 4, 2, 128, 3, 1), (8, 4, 2, 64, 1, 5), (129, 6, 0, 64, 0, 0), (65, 0, 5, 128, 0, 0), (300, 12, 2, 16, 0, 0),
    (40, 2, 1, 6, 0, 0), (2000, 8, 2, 64, 0, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mrope", [False, True])
@pytest.mark.parametrize("n,H,G,hd,pad,offset", CASES)
def test_forward_and_backward(n, H, G, hd, pad, offset, mrope, dtype):
    sec = sections(hd, mrope)
    max_pos = 4097
    # the context's own heads only have to be a valid config of this head size
    eng = engine(dtype, 32, 32, hd, max_pos, sec)
    q, k, gq, gk, pos, rng = make(n, H, G, hd, dtype, 31 * n + hd + H, max_pos, pad, offset)
    p = torch.from_numpy(pos).cuda()
    half = hd // 2
    step = torch.finfo(DT[dtype]).eps / 2
    got = eng.qk_norm_rope(q, k, gq, gk, positions=p)
    dq, dk = (None if t is None else torch.from_numpy(rng.standard_normal(tuple(t.shape)).astype(np.float32))
              .to(DT[dtype]).cuda() for t in (q, k))
    back = eng.qk_norm_rope_backward(q, k, gq, gk, dq, dk, positions=p)
    torch.cuda.synchronize()
    for x, g, y, dy, dx, dg in ((q, gq, got[0], dq, back[0], back[2]), (k, gk, got[1], dk, back[1], back[3])):
        if x is None:
            assert y is None and dx is None and dg is None
            continue
        x, dy = f64(x, n, hd), f64(dy, n, hd)
        g = g.double().cpu().numpy()
        ref = qk_ref(x, g, pos, sec)
        r = 1 / np.sqrt(np.mean(x * x, 2, keepdims=True) + 1e-6)
        a = np.abs(x * r * g)
        pair = np.tile(a[..., :half] + a[..., half:], 2)
        close(f64(y, n, hd), ref, 26 * H_ * pair + step * np.abs(ref) + 1e-30)
        rx, rg, sg = qk_back_ref(x, g, pos, sec, dy)
        ad = np.abs(dy)
        d = np.tile(ad[..., :half] + ad[..., half:], 2)  # at least what is turned back
        t = r * (np.abs(g) * d + np.abs(x * r) * np.mean(np.abs(g) * d * np.abs(x * r), 2, keepdims=True))
        close(f64(dx, n, hd), rx, 64 * H_ * t + step * np.abs(rx) + 1e-30)
        m = n * x.shape[1]
        close(dg.double().cpu().numpy(), rg, (26 + m) * H_ * np.sum(d * np.abs(x * r), (0, 1)) + 1e-30)
    eng.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128, 50])
def test_in_place_row_index_positions_and_repeats(dtype, hd):
    n, H, G = 70, 6, 2
    eng = engine(dtype, 32, 32, hd, 70)
    q, k, gq, gk, _, rng = make(n, H, G, hd, dtype, 3, 70, pad=2 * hd)
    idx = torch.arange(n, dtype=torch.int32, device="cuda")[:, None].expand(n, 3).contiguous()
    a = eng.qk_norm_rope(q, k, gq, gk, positions=idx)
    b = eng.qk_norm_rope(q, k, gq, gk)
    dq, dk = torch.randn_like(a[0]), torch.randn_like(a[1])
    c = eng.qk_norm_rope_backward(q, k, gq, gk, dq, dk)
    d = eng.qk_norm_rope_backward(q, k, gq, gk, dq, dk, positions=idx, out=(dq, dk, c[2] * 0, c[3] * 0))
    torch.cuda.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert all(torch.equal(x, y) for x, y in zip(c, d))
    rest = q.as_strided((n, 2 * hd), (q.stride(0), 1), q.storage_offset() + (H + G) * hd).clone()
    eng.qk_norm_rope(q, k, gq, gk, out=(q, k))
    torch.cuda.synchronize()
    assert torch.equal(q, a[0]) and torch.equal(k, a[1])
    assert torch.equal(rest, q.as_strided((n, 2 * hd), (q.stride(0), 1), q.storage_offset() + (H + G) * hd))
    eng.close()


@pytest.mark.parametrize("hd", [128, 36])
def test_zero_heads_and_positions_outside_the_table(hd):
    eng = engine("f32", 32, 32, hd, 50)
    q, k, gq, gk, pos, _ = make(8, 2, 1, hd, "f32", 4, 50)
    q[3] = 0.0
    pos[5, 0], pos[6, 0] = 50, -1
    got = eng.qk_norm_rope(q, k, gq, gk, positions=torch.from_numpy(pos).cuda())
    torch.cuda.synchronize()
    for t in got:
        bad = torch.isnan(t).all(1).cpu().numpy()
        assert bad.tolist() == [False] * 5 + [True, True, False]
        assert bool(torch.isfinite(t[~torch.from_numpy(bad).cuda()]).all())
    assert bool((got[0][3] == 0).all())
    eng.close()


def test_gradient_against_differences():
    n, H, hd = 4, 2, 32
    eng = engine("f32", 32, 32, hd, 100)
    q, _, gq, _, pos, rng = make(n, H, 0, hd, "f32", 5, 100)
    dy = rng.standard_normal((n, H, hd))
    b = eng.qk_norm_rope_backward(q, None, gq, None, torch.from_numpy(dy.reshape(n, -1).astype(np.float32)).cuda(),
                                  None, positions=torch.from_numpy(pos).cuda())
    torch.cuda.synchronize()
    dy = dy.astype(np.float32).astype(np.float64)
    x, g = f64(q, n, hd), gq.double().cpu().numpy()
    dx, dg = f64(b[0], n, hd), b[2].double().cpu().numpy()
    h = 1e-5
    for _ in range(5):
        u, v = rng.standard_normal(x.shape), rng.standard_normal(hd)
        fx = np.sum(dy * (qk_ref(x + h * u, g, pos, (0, 0, 0)) - qk_ref(x - h * u, g, pos, (0, 0, 0)))) / (2 * h)
        fg = np.sum(dy * (qk_ref(x, g + h * v, pos, (0, 0, 0)) - qk_ref(x, g - h * v, pos, (0, 0, 0)))) / (2 * h)
        # truncation: h^2 / 6 times a third derivative below 1e3 of the values; fp32 gradient: 2^-18 of its terms
        assert abs(fx - np.sum(dx * u)) <= 2.0 ** -18 * np.sum(np.abs(dx * u)) + 1e-6
        assert abs(fg - np.sum(dg * v)) <= 2.0 ** -18 * np.sum(np.abs(dg * v)) + 1e-6


def test_captured_replays_and_another_stream():
    n, H, G, hd = 90, 8, 2, 128
    st = torch.cuda.Stream()
    eng = engine("bf16", 32, 32, hd, 100)
    q, k, gq, gk, pos, rng = make(n, H, G, hd, "bf16", 6, 100)
    p = torch.from_numpy(pos).cuda()
    dq, dk = torch.randn(n, H * hd, device="cuda").bfloat16(), torch.randn(n, G * hd, device="cuda").bfloat16()
    st.wait_stream(torch.cuda.current_stream())
    e2 = engine("bf16", 32, 32, hd, 100, stream=st)
    out = (torch.empty_like(dq), torch.empty_like(dk))
    back = (torch.empty_like(dq), torch.empty_like(dk), torch.empty(hd, device="cuda"), torch.empty(hd, device="cuda"))

    def both(e):
        e.qk_norm_rope(q, k, gq, gk, positions=p, out=out)
        e.qk_norm_rope_backward(q, k, gq, gk, dq, dk, positions=p, out=back)

    with torch.cuda.stream(st):
        both(e2)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            both(e2)
    for i in range(3):
        q.mul_(1.1).add_(0.1 * i)
        dk.mul_(-0.7)
        p.copy_((p + 7) % 100)
        both(eng)
        ref = [t.clone() for t in out + back]
        for t in out + back:
            t.fill_(9.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out + back, ref))
    e2.close()
    eng.close()


def test_in_place_needs_the_same_row_stride():
    """A row written at another stride would land on rows that are still read."""
    hd, n = 64, 5
    eng = engine("bf16", 4, 4, hd, 16)
    x = torch.zeros(n, 512, dtype=torch.bfloat16, device="cuda")
    g, dg = torch.ones(hd, dtype=torch.bfloat16, device="cuda"), torch.zeros(hd, device="cuda")
    y = torch.zeros_like(x)
    a, b, gp, dgp, lib, ctx, s = x.data_ptr(), y.data_ptr(), g.data_ptr(), dg.data_ptr(), eng.lib, eng.ctx, eng._sp()

    def fwd(rows, out_stride):
        return lib.alr_qk_norm_rope(ctx, rows, 4, 0, None, a, 512, None, 0, gp, None, a, out_stride, None, 0, s)

    def back(rows, dy, dx, stride):
        return lib.alr_qk_norm_rope_backward(ctx, rows, 4, 0, None, a, 512, None, 0, gp, None, dy, 512, None, 0,
                                             dx, stride, None, 0, dgp, None, s)

    assert fwd(n, 256) == 1 and b"in place" in lib.alr_last_error(ctx)
    assert back(n, b, b, 256) == 1 and back(n, b, a, 256) == 1
    assert fwd(n, 512) == 0 and fwd(1, 256) == 0 and back(n, b, b, 512) == 0 and back(n, b, a, 512) == 0
    torch.cuda.synchronize()
    eng.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_in_the_inputs_place(dtype):
    n, H, G, hd = 37, 6, 2, 128
    eng = engine(dtype, 8, 2, hd, 64)
    q, k, gq, gk, pos, _ = make(n, H, G, hd, dtype, 3, 64)
    p = torch.from_numpy(pos).cuda()
    dq, dk = torch.randn(q.shape, device="cuda").to(q.dtype), torch.randn(k.shape, device="cuda").to(k.dtype)
    ref = eng.qk_norm_rope_backward(q, k, gq, gk, dq, dk, positions=p)
    dg = [torch.empty(hd, device="cuda") for _ in range(2)]
    got = eng.qk_norm_rope_backward(q, k, gq, gk, dq, dk, positions=p, out=(q, k, *dg))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    eng.close()


def test_refusals():
    hd = 64
    eng = engine("bf16", 4, 4, hd, 16)
    q, k, gq, gk, pos, _ = make(5, 4, 2, hd, "bf16", 7, 16)
    p = torch.from_numpy(pos).cuda()
    with pytest.raises(ValueError, match="dtype"):
        eng.qk_norm_rope(q.float(), k, gq, gk, positions=p)
    with pytest.raises(ValueError, match="heads"):
        eng.qk_norm_rope(q[:, :100], k, gq, gk, positions=p)
    with pytest.raises(ValueError, match="shape"):
        eng.qk_norm_rope(q, k[:4], gq, gk, positions=p)
    with pytest.raises(ValueError, match="positions"):
        eng.qk_norm_rope(q, k, gq, gk, positions=p[:, :1].contiguous())
    with pytest.raises(ValueError, match="outputs"):
        eng.qk_norm_rope(q, k, gq, gk, positions=p, out=(k, q[:, :128]))
    with pytest.raises(Exception, match="max_pos"):
        big = torch.zeros(17, hd, dtype=torch.bfloat16, device="cuda")
        eng.qk_norm_rope(big, None, gq, None)
    lib, ctx, s = eng.lib, eng.ctx, eng._sp()
    a, b, ga, gb, pp = (t.data_ptr() for t in (q, k, gq, gk, p))

    def call(n=5, H=4, G=2, q=a, qs=384, gq=ga, qo=a, qos=384):
        return lib.alr_qk_norm_rope(ctx, n, H, G, pp, q, qs, b, 384, gq, gb, qo, qos, b, 384, s)

    assert call(n=-1) == 1 and call(H=-1) == 1 and call(H=0, G=0) == 1 and call(H=70000) == 1
    assert call(q=None) == 1 and call(gq=None) == 1 and call(qo=None) == 1 and call(q=a + 1) == 1
    assert call(qs=255) == 1 and call(qos=255) == 1 and b"stride" in lib.alr_last_error(ctx)
    assert call(n=0, q=None) == 0
    assert lib.alr_qk_norm_rope_backward(ctx, 5, 4, 2, pp, a, 384, b, 384, ga, gb, a, 384, b, 384, a, 384, b,
                                         384, None, ga, s) == 1
    dg = torch.full((2, hd), 5.0, device="cuda")
    none = q[:0], k[:0]
    eng.qk_norm_rope_backward(*none, gq, gk, *none, positions=p[:0],
                              out=(*none, dg[0], dg[1]))  # nothing: gradients of 0
    torch.cuda.synchronize()
    assert bool((dg == 0).all())
    eng.close()
