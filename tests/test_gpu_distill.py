"""The distillation loss and its gradient (alr_distill_loss) against its definition in float64.

Tolerances.  A row's two sums of exponentials are formed in fp32: a term at distance x below the maximum
is off by (|x| log2(e) + 2) half steps (2^-24) of itself, whose weighted mean over a row is below 40 half steps
here, and a thread adds at most ceil(V / 64) terms in turn before a tree of at most 16 levels, so the sums are
off by E = (ceil(V / 64) + 64) 2^-24 relative at most (bounds that assume a workgroup of one wave).
A row loss, sum of masses <= 1.1 times log-probabilities, is off by 2 E (both logarithms) plus
4 half steps of the log-probabilities' size.  A gradient entry, P q_v - tail q_v / q_tail - pi_v times a
factor, is off by 2 E + 8 half steps of the sum of its terms' sizes, plus half a step of its type.
"""
import math

import numpy as np
import pytest

from op_util import distill_ref, engine

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
H = 2.0 ** -24


@pytest.fixture(scope="module")
def eng():
    e = engine()
    yield e
    e.close()


def make(n, V, dtype, seed, pad=0, offset=0, spread=2.0):
    """Logits rows inside a larger buffer, labels of a teacher, slot weights with zeros."""
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((n, V)).astype(np.float32) * spread
    t = torch.from_numpy(z).to(dtype)
    buf = torch.zeros(n * (V + pad) + offset, dtype=dtype, device="cuda")
    rows = buf[offset:].view(n, V + pad)[:, :V]
    rows.copy_(t)
    k = min(8, V)
    teach = z * 0.5 + rng.standard_normal((n, V))
    ids = np.full((n, 8), -1, np.int32)
    logp = np.full((n, 8), -np.inf, np.float32)
    lse = np.log(np.exp(teach).sum(1))
    top = np.argsort(-teach, axis=1)[:, :k]
    ids[:, :k] = top
    logp[:, :k] = np.take_along_axis(teach, top, 1) - lse[:, None]
    tail = np.maximum(0, 1 - np.exp(logp.astype(np.float64)).sum(1)).astype(np.float32)
    if k == V:
        tail[:] = 0
    w = np.exp(-(np.arange(n) % 16) / 2.0).astype(np.float32)
    w[rng.random(n) < 0.2] = 0
    if n > 0 and not w.any():
        w[0] = 1
    return rows, ids, logp, tail, w


def dev(*arrays):
    return [None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in arrays]


def check(eng, rows, ids, logp, tail, w, scale=1.013441, up=0.75, dz=None, want_grad=True):
    n, V = rows.shape
    z = rows.double().cpu().numpy()
    loss, Wsum, row_ref, grad_ref = distill_ref(z, ids, logp, tail, w, scale, up)
    d = dev(ids, logp, tail, w)
    out = None
    if dz is not None:
        out = (torch.full((2,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda"), dz)
    got = eng.distill_loss(rows, *d, scale=scale, want_grad=want_grad, out=out,
                           grad_out=torch.tensor([up], device="cuda"))
    torch.cuda.synchronize()
    g_loss, g_row = got[0].double().cpu().numpy(), got[1].double().cpu().numpy()
    E = (math.ceil(V / 64) + 64) * H
    m = z.max(1)
    # distances that matter: below -200 an exponential is 0 in fp32 whatever its argument's last bits
    size = np.abs(z - m[:, None]).max(1, initial=0, where=z > m[:, None] - 200) + math.log(V) + 1
    # a log-probability may lie further down than that: -log q = (m - z) + log(sum) is rounded at each of
    # its two operations and once in the product with its mass, by half a step of its own size, and
    # the masses times those sizes add up to the row's loss
    tol = 2 * E * 1.1 + 4 * H * (size + np.where(np.isfinite(row_ref), np.abs(row_ref), 0))
    fin = np.isfinite(row_ref)
    assert (np.isfinite(g_row) == fin).all()
    assert (np.abs(g_row - row_ref)[fin] <= tol[fin]).all(), np.abs(g_row - row_ref).max()
    assert g_loss[1] == np.float32(Wsum)
    if fin.all():
        assert abs(g_loss[0] - loss) <= scale * tol.max() + 2 * H * abs(loss)
    if not want_grad:
        assert got[2] is None
        return got
    g = got[2].double().cpu().numpy()
    # sizes of a gradient entry's terms
    e = np.exp(z - m[:, None])
    q = e / e.sum(1, keepdims=True)
    terms = np.zeros_like(z)
    half = torch.finfo(rows.dtype).eps / 2
    for r in range(n):
        if w[r] == 0:
            assert (g[r] == 0).all()
            continue
        ok = (ids[r] >= 0) & (ids[r] < V)
        out_ = np.ones(V, bool)
        out_[ids[r][ok]] = False
        pi = np.exp(logp[r].astype(np.float64))
        tz = np.where(out_, z[r], -np.inf)
        te = np.exp(tz - tz.max()) if np.isfinite(tz.max()) else np.zeros(V)
        cond = te / te.sum() if te.sum() else te
        terms[r] = (pi[ok].sum() + tail[r]) * q[r] + tail[r] * cond
        np.add.at(terms[r], ids[r][ok], pi[ok])
        terms[r] *= abs(up * scale * w[r] / Wsum) if Wsum else 0
    # below fp32's smallest normal number exponentials flush to 0
    tol = (2 * E + 8 * H + 6 * H * size[:, None]) * terms + half * np.abs(grad_ref) + 1e-37
    err = np.abs(g - grad_ref)
    assert (err <= tol).all(), (err - tol).max()
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,V,pad,offset", [
    (1, 1, 0, 0), (3, 5, 0, 0), (2, 8, 0, 1), (5, 9, 2, 0), (33, 63, 1, 3), (16, 512, 0, 0),
    (17, 513, 7, 0), (48, 2047, 0, 5), (9, 4099, 5, 1), (300, 1024, 0, 0), (6, 32000, 64, 0),
    (3, 128256, 0, 0), (2, 152064, 3, 7)])
def test_against_the_definition(eng, n, V, pad, offset, dtype):
    rows, ids, logp, tail, w = make(n, V, dtype, 11 * n + V, pad, offset)
    check(eng, rows, ids, logp, tail, w)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_labels_that_are_short_double_or_cut(eng, dtype):
    n, V = 12, 700
    rows, ids, logp, tail, w = make(n, V, dtype, 5)
    w[:] = 1
    ids[0], logp[0], tail[0] = -1, -np.inf, 0      # no label at all
    ids[1, 3:], logp[1, 3:] = -1, -np.inf          # three entries
    ids[2, 4] = ids[2, 0]                          # one token twice
    ids[3, :2] = (V, V + 100000)                   # tokens that a cut vocabulary lacks
    ids[4, 0] = 2 ** 31 - 1
    ids[5, 0] = -2 ** 31
    tail[6] = 0
    logp[7, 1:] = -np.inf                          # one-hot, entries of zero probability
    logp[7, 0], tail[7] = 0.0, 0.0
    ids[8, :] = -1                                 # only the tail: all of the vocabulary
    tail[8] = 1
    got = check(eng, rows, ids, logp, tail, w)
    assert float(got[1][0]) == 0 and bool((got[2][0] == 0).all()) and float(got[1][8]) == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_masked_and_extreme_logits(eng, dtype):
    n, V = 10, 1500
    rows, ids, logp, tail, w = make(n, V, dtype, 6)
    w[:] = 1
    low = torch.finfo(dtype).min
    rows[0, 100:900] = -math.inf       # masked columns, some of them maybe listed
    ids[0] = np.arange(8)
    rows[1] = -math.inf                # all but the listed: the tail has no probability
    rows[1, :8] = 1.0
    ids[1], logp[1], tail[1] = np.arange(8), math.log(1 / 8), 0
    rows[2] = low                      # masked by the lowest value
    rows[2, 5:40] = 0.5
    ids[2] = np.arange(5, 13)
    rows[3] = rows[3] * 0 + 7.25       # all alike
    rows[4, 17] = 300.0                # one token holds everything, and is listed
    ids[4, 0] = 17
    rows[5, 17] = 300.0                # ... and is not listed
    ids[5] = np.arange(20, 28)
    rows[6] += 30000.0                 # far from zero
    rows[7] = rows[7] * 0 + low
    check(eng, rows, ids, logp, tail, w)


def test_rows_without_a_probability_for_their_label(eng):
    """A listed token, or the tail, at zero probability: the loss is infinite; gradients stay finite."""
    n, V = 4, 600
    rows, ids, logp, tail, w = make(n, V, torch.float32, 7)
    w[:] = (1, 1, 1, 0)
    rows[0, int(ids[0, 2])] = -math.inf
    rows[1] = -math.inf
    rows[1, :8] = 0.5
    ids[1] = np.arange(8)  # tail > 0 with no mass outside the list
    rows[3] = math.nan     # weight 0: not read
    got = eng.distill_loss(rows, *dev(ids, logp, tail, w))
    torch.cuda.synchronize()
    row = got[1].cpu().numpy()
    assert np.isposinf(row[:2]).all() and np.isfinite(row[2]) and row[3] == 0
    assert math.isinf(float(got[0][0]))
    assert bool(torch.isfinite(got[2]).all()) and bool((got[2][3] == 0).all())
    rows[2, 50] = math.nan
    got = eng.distill_loss(rows, *dev(ids, logp, tail, w))
    assert math.isnan(float(got[1][2])) and bool(torch.isnan(got[2][2]).all())
    assert bool(torch.isfinite(got[2][:2]).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_weights(eng, dtype):
    rows, ids, logp, tail, w = make(40, 777, dtype, 8)
    check(eng, rows, ids, logp, tail, 0 * w)                     # nothing counts: loss 0, gradients 0
    got = eng.distill_loss(rows, *dev(ids, logp, tail), None, scale=2.0)
    ones = eng.distill_loss(rows, *dev(ids, logp, tail, 0 * w + 1), scale=2.0)
    assert all(torch.equal(a, b) for a, b in zip(got, ones))     # no weights: 1 each
    assert float(got[0][1]) == 40
    empty = eng.distill_loss(rows[:0], *dev(ids[:0], logp[:0], tail[:0], w[:0]))
    assert empty[0].tolist() == [0.0, 0.0] and empty[1].numel() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("V,pad,offset", [(1000, 0, 0), (1001, 3, 1), (70001, 0, 0)])
def test_gradient_in_place_and_in_rows_of_another_alignment(eng, V, pad, offset, dtype):
    rows, ids, logp, tail, w = make(21, V, dtype, 9, pad, offset)
    d = dev(ids, logp, tail, w)
    ref = [t.clone() for t in eng.distill_loss(rows, *d)]
    around = torch.full((21, V + 9), 3.0, dtype=dtype, device="cuda")
    got = eng.distill_loss(rows, *d, out=(torch.empty(2, device="cuda"), torch.empty(21, device="cuda"),
                                          around[:, 4:4 + V]))
    assert torch.equal(got[2], ref[2]) and torch.equal(got[1], ref[1])
    assert bool((around[:, :4] == 3).all()) and bool((around[:, 4 + V:] == 3).all())
    got = eng.distill_loss(rows, *d, out=(torch.empty(2, device="cuda"), torch.empty(21, device="cuda"), rows))
    assert torch.equal(rows, ref[2]) and torch.equal(got[0], ref[0])


def test_rows_by_loss_alone_and_repeats_agree(eng):
    rows, ids, logp, tail, w = make(130, 5000, torch.bfloat16, 10)
    d = dev(ids, logp, tail, w)
    a = eng.distill_loss(rows, *d)
    b = eng.distill_loss(rows, *d)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    check(eng, rows, ids, logp, tail, w, want_grad=False)


def test_gradient_against_differences(eng):
    """The gradient times a direction against central differences of the definition's loss."""
    n, V = 6, 90
    rows, ids, logp, tail, w = make(n, V, torch.float32, 12)
    got = eng.distill_loss(rows, *dev(ids, logp, tail, w), scale=1.5)
    g = got[2].double().cpu().numpy()
    z = rows.double().cpu().numpy()
    rng = np.random.default_rng(3)
    for _ in range(5):
        d = rng.standard_normal(z.shape)
        h = 1e-4
        fd = (distill_ref(z + h * d, ids, logp, tail, w, 1.5)[0] -
              distill_ref(z - h * d, ids, logp, tail, w, 1.5)[0]) / (2 * h)
        # third derivative of a log-sum-exp along d: below 2 max|d|^3; fp32 gradient: 2^-17 of its terms
        tol = h * h / 3 * 1.5 * np.abs(d).max() ** 3 + 2.0 ** -17 * np.sum(np.abs(g * d)) + 2.0 ** -20
        assert abs(fd - np.sum(g * d)) <= tol


def test_many_rows(eng):
    """More rows than any one pass over them in a workgroup, and weights whose sum needs 64 bits."""
    n, V = 70001, 40
    rows, ids, logp, tail, w = make(n, V, torch.float32, 13)
    w[0] = 2.0 ** 22
    check(eng, rows, ids, logp, tail, w)


@pytest.mark.parametrize("n,V,dtype,pad", [
    (2048, 5003, torch.bfloat16, 0), (2049, 4001, torch.float32, 3), (2060, 9001, torch.bfloat16, 5),
    (1024, 700, torch.bfloat16, 0), (1025, 700, torch.float32, 1), (2500, 7, torch.bfloat16, 0)])
def test_many_rows_of_every_length(eng, n, V, dtype, pad):
    """Calls of many rows take workgroups of their own kind."""
    check(eng, *make(n, V, dtype, n + V, pad))


def test_captured_replays_and_another_stream(eng):
    rows, ids, logp, tail, w = make(64, 3001, torch.bfloat16, 14)
    d = dev(ids, logp, tail, w)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    e2 = engine(stream=st)
    out = (torch.empty(2, device="cuda"), torch.empty(64, device="cuda"),
           torch.empty(64, 3001, dtype=torch.bfloat16, device="cuda"))
    with torch.cuda.stream(st):
        e2.distill_loss(rows, *d, out=out)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            e2.distill_loss(rows, *d, out=out)
    for step in range(3):
        rows.copy_(rows * 0.9 + step)
        d[3].mul_(0.5).add_(0.01 * step)
        ref = [t.clone() for t in eng.distill_loss(rows, *d)]
        for t in out:
            t.fill_(5.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
    e2.close()


def test_refusals(eng):
    rows, ids, logp, tail, w = make(4, 100, torch.float32, 15)
    d = dev(ids, logp, tail, w)
    with pytest.raises(ValueError, match="dtype"):
        eng.distill_loss(rows.half(), *d)
    with pytest.raises(ValueError, match="shape"):
        eng.distill_loss(rows, d[0][:3], *d[1:])
    with pytest.raises(ValueError, match="context is on"):
        eng.distill_loss(rows, d[0].cpu(), *d[1:])
    with pytest.raises(ValueError, match="rows"):
        eng.distill_loss(rows.t().contiguous().t(), *d)
    with pytest.raises(ValueError, match="overlap"):
        eng.distill_loss(rows[:1].expand(4, 100), *d)
    lib, ctx, s = eng.lib, eng.ctx, eng._sp()
    p = [t.data_ptr() for t in d]
    loss, row = torch.empty(2, device="cuda"), torch.empty(4, device="cuda")

    def call(n=4, V=100, z=rows.data_ptr(), dt=0, rs=100, p=p, loss=loss.data_ptr(), row=row.data_ptr(),
             dz=None, dzs=100):
        return lib.alr_distill_loss(ctx, n, V, z, dt, rs, *p, 1.0, None, loss, row, dz, dzs, s)

    assert call(n=-1) == 1 and call(V=0) == 1 and call(dt=2) == 1 and call(z=None) == 1
    assert call(rs=99) == 1 and b"stride" in lib.alr_last_error(ctx)
    assert call(z=rows.data_ptr() + 2) == 1 and call(loss=None) == 1 and call(row=None) == 1
    assert call(p=[None, *p[1:]]) == 1 and call(p=[p[0], None, *p[2:]]) == 1
    assert call(dz=rows.data_ptr(), dzs=200) == 1 and call(dz=rows.data_ptr(), dzs=99) == 1
    assert call(dz=row.data_ptr() + 1) == 1
    assert call(z=rows.data_ptr()) == 0
    torch.cuda.synchronize()
