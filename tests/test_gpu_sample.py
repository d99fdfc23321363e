"""Tokens drawn by alr_sample against a full sort in float64, and rollouts under a sampled policy.

Tokens must be equal.  A draw could differ from float64's only where the uniform number lies within about
V 2^-45 of a border between two tokens' shares, and so could a limit; the inputs here are fixed and
have no such draw.  Log-probs are formed in 64 bits and rounded to fp32 once: half a step of them, and
V 2^-44 <= 2^-26 for the weights' units.
"""
import math

import numpy as np
import pytest

from op_util import engine, sample_ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def eng():
    e = engine()
    yield e
    e.close()


def rows_of(z, dtype, pad=0, offset=0):
    n, V = z.shape
    buf = torch.zeros(n * (V + pad) + offset, dtype=dtype, device="cuda")
    rows = buf[offset:].view(n, V + pad)[:, :V]
    rows.copy_(torch.from_numpy(z.astype(np.float32)).to(dtype))
    return rows


def draw(eng, rows, u, temperature=None, top_k=None, top_p=None, min_p=None):
    c = lambda a, dt: None if a is None else torch.from_numpy(np.ascontiguousarray(a, dt)).cuda()  # noqa: E731
    tok, lp = eng.sample(rows, c(u, np.float32), c(temperature, np.float32), c(top_k, np.int32),
                         c(top_p, np.float32), c(min_p, np.float32))
    torch.cuda.synchronize()
    return tok.cpu().numpy(), lp.double().cpu().numpy()


def check(eng, rows, u, **lim):
    z = rows.double().cpu().numpy()
    got, lp = draw(eng, rows, u, **lim)
    at = lambda name, r, off: off if lim.get(name) is None else lim[name][r]  # noqa: E731
    for r in range(len(z)):
        tok, ref = sample_ref(z[r], u[r], at("temperature", r, 1.0), at("top_k", r, 0),
                              at("top_p", r, 1.0), at("min_p", r, 0.0))
        assert got[r] == tok, (r, got[r], tok, {k: v[r] for k, v in lim.items()}, u[r])
        if math.isfinite(ref):
            assert abs(lp[r] - ref) <= 2.0 ** -24 * abs(ref) + 2.0 ** -25, (r, lp[r], ref)
        else:
            assert lp[r] == ref
    return got


def logits(n, V, seed):
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((n, V)) * 2
    for r in range(n):
        z[r, rng.integers(0, V, min(12, V))] += rng.random(min(12, V)) * 10
    return z, rng


LIMITS = {
    "free": lambda rng, n: {},
    "temperature": lambda rng, n: dict(temperature=rng.choice([0.0, 0.3, 0.7, 1.0, 2.5], n)),
    "top_k": lambda rng, n: dict(top_k=rng.choice([0, 1, 2, 7, 50, 1000, 10 ** 9, -3], n),
                                 temperature=rng.random(n) + 0.5),
    "top_p": lambda rng, n: dict(top_p=rng.choice([0.0, 0.01, 0.5, 0.9, 0.95, 0.999, 1.0, 1.5], n)),
    "min_p": lambda rng, n: dict(min_p=rng.choice([0.0, 1e-6, 0.01, 0.1, 0.5, 1.0], n)),
    "all": lambda rng, n: dict(temperature=rng.choice([0.0, 0.6, 1.0, 1.4], n),
                               top_k=rng.choice([0, 3, 40, 500], n),
                               top_p=rng.choice([0.3, 0.8, 0.95, 1.0], n),
                               min_p=rng.choice([0.0, 0.001, 0.05], n)),
}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("limits", list(LIMITS))
@pytest.mark.parametrize("n,V,pad,offset", [
    (40, 1, 0, 0), (40, 2, 1, 1), (40, 63, 0, 0), (40, 64, 0, 3), (64, 513, 3, 0), (33, 4099, 5, 1),
    (12, 32000, 0, 0), (5, 128256, 0, 0), (3, 152064, 3, 5)])
def test_against_a_full_sort(eng, n, V, pad, offset, limits, dtype):
    z, rng = logits(n, V, 7 * n + V)
    check(eng, rows_of(z, dtype, pad, offset), rng.random(n, np.float32), **LIMITS[limits](rng, n))


@pytest.mark.parametrize("V", [50, 700, 20000])
@pytest.mark.parametrize("kind", ["alike", "few_values", "two_zeros"])
def test_ties(eng, V, kind):
    """Equal logits: the limits count them by id, +0 and -0 are equal."""
    rng = np.random.default_rng(V)
    n = 48
    z = {"alike": np.full((n, V), 1.5), "few_values": rng.integers(0, 4, (n, V)) * 0.5,
         "two_zeros": np.where(rng.random((n, V)) < 0.5, 0.0, -0.0)}[kind]
    for name in ("top_k", "top_p", "all"):
        lim = LIMITS[name](rng, n)
        check(eng, rows_of(z, torch.float32), rng.random(n, np.float32), **lim)


def test_ends_of_the_uniform_range(eng):
    z, rng = logits(6, 3000, 3)
    rows = rows_of(z, torch.float32)
    top = np.float32(1 - 2.0 ** -24)
    check(eng, rows, np.zeros(6, np.float32))
    check(eng, rows, np.full(6, top))
    ref, _ = draw(eng, rows, np.full(6, top))
    got, _ = draw(eng, rows, np.array([1.0, 2.0, np.inf, 1.0, 1.0, 1.0], np.float32))
    assert (got == ref).all()
    ref, _ = draw(eng, rows, np.zeros(6))
    got, _ = draw(eng, rows, np.array([-1.0, -np.inf, -0.0, -1e-30, -5, -1], np.float32))
    assert (got == ref).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("V", [300, 9000])
def test_masked_and_extreme_logits(eng, V, dtype):
    n = 24
    z, rng = logits(n, V, 4)
    z[0] = -np.inf
    z[1] = np.nan
    z[2, 10:] = -np.inf
    z[3] = -np.inf
    z[3, 77] = -5.0
    z[4, ::2] = np.nan
    z[5, [9, 4, 200]] = np.inf
    z[6] = float(torch.finfo(dtype).min)
    z[7] = float(torch.finfo(dtype).min)
    z[7, 55] = 1.0
    z[8] = float(torch.finfo(dtype).max)
    z[9, 5] = 500.0
    z[10, 1::2] = -np.inf
    u = rng.random(n, np.float32)
    rows = rows_of(z, dtype)
    for name in LIMITS:
        lim = LIMITS[name](np.random.default_rng(5), n)
        got = check(eng, rows, u, **lim)
        assert got[0] == -1 and got[1] == -1 and got[3] == 77 and got[5] == 4 and got[7] == 55


def test_extreme_limits(eng):
    n, V = 12, 5000
    z, rng = logits(n, V, 6)
    rows = rows_of(z, torch.float32)
    u = rng.random(n, np.float32)
    big = np.float32(3e38)
    check(eng, rows, u, temperature=np.full(n, 1e-40, np.float32))
    check(eng, rows, u, temperature=np.full(n, 1e-6, np.float32), top_p=np.full(n, 0.9))
    check(eng, rows, u, temperature=np.full(n, big))          # uniform over all tokens
    check(eng, rows, u, temperature=np.full(n, 1e5), top_p=np.full(n, 0.37), top_k=np.full(n, 4321))
    ref, _ = draw(eng, rows, u)
    nan = np.full(n, np.nan)
    got, _ = draw(eng, rows, u, top_p=nan, min_p=nan)          # off
    assert (got == ref).all()
    got, _ = draw(eng, rows, u, temperature=nan)               # greedy
    assert (got == z.astype(np.float32).argmax(1)).all()
    got, _ = draw(eng, rows, u, temperature=np.full(n, -1.0))
    assert (got == z.astype(np.float32).argmax(1)).all()
    got, _ = draw(eng, rows, u, min_p=np.full(n, 7.0))
    assert (got == z.astype(np.float32).argmax(1)).all()


def test_frequencies(eng):
    """Evenly spaced uniform numbers give every token its share of the rows, to within one row and one
    for each end of its interval."""
    n, V = 4096, 9
    z = np.random.default_rng(1).standard_normal(V)
    rows = rows_of(np.tile(z, (n, 1)), torch.float32)
    got, _ = draw(eng, rows, (np.arange(n) + 0.5) / n)
    z = rows[0].double().cpu().numpy()
    p = np.exp(z) / np.exp(z).sum()
    assert (np.abs(np.bincount(got, minlength=V) - n * p) <= 2).all()


def test_rows_do_not_depend_on_their_neighbours(eng):
    z, rng = logits(300, 2500, 8)
    rows = rows_of(z, torch.bfloat16)
    u = rng.random(300, np.float32)
    lim = LIMITS["all"](rng, 300)
    a, la = draw(eng, rows, u, **lim)
    b, lb = draw(eng, rows, u, **lim)
    assert (a == b).all() and (la == lb).all()
    at = [299, 4, 150, 4]
    c, lc = draw(eng, rows[at].contiguous(), u[at], **{k: v[at] for k, v in lim.items()})
    assert (c == a[at]).all() and (lc == la[at]).all()


@pytest.mark.parametrize("V", [70, 3000])
def test_more_rows_than_the_scratch_holds(eng, V):
    """The workspace holds the scans of 1024 rows here: a call of more comes in several."""
    z, rng = logits(2300, V, V)
    rows = rows_of(z, torch.bfloat16)
    u = rng.random(2300, np.float32)
    lim = LIMITS["all"](rng, 2300)
    a, la = draw(eng, rows, u, **lim)
    for at in (slice(0, 9), slice(1020, 1030), slice(2290, 2300)):
        b, lb = draw(eng, rows[at], u[at], **{k: v[at] for k, v in lim.items()})
        assert (a[at] == b).all() and (la[at] == lb).all()
    pick = np.r_[0:40, 1000:1060, 2040:2060, 2280:2300]
    z = rows.double().cpu().numpy()
    for r in pick:
        assert a[r] == sample_ref(z[r], u[r], **{k: v[r] for k, v in lim.items()})[0]


@pytest.mark.parametrize("kind", ["alike", "spread"])
def test_largest_vocabulary(eng, kind):
    """The sums of weights at their largest (2^62 units), rows of 2 MiB."""
    n, V = 6, 524288
    z, rng = logits(n, V, 31)
    if kind == "alike":
        z[:] = -3.25
    lim = dict(top_k=np.array([0, 0, 300000, 0, 5000, 60]), top_p=np.array([1, 0.9, 0.5, 1, 1, 0.99]),
               min_p=np.array([0, 0, 0, 1e-3, 0, 0]))
    rows = rows_of(z, torch.float32)
    check(eng, rows, rng.random(n, np.float32), **lim)
    check(eng, rows, rng.random(n, np.float32))


def test_captured_replays_and_another_stream(eng):
    n, V = 50, 6001
    z, rng = logits(n, V, 9)
    rows = rows_of(z, torch.float32)
    u = torch.rand(n, device="cuda")
    p = torch.full((n,), 0.8, device="cuda")
    k = torch.full((n,), 60, dtype=torch.int32, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    e2 = engine(stream=st)
    out = (torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda"))
    with torch.cuda.stream(st):
        e2.sample(rows, u, top_p=p, top_k=k, out=out)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            e2.sample(rows, u, top_p=p, top_k=k, out=out)
    for step in range(3):
        rows.mul_(0.8).add_(step)
        u.copy_(torch.rand(n, device="cuda"))
        p.sub_(0.1)
        ref = [t.clone() for t in eng.sample(rows, u, top_p=p, top_k=k)]
        out[0].fill_(-9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], ref[0]) and torch.equal(out[1], ref[1])
    e2.close()


def test_refusals(eng):
    rows = torch.zeros(4, 100, device="cuda")
    u = torch.zeros(4, device="cuda")
    with pytest.raises(ValueError, match="dtype"):
        eng.sample(rows, u, top_k=u)
    with pytest.raises(ValueError, match="shape"):
        eng.sample(rows, u[:3])
    with pytest.raises(ValueError, match="context is on"):
        eng.sample(rows.cpu(), u)
    with pytest.raises(ValueError, match="rows"):
        eng.sample(rows.t(), torch.zeros(100, device="cuda"))
    tok, _ = eng.sample(rows[:0], u[:0])
    assert tok.numel() == 0
    lib, ctx, s = eng.lib, eng.ctx, eng._sp()
    t = torch.empty(4, dtype=torch.int32, device="cuda")

    def call(n=4, V=100, z=rows.data_ptr(), dt=0, rs=100, u=u.data_ptr(), t=t.data_ptr()):
        return lib.alr_sample(ctx, n, V, z, dt, rs, None, u, t, None, s)

    assert call(n=-1) == 1 and call(V=0) == 1 and call(dt=3) == 1 and call(z=None) == 1
    assert call(rs=99) == 1 and call(z=rows.data_ptr() + 2) == 1 and call(u=None) == 1 and call(t=None) == 1
    assert call(V=524289, rs=1 << 20) == 5 and b"vocab" in lib.alr_last_error(ctx)
    assert call() == 0
    torch.cuda.synchronize()
    assert (t == 0).all()
