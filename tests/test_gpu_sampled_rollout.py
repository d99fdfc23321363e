"""Models with per-head q/k norms, rollouts under a sampled policy, and the whole chain: such a model's
sampled rollouts, their labels and weights, and a drafter's loss and gradient on them."""
import numpy as np
import pytest

from oracle import labels as LB
from op_util import distill_ref, sample_ref
from paper_2609_38795_amd import binding, workloads as W
from parity import compare
from gpu_util import make_engine, prefill, runner

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _inputs(dtype, hd, H, G, seed, norms=True, sections=(0, 0, 0), seq_len=160, anchors=6, block=6,
            vocab=1024, d_model=256):
    base = W.get("tiny_fp32")
    w = W.scaled(base, f"qkn_{dtype}_{hd}_{H}_{seed}", n_layers=2, d_model=d_model, n_heads=H,
                 n_kv_heads=G, head_dim=hd, d_ffn=512, vocab=vocab, feat_layers=(0, 1), dtype=dtype,
                 mrope_sections=sections, n_seq=2, seq_len=seq_len, anchors_per_seq=anchors,
                 anchor_lo=10, anchor_hi=seq_len - 1, block=block)
    wt = W.random_weights(w.shape, seed + 3, scale=0.05, norm_gain="random")
    if norms:
        rng = np.random.default_rng(seed + 4)
        for ld in wt["layers"]:
            for name in ("q_norm", "k_norm"):
                g = (1.0 + 0.3 * rng.standard_normal(hd)).astype(np.float32)
                ld[name] = W.f32_to_bf16_bits(g) if dtype == "bf16" else g
    a_seq, a_pos = W.random_anchors(2, seq_len, anchors, 10, seq_len - 1, seed)
    return W.Inputs(w, wt, W.random_tokens(vocab, (2, seq_len), seed + 1, dist="zipf"), a_seq, a_pos,
                    None, None)


def _grid(inp, side=6):
    pos = np.stack([W.grid_positions(inp.workload.seq_len, side)] * 2)
    return pos


def _fill(eng, inp, pos=None):
    w = inp.workload
    toks = torch.from_numpy(inp.tokens.reshape(-1).astype(np.int32)).to(eng.device)
    eng.prefill(toks, [w.seq_len] * w.n_seq, positions=None if pos is None else pos.reshape(-1, 3))


@pytest.mark.parametrize("dtype,hd,H,G,sections,d_model", [
    ("f32", 32, 4, 2, (0, 0, 0), 256), ("f32", 36, 16, 16, (0, 0, 0), 256),
    ("bf16", 128, 4, 2, (16, 24, 24), 256), ("bf16", 64, 8, 2, (0, 0, 0), 256),
    ("bf16", 64, 8, 2, (6, 13, 13), 2048), ("bf16", 50, 32, 32, (0, 0, 0), 256)])
def test_model_with_qk_norms_matches_the_oracle(dtype, hd, H, G, sections, d_model):
    inp = _inputs(dtype, hd, H, G, hd + H, sections=sections, d_model=d_model)
    w = inp.workload
    pos = _grid(inp) if sum(sections) else None
    eng = make_engine(inp)
    _fill(eng, inp, pos)
    rep = compare(inp, w.shape, np.arange(len(inp.anchor_seq)),
                  runner(eng, inp.anchor_seq, inp.anchor_pos, w.block), w.block, positions=pos)
    print(f"q/k norms {dtype} hd {hd}: {rep}", flush=True)
    assert rep.ok(), rep
    eng.close()


def test_turning_the_norms_on_and_off():
    inp, plain = (_inputs("bf16", 64, 8, 2, 3, norms=n) for n in (True, False))
    gains = [[ld[k] for ld in inp.weights["layers"]] for k in ("q_norm", "k_norm")]
    a, b = make_engine(inp), make_engine(plain)
    for e in (a, b):
        _fill(e, inp)
    run = lambda e: e.rollout(inp.anchor_seq, inp.anchor_pos, inp.workload.block)  # noqa: E731
    with_norms, without = run(a), run(b)
    assert not torch.equal(with_norms[1], without[1])
    b.set_rollout_graphs(True)
    run(b)
    b.set_qk_norm(*gains)
    with pytest.raises(binding.AlrError) as e:  # the cache was filled without norms
        run(b)
    assert e.value.status == 4
    _fill(b, inp)
    for _ in range(2):  # recorded, then replayed
        assert all(torch.equal(x, y) for x, y in zip(run(b), with_norms))
    b.set_qk_norm()
    _fill(b, inp)
    assert all(torch.equal(x, y) for x, y in zip(run(b), without))
    with pytest.raises(ValueError, match="gains"):
        b.set_qk_norm(gains[0][:1], gains[1])
    assert b.lib.alr_set_qk_norm(b.ctx, None, None, b._sp()) == 0
    arr = binding.ctypes.cast((binding.ctypes.c_void_p * 2)(None, None), binding._PP)
    assert b.lib.alr_set_qk_norm(b.ctx, arr, None, b._sp()) == 1
    assert b.lib.alr_set_qk_norm(b.ctx, arr, arr, b._sp()) == 1
    a.close()
    b.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_temperature_zero_is_the_greedy_rollout(dtype):
    inp = _inputs(dtype, 64, 8, 2, 5)
    w = inp.workload
    eng = make_engine(inp)
    _fill(eng, inp)
    n, B = len(inp.anchor_seq), w.block
    ref = eng.rollout_topk(inp.anchor_seq, inp.anchor_pos, B, want_logprobs=True)
    u = torch.rand(n, B, device="cuda")
    got = eng.rollout_sampled(inp.anchor_seq, inp.anchor_pos, B, u, temperature=torch.zeros(n, device="cuda"),
                              want_logprobs=True)
    torch.cuda.synchronize()
    assert bool((got[1] == 0).all())
    assert all(torch.equal(x, y) for x, y in zip((got[0], *got[2:]), ref))
    eng.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sampled_tokens_are_draws_from_the_rollouts_own_distribution(dtype):
    """Fed the drawn tokens, the greedy entry point gives each slot's log-probs; a draw from those in
    float64 gives the same token.  They are the logits minus an fp32 log-sum, so off by 2^-20 at most (half a
    step at 16): draws and limits within 2^-17 of a border are left out, a few in a thousand."""
    inp = _inputs(dtype, 64, 8, 2, 7, anchors=40, block=8)
    w = inp.workload
    eng = make_engine(inp)
    _fill(eng, inp)
    n, B, rng = len(inp.anchor_seq), w.block, np.random.default_rng(0)
    u = torch.from_numpy(rng.random((n, B), np.float32)).cuda()
    lim = dict(temperature=rng.choice([0.0, 0.7, 1.0, 1.3], n).astype(np.float32),
               top_k=rng.choice([0, 20, 200], n).astype(np.int32),
               top_p=rng.choice([0.6, 0.95, 1.0], n).astype(np.float32))
    dl = {k: torch.from_numpy(v).cuda() for k, v in lim.items()}
    tok, lp, ids, tl, tt, full, ft = eng.rollout_sampled(inp.anchor_seq, inp.anchor_pos, B, u, want_logprobs=True,
                                                         **dl)
    g = eng.rollout_topk(inp.anchor_seq, inp.anchor_pos, B, forced=tok, want_logprobs=True)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((ids, tl, tt, full, ft), g[1:]))
    z, t, uu = full.double().cpu().numpy(), tok.cpu().numpy(), u.cpu().numpy()
    same = 0
    for r in range(n):
        for s in range(B):
            at = {k: v[r] for k, v in lim.items()}
            draws = set()
            for d in (-2.0 ** -17, 0.0, 2.0 ** -17):
                a = dict(at)
                a["top_p"] = at["top_p"] + d if at["top_p"] < 1 else 1.0
                for du in (-2.0 ** -17, 0.0, 2.0 ** -17):
                    draws.add(sample_ref(z[r, s], uu[r, s] + du, **a)[0])
            assert t[r, s] in draws
            same += len(draws) == 1
    assert same >= 0.97 * n * B
    # the same tokens whatever else is asked for, with graphs, and in another order of the anchors
    less = eng.rollout_sampled(inp.anchor_seq, inp.anchor_pos, B, u, want_topk=False, want_feats=False, **dl)
    assert torch.equal(less[0], tok) and torch.equal(less[1], lp) and less[2] is None
    p = rng.permutation(n)
    pd = torch.from_numpy(p).cuda()
    perm = eng.rollout_sampled(inp.anchor_seq[p], inp.anchor_pos[p], B, u[pd].contiguous(),
                               **{k: v[pd].contiguous() for k, v in dl.items()})
    assert torch.equal(perm[0], tok[pd]) and torch.equal(perm[2], ids[pd])
    eng.set_rollout_graphs(True)
    out = tuple(None if x is None else torch.empty_like(x) for x in less)
    for step in range(3):  # recorded, then replayed with other numbers in the same arrays
        ref = eng.rollout_topk(inp.anchor_seq, inp.anchor_pos, B, want_feats=False)
        eng.rollout_sampled(inp.anchor_seq, inp.anchor_pos, B, u, out=out, **dl)
        eng.set_rollout_graphs(False)
        plain = eng.rollout_sampled(inp.anchor_seq, inp.anchor_pos, B, u, want_topk=False, want_feats=False, **dl)
        eng.set_rollout_graphs(True)
        eng.rollout_sampled(inp.anchor_seq, inp.anchor_pos, B, u, out=out, **dl)
        assert torch.equal(out[0], plain[0]) and torch.equal(out[1], plain[1])
        u.copy_(torch.rand_like(u))
        dl["top_k"].add_(3)
        eng.rollout_sampled(inp.anchor_seq, inp.anchor_pos, B, u, out=out, **dl)
        again = tuple(x.clone() for x in out[:2])
        eng.set_rollout_graphs(False)
        plain = eng.rollout_sampled(inp.anchor_seq, inp.anchor_pos, B, u, want_topk=False, want_feats=False, **dl)
        eng.set_rollout_graphs(True)
        assert torch.equal(again[0], plain[0]) and torch.equal(again[1], plain[1])
        del ref
    eng.close()


def test_forced_tokens_and_refusals():
    inp = _inputs("f32", 64, 8, 2, 9, norms=False)
    eng = make_engine(inp)
    _fill(eng, inp)
    n, B = len(inp.anchor_seq), inp.workload.block
    u = torch.rand(n, B, device="cuda")
    forced = torch.full((n, B), -1, dtype=torch.int32, device="cuda")
    forced[::2, 1] = 5
    got = eng.rollout_sampled(inp.anchor_seq, inp.anchor_pos, B, u, forced=forced, want_logprobs=True)
    feed = torch.where(forced >= 0, forced, got[0])
    ref = eng.rollout_topk(inp.anchor_seq, inp.anchor_pos, B, forced=feed, want_logprobs=True)
    torch.cuda.synchronize()
    assert torch.equal(got[5], ref[4]) and torch.equal(got[6], ref[5])
    with pytest.raises(ValueError, match="uniform"):
        eng.rollout_sampled(inp.anchor_seq, inp.anchor_pos, B, u[:, :2].contiguous())
    with pytest.raises(ValueError, match="top_k"):
        eng.rollout_sampled(inp.anchor_seq, inp.anchor_pos, B, u, top_k=u[:, 0].contiguous())
    with pytest.raises(binding.AlrError) as e:
        eng.rollout_sampled(inp.anchor_seq, inp.anchor_pos + 1000, B, u)
    assert e.value.status == 2
    out = list(got)
    out[3] = None
    with pytest.raises(binding.AlrError) as e:
        eng.rollout_sampled(inp.anchor_seq, inp.anchor_pos, B, u, out=tuple(out))
    assert e.value.status == 1
    eng.close()


def test_the_whole_chain():
    """A q/k-normed bf16 target's sampled rollout, its labels and slot weights, and a drafter's loss and
    gradient on them, all on one stream; the drafter's own heads go through the norms and back."""
    inp = _inputs("bf16", 64, 8, 2, 11, anchors=20, block=8)
    w = inp.workload
    eng = make_engine(inp)
    _fill(eng, inp)
    n, B, V = len(inp.anchor_seq), w.block, w.shape.vocab
    u = torch.rand(n, B, device="cuda")
    tok, _, ids, tl, tt, full, ft = eng.rollout_sampled(inp.anchor_seq, inp.anchor_pos, B, u, want_logprobs=True,
                                                        top_p=torch.full((n,), 0.9, device="cuda"))
    eos = int(tok[0, 2])
    wt = eng.slot_weights(tok, eos_id=eos)
    drafter = full.view(n * B, V).bfloat16()  # a drafter that agrees with its target up to rounding
    loss, row, grad = eng.distill_loss(drafter, ids, tl, tt, wt, scale=1.013441)
    torch.cuda.synchronize()
    np.testing.assert_allclose(wt.cpu().numpy(), LB.slot_weights(tok.cpu().numpy(), eos, gamma=2.0), rtol=1e-6)
    args = (ids.view(-1, 8).cpu().numpy(), tl.view(-1, 8).cpu().numpy(), tt.view(-1).cpu().numpy(),
            wt.view(-1).cpu().numpy())
    rl, rW, rr, rg = distill_ref(drafter.double().cpu().numpy(), *args, 1.013441)
    # as in the loss's own tests: (ceil(V / 64) + 64) half steps for the sums, half a step of bf16
    E = 2 * (V / 64 + 64) * 2.0 ** -24
    assert abs(float(loss[0]) - rl) <= 4 * E and np.abs(row.cpu().numpy() - rr).max() <= 2 * E + 2.0 ** -20
    g = grad.double().cpu().numpy()
    share = args[3][:, None] / rW
    assert (np.abs(g - rg) <= 2 * E * share * 4 + 2.0 ** -8 * np.abs(rg) + 1e-30).all()
    # the loss is the cross-entropy with the target itself: no direction lowers it by more than rounding
    assert np.abs(g).sum() < 0.05
    hd, H = w.shape.head_dim, w.shape.n_heads
    gain = torch.ones(hd, dtype=torch.bfloat16, device="cuda")
    q = ft[:, :, 0, :].reshape(n * B, -1).bfloat16()[:, :4 * hd]
    pos = torch.randint(0, w.max_pos, (n * B, 3), dtype=torch.int32, device="cuda")
    y, _ = eng.qk_norm_rope(q, None, gain, None, positions=pos)
    dq, _, dg, _ = eng.qk_norm_rope_backward(q, None, gain, None, y, None, positions=pos)
    torch.cuda.synchronize()
    # y has fixed length, so its own direction changes nothing: d |y|^2 / 2 = 0 but for eps and rounding
    x = q.double().view(n * B, 4, hd)
    r = 1 / torch.sqrt(x.square().mean(2, keepdim=True) + w.shape.rms_eps)
    assert bool((dq.double().view(n * B, 4, hd).abs() <= r * (r * r * w.shape.rms_eps + 2.0 ** -6) *
                 (1 + (x * r).abs())).all())
    assert H == 8 and bool((dg.double() - (x * r).square().sum((0, 1))).abs().max() <= 2.0 ** -6 * n * B * 4 * 2)
    eng.close()


def test_weights_with_one_of_the_two_norms_are_refused():
    inp = _inputs("f32", 64, 8, 2, 13)
    del inp.weights["layers"][1]["k_norm"]
    with pytest.raises(ValueError, match="gains"):
        make_engine(inp)
    for ld in inp.weights["layers"]:
        ld.pop("k_norm", None)
    with pytest.raises(ValueError, match="gains"):
        make_engine(inp)
