"""The operators around the target's logits and attention inputs, as cases that can be timed and compared.

* ``distill``: the paper's distillation loss on top-8 + tail labels and its gradient, on a drafter's
  logits (``Engine.distill_loss``);
* ``sample``: one token per row of logits, by temperature, top-k, top-p and min-p, from given random
  numbers (``Engine.sample``);
* ``qk``: the norms of queries and keys per head with the position rotation in the same pass, and its
  gradient (``Engine.qk_norm_rope``, ``Engine.qk_norm_rope_backward``).

``run`` computes a case in plain torch operations, or, where ``own`` is set, by this package's calls.
Sizes are those of the package's workloads: vocabularies of 512 to 152064, 16-slot blocks, 32/8, 28/4 and
16/4 heads of 64 or 128, sequences of up to 8192 tokens.
"""
import math

import torch

own = False

BLOCK = 16


def listed():
    return [
        # one fp32 micro-batch of the tiny model, loss and gradient: latency
        dict(name="distill_tiny_f32", op="distill", n=32, vocab=512, pad=0, dtype="f32", grad=True),
        # a validation pass: the loss alone, at the vision-language vocabulary, rows of a padded fp32 buffer
        dict(name="distill_eval_152k_f32", op="distill", n=768, vocab=152064, pad=64, dtype="f32", grad=False),
        # the 1B-like model's 256 anchors, a training step in bf16
        dict(name="distill_32k", op="distill", n=4096, vocab=32000, pad=0, dtype="bf16", grad=True),
        # one sample's 128 anchors at the 8B-like vocabulary: the training step the paper's recipe takes
        dict(name="distill_128k", op="distill", n=2048, vocab=128256, pad=0, dtype="bf16", grad=True),
        # one token of one stream, nucleus sampling: latency
        dict(name="sample_one", op="sample", n=1, vocab=128256, pad=0, dtype="f32", mode="top_p"),
        # a few streams of a drafter with a cut, odd vocabulary, all limits at once
        dict(name="sample_few_odd", op="sample", n=37, vocab=31999, pad=0, dtype="bf16", mode="mixed"),
        # one rollout step of one sample per device: 128 anchors, by temperature alone
        dict(name="sample_128k_free", op="sample", n=128, vocab=128256, pad=0, dtype="f32", mode="temperature"),
        # one rollout step of the 8B-like workload's 1024 anchors, all limits at once
        dict(name="sample_128k", op="sample", n=1024, vocab=128256, pad=0, dtype="f32", mode="mixed"),
        # a decode step of seven anchors: latency
        dict(name="qk_decode", op="qk", n=7, q_heads=32, k_heads=8, hd=128, dtype="bf16", mrope=False,
             max_pos=8192, back=False),
        # a prefill of 8 x 4096 tokens
        dict(name="qk_prefill", op="qk", n=32768, q_heads=32, k_heads=8, hd=128, dtype="bf16", mrope=False,
             max_pos=4096, back=False),
        # gradients over a drafter's blocks: 512 blocks of 16 slots, M-RoPE positions
        dict(name="qk_grad_mrope", op="qk", n=8192, q_heads=28, k_heads=4, hd=128, dtype="bf16", mrope=True,
             max_pos=1600, back=True),
        # gradients in fp32 at the 1B-like heads, an odd number of rows
        dict(name="qk_grad_f32", op="qk", n=2047, q_heads=16, k_heads=4, hd=64, dtype="f32", mrope=False,
             max_pos=2048, back=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("distill", "sample", "qk"))
    dtype = rng.choice(("bf16", "f32"))
    if op == "qk":
        q_heads, k_heads = rng.choice(((32, 8), (28, 4), (16, 4), (4, 4)))
        return dict(op=op, n=_log(rng, 1, 16384), q_heads=q_heads, k_heads=k_heads,
                    hd=rng.choice((32, 64, 128)), dtype=dtype, mrope=rng.random() < 0.4,
                    max_pos=_log(rng, 64, 8192), back=rng.random() < 0.5)
    vocab = _log(rng, 500, 152064)
    if rng.random() < 0.6:
        vocab = vocab // 64 * 64  # an output head's own size; else one cut anywhere
    pad = rng.choice((0, 0, 8, 3))
    if op == "distill":
        return dict(op=op, n=_log(rng, 1, max(2, min(8192, 100_000_000 // vocab))), vocab=vocab, pad=pad,
                    dtype=dtype, grad=rng.random() < 0.75)
    return dict(op=op, n=_log(rng, 1, max(2, min(2048, 60_000_000 // vocab))), vocab=vocab, pad=pad,
                dtype=dtype, mode=rng.choice(("temperature", "top_k", "top_p", "mixed")))


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _engine(dtype, q_heads=1, k_heads=1, hd=64, max_pos=1, sections=(0, 0, 0)):
    """The library context that a program of these calls holds: of the model's head shape, here
    without layers (the operators read none of a model's weights)."""
    import numpy as np

    from paper_2609_38795_amd import binding, workloads

    d = 64
    shape = workloads.ModelShape(0, d, q_heads, k_heads, hd, 64, 64, 1e-6, 1000000.0, dtype, (),
                                 mrope_sections=sections)
    z = np.zeros((64, d), np.uint16 if dtype == "bf16" else np.float32)
    weights = {"tok_embed": z, "lm_head": z, "final_norm": z[0], "layers": []}
    return binding.Engine(shape, weights, max_pos, binding.make_limits(1, 1, 1, 1))


def _logits(g, n, vocab, pad, dtype):
    """Rows of next-token logits: a broad floor and a dozen tokens that stand out of it."""
    z = torch.randn((n, vocab + pad), generator=g, device="cuda") * 2.0
    at = torch.randint(0, vocab, (n, 12), generator=g, device="cuda")
    z.scatter_add_(1, at, torch.rand((n, 12), generator=g, device="cuda") * 10.0)
    return z.to(dtype)[:, :vocab]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, n, f32 = _dtype(case), case["n"], dict(dtype=torch.float32, device="cuda")
    s = dict(case)
    if case["op"] == "qk":
        H, G, hd, P = case["q_heads"], case["k_heads"], case["hd"], case["max_pos"]
        # the projection's output, [q | k | v] per token; q and k are read in place
        s["qkv"] = torch.randn((n, (H + 2 * G) * hd), generator=g, device="cuda").to(dt)
        s["gq"] = (1 + 0.25 * torch.randn(hd, generator=g, device="cuda")).to(dt)
        s["gk"] = (1 + 0.25 * torch.randn(hd, generator=g, device="cuda")).to(dt)
        s["sections"] = (hd // 8, 3 * hd // 16, 3 * hd // 16) if case["mrope"] else (0, 0, 0)
        p = torch.randint(0, P, (n, 3), generator=g, device="cuda", dtype=torch.int32)
        s["pos"] = p if case["mrope"] else p[:, :1].expand(n, 3).contiguous()
        if case["back"]:
            s["dq"] = torch.randn((n, H * hd), generator=g, device="cuda").to(dt)
            s["dk"] = torch.randn((n, G * hd), generator=g, device="cuda").to(dt)
        if own:  # the context, and the buffers that the calls fill
            s["engine"] = _engine(case["dtype"], H, G, hd, P, s["sections"])
            s["out"] = (torch.empty((n, H * hd), dtype=dt, device="cuda"),
                        torch.empty((n, G * hd), dtype=dt, device="cuda"))
            if case["back"]:
                s["out"] += (torch.empty(hd, **f32), torch.empty(hd, **f32))
        return s
    V = case["vocab"]
    s["logits"] = _logits(g, n, V, case["pad"], dt)
    if case["op"] == "distill":
        t = s["logits"].float() * 0.8
        t += torch.randn((n, V), generator=g, device="cuda")
        top = torch.topk(t, 8, dim=1)
        lse = torch.logsumexp(t, 1)
        s["ids"] = top.indices.to(torch.int32)
        s["logp"] = top.values - lse[:, None]
        s["tail"] = (1 - s["logp"].double().exp().sum(1)).clamp(min=0).float()
        del t
        # the slots' envelope, over for blocks whose rollout ended early; the last rows have no label
        slot = torch.arange(n, device="cuda") % BLOCK
        w = torch.exp(-slot.float() / 2.0)
        ends = torch.randint(1, 3 * BLOCK, (n // BLOCK + 1,), generator=g, device="cuda")
        s["weight"] = torch.where(slot < ends[torch.arange(n, device="cuda") // BLOCK], w, 0.0 * w)
        if n > 40:
            s["ids"][-3:], s["logp"][-3:], s["tail"][-3:], s["weight"][-3:] = -1, -math.inf, 0, 0
        s["scale"] = 1.013441
        s["up"] = torch.full((1,), 0.5, **f32)  # the gradient that arrives at the loss
        if own:
            s["engine"] = _engine(case["dtype"])
            s["out"] = (torch.empty(2, **f32), torch.empty(n, **f32),
                        torch.empty((n, V), dtype=dt, device="cuda") if case["grad"] else None)
        return s
    mode, row = case["mode"], torch.arange(n, device="cuda")
    rand = lambda: torch.rand(n, generator=g, device="cuda")  # noqa: E731
    s["uniform"] = rand()
    s["temperature"] = 0.5 + rand()
    s["top_k"] = s["top_p"] = s["min_p"] = None
    if mode == "mixed":  # every 16th row is greedy, some limits are off
        s["temperature"] = torch.where(row % 16 == 5, 0.0 * row, s["temperature"]).float()
    if mode in ("top_k", "mixed"):
        k = torch.exp(rand() * math.log(1000.0)).to(torch.int32)
        s["top_k"] = torch.where(row % 4 == 1, 0 * k, k)
    if mode in ("top_p", "mixed"):
        p = 0.5 + 0.5 * rand()
        s["top_p"] = torch.where(row % 8 == 3, 1 + 0 * p, p)
    if mode == "mixed":
        s["min_p"] = torch.where(row % 2 == 1, 0 * rand(), 0.1 * rand())
    if own:
        s["engine"] = _engine(case["dtype"])
        s["out"] = (torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, **f32))
    return s


def run(s):
    if s["op"] == "distill":
        if own:
            return s["engine"].distill_loss(s["logits"], s["ids"], s["logp"], s["tail"], s["weight"],
                                            scale=s["scale"], grad_out=s["up"], want_grad=s["grad"],
                                            out=s["out"])
        return _distill(s)
    if s["op"] == "sample":
        if own:
            return s["engine"].sample(s["logits"], s["uniform"], temperature=s["temperature"],
                                      top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], out=s["out"])
        return _sample(s)
    if own:
        H, hd = s["q_heads"], s["hd"]
        q, k = s["qkv"][:, :H * hd], s["qkv"][:, H * hd:(H + s["k_heads"]) * hd]
        if s["back"]:
            return s["engine"].qk_norm_rope_backward(q, k, s["gq"], s["gk"], s["dq"], s["dk"],
                                                     positions=s["pos"], out=s["out"])
        return s["engine"].qk_norm_rope(q, k, s["gq"], s["gk"], positions=s["pos"], out=s["out"])
    return _qk(s)


def _distill(s):
    z, V = s["logits"].float(), s["vocab"]
    ids, w = s["ids"].long(), s["weight"]
    have = (ids >= 0) & (ids < V)
    pi = torch.where(have, s["logp"].exp(), 0.0)
    tau = s["tail"]
    col = torch.where(have, ids, V)  # a column of its own for entries without a token
    listed = torch.zeros((z.shape[0], V + 1), dtype=torch.bool, device=z.device).scatter_(1, col, True)[:, :V]
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    sums = e.sum(1, keepdim=True)
    lse = m + torch.log(sums)
    zt = torch.where(listed, -math.inf, z)  # the tail bucket: every token not listed
    mt = zt.amax(1, keepdim=True)
    et = torch.exp(zt - mt)
    st = et.sum(1, keepdim=True)
    lse_t = mt + torch.log(st)
    zi = z.gather(1, ids.clamp(0, V - 1))
    row = -torch.where(pi > 0, pi * (zi - lse), 0.0).sum(1) - torch.where(tau > 0, tau * (lse_t - lse)[:, 0], 0.0)
    row = torch.where(w == 0, 0.0, row)
    W = w.sum()
    inv = torch.where(W == 0, 0.0, 1 / W)
    loss = torch.stack((s["scale"] * (w * row).sum() * inv, W))
    if not s["grad"]:
        return loss, row, None
    mass = (pi.sum(1) + tau)[:, None]
    d = torch.zeros((z.shape[0], V + 1), device=z.device)
    d[:, :V] = mass * (e / sums) - tau[:, None] * (et / st)
    d.scatter_add_(1, col, -pi)
    d = d[:, :V] * (s["up"] * s["scale"] * w * inv)[:, None]
    return loss, row, d.to(s["logits"].dtype)


def _sample(s):
    # in 64 bits: a token's share of the cumulative weight is narrower than 32 bits resolve
    z, n, V = s["logits"].double(), s["n"], s["vocab"]
    zs, order = torch.sort(z, dim=1, descending=True, stable=True)
    rank = torch.arange(V, device=z.device)[None, :]
    T = s["temperature"].double()[:, None]
    greedy = T == 0
    w = torch.exp((zs - zs[:, :1]) / torch.where(greedy, 1.0, T))
    keep = (rank == 0) | ~greedy
    if s["top_k"] is not None:
        k = s["top_k"][:, None]
        keep = keep & ((k <= 0) | (rank < k))
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        cum = torch.cumsum(w * keep, 1)
        before = cum - w
        keep = keep & ((p >= 1) | (rank == 0) | (before < p * cum[:, -1:]))
    if s["min_p"] is not None:
        keep = keep & ((rank == 0) | (w >= s["min_p"].double()[:, None]))
    kept = torch.zeros_like(z).scatter_(1, order, w * keep)  # back in the order of the ids
    cum = torch.cumsum(kept, 1)
    total = cum[:, -1:]
    tok = (cum <= s["uniform"].double()[:, None] * total).sum(1).clamp(max=V - 1)
    logp = torch.log(kept.gather(1, tok[:, None])[:, 0] / total[:, 0])
    return tok.to(torch.int32), logp.float()


def _angles(s):
    """cos and sin of every row's angles, [n, hd / 2], from 64-bit angles."""
    half = s["hd"] // 2
    i = torch.arange(half, device="cuda")
    a, b, _ = s["sections"]
    axis = (i >= a).long() + (i >= a + b).long() if sum(s["sections"]) else 0 * i
    ang = s["pos"].double()[:, axis] * torch.pow(1000000.0, -2.0 * i.double() / s["hd"])
    return torch.cos(ang).float()[:, None, :], torch.sin(ang).float()[:, None, :]


def _qk(s):
    n, hd, H, G = s["n"], s["hd"], s["q_heads"], s["k_heads"]
    half, dt = hd // 2, s["qkv"].dtype
    cos, sin = _angles(s)
    x = s["qkv"][:, :(H + G) * hd].float().view(n, H + G, hd)
    gain = torch.cat((s["gq"].float().expand(H, hd), s["gk"].float().expand(G, hd)))
    r = torch.rsqrt(x.square().mean(2, keepdim=True) + 1e-6)
    if not s["back"]:
        y = x * r * gain
        lo, hi = y[..., :half], y[..., half:]
        y = torch.cat((lo * cos - hi * sin, hi * cos + lo * sin), 2).to(dt)
        return y[:, :H].reshape(n, H * hd), y[:, H:].reshape(n, G * hd)
    dy = torch.cat((s["dq"], s["dk"]), 1).float().view(n, H + G, hd)
    lo, hi = dy[..., :half], dy[..., half:]
    dy = torch.cat((lo * cos + hi * sin, hi * cos - lo * sin), 2)  # the rotation undone
    xh = x * r
    dgain = (dy * xh).sum(0)
    dn = dy * gain
    dx = (r * (dn - xh * (dn * xh).mean(2, keepdim=True))).to(dt)
    return (dx[:, :H].reshape(n, H * hd), dx[:, H:].reshape(n, G * hd), dgain[:H].sum(0), dgain[H:].sum(0))


def work(case):
    n, es = case["n"], 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "qk":
        vals = n * (case["q_heads"] + case["k_heads"]) * case["hd"]
        # forward: read, write; backward: two reads, one write
        return {"bytes": vals * es * (3 if case["back"] else 2) + n * 12, "flops": vals * (20 if case["back"] else 8)}
    vals = n * case["vocab"]
    if case["op"] == "distill":
        return {"bytes": vals * es * (2 if case["grad"] else 1) + n * 76, "flops": vals * (8 if case["grad"] else 4)}
    return {"bytes": vals * es + n * 28, "flops": vals * 4}


def exact(case, seed):
    s = prepare(case, seed)
    return {"distill": _exact_distill, "sample": _exact_sample, "qk": _exact_qk}[case["op"]](s)


def _exact_distill(s):
    # from the definition, a few rows at a time: the cross-entropy of the nine buckets, and the
    # derivative of log q_v (a listed token) and log sum q_v (the tail) by every logit
    V, n, w = s["vocab"], s["n"], s["weight"].double()
    W = float(w.sum())
    rows, grads = [], []
    step = max(1, 40_000_000 // V)
    for r0 in range(0, n, step):
        z = s["logits"][r0:r0 + step].double()
        q = torch.softmax(z, 1)
        logq = torch.log_softmax(z, 1)
        tail_q = q.clone()
        loss = torch.zeros(z.shape[0], dtype=torch.float64, device=z.device)
        d = torch.zeros_like(z)
        at = torch.arange(z.shape[0], device=z.device)
        for j in range(8):
            i = s["ids"][r0:r0 + step, j].long()
            p = torch.where((i >= 0) & (i < V), s["logp"][r0:r0 + step, j].double().exp(), 0.0)
            i = i.clamp(0, V - 1)
            loss -= p * logq[at, i]
            d += p[:, None] * q
            d[at, i] -= p
            tail_q[at, i] = torch.where(p > 0, 0.0, tail_q[at, i])
        t = s["tail"][r0:r0 + step].double()
        mass = tail_q.sum(1)
        loss -= torch.where(t > 0, t * torch.log(mass), 0.0)
        d += t[:, None] * (q - tail_q / mass[:, None])
        ww = w[r0:r0 + step]
        rows.append(torch.where(ww == 0, 0.0, loss))
        if s["grad"]:
            grads.append(d * (float(s["up"]) * s["scale"] * ww / W if W else 0 * ww)[:, None])
    row = torch.cat(rows)
    total = torch.tensor([s["scale"] * float((w * row).sum()) / W if W else 0.0, W], dtype=torch.float64)
    return total, row, torch.cat(grads) if s["grad"] else None


def _exact_sample(s):
    # row by row: the limits as a threshold on (logit, id), then the walk over the kept tokens by id
    tok, logp = [], []
    opt = {k: (s[k].tolist() if s[k] is not None else None) for k in ("temperature", "top_k", "top_p", "min_p")}
    u = s["uniform"].double().tolist()
    if s["n"] > 2048:
        return None
    for r in range(s["n"]):
        z = s["logits"][r].double()
        T = opt["temperature"][r]
        if T == 0:
            tok.append((z == z.max()).nonzero()[0, 0])
            logp.append(torch.zeros((), dtype=torch.float64, device=z.device))
            continue
        k = opt["top_k"][r] if opt["top_k"] else 0
        size = k if 0 < k < z.numel() else z.numel()
        order = torch.argsort(z, descending=True, stable=True)[:size]
        x = z[order] / T
        w = torch.exp(x - x[0])
        c = torch.cumsum(w, 0)
        if opt["top_p"] and opt["top_p"][r] < 1:
            short = int((c < opt["top_p"][r] * c[-1]).sum()) + 1
            order, w = order[:short], w[:short]
        if opt["min_p"]:
            order = order[(w >= opt["min_p"][r]) | (w == 1)]
        ids = torch.sort(order).values
        w = torch.exp((z[ids] - z.max()) / T)
        c = torch.cumsum(w, 0)
        j = torch.searchsorted(c, (u[r] * c[-1]).reshape(1), right=True)[0].clamp(max=ids.numel() - 1)
        tok.append(ids[j])
        logp.append(torch.log(w[j]) - torch.log(c[-1]))
    return torch.stack(tok).to(torch.int32), torch.stack(logp)


def _exact_qk(s):
    # pairs (i, i + hd/2) as complex numbers, the rotation as a product
    n, hd = s["n"], s["hd"]
    half, ax = hd // 2, []
    for i in range(half):
        a, b, _ = s["sections"]
        ax.append(0 if not sum(s["sections"]) else 0 if i < a else 1 if i < a + b else 2)
    freq = torch.tensor([1000000.0 ** (-2.0 * i / hd) for i in range(half)], dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["pos"].double()[:, ax] * freq)[:, None, :]
    out, first = [], 0
    for heads, gain, dy in ((s["q_heads"], s["gq"], s.get("dq")), (s["k_heads"], s["gk"], s.get("dk"))):
        x = s["qkv"][:, first:first + heads * hd].double().reshape(n, heads, hd)
        first += heads * hd
        g = gain.double()
        ms = torch.linalg.vector_norm(x, dim=2, keepdim=True) ** 2 / hd + 1e-6
        if not s["back"]:
            y = x / torch.sqrt(ms) * g
            y = torch.complex(y[..., :half], y[..., half:]) * turn
            out.append(torch.cat((y.real, y.imag), 2).reshape(n, heads * hd))
            continue
        d = dy.double().reshape(n, heads, hd)
        d = torch.complex(d[..., :half], d[..., half:]) * turn.conj()
        d = torch.cat((d.real, d.imag), 2)
        out.append(((d * g) / torch.sqrt(ms) - x * (d * g * x).sum(2, keepdim=True) / (hd * ms ** 1.5)).reshape(n, heads * hd))
        out.append((d * x / torch.sqrt(ms)).sum((0, 1)))
    return (out[0], out[2], out[1], out[3]) if s["back"] else tuple(out)
