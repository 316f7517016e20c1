"""Training on drafts, trajectories and prompts, as measurable cases through the library's public entry points: causal
attention of a packed batch of texts (packed.attention), the same with its backward pass (packed.attention_grad), and the
clipped policy loss with its KL and entropy terms and its gradient by the logits (logprobs.policy_loss).

Sizes are those of the model shapes in paper_2512_14681_gb300/inputs.py (28 query heads on 4 key/value heads of 128 and 12
on 2 for the bf16 shapes, 4 on 2 of 64 for the tiny fp32 one, and their vocabularies) and of bench.py's workloads (drafts
of 8 to 128 tokens, prompts up to the sweep's), or generic odd ones between them.

Attention. The texts of a batch lie one behind the other in the rows of q, k and v; row i of a text sees its rows 0 .. i.
Rows behind the last text belong to none: their output and gradients are 0, their log-sum-exp -infinity.

Policy loss of a row, lp the log probability of its target, x = lp - old, r = e^x, d = ref - lp, H the row's entropy:
  loss = weight (-min(r A, min(max(r, 1 - below), 1 + above) A) + kl (e^d - 1 - d) - entropy H)
for an advantage A; a row with a negative target has no loss.
"""
from __future__ import annotations

import math

import torch

own = False

ABOVE, BELOW = 0.28, 0.2  # how far a ratio counts on either side of 1


def listed():
    return [
        # a text of one token: the smallest call, launch and latency
        dict(name="attn-1tok", kind="attn", Hq=28, Hkv=4, hd=128, lens="1", tail=0, src="bf16"),
        # sixteen drafts of odd lengths packed together, 1.5B heads
        dict(name="attn-drafts", kind="attn", Hq=12, Hkv=2, hd=128, lens="32 17 64 8 128 33 1 100 16 31 65 2 48 127 32 90", tail=6, src="bf16"),
        # prompts of very different lengths in one pass, 7B heads
        dict(name="attn-packed", kind="attn", Hq=28, Hkv=4, hd=128, lens="1023 2048 1 301 4096 0 777", tail=20, src="bf16"),
        # one long prompt (the sweep's 16384): bound by the products
        dict(name="attn-prompt-16k", kind="attn", Hq=28, Hkv=4, hd=128, lens="16384", tail=0, src="bf16"),
        # the tiny fp32 model's heads
        dict(name="attn-f32", kind="attn", Hq=4, Hkv=2, hd=64, lens="777 90 1 300", tail=0, src="f32"),
        # a training step's pass over sixteen drafts, 7B heads: forward and backward
        dict(name="grad-drafts", kind="grad", Hq=28, Hkv=4, hd=128, lens="32 17 64 8 128 33 1 100 16 31 65 2 48 127 32 90", tail=0, src="bf16"),
        # packed trajectories of odd lengths, 1.5B heads, rows to spare behind them
        dict(name="grad-packed", kind="grad", Hq=12, Hkv=2, hd=128, lens="1001 512 2000 3 640", tail=12, src="bf16"),
        # one long text, 7B heads: bound by the products
        dict(name="grad-prompt-8k", kind="grad", Hq=28, Hkv=4, hd=128, lens="8192", tail=0, src="bf16"),
        # the tiny fp32 model's heads, forward and backward
        dict(name="grad-f32", kind="grad", Hq=4, Hkv=2, hd=64, lens="301 64 1 150", tail=3, src="f32"),
        # one short draft's loss on the tiny shape's vocabulary: launch and latency
        dict(name="policy-16", kind="policy", rows=16, vocab=4096, pad=0, src="f32", masked=False, scale=1.0, ref=False, kl=0.0, entropy=0.0),
        # a batch of drafts with bf16 logits, an odd vocabulary and row stride, part of it masked out, every term of the loss
        dict(name="policy-512", kind="policy", rows=512, vocab=152063, pad=2, src="bf16", masked=True, scale=1.25, ref=True, kl=0.05, entropy=0.01),
        # a training step's rows with fp32 logits, all of the vocabulary: bound by the bytes
        dict(name="policy-2048", kind="policy", rows=2048, vocab=152064, pad=0, src="f32", masked=False, scale=1.0, ref=True, kl=0.02, entropy=0.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _ints(text):
    """Per-text numbers of a case ("512 301")."""
    return [int(v) for v in text.split()]


def draw(rng):
    kind = rng.choice(["attn", "attn", "grad", "grad", "policy"])
    if kind == "policy":
        ref = rng.random() < 0.7
        return dict(kind=kind, rows=_log_int(rng, 1, 1024), vocab=_log_int(rng, 100, 152064), pad=rng.choice([0, 0, 1, 2, 8]),
                    src=rng.choice(["f32", "bf16"]), masked=rng.random() < 0.5, scale=rng.choice([1.0, 0.7, 1.25]), ref=ref,
                    kl=rng.choice([0.02, 0.1]) if ref else 0.0, entropy=rng.choice([0.0, 0.01]))
    Hq, Hkv, hd, src = rng.choice([(28, 4, 128, "bf16"), (28, 4, 128, "bf16"), (12, 2, 128, "bf16"), (12, 2, 128, "bf16"), (8, 8, 64, "bf16"),
                                   (16, 1, 128, "bf16"), (10, 2, 64, "bf16"), (4, 2, 64, "f32"), (12, 2, 128, "f32")])
    most = (2000 if kind == "attn" else 1000) if src == "f32" else (12000 if kind == "attn" else 6000)
    n = rng.choice([1, 1, 2, 3, 5, 16, 40])
    lens = [_log_int(rng, 1, max(2, 2 * most // (n + 1))) for _ in range(n)]
    while sum(lens) > most:
        lens[lens.index(max(lens))] //= 2
    return dict(kind=kind, Hq=Hq, Hkv=Hkv, hd=hd, lens=" ".join(str(v) for v in lens), tail=rng.choice([0, 0, 1, 30]), src=src)


_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------
def _groups(lens):
    """Texts of like lengths (within a factor of two of each other) as padded batches: [(rows [texts][longest], real)].
    Padding repeats the text's last row, behind everything that its rows see."""
    start, at = [], 0
    for n in lens:
        start.append(at)
        at += n
    by = {}
    for s, n in zip(start, lens):
        if n:
            by.setdefault((n - 1).bit_length(), []).append((s, n))
    out = []
    for texts in by.values():
        s, n = torch.tensor(texts, device="cuda").T
        i = torch.arange(int(n.max()), device="cuda")[None, :]
        out.append((s[:, None] + torch.minimum(i, n[:, None] - 1), i < n[:, None]))
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.rand(*shape, generator=g, device="cuda")
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    src = _TYPES[case["src"]]
    if case["kind"] == "policy":
        rows, V, ld = case["rows"], case["vocab"], case["vocab"] + case["pad"]
        z = randn(rows, ld) * 2.5
        peaks = torch.randint(0, V, (rows, 8), generator=g, device="cuda")
        z.scatter_(1, peaks, z.gather(1, peaks) + 9.0)
        if case["masked"]:  # tokens that a grammar forbids, some by -inf and some by the type's lowest value
            forbidden = rand(rows, ld)
            z = torch.where(forbidden < 0.2, torch.full_like(z, -math.inf), z)
            z = torch.where(forbidden > 0.9, torch.full_like(z, torch.finfo(src).min), z)
            z.scatter_(1, peaks[:, :1], 5.0)
        z = z.to(src)
        target = peaks[:, 0].clone()
        target[1::2] = torch.randint(0, V, (rows // 2,), generator=g, device="cuda")
        zt = z.gather(1, target[:, None])[:, 0].float()
        target = torch.where(zt < -1e4, peaks[:, 0], target)  # a token that was sampled
        zt = z.gather(1, target[:, None])[:, 0].float()
        lp = zt * case["scale"] - torch.logsumexp(z[:, :V].float() * case["scale"], 1)
        # the policy that sampled is a little older; ratios of 1 +- 0.2 and a few beyond, none within rounding of a border
        ratio = torch.exp(randn(rows) * 0.2)
        for border in (1 - BELOW, 1 + ABOVE):
            ratio = torch.where((ratio - border).abs() < 1e-3, ratio * 1.01, ratio)
        target[7::23] = -1
        return dict(kind="policy", logits=z[:, :V], target=target.int(), old=lp - torch.log(ratio), ref=lp + randn(rows) * 0.4 if case["ref"] else None,
                    advantage=randn(rows), weight=(0.5 + rand(rows)) / rows, scale=case["scale"], kl=case["kl"], entropy=case["entropy"])
    lens = _ints(case["lens"])
    Hq, Hkv, hd = case["Hq"], case["Hkv"], case["hd"]
    R = sum(lens) + case["tail"]
    # one row of the fused projection: queries, keys with channels of different size, values of different size by token
    channel = 0.5 + rand(Hkv, hd)
    channel = torch.where(rand(Hkv, hd) < 0.03, channel * 4, channel)
    qkv = torch.cat([randn(R, Hq * hd) * 1.2, (randn(R, Hkv, hd) * channel).view(R, -1), randn(R, Hkv * hd) * torch.exp(randn(R, 1) * 0.5)], 1).to(src)
    st = dict(kind=case["kind"], lens=lens, heads=(Hq, Hkv, hd), qkv=qkv, softmax_scale=1.0 / math.sqrt(hd), src=src, groups=_groups(lens))
    if case["kind"] == "grad":
        st["d_out"] = (randn(R, Hq, hd) * torch.exp(randn(R, 1, 1)) * 1e-2).to(src)
    if own:
        from paper_2512_14681_gb300 import packed

        st["texts"] = packed.Packed.of(lens, n_rows=R)
    return st


# ---------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------
def _heads(st):
    """q [rows][Hq][hd], k and v [rows][Hkv][hd] as views of the projection's rows."""
    Hq, Hkv, hd = st["heads"]
    q, k, v = st["qkv"].split([Hq * hd, Hkv * hd, Hkv * hd], 1)
    return q.unflatten(1, (Hq, hd)), k.unflatten(1, (Hkv, hd)), v.unflatten(1, (Hkv, hd))


def _plain_attention(st):
    Hq, Hkv, hd = st["heads"]
    G, c = Hq // Hkv, st["softmax_scale"]
    q, k, v = _heads(st)
    R = q.shape[0]
    f32 = dict(dtype=torch.float32, device="cuda")
    out, lse = torch.zeros(R, Hq, hd, **f32), torch.full((R, Hq), -math.inf, **f32)
    grads = [torch.zeros(R, H, hd, **f32) for H in (Hq, Hkv, Hkv)] if st["kind"] == "grad" else []
    for rows, real in st["groups"]:
        B, L = rows.shape
        by_head = lambda x, H: x[rows].float().view(B, L, Hkv, H // Hkv, hd).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, hd)
        by_row = lambda x, H: x.view(B, Hkv, H // Hkv, L, hd).permute(0, 3, 1, 2, 4).reshape(B, L, H, hd)[real]
        Q, K, V = by_head(q, Hq), by_head(k, Hkv), by_head(v, Hkv)
        s = (torch.matmul(Q, K.transpose(2, 3)) * c).view(B, Hkv, G, L, L)
        i = torch.arange(L, device="cuda")
        s.masked_fill_(i[None, :] > i[:, None], -math.inf)
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(-1, keepdim=True)
        p = p / total
        del s
        O = torch.matmul(p.view(B, Hkv, G * L, L), V)
        at = rows[real]
        out[at] = by_row(O, Hq)
        lse[at] = (top + torch.log(total)).view(B, Hq, L).transpose(1, 2)[real]
        if grads:
            dO = by_head(st["d_out"], Hq)
            dO = dO * real[:, None, None, :, None].expand(B, Hkv, G, L, 1).reshape(B, Hkv, G * L, 1)  # nothing comes back from padding
            P = p.view(B, Hkv, G * L, L)
            dV = torch.matmul(P.transpose(2, 3), dO)
            ds = torch.matmul(dO, V.transpose(2, 3)) - (dO * O).sum(-1, keepdim=True)
            ds = ds * P * c
            grads[0][at] = by_row(torch.matmul(ds, K), Hq)
            grads[1][at] = by_row(torch.matmul(ds.transpose(2, 3), Q), Hkv)
            grads[2][at] = by_row(dV, Hkv)
    if grads:
        return [x.to(st["src"]) for x in [out, *grads]]
    return [out.to(st["src"]), lse]


def _plain_policy(st):
    scale, t = st["scale"], st["target"].long()
    z = st["logits"].float() * scale
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    p = e / total
    logp = (z - top) - torch.log(total)
    H = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    has, at = t >= 0, t.clamp(min=0)[:, None]
    zero = torch.zeros_like(H)
    lp = torch.where(has, logp.gather(1, at)[:, 0], zero)
    A, w = st["advantage"], torch.where(has, st["weight"], zero)
    r = torch.where(has, torch.exp(lp - st["old"]), zero)
    free, held = r * A, r.clamp(1 - BELOW, 1 + ABOVE) * A
    loss = -torch.minimum(free, held)
    g = -torch.where(free <= held, free, zero)
    kl = zero
    if st["ref"] is not None:
        d = st["ref"] - lp
        kl = torch.where(has, torch.expm1(d) - d, zero)
        loss = loss + st["kl"] * kl
        g = g - st["kl"] * torch.expm1(d)
    loss = w * (loss - st["entropy"] * H)
    g = w * g
    dz = -g[:, None] * p
    if st["entropy"]:
        dz = dz + (w * st["entropy"])[:, None] * torch.where(p > 0, p * (logp + H[:, None]), torch.zeros_like(p))
    dz.scatter_add_(1, at, g[:, None])
    return [loss, lp, H, r, kl, (dz * scale).to(st["logits"].dtype)]


def run(state):
    if not own:
        return _plain_policy(state) if state["kind"] == "policy" else _plain_attention(state)
    if state["kind"] == "policy":
        from paper_2512_14681_gb300 import logprobs

        r = logprobs.policy_loss(state["logits"], state["target"], state["old"], state["advantage"], weight=state["weight"],
                                 ref_logprob=state["ref"], below=BELOW, above=ABOVE, kl=state["kl"], entropy=state["entropy"], scale=state["scale"])
        return [r.loss, r.logprob, r.entropy, r.ratio, r.kl, r.grad]
    from paper_2512_14681_gb300 import packed

    q, k, v = _heads(state)
    out, lse = packed.attention(state["texts"], q, k, v, state["softmax_scale"], want_lse=True)
    if state["kind"] == "attn":
        return [out, lse]
    return [out, *packed.attention_grad(state["texts"], q, k, v, out, lse, state["d_out"], state["softmax_scale"])]


# ---------------------------------------------------------------------------------------------
# Work and 64-bit results
# ---------------------------------------------------------------------------------------------
def work(case):
    es = {"bf16": 2, "f32": 4}[case["src"]]
    if case["kind"] == "policy":
        n = float(case["rows"]) * case["vocab"]
        return dict(bytes=2 * n * es + case["rows"] * 44, flops=n * 8)
    lens, Hq, Hkv, hd = _ints(case["lens"]), case["Hq"], case["Hkv"], case["hd"]
    R = sum(lens) + case["tail"]
    pairs = sum(n * (n + 1) // 2 for n in lens)
    if case["kind"] == "attn":  # q, k, v in; out and lse out
        return dict(bytes=R * ((2 * Hq + 2 * Hkv) * hd * es + Hq * 4), flops=4.0 * pairs * Hq * hd)
    return dict(bytes=R * (4 * Hq + 4 * Hkv) * hd * es, flops=14.0 * pairs * Hq * hd)  # and the output's gradient in; dq, dk, dv out


def _exact_attention(case, seed):
    st = prepare(case, seed)
    q, k, v = (x.double() for x in _heads(st))
    Hq, Hkv, hd = st["heads"]
    back = case["kind"] == "grad"
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    at = 0
    for n in st["lens"]:
        rows = slice(at, at + n)
        at += n
        hidden = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
        for h in range(Hq if n else 0):
            one = [x.detach().clone().requires_grad_(back) for x in (q[rows, h], k[rows, h * Hkv // Hq], v[rows, h * Hkv // Hq])]
            s = (one[0] @ one[1].T * st["softmax_scale"]).masked_fill(hidden, -math.inf)
            o = torch.softmax(s, 1) @ one[2]
            out[rows, h], lse[rows, h] = o.detach(), torch.logsumexp(s.detach(), 1)
            if back:
                d = torch.autograd.grad(o, one, st["d_out"][rows, h].double())
                dq[rows, h] = d[0]
                dk[rows, h * Hkv // Hq] += d[1]
                dv[rows, h * Hkv // Hq] += d[2]
    return [out, dq, dk, dv] if back else [out, lse]


def _exact_policy(case, seed):
    st = prepare(case, seed)
    z = st["logits"].double().requires_grad_()
    t = st["target"].long()
    logp = torch.log_softmax(z * st["scale"], 1)
    H = torch.special.entr(torch.softmax(z * st["scale"], 1)).sum(1)
    on = t >= 0
    lp = torch.where(on, logp.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
    ratio = torch.where(on, torch.exp(lp - st["old"].double()), 0.0)
    A = st["advantage"].double()
    surrogate = torch.where(A >= 0, -torch.where(ratio > 1 + ABOVE, 1 + ABOVE, ratio) * A, -torch.where(ratio < 1 - BELOW, 1 - BELOW, ratio) * A)
    kl = torch.zeros_like(lp)
    if st["ref"] is not None:
        behind = st["ref"].double() - lp
        kl = torch.where(on, torch.exp(behind) - behind - 1, 0.0)
    p = torch.softmax(z.detach() * st["scale"], 1)
    loss = torch.where(on, st["weight"].double(), 0.0) * (surrogate + st["kl"] * kl - st["entropy"] * H.detach())
    dz, = torch.autograd.grad((torch.where(on, st["weight"].double(), 0.0) * (surrogate + st["kl"] * kl)).sum(), z)
    dz = torch.nan_to_num(dz)
    if st["entropy"]:  # d(-H) / dz by hand: the logit of probability 0 has no share
        d = torch.where(p > 0, p * (torch.where(p > 0, logp.detach(), 0.0) + H.detach()[:, None]), 0.0)
        dz = dz + torch.where(on, st["weight"].double(), 0.0)[:, None] * st["entropy"] * d * st["scale"]
    return [x.detach() for x in (loss, lp, H, ratio, kl)] + [dz]


def exact(case, seed):
    return _exact_policy(case, seed) if case["kind"] == "policy" else _exact_attention(case, seed)
