"""Scoring tokens over a cache held in 8 bits, as measurable cases through the library's public entry points:
appending keys and values to a paged 8-bit cache with the rotary embedding applied on the way (kv8.Kv8Cache.append,
with .read for the values that the cache then stands for), attention of a batch's new rows over that cache
(Kv8Cache.attention), and log probabilities of given tokens with entropy and top alternatives (logprobs.token_logprobs)
and their gradient (logprobs.token_logprobs_grad).

Sizes are those of the model shapes in paper_2512_14681_gb300/inputs.py (28 query heads on 4 key/value heads of 128
and 12 on 2 for the bf16 shapes, 4 on 2 of 64 for the tiny fp32 one, and their vocabularies) and of bench.py's
workloads, or generic odd ones between them.

The cache. A block is one page of 16 tokens and one head. It holds x as e4m3 values c with one exponent e:
x ~ c 2^e, with e the smallest integer for which the block's largest |x| is at most 448 2^e (-120 <= e <= 119; -120
for a block of zeros). Rows appended to a block that already holds tokens keep max(e, what the new rows need) and
round what was there again where e grew.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 16
E_MIN, E_MAX = -120, 119
NAN_CODE = 0x7F  # what memory that no token was written to may hold


def listed():
    return [
        # one decode step's append: one token of one sequence into a page that holds some; launch and latency
        dict(name="append-1tok", kind="append", Hq=28, Hkv=4, hd=128, lens="1003", new="1", cands=0, src="bf16", dst="bf16"),
        # four sequences' Jacobi drafts of odd lengths behind odd contexts, the last 3 x 8 rows of each recycled
        # candidates (positions that start over); projections hand over fp32 sums, queries go on in bf16
        dict(name="append-drafts", kind="append", Hq=12, Hkv=2, hd=128, lens="777 1200 0 4093", new="43 56 51 40", cands=3,
             src="f32", dst="bf16"),
        # prompts of three sequences at once, 7B heads, the largest append
        dict(name="append-prefill", kind="append", Hq=28, Hkv=4, hd=128, lens="0 512 0", new="4000 2777 1415", cands=0,
             src="bf16", dst="bf16"),
        # one token over a short context, 7B heads: the smallest call
        dict(name="attend-1tok-1k", kind="attend", Hq=28, Hkv=4, hd=128, lens="1024", new="1", cands=0, src="bf16"),
        # single-token serving of 16 sequences of very different lengths: the cache's bytes
        dict(name="attend-1tok-16seq", kind="attend", Hq=28, Hkv=4, hd=128, lens="32768 301 1200 17 31999 8192 640 25000 "
             "32001 4096 777 16383 12345 30000 2048 28001", new="1 " * 15 + "1", cands=0, src="bf16"),
        # one Jacobi draft of 32 tokens over a long context (the sweep's P = 32768)
        dict(name="attend-draft-32k", kind="attend", Hq=28, Hkv=4, hd=128, lens="32768", new="32", cands=0, src="bf16"),
        # drafts with recycled candidates under the tree mask, 1.5B heads, one sequence without a context and
        # rows that see nothing at all
        dict(name="attend-tree-4seq", kind="attend", Hq=12, Hkv=2, hd=128, lens="5003 0 777 12001", new="67 40 51 88", cands=4,
             src="bf16"),
        # a prompt's 512-row chunk over what is already cached: bound by the products
        dict(name="attend-chunk-8k", kind="attend", Hq=28, Hkv=4, hd=128, lens="8192", new="512", cands=0, src="bf16"),
        # the tiny fp32 model's heads of 64 dimensions
        dict(name="attend-f32", kind="attend", Hq=4, Hkv=2, hd=64, lens="777 90", new="19 8", cands=0, src="f32"),
        # the log probability of one sampled token with five alternatives: latency
        dict(name="logprobs-1row", kind="logprobs", rows=1, vocab=151936, pad=0, top=5, src="f32", masked=False, scale=1.0),
        # scoring a chunk of bf16 logits (ties everywhere), an odd vocabulary and row stride, part of it masked out
        dict(name="logprobs-512", kind="logprobs", rows=512, vocab=152063, pad=2, top=20, src="bf16", masked=True, scale=1.25),
        # a training step's loss on a draft's rows: values, and the gradient of every logit
        dict(name="logprobs-grad-512", kind="grad", rows=512, vocab=152064, pad=0, top=0, src="f32", masked=False, scale=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _text(values):
    return " ".join(str(v) for v in values)


def _ints(text):
    """Per-sequence numbers of a case ("512 301")."""
    return [int(v) for v in text.split()]


def draw(rng):
    kind = rng.choice(["append", "append", "attend", "attend", "attend", "attend", "logprobs", "logprobs", "grad"])
    if kind in ("logprobs", "grad"):
        vocab = _log_int(rng, 100, 152064)
        return dict(kind=kind, rows=_log_int(rng, 1, 512), vocab=vocab, pad=rng.choice([0, 0, 1, 2, 8]),
                    top=0 if kind == "grad" else rng.choice([0, 1, 5, 20, 32]), src=rng.choice(["f32", "bf16"]),
                    masked=rng.random() < 0.5, scale=rng.choice([1.0, 0.7, 1.25]))
    Hq, Hkv, hd, src = rng.choice([(28, 4, 128, "bf16"), (28, 4, 128, "bf16"), (12, 2, 128, "bf16"), (8, 8, 64, "bf16"),
                                   (16, 1, 128, "bf16"), (4, 2, 64, "f32"), (12, 2, 128, "f32")])
    n_seqs = rng.choice([1, 1, 2, 3, 5, 16])
    cands = rng.choice([0, 0, 2, 4])
    if kind == "append":
        new = [_log_int(rng, 1, 4000 // n_seqs) for _ in range(n_seqs)]
        lens = [rng.choice([0, _log_int(rng, 1, 16384)]) for _ in range(n_seqs)]
        return dict(kind=kind, Hq=Hq, Hkv=Hkv, hd=hd, lens=_text(lens), new=_text(new), cands=cands, src=src,
                    dst=rng.choice(["bf16", src]))
    shape = rng.choice(["token", "draft", "draft", "chunk"])
    most = 2000 if src == "f32" else 32768
    lens = [_log_int(rng, 1, most) for _ in range(n_seqs)]
    if shape == "token":
        new, cands = [1] * n_seqs, 0
    elif shape == "draft":
        new = [_log_int(rng, 2, 128 if n_seqs < 5 else 40) for _ in range(n_seqs)]
    else:
        new, lens, cands = [_log_int(rng, 64, 512 // n_seqs + 64) for _ in range(n_seqs)], [min(v, 8192) for v in lens], 0
        if n_seqs > 3:
            new, lens = new[:3], lens[:3]
    return dict(kind=kind, Hq=Hq, Hkv=Hkv, hd=hd, lens=_text(lens), new=_text(new), cands=cands, src=src)


_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------
CAND = 8  # rows of a recycled candidate


def _main_rows(n, cands):
    """Rows of a sequence's draft before its candidates (of CAND rows each, as many as fit behind a row of draft)."""
    return n - CAND * min(cands, max(0, (n - 1) // CAND))


def _offsets(n, cands):
    """Position of each new row behind the context: the draft counts up, every candidate starts over."""
    main = _main_rows(n, cands)
    return list(range(main)) + [i % CAND for i in range(n - main)]


def _tree(n, cands, words):
    """Visibility of a sequence's new rows as bits, [n][words] int32: the draft's rows see the draft up to
    themselves, a candidate's rows their own candidate up to themselves, and the last row of the last candidate
    (padding) sees no new row."""
    main = _main_rows(n, cands)
    i, j = torch.arange(n)[:, None], torch.arange(n)[None, :]
    chain = torch.where(torch.arange(n) < main, -1, (torch.arange(n) - main) // CAND)
    see = (j <= i) & (chain[:, None] == chain[None, :])
    if main < n:
        see[n - 1] = False
    bits = torch.zeros(n, words * 32, dtype=torch.int64)
    bits[:, :n] = see.long()
    packed = (bits.view(n, words, 32) << torch.arange(32)).sum(-1)
    return torch.where(packed >= 1 << 31, packed - (1 << 32), packed).to(torch.int32)


def _rope(n, hd):
    """(cos, sin) of every position, [n][hd / 2][2]: rotate-half pairing, frequency 1e6^(-2i/hd)."""
    ang = torch.arange(n, device="cuda").double()[:, None] * 1e6 ** (-torch.arange(hd // 2, device="cuda").double() * 2 / hd)
    return torch.stack([torch.cos(ang), torch.sin(ang)], -1).float()


def _exponent(amax):
    """Smallest e with amax <= 448 2^e (448 = 0.875 * 2^9), within the format's range."""
    m, x = torch.frexp(amax)
    e = torch.where(m <= 0.875, x - 9, x - 8)
    return torch.where(amax > 0, e, torch.full_like(e, E_MIN)).clamp(E_MIN, E_MAX)


def _pow2(e):
    """2^e in fp32, exact (e within -126 .. 127)."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _to_e4m3(y):
    """Codes of values within +-448, rounded to the nearest (even)."""
    return y.to(torch.float8_e4m3fn).view(torch.uint8)


def _values(codes):
    return codes.view(torch.float8_e4m3fn).float()


def _batch(case):
    lens, new = _ints(case["lens"]), _ints(case["new"])
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    return lens, new, start


def _pages_of(total):
    return (total + PAGE - 1) // PAGE


def _cache(case, g, filled):
    """A pool of pages in scrambled order whose sequences hold `filled` tokens each; memory without a token holds
    arbitrary codes. Keys have channels of different size and a few large ones, values differ from token to token."""
    lens, new, _ = _batch(case)
    Hkv, hd = case["Hkv"], case["hd"]
    per_seq = [_pages_of(a + b) for a, b in zip(lens, new)]
    n_pages = sum(per_seq) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda")
    table = torch.full((len(lens), max(per_seq)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(per_seq):
        table[b, :n] = order[at:at + n].int()
        at += n
    st = dict(table=table, lens=lens, new=new)
    channel = 0.5 + torch.rand(Hkv, 1, hd, generator=g, device="cuda")
    channel = torch.where(torch.rand(Hkv, 1, hd, generator=g, device="cuda") < 0.03, channel * 8, channel)
    for name in ("k", "v"):
        pool = torch.full((n_pages, Hkv, PAGE, hd), NAN_CODE, dtype=torch.uint8, device="cuda")
        exps = torch.full((n_pages, Hkv), 85, dtype=torch.int8, device="cuda")
        for b, n in enumerate(filled):
            if n == 0:
                continue
            pages = table[b, :_pages_of(n)].long()
            x = torch.randn(pages.numel(), Hkv, PAGE, hd, generator=g, device="cuda")
            x = x * channel if name == "k" else x * torch.exp(torch.randn(pages.numel(), Hkv, PAGE, 1, generator=g, device="cuda") * 0.5)
            e = _exponent(x.abs().amax((2, 3)))
            codes = _to_e4m3(x * _pow2(-e)[:, :, None, None])
            if n % PAGE:
                codes[-1, :, n % PAGE:] = NAN_CODE
            pool[pages], exps[pages] = codes, e.to(torch.int8)
        st[name], st[name + "_exp"] = pool, exps
    return st


def prepare(case, seed):
    g = _generator(seed)
    kind, src = case["kind"], _TYPES[case["src"]]
    if kind in ("logprobs", "grad"):
        rows, V, ld = case["rows"], case["vocab"], case["vocab"] + case["pad"]
        z = torch.randn(rows, ld, generator=g, device="cuda") * 2.5
        peaks = torch.randint(0, V, (rows, 8), generator=g, device="cuda")
        z.scatter_(1, peaks, z.gather(1, peaks) + 9.0)
        if case["masked"]:  # tokens that a grammar forbids, some by -inf and some by the type's lowest value
            forbidden = torch.rand(rows, ld, generator=g, device="cuda")
            z = torch.where(forbidden < 0.2, torch.full_like(z, -math.inf), z)
            z = torch.where(forbidden > 0.9, torch.full_like(z, torch.finfo(src).min), z)
        z = z.to(src)
        target = peaks[:, 0].clone()
        target[1::2] = torch.randint(0, V, (rows // 2,), generator=g, device="cuda")
        target = torch.where(z.gather(1, target[:, None])[:, 0] == -math.inf, -1, target)  # a target is a token that may occur
        target[7::23] = -1
        st = dict(kind=kind, logits=z[:, :V], target=target.int(), top=case["top"], scale=case["scale"])
        if kind == "grad":
            st["g_logprob"] = -torch.rand(rows, generator=g, device="cuda") / rows
            st["g_entropy"] = 0.01 * torch.rand(rows, generator=g, device="cuda") / rows
        return st
    lens, new, start = _batch(case)
    Hq, Hkv, hd, cands = case["Hq"], case["Hkv"], case["hd"], case["cands"]
    R = start[-1]
    attend = kind == "attend"
    st = _cache(case, g, [a + b for a, b in zip(lens, new)] if attend else lens)
    st.update(kind=kind, src=src, len=_i32(lens), row_start=_i32(start), max_rows=max(new))
    if attend:
        st["q"] = (torch.randn(R, Hq, hd, generator=g, device="cuda") * 1.2).to(src)
        st["softmax_scale"] = 1.0 / math.sqrt(hd)
        st["mask"] = None
        if cands:
            words = (max(new) + 31) // 32
            st["mask"] = torch.cat([_tree(n, cands, words) for n in new]).cuda()
    else:
        # one row of the fused projection: queries, keys, values
        st["qkv"] = (torch.randn(R, (Hq + 2 * Hkv) * hd, generator=g, device="cuda") *
                     torch.exp(torch.randn(R, 1, generator=g, device="cuda") * 0.3)).to(src)
        st["dst"] = _TYPES[case["dst"]]
        st["heads"] = (Hq, Hkv, hd)
        st["rope"] = _rope(max(a + b for a, b in zip(lens, new)), hd)
        st["positions"] = _i32([a + o for a, n in zip(lens, new) for o in _offsets(n, cands)]) if cands else None
        # the pages that the new rows touch, from their first slot on
        first = [a // PAGE * PAGE for a in lens]
        back = [a + n - f for a, n, f in zip(lens, new, first)]
        back_start = [0]
        for n in back:
            back_start.append(back_start[-1] + n)
        st["read_rows"] = (_i32(back_start), _i32(first), max(back), back_start[-1])
    if own:
        from paper_2512_14681_gb300 import kv8

        st["cache"] = kv8.Kv8Cache(st["k"], st["v"], st["k_exp"], st["v_exp"], st["table"])
        st["rows"] = kv8.Rows(st["row_start"], st["len"], R, st["max_rows"])
        if not attend:
            st["back"] = kv8.Rows(st["read_rows"][0], st["read_rows"][1], st["read_rows"][3], st["read_rows"][2])
    return st


# ---------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------
def _rotate(x, cs):
    """Rotary embedding in fp32, rotate-half pairing: x [R][H][hd], cs [R][hd / 2][2]."""
    half = x.shape[-1] // 2
    a, b = x[..., :half], x[..., half:]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _plain_append(st):
    Hq, Hkv, hd = st["heads"]
    qkv = st["qkv"].float()
    R = qkv.shape[0]
    q, k, v = qkv.split([Hq * hd, Hkv * hd, Hkv * hd], 1)
    q, k, v = q.view(R, Hq, hd), k.view(R, Hkv, hd), v.view(R, Hkv, hd)
    back_k, back_v, q_out = [], [], []
    r = 0
    for b, (n0, n) in enumerate(zip(st["lens"], st["new"])):
        pos = torch.arange(n0, n0 + n, device="cuda") if st["positions"] is None else st["positions"][r:r + n].long()
        cs = st["rope"][pos]
        q_out.append(_rotate(q[r:r + n], cs))
        p0, old = n0 // PAGE, n0 % PAGE
        pages = st["table"][b, p0:_pages_of(n0 + n)].long()
        for x, name, back in ((_rotate(k[r:r + n], cs), "k", back_k), (v[r:r + n], "v", back_v)):
            full = torch.zeros(pages.numel() * PAGE, Hkv, hd, device="cuda")
            full[old:old + n] = x
            full = full.view(-1, PAGE, Hkv, hd).transpose(1, 2)  # [page][head][slot][dim]
            e = _exponent(full.abs().amax((2, 3)))
            codes = st[name][pages]
            if old:  # the first page's tokens stay, at the larger of the two exponents
                e_old = st[name + "_exp"][pages[0]].int()
                e[0] = torch.maximum(e[0], e_old)
                kept = _values(codes[0, :, :old]) * _pow2(e_old - e[0])[:, None, None]
                codes[0, :, :old] = _to_e4m3(kept)
            fresh = _to_e4m3(full * _pow2(-e)[:, :, None, None])
            slot = torch.arange(pages.numel() * PAGE, device="cuda").view(-1, 1, PAGE, 1)
            written = (slot >= old) & (slot < old + n)
            codes = torch.where(written, fresh, codes)
            st[name][pages], st[name + "_exp"][pages] = codes, e.to(torch.int8)
            values = _values(codes) * _pow2(e)[:, :, None, None]
            back.append(values.transpose(1, 2).reshape(-1, Hkv, hd)[:old + n])
        r += n
    return [torch.cat(q_out).to(st["dst"]), torch.cat(back_k).bfloat16(), torch.cat(back_v).bfloat16()]


def _visible(st, b, r, n, n0):
    """[n][n0 + n]: which keys each new row of sequence b sees."""
    key = torch.arange(n0 + n, device="cuda")
    if st["mask"] is None:
        return key[None, :] <= n0 + torch.arange(n, device="cuda")[:, None]
    bits = (st["mask"][r:r + n, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
    return torch.cat([torch.ones(n, n0, dtype=torch.bool, device="cuda"), bits.view(n, -1)[:, :n].bool()], 1)


def _plain_attend(st):
    out = []
    R, Hq, hd = st["q"].shape
    Hkv = st["k"].shape[1]
    G = Hq // Hkv
    r = 0
    for b, (n0, n) in enumerate(zip(st["lens"], st["new"])):
        total = n0 + n
        pages = st["table"][b, :_pages_of(total)].long()

        def held(name):
            x = _values(st[name][pages]) * _pow2(st[name + "_exp"][pages])[:, :, None, None]
            return x.transpose(0, 1).reshape(Hkv, -1, hd)[:, :total]

        q = st["q"][r:r + n].float().view(n, Hkv, G, hd).permute(1, 2, 0, 3).reshape(Hkv, G * n, hd)
        s = torch.matmul(q, held("k").transpose(1, 2)).view(Hkv, G, n, total) * st["softmax_scale"]
        s = torch.where(_visible(st, b, r, n, n0), s, torch.full_like(s, -math.inf))
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
        total_p = p.sum(-1, keepdim=True)
        p = p / torch.where(total_p > 0, total_p, torch.ones_like(total_p))
        o = torch.matmul(p.view(Hkv, G * n, total), held("v"))
        out.append(o.view(Hkv, G, n, hd).permute(2, 0, 1, 3).reshape(n, Hq, hd))
        r += n
    return torch.cat(out).to(st["src"])


def _statistics(z):
    """(z - lse, lse, entropy) of rows of scaled logits; a logit of -inf has no share."""
    m = z.amax(-1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(-1, keepdim=True)
    lse = m + torch.log(total)
    lp = z - lse
    p = e / total
    entropy = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(-1)
    return lp, p, lse[:, 0], entropy


def _of_targets(lp, target):
    t = target.long()
    return torch.where(t >= 0, lp.gather(1, t.clamp(min=0)[:, None])[:, 0], torch.zeros_like(lp[:, 0]))


def _tops(z, lp, k):
    """The k most probable tokens, ties to the lowest index (at most as many as may occur)."""
    order = torch.sort(z, dim=-1, descending=True, stable=True).indices[:, :k]
    values = lp.gather(1, order)
    none = values == -math.inf
    order = torch.where(none, torch.full_like(order, 0x7FFFFFFF), order).int()
    if k > z.shape[1]:
        pad = k - z.shape[1]
        order = torch.nn.functional.pad(order, (0, pad), value=0x7FFFFFFF)
        values = torch.nn.functional.pad(values, (0, pad), value=-math.inf)
    return order, values


def _plain_logprobs(st):
    z = st["logits"].float()
    lp, p, lse, entropy = _statistics(z * st["scale"])
    out = [_of_targets(lp, st["target"]), entropy, lse]
    if st["kind"] == "logprobs":
        return out + (list(_tops(z, lp, st["top"])) if st["top"] else [])
    d = -st["g_entropy"][:, None] * torch.where(p > 0, p * (lp + entropy[:, None]), torch.zeros_like(p))
    g = torch.where(st["target"] >= 0, st["g_logprob"], torch.zeros_like(st["g_logprob"]))
    d = d - g[:, None] * p
    d.scatter_add_(1, st["target"].long().clamp(min=0)[:, None], g[:, None])
    return out + [(d * st["scale"]).to(st["logits"].dtype)]


def run(state):
    kind = state["kind"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend}.get(kind, _plain_logprobs)(state)
    from paper_2512_14681_gb300 import logprobs

    if kind == "append":
        Hq, Hkv, hd = state["heads"]
        q, k, v = state["qkv"].split([Hq * hd, Hkv * hd, Hkv * hd], 1)
        rotated = state["cache"].append(state["rows"], k, v, q=q, rope=state["rope"], positions=state["positions"],
                                        q_dtype=state["dst"])
        return [rotated, *state["cache"].read(state["back"], torch.bfloat16)]
    if kind == "attend":
        return state["cache"].attention(state["rows"], state["q"], state["softmax_scale"], mask=state["mask"])
    r = logprobs.token_logprobs(state["logits"], state["target"], top=state["top"], scale=state["scale"])
    out = [r.logprob, r.entropy, r.lse]
    if kind == "logprobs":
        return out + ([r.top_ids, r.top_logprobs] if state["top"] else [])
    return out + [logprobs.token_logprobs_grad(state["logits"], state["target"], r.row_stats, r.entropy, state["g_logprob"],
                                               state["g_entropy"], scale=state["scale"])]


# ---------------------------------------------------------------------------------------------
# Work and 64-bit results
# ---------------------------------------------------------------------------------------------
def work(case):
    es = {"bf16": 2, "f32": 4}
    if case["kind"] in ("logprobs", "grad"):
        n = float(case["rows"]) * case["vocab"]
        grad = case["kind"] == "grad"
        return dict(bytes=n * es[case["src"]] * (2 if grad else 1) + case["rows"] * (16 + 8 * case["top"]),
                    flops=n * (8 if grad else 5))
    lens, new, start = _batch(case)
    Hq, Hkv, hd, R = case["Hq"], case["Hkv"], case["hd"], start[-1]
    if case["kind"] == "append":
        touched = sum(a % PAGE + n for a, n in zip(lens, new))
        return dict(bytes=R * (Hq + 2 * Hkv) * hd * es[case["src"]] + R * Hq * hd * es[case["dst"]] + R * hd * 4 +
                    2 * touched * Hkv * hd * (1 + 1 + 2), flops=R * (4 * Hq + 6 * Hkv) * hd)
    keys = sum(a + n for a, n in zip(lens, new))
    pairs = sum(n * a + n * (n + 1) // 2 for a, n in zip(lens, new))
    return dict(bytes=2 * keys * Hkv * hd + 2 * R * Hq * hd * es[case["src"]], flops=4.0 * pairs * Hq * hd)


def _nearest_e4m3(y):
    """The e4m3 value nearest to y, ties to even, in 64 bits (|y| <= 448)."""
    _, x = torch.frexp(y)
    step = torch.pow(torch.full_like(y, 2.0), (x.double() - 1).clamp(min=-6) - 3)
    return torch.round(y / step) * step


def _decoded(codes):
    """Values of e4m3 codes in 64 bits: sign, 4 bits of exponent (bias 7), 3 of mantissa."""
    c = codes.long()
    x, m = (c >> 3) & 15, (c & 7).double()
    mag = torch.where(x > 0, (1 + m / 8) * torch.pow(2.0, x.double() - 7), m / 8 * 2.0 ** -6)
    return torch.where(c >= 128, -mag, mag)


def _exact_append(case, seed):
    st = prepare(case, seed)
    Hq, Hkv, hd = case["Hq"], case["Hkv"], case["hd"]
    x = st["qkv"].double().view(-1, Hq + 2 * Hkv, hd)
    offsets = st["positions"].tolist() if st["positions"] is not None else \
        [p for a, n in zip(st["lens"], st["new"]) for p in range(a, a + n)]
    cs = st["rope"].double()[torch.tensor(offsets, device="cuda")][:, None]
    turn = torch.complex(x[..., :hd // 2], x[..., hd // 2:]) * torch.complex(cs[..., 0], cs[..., 1])
    turned = torch.cat([turn.real, turn.imag], -1)
    parts = {"k": turned[:, Hq:Hq + Hkv], "v": x[:, Hq + Hkv:]}
    outs = {"k": [], "v": []}
    for name, rows in parts.items():
        r = 0
        for b, (a, n) in enumerate(zip(st["lens"], st["new"])):
            slot = a
            while slot < a + n:
                page, first, last = slot // PAGE, slot % PAGE, min(PAGE, a + n - slot // PAGE * PAGE)
                block = rows[r + slot - a:r + slot - a + last - first]
                amax = block.abs().amax((0, 2))
                e = torch.ceil(torch.log2(amax / 448)).clamp(E_MIN, E_MAX)
                if first:
                    phys = int(st["table"][b, page])
                    e_old = st[name + "_exp"][phys].double()
                    e = torch.maximum(e, e_old)
                    kept = _decoded(st[name][phys, :, :first]) * torch.pow(2.0, e_old - e)[:, None, None]
                    outs[name].append((_nearest_e4m3(kept) * torch.pow(2.0, e)[:, None, None]).transpose(0, 1))
                unit = torch.pow(2.0, e)[None, :, None]
                outs[name].append(_nearest_e4m3(block / unit) * unit)
                slot += last - first
            r += n
    return [turned[:, :Hq], torch.cat(outs["k"]), torch.cat(outs["v"])]


def _exact_attend(case, seed):
    st = prepare(case, seed)
    Hq, Hkv, hd = case["Hq"], case["Hkv"], case["hd"]
    q = st["q"].double()
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    r = 0
    for b, (a, n) in enumerate(zip(st["lens"], st["new"])):
        see = torch.zeros(n, a + n, dtype=torch.bool, device="cuda")
        see[:, :a] = True
        new = torch.ones(n, n, device="cuda").tril().bool() if st["mask"] is None else \
            torch.stack([(st["mask"][r:r + n, j // 32] >> (j % 32)) & 1 for j in range(n)], 1).bool()
        see[:, a:] = new
        pages = st["table"][b, :(a + n + PAGE - 1) // PAGE].long()
        for h in range(Hkv):
            k, v = ((_decoded(st[x][pages, h]) * torch.pow(2.0, st[x + "_exp"][pages, h].double())[:, None, None])
                    .reshape(-1, hd)[:a + n] for x in ("k", "v"))
            for i in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                s = (q[r:r + n, i] @ k.T / math.sqrt(hd)).masked_fill(~see, -math.inf)
                out[r:r + n, i] = torch.nan_to_num(torch.softmax(s, -1)) @ v  # (a row that sees nothing is 0)
        r += n
    return out


def _exact_logprobs(case, seed):
    st = prepare(case, seed)
    z = st["logits"].double()
    lp = torch.log_softmax(z * st["scale"], -1)
    p = torch.exp(lp)
    entropy = torch.special.entr(p).sum(-1)
    t = st["target"].long()
    picked = torch.zeros(len(t), dtype=torch.float64, device="cuda")
    picked[t >= 0] = lp[t >= 0, t[t >= 0]]
    out = [picked, entropy, torch.logsumexp(z * st["scale"], -1)]
    if case["kind"] == "logprobs":
        return out + ([None, _tops(st["logits"].float(), lp, st["top"])[1]] if st["top"] else [])
    d = -st["g_entropy"].double()[:, None] * torch.nan_to_num(p * (lp + entropy[:, None]))
    hot = torch.zeros_like(p)
    hot[t >= 0, t[t >= 0]] = 1.0
    d += torch.where(t >= 0, st["g_logprob"].double(), 0.0)[:, None] * (hot - p)
    return out + [d * st["scale"]]


def exact(case, seed):
    return {"append": _exact_append, "attend": _exact_attend}.get(case["kind"], _exact_logprobs)(case, seed)
