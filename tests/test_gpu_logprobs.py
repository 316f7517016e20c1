"""Log probabilities of given tokens with entropy and top alternatives, and their gradient (jf_op_token_logprobs*),
against plain 64-bit arithmetic.

Tolerances. An exponential is off by 2^-22 + |d| 2^-23 (its argument d = scale (x - max), rounded twice), a sum of V of
them by at most about 2^-20 in the order that threads add (a few hundred terms each); lse, log p and the entropy follow with
that plus their own rounding 2^-23 of their magnitude: 4e-6 (1 + |value|) covers them for |d| that carry weight. Gradients:
scale * (|g| + |gH| (|log p| + H)) * (p * 2e-5 + rounding of the output's type).
"""
import numpy as np
import pytest

from tests.parity import need_gpu

pytestmark = pytest.mark.gpu
NO_TOKEN = 0x7FFFFFFF


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


def place(torch, x, dtype, pad, shift):
    """x [rows][V] as rows V + pad elements apart, starting `shift` elements into an allocation; NaN around them."""
    rows, V = x.shape
    store = torch.full((rows * (V + pad) + shift + 16,), float("nan"), dtype=dtype, device="cuda")
    view = store[shift:shift + rows * (V + pad)].view(rows, V + pad)[:, :V]
    view.copy_(torch.from_numpy(x))
    return view


def reference(z, targets, scale, k):
    """lse, entropy, logprob, log p of every token, top ids: 64 bits."""
    rows, V = z.shape
    with np.errstate(all="ignore"):
        m = z.max(1, keepdims=True)
        d = np.where(m == -np.inf, -np.inf, (z - np.where(m == -np.inf, 0, m)) * scale)
        s = np.exp(d).sum(1, keepdims=True)
        lp = d - np.log(s)
        p = np.where(s > 0, np.exp(lp), 0)
        lse = (m * scale + np.log(s))[:, 0]
        lse[m[:, 0] == -np.inf] = -np.inf
        entropy = -np.where(p > 0, p * lp, 0).sum(1)
    lp[(m == -np.inf)[:, 0]] = -np.inf
    picked = np.array([lp[i, t] if t >= 0 else 0.0 for i, t in enumerate(targets)])
    ids = np.full((rows, k), NO_TOKEN)
    for i in range(rows):
        order = np.argsort(-z[i], kind="stable")[:k]
        order = order[z[i, order] > -np.inf]
        ids[i, :len(order)] = order
    return lse, entropy, picked, lp, p, ids


def logits(rng, rows, V, dtype, kind):
    x = rng.standard_normal((rows, V)) * 3
    if kind == "ties":
        x = np.round(x)
    if kind == "flat":
        x = np.zeros((rows, V))
    if kind == "rising":
        x = np.sort(x, 1)
    if kind == "masked":
        x[rng.random((rows, V)) < 0.3] = -np.inf
        x[rng.random((rows, V)) < 0.2] = -3.0e38
    if kind == "large":
        x = x * 1e4 + 1e5
    return x


KINDS = ["plain", "ties", "flat", "rising", "masked", "large"]
SHAPES = [  # rows, vocab, pad, shift, top, scale
    (1, 1, 0, 0, 1, 1.0), (3, 2, 1, 1, 5, 0.5), (2, 7, 0, 3, 3, 1.0), (5, 100, 0, 0, 64, 2.0), (1, 4096, 0, 0, 5, 1.0),
    (4, 4097, 3, 1, 20, 1.25), (1, 50001, 0, 5, 33, 1.0), (2, 151936, 0, 0, 1, 1.0), (77, 8191, 1, 0, 20, 0.7),
    (700, 1000, 0, 2, 8, 1.0), (310, 9001, 7, 0, 0, 1.0),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
def test_values_and_top_lists(torch, dtype, kind):
    from paper_2512_14681_gb300 import logprobs as L

    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    for n, (rows, V, pad, shift, top, scale) in enumerate(SHAPES):
        rng = np.random.default_rng(n)
        x = place(torch, logits(rng, rows, V, dtype, kind), t, pad, shift)
        z = x.double().cpu().numpy()
        targets = rng.integers(-1, V, rows)
        r = L.token_logprobs(x, torch.from_numpy(targets.astype(np.int32)).cuda(), top=top, scale=scale)
        L.check()
        lse, entropy, picked, lp, p, ids = reference(z, targets, np.float32(scale).astype(np.float64), top)
        for got, want, what in ((r.lse, lse, "lse"), (r.entropy, entropy, "entropy"), (r.logprob, picked, "logprob")):
            got = got.double().cpu().numpy()
            fin = np.isfinite(want) & (np.abs(want) < 3.4e38)
            assert (np.abs(got - want)[fin] <= 4e-6 * (1 + np.abs(want[fin]))).all(), (what, rows, V)
            assert (got[~fin] == np.where(np.isfinite(want), np.sign(want) * np.inf, want)[~fin]).all(), (what, rows, V)
        if top:
            assert (r.top_ids.cpu().numpy() == ids).all(), (rows, V)
            got = r.top_logprobs.double().cpu().numpy()
            want = np.where(ids == NO_TOKEN, -np.inf, np.take_along_axis(lp, np.minimum(ids, V - 1), 1))
            fin = np.isfinite(want) & (np.abs(want) < 3.4e38)
            assert (np.abs(got - want)[fin] <= 4e-6 * (1 + np.abs(want[fin]))).all()
            assert (got[~fin] == -np.inf).all()
        again = L.token_logprobs(x, torch.from_numpy(targets.astype(np.int32)).cuda(), top=top, scale=scale)
        assert torch.equal(again.entropy, r.entropy) and torch.equal(again.lse, r.lse)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 400])
def test_rows_that_are_empty_or_hold_no_numbers(torch, dtype, rows):
    from paper_2512_14681_gb300 import logprobs as L

    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    V = 5000
    base = torch.randn(rows, V, device="cuda").to(t)
    target = torch.full((rows,), 17, dtype=torch.int32, device="cuda")
    low = float(torch.finfo(t).min)
    for name, edit in {"empty": lambda x: x.fill_(-float("inf")), "lowest": lambda x: x.fill_(low),
                       "nan": lambda x: x[-1, 4000].fill_(float("nan")), "all nan": lambda x: x.fill_(float("nan")),
                       "inf": lambda x: x[-1, 3000].fill_(float("inf")),
                       "one": lambda x: (x.fill_(-float("inf")), x[:, 4999].fill_(2.0))}.items():
        x = base.clone()
        edit(x)
        r = L.token_logprobs(x, target, top=3)
        d = L.token_logprobs_grad(x, target, r.row_stats, r.entropy, 1.0, 0.5)
        lp, h, lse, ids, lps = (v[-1].tolist() for v in (r.logprob, r.entropy, r.lse, r.top_ids, r.top_logprobs))
        if name == "empty":
            assert (lp, h, lse) == (-float("inf"), 0.0, -float("inf")) and ids == [NO_TOKEN] * 3 and not d[-1].any()
        elif name == "lowest":  # every token as likely as another
            assert abs(lp + np.log(V)) < 1e-5 and abs(h - np.log(V)) < 1e-4 and ids == [0, 1, 2]
            want = np.full(V, -1 / V)
            want[17] += 1
            assert np.abs(d[-1].double().cpu().numpy() - want).max() < (1e-3 if dtype == "bf16" else 1e-6)
        elif name == "nan":
            assert np.isnan([lp, h, lse] + lps).all() and 4000 not in ids and d[-1].isnan().all()
            good = torch.topk(base[-1].float().index_fill(0, torch.tensor([4000], device="cuda"), -9e9), 3).values
            assert torch.equal(base[-1].float()[r.top_ids[-1].long()], good)
        elif name == "all nan":
            assert np.isnan([lp, h, lse]).all() and ids == [NO_TOKEN] * 3
        elif name == "inf":
            assert np.isnan([lp, h, lse]).all() and ids[0] == 3000
        else:
            assert (lp, h, ids, lps[0]) == (-float("inf"), 0.0, [4999, NO_TOKEN, NO_TOKEN], 0.0) and abs(lse - 2) < 1e-6
            want = torch.zeros(V, device="cuda")
            want[17] = 1.0  # (the target cannot occur, but its logit is asked to grow)
            want[4999] = -1.0
            assert torch.equal(d[-1].float(), want)
        if rows > 1 and name in ("nan", "inf"):  # the other rows are as they were
            clean = L.token_logprobs(base, target, top=3)
            assert torch.equal(clean.entropy[:-1], r.entropy[:-1]) and torch.equal(clean.top_ids[:-1], r.top_ids[:-1])
    L.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "masked", "flat", "large"])
def test_gradient_against_its_formula(torch, dtype, kind):
    from paper_2512_14681_gb300 import logprobs as L

    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    for n, (rows, V, pad, shift, _, scale) in enumerate(SHAPES):
        rng = np.random.default_rng(100 + n)
        x = place(torch, logits(rng, rows, V, dtype, kind), t, pad, shift)
        z = x.double().cpu().numpy()
        targets = rng.integers(-1, V, rows)
        g, gh = rng.standard_normal(rows).astype(np.float32), rng.standard_normal(rows).astype(np.float32)
        tt, tg, th = (torch.from_numpy(v).cuda() for v in (targets.astype(np.int32), g, gh))
        r = L.token_logprobs(x, tt, scale=scale)
        _, H, _, lp, p, _ = reference(z, targets, np.float32(scale).astype(np.float64), 0)
        some = (z.max(1) > -np.inf)[:, None]
        hot = np.zeros_like(p)
        hot[np.arange(rows)[targets >= 0], targets[targets >= 0]] = 1
        gt = np.where(targets >= 0, g, 0)[:, None]
        for mine_g, mine_h in ((tg, th), (tg, None), (None, th)):
            a, b = (gt if mine_g is not None else 0 * gt), (gh[:, None] if mine_h is not None else 0 * gt)
            with np.errstate(all="ignore"):
                plogp = np.where(p > 0, p * (lp + H[:, None]), 0)
                want = scale * np.where(some, a * (hot - p) - b * plogp, 0)
                size = scale * (np.abs(a) * (hot + p) + np.abs(b) * np.where(p > 0, p * (np.abs(lp) + H[:, None] + 1), 0))
            tol = size * (2e-5 + (2.0 ** -8 if dtype == "bf16" else 0)) + 1e-37
            # into fresh memory, into rows that lie differently, and in place
            out = place(torch, np.zeros((rows, V)), t, 5, 2)
            for o in (None, out, x.clone()):
                src = o if o is not None and o.shape == x.shape and o is not out else x
                d = L.token_logprobs_grad(src, tt, r.row_stats, r.entropy, mine_g, mine_h, scale=scale, out=o)
                assert (np.abs(d.double().cpu().numpy() - want) <= tol).all(), (rows, V)
    L.check()


def test_gradient_against_differences(torch):
    """Central differences of the kernel's own logprob and entropy, step 2^-6: their error is 2^-12 / 6 of the third
    derivative (at most 1 / 4 here) plus 2 * 4e-6 / 2^-5 of the values' rounding."""
    from paper_2512_14681_gb300 import logprobs as L

    V, h = 40, 2.0 ** -6
    x = torch.randn(1, V, device="cuda") * 1.5
    target = torch.tensor([7], dtype=torch.int32, device="cuda")
    r = L.token_logprobs(x, target, scale=0.8)
    for g, gh in ((1.0, None), (None, 1.0), (0.7, -0.4)):
        d = L.token_logprobs_grad(x, target, r.row_stats, r.entropy, g, gh, scale=0.8)[0]
        up, down = x.repeat(V, 1) + h * torch.eye(V, device="cuda"), x.repeat(V, 1) - h * torch.eye(V, device="cuda")
        a, b = (L.token_logprobs(v, target.repeat(V), scale=0.8) for v in (up, down))
        num = ((g or 0) * (a.logprob - b.logprob) + (gh or 0) * (a.entropy - b.entropy)) / (2 * h)
        assert (num - d).abs().max() < 2.0 ** -12 / 6 + 2 * 4e-6 * (1 + float(r.lse.abs())) / (2 * h)


def test_other_streams_and_padding_stays(torch):
    from paper_2512_14681_gb300 import logprobs as L

    x = torch.randn(3, 9000, device="cuda")
    target = torch.tensor([5, -1, 8999], dtype=torch.int32, device="cuda")
    want = L.token_logprobs(x, target, top=4)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        late = torch.zeros_like(x)
        torch.cuda._sleep(2_000_000)
        late.copy_(x)
    got = L.token_logprobs(late, target, top=4, stream=st)
    out = torch.full((3, 9003), 7.0, device="cuda")
    st.wait_stream(torch.cuda.current_stream())
    L.token_logprobs_grad(late, target, got.row_stats, got.entropy, 1.0, out=out[:, 1:9001], stream=st)
    st.synchronize()
    assert torch.equal(got.logprob, want.logprob) and torch.equal(got.top_ids, want.top_ids)
    assert (out[:, 0] == 7).all() and (out[:, 9001:] == 7).all() and not out[1, 1:9001].any()


def test_refusals_and_targets_beyond_the_vocabulary(torch):
    from paper_2512_14681_gb300 import _lib as J
    from paper_2512_14681_gb300 import logprobs as L

    x = torch.randn(2, 50, device="cuda")
    target = torch.tensor([3, 50], dtype=torch.int32, device="cuda")
    r = L.token_logprobs(x, target)
    with pytest.raises(J.JfError, match="vocabulary"):
        L.check()
    L.check()
    assert r.logprob.isnan().tolist() == [False, True] and not r.entropy.isnan().any()
    L.token_logprobs_grad(x, target, r.row_stats, r.entropy, 1.0)
    with pytest.raises(J.JfError, match="vocabulary"):
        L.check()
    good = torch.tensor([3, 4], dtype=torch.int32, device="cuda")

    def refused(status, f):
        with pytest.raises(J.JfError) as e:
            f()
        assert e.value.status == status, e.value

    inv = J.JF_EINVAL
    refused(inv, lambda: L.token_logprobs(x, good[:1]))
    refused(inv, lambda: L.token_logprobs(x, good.long()))
    refused(inv, lambda: L.token_logprobs(x.t(), good))
    refused(inv, lambda: L.token_logprobs(x, good, top=65))
    refused(inv, lambda: L.token_logprobs(x, good, scale=0.0))
    refused(inv, lambda: L.token_logprobs(x, good, scale=float("nan")))
    refused(J.JF_EUNSUPPORTED, lambda: L.token_logprobs(x.half(), good))
    refused(inv, lambda: L.token_logprobs_grad(x, good, r.row_stats, r.entropy[:1], 1.0, 1.0))
    refused(inv, lambda: L.token_logprobs_grad(x, good, r.row_stats, r.entropy, 1.0, out=x.bfloat16()))
    assert L.token_logprobs(x[:0], good[:0], top=2).top_ids.shape == (0, 2)
    torch.cuda.synchronize()
    L.check()
