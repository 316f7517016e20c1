"""The clipped policy loss and its gradient against plain 64-bit arithmetic.

u = 2^-24. With z = scale * logit, m its largest and S = sum e^(z - m): a term is off by |z - m| 3 u (product, difference, base of
the logarithm) and 2^-22 (the exponential), the sum by (V / 256 + 32) u, whichever way it is split, so
  ln S: E = sum p |z - m| 3 u + 2^-22 + (V / 256 + 32) u;   lp: E + 4 u (|z_t - m| + ln S);   H: E + sum p |z - m| (|z - m| 3 u + E') + 8 u (H + ln S)
ratio, kl and loss take lp's error with their slopes and a few u of their parts; the gradient that of p (relative: E + 4 u |ln p| + 2^-22)."""
import math

import pytest

from tests.packed_ref import U, half_step, inside
from tests.parity import need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


def make(torch, rows, vocab, dtype, seed=0, pad=0, masked=False, scale=1.0, first=0, below=0.2, above=0.28):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.randn(rows * (vocab + pad) + first, generator=g, device="cuda") * 3
    z = buf[first:].view(rows, vocab + pad)
    if masked:
        f = torch.rand(z.shape, generator=g, device="cuda")
        z[f < 0.3] = -math.inf
        z[f > 0.9] = torch.finfo(dtype).min
    target = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    z.scatter_(1, target[:, None], torch.rand(rows, 1, generator=g, device="cuda") * 4)
    buf = buf.to(dtype)
    z = buf[first:].view(rows, vocab + pad)[:, :vocab]
    lp = torch.log_softmax(z.double() * scale, 1).gather(1, target[:, None])[:, 0]
    x = torch.randn(rows, generator=g, device="cuda", dtype=torch.float64) * 0.3
    for border in (math.log(max(1 - below, 1e-9)), math.log(1 + above)):
        x = torch.where((x - border).abs() < 1e-3, x + 3e-3, x)
    f32 = lambda t: t.float()
    target[5::7] = -1
    return dict(logits=z, targets=target.int(), old=f32(lp - x), ref=f32(lp + torch.randn(rows, generator=g, device="cuda", dtype=torch.float64) * 0.5),
                adv=torch.randn(rows, generator=g, device="cuda"), weight=torch.rand(rows, generator=g, device="cuda"))


def reference(torch, s, below, above, kl, eta, scale, weight=True, ref=True, old=True):
    """(values, bounds) of loss, logprob, entropy, ratio, kl and the gradient."""
    z = s["logits"].double() * scale
    V = z.shape[1]
    t = s["targets"].long()
    on = t >= 0
    m = z.amax(1, keepdim=True)
    lse = torch.logsumexp(z, 1, keepdim=True)
    logp = z - lse
    p = torch.exp(logp)
    few = torch.where(p > 0, (z - m).abs(), 0.0)
    H = torch.special.entr(p).sum(1)
    lnS = (lse - m)[:, 0]
    sums = (V / 256 + 32) * U
    E = (p * few).sum(1) * 3 * U + 2.0 ** -22 + sums
    E_H = E + (p * few * (few * 3 * U + 2.0 ** -22 + 2 * sums)).sum(1) + 8 * U * (H + lnS)
    at = t.clamp(min=0)[:, None]
    lp = torch.where(on, logp.gather(1, at)[:, 0], 0.0)
    E_lp = torch.where(on, E + 4 * U * ((z - m).gather(1, at)[:, 0].abs() + lnS), 0.0)
    A = s["adv"].double()
    w = torch.where(on, s["weight"].double() if weight else torch.ones_like(A), 0.0)
    x = lp - s["old"].double() if old else torch.zeros_like(lp)
    r = torch.where(on, torch.exp(x), 0.0)
    E_r = r * (E_lp + 2 * U * x.abs() + 8 * U) if old else torch.zeros_like(r)
    free, held = r * A, r.clamp(1 - below, 1 + above) * A
    runs = free <= held
    loss, E_loss = -torch.minimum(free, held), torch.where(runs, A.abs() * E_r, 0.0) + 4 * U * held.abs() + 4 * U * free.abs()
    g, E_g = -torch.where(runs, free, 0.0), torch.where(runs, A.abs() * E_r + 4 * U * free.abs(), 0.0)
    k, E_k = torch.zeros_like(lp), torch.zeros_like(lp)
    if ref:
        d = s["ref"].double() - lp
        e = torch.expm1(d)
        k = torch.where(on, e - d, 0.0)
        E_d = E_lp + U * d.abs()
        E_k = torch.where(on, e.abs() * E_d + 4 * U * (e.abs() + d.abs()), 0.0)
        loss, E_loss = loss + kl * k, E_loss + kl * (E_k + 4 * U * k)
        g, E_g = g - kl * e, E_g + kl * ((1 + e.abs()) * E_d + 4 * U * e.abs())
    E_loss = E_loss + abs(eta) * E_H + 4 * U * (loss.abs() + abs(eta) * H)
    loss = w * (loss - eta * H)
    g, E_g = w * g, w * (E_g + 4 * U * g.abs())
    P = p * (E[:, None] + 4 * U * torch.where(p > 0, logp.abs(), 0.0) + 2.0 ** -22)
    hot = torch.zeros_like(p).scatter_(1, at, on.double()[:, None])
    share = torch.where(p > 0, p * (logp + H[:, None]), 0.0)
    dz = scale * (g[:, None] * (hot - p) + (w * eta)[:, None] * share)
    lpf = torch.where(p > 0, logp.abs(), 0.0)
    t_dz = scale * (E_g[:, None] * (hot + p) + g.abs()[:, None] * (P + 4 * U * (hot + p)) +
                    (w * abs(eta))[:, None] * (P * (lpf + H[:, None]) + p * (E[:, None] + 4 * U * lpf + E_H[:, None]) + 4 * U * p * (lpf + H[:, None])))
    t_dz = t_dz + half_step(torch, s["logits"].dtype) * dz.abs() + 1e-37
    values = [loss, lp, H, r, k, dz]
    bounds = [w * E_loss + 4 * U * loss.abs() + 1e-37, E_lp, E_H, E_r + 1e-37, E_k, t_dz]
    return values, bounds


NAMES = ("loss", "logprob", "entropy", "ratio", "kl", "grad")


def call(torch, s, below=0.2, above=0.28, kl=0.05, eta=0.01, scale=1.0, weight=True, ref=True, old=True, **more):
    from paper_2512_14681_gb300 import logprobs as L

    return L.policy_loss(s["logits"], s["targets"], s["old"] if old else None, s["adv"], weight=s["weight"] if weight else None,
                         ref_logprob=s["ref"] if ref else None, below=below, above=above, kl=kl, entropy=eta, scale=scale, **more)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,vocab,pad,first,masked,scale", [(1, 1, 0, 0, False, 1.0), (3, 7, 0, 0, False, 1.0), (9, 100, 3, 1, True, 0.7), (16, 4096, 0, 0, False, 1.0),
                                                               (40, 5001, 2, 3, True, 1.25), (5, 32769, 1, 0, False, 1.0), (33, 151936, 0, 0, True, 1.0), (30, 152063, 2, 0, False, 1.25),
                                                               (300, 20011, 0, 1, False, 1.0), (700, 40000, 0, 0, True, 1.0), (2, 400003, 1, 1, False, 1.0), (3, 1100000, 0, 0, False, 1.0)])
def test_against_64_bits(torch, dtype, rows, vocab, pad, first, masked, scale):
    from paper_2512_14681_gb300 import logprobs as L

    s = make(torch, rows, vocab, getattr(torch, dtype), pad=pad, first=first, masked=masked, scale=scale)
    for terms in (dict(kl=0.0, eta=0.0), dict(kl=0.05, eta=0.01), dict(kl=0.0, eta=0.02, weight=False, ref=False), dict(kl=0.1, eta=0.0, old=False)):
        kw = dict(below=0.2, above=0.28, scale=scale, **terms)
        got = call(torch, s, **kw)
        want, bounds = reference(torch, s, **kw)
        for x, v, b, name in zip(got, want, bounds, NAMES):
            inside(torch, x, v, b, f"{name} {terms}")
    L.check()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("below,above", [(0.0, 0.0), (1.0, 1e30), (0.2, 0.2)])
def test_borders(torch, dtype, below, above):
    """Nothing counts beyond 1, everything does, and both signs of the advantage beyond either border."""
    s = make(torch, 60, 3001, getattr(torch, dtype), seed=1, below=below, above=above if above < 1e9 else 0.2)
    got = call(torch, s, below=below, above=above, kl=0.0, eta=0.0)
    want, bounds = reference(torch, s, below, above, 0.0, 0.0, 1.0)
    for x, v, b, name in zip(got, want, bounds, NAMES):
        inside(torch, x, v, b, name)
    if below == 0.2:
        on, r, A = s["targets"] >= 0, want[3], s["adv"]
        still = on & (((r > 1.2) & (A > 0)) | ((r < 0.8) & (A < 0)))
        assert still.any() and (got.grad[still] == 0).all()


def test_without_a_gradient_and_in_place(torch):
    s = make(torch, 20, 2000, torch.float32, seed=2, pad=5)
    want = call(torch, s)
    alone = call(torch, s, want_grad=False)
    assert alone.grad is None and all(torch.equal(a, b) for a, b in zip(alone[:5], want[:5]))
    room = torch.full((20, 2003), 9.0, device="cuda")
    got = call(torch, s, out=room[:, 1:2001])
    assert torch.equal(got.grad, want.grad) and (room[:, 0] == 9).all() and (room[:, 2001:] == 9).all()
    got = call(torch, s, out=s["logits"])
    assert got.grad is s["logits"] and torch.equal(s["logits"], want.grad) and all(torch.equal(a, b) for a, b in zip(got[:5], want[:5]))


@pytest.mark.parametrize("dtype,vocab", [("float32", 500000), ("float32", 460803), ("bfloat16", 930001), ("bfloat16", 300000), ("float32", 11)])
def test_in_place_at_any_length(torch, dtype, vocab):
    """... beside rows that a cluster holds as well; 2 rows whose distance passes the vocabulary by an odd number."""
    s = make(torch, 2, vocab, getattr(torch, dtype), seed=8, pad=3)
    beside = s["logits"].as_strided((2, 3), (vocab + 3, 1), s["logits"].storage_offset() + vocab)[:1].clone()
    want = call(torch, s)
    got = call(torch, s, out=s["logits"])
    assert torch.equal(s["logits"], want.grad) and all(torch.equal(a, b) for a, b in zip(got[:5], want[:5]))
    assert torch.equal(s["logits"].as_strided((2, 3), (vocab + 3, 1), s["logits"].storage_offset() + vocab)[:1], beside)


@pytest.mark.parametrize("vocab", [1000, 500000])
def test_rows_further_apart_than_31_bits(torch, vocab):
    """Within the bounds, which hold for any split of a sum (the same bits only at the same alignment: a row's 16-byte vectors, and so the
    order of its sums, begin elsewhere)."""
    s = make(torch, 4, vocab, torch.bfloat16, seed=9)
    want, bounds = reference(torch, s, 0.2, 0.28, 0.05, 0.01, 1.0)
    apart = (1 << 30) + 3
    room = torch.empty(3 * apart + vocab, dtype=torch.bfloat16, device="cuda")
    far = room.as_strided((4, vocab), (apart, 1))
    far.copy_(s["logits"])
    got = call(torch, {**s, "logits": far}, out=far)
    for x, v, b, name in zip(got, want, bounds, NAMES):
        inside(torch, x, v, b, name)


@pytest.mark.parametrize("dtype,top", [("float32", 1e32), ("float32", 3.4e38), ("float32", -1e32), ("float32", 1e29), ("bfloat16", 1e31), ("bfloat16", -2e30), ("bfloat16", 3.3e38)])
@pytest.mark.parametrize("vocab", [9, 5000, 300000])
def test_logits_of_any_size(torch, dtype, top, vocab):
    """Two equal largest logits, the others lower by a step of the type or more (and so by more than e^-10000): halves and zeros. Also with
    a scale of 1e7 and logits around 1."""
    dtype = getattr(torch, dtype)
    z = torch.full((3, vocab), top, dtype=dtype, device="cuda")
    for row, scale in ((0, 1.0), (1, 1.0), (2, 1.0)):
        z[row] = z[row] - (abs(top) / 16 if row else abs(top) / 2)
        z[row, row], z[row, vocab - 1 - row] = top, top
    t = torch.arange(3, device="cuda").int()
    half = torch.full((3,), -math.log(2), device="cuda")
    for logits, scale in ((z, 1.0), ((z.float() / abs(top)).to(dtype), 1e7)):
        got = call(torch, dict(logits=logits, targets=t, old=half, ref=half, adv=torch.ones(3, device="cuda"), weight=torch.ones(3, device="cuda")), kl=0.0, eta=0.0,
                   scale=scale)
        # old rounds ln 2, log2 and its product with ln 2 round twice
        assert (got.logprob + math.log(2)).abs().max() <= 4 * U and (got.entropy - math.log(2)).abs().max() <= 4 * U and (got.ratio - 1).abs().max() <= 8 * U
        want = torch.zeros(3, vocab, dtype=torch.float64, device="cuda")
        for row in range(3):
            want[row, row], want[row, vocab - 1 - row] = -0.5 * scale, 0.5 * scale
        off = (got.grad.double() - want).abs().max()
        assert off <= scale * (16 * U + half_step(torch, dtype) * 0.5), (scale, off.item())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab", [50, 6001, 160000, 1000003])
def test_rows_that_are_left_out_or_are_no_numbers(torch, dtype, vocab):
    from paper_2512_14681_gb300 import _lib as J
    from paper_2512_14681_gb300 import logprobs as L

    s = make(torch, 12, vocab, getattr(torch, dtype), seed=3)
    s["targets"].copy_(torch.tensor([-1, 3, 3, 3, 3, 3, 3, 3, vocab, 3, 3, -7], dtype=torch.int32))
    z, inf = s["logits"], math.inf
    z[1] = -inf                      # no token can occur
    z[2, 3] = -inf                   # the target cannot
    z[3, 0] = math.nan
    z[4, vocab - 1] = inf
    s["weight"][5] = 0.0
    s["old"][5] = math.nan
    s["adv"][6] = 0.0
    s["old"][6] = -1e30              # ratio infinite
    z[7] = torch.finfo(z.dtype).min  # all equal, at the type's lowest value
    s["old"][7] = -math.log(vocab)
    s["ref"][7] = -math.log(vocab)
    s["old"][9], s["adv"][9] = -1e30, 1.0   # infinite, held at 1 + above
    s["old"][10], s["adv"][10] = -1e30, -1.0
    s["ref"][10] = -3.0
    got = call(torch, s, kl=0.05, eta=0.01)
    with pytest.raises(J.JfError, match="vocabulary"):
        L.check()
    loss, lp, H, r, k, g = got
    for row in (0, 11):
        assert loss[row] == lp[row] == r[row] == k[row] == 0 and H[row] > 0 and (g[row] == 0).all()
    assert (g[1] == 0).all() and lp[1] == -inf and H[1] == 0
    assert lp[2] == -inf and r[2] == 0 and k[2] == inf and loss[2] == inf and not torch.isnan(g[2]).any()
    for row in (3, 4):
        assert math.isnan(loss[row]) and math.isnan(lp[row]) and math.isnan(H[row])
    assert loss[5] == 0 and (g[5] == 0).all() and math.isfinite(lp[5]) and math.isnan(r[5])
    assert r[6] == inf and math.isfinite(loss[6]) and torch.isfinite(g[6]).all()
    assert abs(lp[7].item() + math.log(vocab)) < 1e-4 and abs(r[7].item() - 1) < 1e-4 and torch.isfinite(g[7]).all()
    assert math.isnan(loss[8]) and math.isnan(lp[8])
    assert r[9] == inf and math.isfinite(loss[9]) and torch.isfinite(g[9]).all()
    assert r[10] == inf and loss[10] == inf
    clean = call(torch, {**s, "targets": s["targets"].clamp(max=vocab - 1)}, kl=0.05, eta=0.01)
    for row in (0, 1, 2, 5, 6, 7, 9, 11):  # what a row holds reaches no other
        assert torch.equal(clean.grad[row], g[row])
    L.check()


def test_the_sum_s_gradient_by_differences(torch):
    """Along a direction, with steps h and 2 h: as in the attention's test; rounding of the losses counts over the step."""
    s = make(torch, 30, 700, torch.float32, seed=4)
    kw = dict(kl=0.2, eta=0.05)
    got = call(torch, s, **kw)
    _, bounds = reference(torch, s, 0.2, 0.28, 0.2, 0.05, 1.0)
    way = torch.randn(30, 700, device="cuda")
    way[(got.ratio - 0.8).abs() < 0.1] = 0  # (rows whose ratio meets a border on the way)
    way[(got.ratio - 1.28).abs() < 0.1] = 0
    z = s["logits"]
    loss = lambda t: call(torch, {**s, "logits": z + t * way}, want_grad=False, **kw).loss.double().sum().item()
    h = 2.0 ** -8
    near, wide = (loss(h) - loss(-h)) / (2 * h), (loss(2 * h) - loss(-2 * h)) / (4 * h)
    noise = bounds[0].sum().item() + (got.grad.double().abs() * (z.abs() + 1) * U).sum().item()
    assert abs((got.grad.double() * way).sum().item() - near) <= abs(near - wide) * 2 / 3 + 2 * noise / (2 * h)


@pytest.mark.parametrize("rows,vocab", [(2, 100), (200, 30000), (4, 152064)])
def test_the_same_bits_every_time(torch, rows, vocab):
    """Also from threads on streams of their own, and captured twice with an eager call in between."""
    import threading

    from paper_2512_14681_gb300 import logprobs as L

    s = make(torch, rows, vocab, torch.bfloat16, seed=5)
    want = call(torch, s)
    for _ in range(10):
        assert all(torch.equal(a, b) for a, b in zip(call(torch, s), want))
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        st = torch.cuda.Stream()
        for _ in range(20):
            got = call(torch, s, stream=st)
            st.synchronize()
            if not all(torch.equal(a, b) for a, b in zip(got, want)):
                wrong.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
    graphs, res = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            res.append(call(torch, s))
    s["adv"].neg_()
    want = call(torch, s)
    for g in graphs:
        g.replay()
    call(torch, s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for r in res for a, b in zip(r, want))
    L.check()


def test_calls_that_are_refused(torch):
    from paper_2512_14681_gb300 import _lib as J
    from paper_2512_14681_gb300 import logprobs as L

    s = make(torch, 4, 100, torch.float32, seed=6)
    z, t, old, A = s["logits"], s["targets"], s["old"], s["adv"]
    bad = [(J.JF_EINVAL, lambda: L.policy_loss(z, t, old[:3], A)), (J.JF_EINVAL, lambda: L.policy_loss(z, t, old.double(), A)),
           (J.JF_EINVAL, lambda: L.policy_loss(z, t.long(), old, A)), (J.JF_EINVAL, lambda: L.policy_loss(z, t, old, A, kl=0.1)),
           (J.JF_EINVAL, lambda: L.policy_loss(z, t, old, A, below=1.5)), (J.JF_EINVAL, lambda: L.policy_loss(z, t, old, A, above=-0.1)),
           (J.JF_EINVAL, lambda: L.policy_loss(z, t, old, A, entropy=math.nan)), (J.JF_EINVAL, lambda: L.policy_loss(z, t, old, A, scale=0.0)),
           (J.JF_EUNSUPPORTED, lambda: L.policy_loss(z.half(), t, old, A)), (J.JF_EINVAL, lambda: L.policy_loss(z.cpu(), t, old, A)),
           (J.JF_EINVAL, lambda: L.policy_loss(z, t, old, A, want_grad=False, out=z)), (J.JF_EINVAL, lambda: L.policy_loss(z, t, old, A, out=z.bfloat16())),
           (J.JF_EINVAL, lambda: L.policy_loss(z[:1].expand(4, 100), t, old, A)), (J.JF_EINVAL, lambda: L.policy_loss(z, t, old, A, out=z.new_empty(1, 100).expand(4, 100))),
           (J.JF_EUNSUPPORTED, lambda: L.policy_loss(z.detach().requires_grad_(), t, old, A))]
    for i, (status, f) in enumerate(bad):
        with pytest.raises(J.JfError) as e:
            f()
        assert e.value.status == status, i
    none = L.policy_loss(z[:0], t[:0], old[:0], A[:0])
    assert none.loss.shape == (0,) and none.grad.shape == (0, 100)
