"""The policy loss over the whole range of its arguments, against plain 64-bit arithmetic (bounds: tests/test_gpu_policy.py).

fp32 rows of up to 230,400 logits (bf16 460,800) are one kernel's, longer ones three kernels': every case runs on both."""
import math

import pytest

from tests.packed_ref import U, half_step, inside
from tests.parity import need_gpu
from tests.test_gpu_policy import NAMES, call, make, reference

pytestmark = pytest.mark.gpu
DTYPES = ["float32", "bfloat16"]


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


def on(torch, logits, target, old=0.0, ref=0.0, adv=1.0, weight=1.0):
    """A call's inputs; what is a number is every row's."""
    rows = logits.shape[0]
    f = lambda x: x if isinstance(x, torch.Tensor) else torch.full((rows,), float(x), device="cuda")
    t = target if isinstance(target, torch.Tensor) else torch.full((rows,), target, dtype=torch.int32, device="cuda")
    return dict(logits=logits, targets=t, old=f(old), ref=f(ref), adv=f(adv), weight=f(weight))


def apart(z):
    """Logits as 64-bit differences from their row's largest (beside which 64 bits may hold no logarithm of a sum)."""
    return z.double() - z.double().amax(1, keepdim=True)


def held(torch, s, what, **kw):
    got = call(torch, s, **kw)
    want, bounds = reference(torch, {**s, "logits": apart(s["logits"])}, 0.2, 0.28, kw["kl"], kw["eta"], kw["scale"])
    bounds[5] = bounds[5] + half_step(torch, s["logits"].dtype) * want[5].abs()
    for x, v, b, name in zip(got, want, bounds, NAMES):
        inside(torch, x, v, b, f"{name} {what}")
    return got


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("top", [1.1e7, 1.2e7, 2.3e7, 2.4e7, 1e9, 4e9, 1.3e10, 7.7e12, 3e20, 9e28, 2e29, 9e37, 2e38])
@pytest.mark.parametrize("vocab", [9, 5001, 300001, 470001])
def test_large_logits(torch, dtype, top, vocab):
    """Logits a few of the type's steps apart, as far as a step still counts beside the largest; of either sign, at scale 1 and at one
    that brings them to 2^24 or below."""
    dtype = getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(vocab)
    step = torch.finfo(dtype).eps * 2.0 ** math.floor(math.log2(top))
    for sign in (1, -1):
        z = (sign * top - step * torch.randint(0, 30, (4, vocab), generator=g, device="cuda").double()).to(dtype)
        z[1, ::3] = -math.inf
        target = z.float().argmax(1)
        lp = lambda scale: torch.log_softmax(apart(z) * scale, 1).gather(1, target[:, None])[:, 0]
        for scale in (1.0, max(2.0 ** -math.ceil(math.log2(step)), 2.0 ** -92)):
            s = on(torch, z, target.int(), old=(lp(scale) + 0.05).float(), ref=(lp(scale) - 0.1).float(), adv=torch.tensor([1.0, -1.0, 0.5, 2.0], device="cuda"))
            held(torch, s, (sign, scale), kl=0.05, eta=0.01, scale=scale)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [1e-28, 1e-10, 1e3, 1e4, 1e5, 6e5, 1e7, 1e12, 1e30])
@pytest.mark.parametrize("vocab", [11, 5001, 300001, 470001])
def test_masks_at_any_scale(torch, dtype, scale, vocab):
    """Scores around 1 whatever the scale, a third of them masked out, with an entropy term of weight 0.1."""
    dtype = getattr(torch, dtype)
    scale = torch.tensor(scale, dtype=torch.float32).item()
    g = torch.Generator(device="cuda").manual_seed(vocab)
    z = (torch.randn(6, vocab, generator=g, device="cuda").double() * 2 / scale).to(dtype)
    f = torch.rand(6, vocab, generator=g, device="cuda")
    z[f < 0.3] = -math.inf
    z[f > 0.95] = torch.finfo(dtype).min
    target = z.float().argmax(1)
    lp = torch.log_softmax(apart(z) * scale, 1).gather(1, target[:, None])[:, 0]
    s = on(torch, z, target.int(), old=(lp + 0.05).float(), ref=(lp - 0.1).float(), adv=torch.tensor([1.0, -1.0, 0.5, 2.0, 0.0, 1.0], device="cuda"))
    got = held(torch, s, scale, kl=0.05, eta=0.1, scale=scale)
    assert (got.grad[z == -math.inf] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [1e-28, 3e-28, 1e-20, 1.0, 1e5])
@pytest.mark.parametrize("vocab", [11, 5001, 300001, 470001])
def test_small_logits_beside_large_ones(torch, dtype, scale, vocab):
    """Rows of scores around -9, 0 and 9 whose every 16-byte vector but one lies 10 to 40 lower: what they add counts, at any scale. Targets
    that are the type's lowest value are as far as they are."""
    dtype = getattr(torch, dtype)
    scale = torch.tensor(scale, dtype=torch.float32).item()
    g = torch.Generator(device="cuda").manual_seed(vocab)
    z = -10 - 30 * torch.rand(6, vocab, generator=g, device="cuda", dtype=torch.float64)
    z[:, :4] = torch.rand(6, 4, generator=g, device="cuda", dtype=torch.float64)
    z += torch.tensor([-9, 0, 9, -9, 0, 9], device="cuda")[:, None]
    z = (z / scale).to(dtype)
    target = torch.tensor([0, 1, 2, 3, 0, 5], device="cuda")
    z[5, 5] = torch.finfo(dtype).min
    lp = torch.log_softmax(apart(z) * scale, 1).gather(1, target[:, None])[:, 0]
    s = on(torch, z, target.int(), old=(lp + 0.05).float(), ref=(lp - 0.1).float(), adv=torch.tensor([1.0, -1.0, 0.5, 2.0, 0.0, 1.0], device="cuda"))
    first = {k: x[:5] for k, x in s.items()}
    held(torch, first, scale, kl=0.05, eta=0.1, scale=scale)
    got, want = call(torch, s, kl=0.0, eta=0.0, scale=scale).logprob[5].item(), lp[5].item()
    assert abs(got - want) <= 8 * U * abs(want) + 2.0 ** -18 or (want < -3.4e38 and got == -math.inf), (got, want)
    if vocab < 200000 and scale < 1e-20:  # a target as far below as the type goes
        z[5, 1] = 2e38
        got, want = call(torch, s, kl=0.0, eta=0.0, scale=scale).logprob[5].item(), (z[5, 5].double() - z[5, 1].double()).item() * scale
        assert abs(got - want) <= 8 * U * abs(want), (got, want)


def masked(torch, dtype, vocab, first=1):
    """Rows at an odd address, a third of them masked out by -infinity and by the type's lowest value, on tokens from 8 on."""
    s = make(torch, 8, vocab, dtype, seed=21, pad=2, first=first, masked=True)
    z = s["logits"]
    z[:, :8] = torch.linspace(-1, 1, 8, device="cuda").to(dtype)
    s["targets"].fill_(3)
    out = (z == -math.inf) | (z == torch.finfo(dtype).min)
    assert out[:, vocab - 8:].any() and (vocab < 100 or out[:, -2:].any())
    return s, out


LONG = [60, 5001, 300001, 470001]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", LONG)
@pytest.mark.parametrize("eta", [0.0, 0.01])
def test_an_infinite_ratio_moves_no_token_of_probability_0(torch, dtype, vocab, eta):
    """A < 0: the gradient is infinite, towards the target and away from the others that can occur, and 0 at those that cannot. (Of a row with
    one token that can occur, what rounding of its entropy leaves: the exponential's 2^-22 and a few steps of fp32.)"""
    dtype = getattr(torch, dtype)
    s, out = masked(torch, dtype, vocab)
    s["old"].fill_(-1e30), s["adv"].fill_(-1.0)
    got = call(torch, s, kl=0.0, eta=eta)
    assert (got.ratio == math.inf).all() and (got.loss == math.inf).all()
    assert (got.grad[out] == 0).all() and (got.grad[:, 3] == math.inf).all()
    assert (got.grad[:, :3] == -math.inf).all() and not torch.isnan(got.grad).any()
    s["logits"][:, 4:] = -math.inf  # one token that can occur has probability 1: nothing moves it
    s["logits"][:, :3] = -math.inf
    got = call(torch, s, kl=0.0, eta=eta)
    assert got.grad.abs().max() <= eta * 16 * U and got.logprob.abs().max() <= 8 * U


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", LONG)
@pytest.mark.parametrize("scale", [1.0, 1.25])
def test_an_infinite_kl_has_no_gradient(torch, dtype, vocab, scale):
    """A target that the type's lowest value, -infinity or a distance of more than 88 puts out of fp32's range of e^d."""
    dtype = getattr(torch, dtype)
    s, out = masked(torch, dtype, vocab)
    z = s["logits"]
    z[0, 3], z[1, 3], z[2, 3], z[3, 3], z[4, 3] = torch.finfo(dtype).min, -math.inf, -95.0, -1000.0, -1e30
    s["ref"].fill_(0.0)
    for eta in (0.0, 0.01):
        got = call(torch, s, kl=0.05, eta=eta, scale=scale)
        without = call(torch, s, kl=0.0, eta=eta, scale=scale)
        assert (got.kl[:5] == math.inf).all() and (got.loss[:5] == math.inf).all()
        assert torch.equal(got.grad[:5], without.grad[:5]) and torch.isfinite(got.grad).all() and (got.grad[out] == 0).all()
    s["ref"][5:] = got.logprob[5:] + 80.0  # a large one that is not: held to the same bounds as any
    assert torch.isfinite(held(torch, {k: x[5:] for k, x in s.items()}, "80", kl=0.05, eta=0.01, scale=scale).loss).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", LONG)
def test_terms_that_are_no_numbers_reach_the_gradient(torch, dtype, vocab):
    """A loss of NaN goes with a gradient of NaN (at tokens that can occur), also without KL and entropy terms; a row's neighbours
    keep theirs."""
    dtype = getattr(torch, dtype)
    s, out = masked(torch, dtype, vocab)
    clean = call(torch, s, kl=0.0, eta=0.0)
    s["old"][1] = math.nan
    s["adv"][2] = math.nan
    s["logits"][3, 5] = math.nan
    s["logits"][4, vocab - 1] = math.inf
    s["weight"][5] = math.nan
    for eta in (0.0, 0.01):
        got = call(torch, s, kl=0.0, eta=eta)
        for row in range(1, 6):
            assert math.isnan(got.loss[row]) and torch.isnan(got.grad[row, :8]).all(), row
        assert not torch.isnan(got.loss[[0, 6, 7]]).any() and not torch.isnan(got.grad[[0, 6, 7]]).any()
        if eta == 0:
            assert torch.equal(got.grad[[0, 6, 7]], clean.grad[[0, 6, 7]])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", LONG)
def test_rows_that_are_left_out_hold_anything(torch, dtype, vocab):
    """A negative target or a weight of 0 makes a row's gradient 0 where its logits, its advantage or its old and reference log
    probabilities are NaN or infinite."""
    dtype = getattr(torch, dtype)
    s, _ = masked(torch, dtype, vocab)
    z = s["logits"]
    s["targets"][:4], s["weight"][4:] = -1, 0.0
    for row, bad in ((0, math.nan), (1, math.inf), (2, math.nan), (4, math.nan), (5, math.inf), (6, math.nan)):
        z[row, 2], z[row, vocab - 1], z[row, vocab // 2] = bad, bad, bad
    z[2], z[6] = math.nan, math.nan
    for name in ("old", "ref", "adv"):
        s[name][3], s[name][7] = math.nan, math.nan
    got = call(torch, s, kl=0.05, eta=0.01)
    assert (got.grad == 0).all() and (got.loss == 0).all()


@pytest.mark.parametrize("first", [0, 1, 3])
@pytest.mark.parametrize("dtype,vocab", [("float32", v) for v in (230400, 230403, 230404)] + [("bfloat16", v) for v in (460800, 460807, 460808)])
def test_both_sides_of_the_longest_row_of_one_kernel(torch, dtype, vocab, first):
    """Rows that fill a cluster's shared memory to the last vector, with elements beside it, and the first that do not fit."""
    s = make(torch, 3, vocab, getattr(torch, dtype), seed=22, pad=1, first=first, masked=True)
    held(torch, s, vocab, kl=0.05, eta=0.01, scale=1.0)
    want = call(torch, s)
    got = call(torch, s, out=s["logits"])
    assert torch.equal(got.grad, want.grad) and all(torch.equal(a, b) for a, b in zip(got[:5], want[:5]))


@pytest.mark.parametrize("which", ["token_logprobs", "policy_loss"])
def test_a_first_call_that_is_captured(torch, monkeypatch, which):
    """The error word of a device is there before the call that a graph keeps, and reports what a replay met."""
    from paper_2512_14681_gb300 import _lib as J
    from paper_2512_14681_gb300 import logprobs as L

    s = make(torch, 4, 300, torch.float32, seed=23)
    run = (lambda: call(torch, s)) if which == "policy_loss" else (lambda: L.token_logprobs(s["logits"], s["targets"]))
    want = run()
    torch.cuda.synchronize()
    monkeypatch.setattr(L, "_err", {})
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    graph.replay()
    L.check()
    for a, b in zip(got, want):
        assert a is b is None or torch.equal(a, b)
    s["targets"][1] = 300
    graph.replay()
    with pytest.raises(J.JfError, match="vocabulary"):
        L.check()
    L.check()
    del graph, got  # the word outlives the graph
    torch.cuda.empty_cache()
    run()
    with pytest.raises(J.JfError, match="vocabulary"):
        L.check()
    L.check()


def test_check_names_what_was_reported(torch, monkeypatch):
    """A wait that ran out is not a target beyond the vocabulary. (The codes are written into the word by hand.)"""
    from paper_2512_14681_gb300 import _lib as J
    from paper_2512_14681_gb300 import logprobs as L

    dev = torch.device("cuda", torch.cuda.current_device())
    for code, status, what in ((4, J.JF_EDEVICE, "vocabulary"), (1, J.JF_ETIMEOUT, "wait")):
        L._error_word(dev).fill_(code)
        with pytest.raises(J.JfError, match=what) as e:
            L.check()
        assert e.value.status == status
        L.check()
