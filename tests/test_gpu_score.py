"""The scoring path (append -> attention -> head -> log probabilities) run together on small decoders.

The 8-bit cache changes keys and values by up to 2^-4 of themselves (half a step of 3 mantissa bits), at random: the small
random models' log probabilities then differ from the 16-bit cache's by a few hundredths (attention adds a fraction of the
residual stream here, N(0, 0.02) weights); 0.25 nats on any token would be another computation.
"""
import numpy as np
import pytest

from paper_2512_14681_gb300 import inputs as I
from tests.parity import need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", params=[I.SMALL_BF16, I.SMALL_BF16_BT, I.TINY_F32, I.TINY_F32_BT], ids=lambda s: s.name)
def models(request):
    need_gpu()
    from paper_2512_14681_gb300.jacobi import Context
    from paper_2512_14681_gb300.score import Scorer

    shape = request.param
    ctx = Context(shape, max_ctx=160, max_rows=128, logits_rows=128)
    ctx.init_random_weights(I.WEIGHT_SEED, I.WEIGHT_STD)
    make = lambda **kw: Scorer(shape, lambda tid, n: ctx.get_weights(tid, 0, n), max_ctx=160, **kw)
    yield ctx, make
    ctx.close()


def log_softmax64(x):
    x = x.astype(np.float64)
    m = x.max(-1, keepdims=True)
    return x - m - np.log(np.exp(x - m).sum(-1, keepdims=True))


def test_scores_follow_the_16_bit_cache(models):
    ctx, make = models
    text = I.prompt_tokens(ctx.shape.vocab, 101).tolist()
    s = make()
    ctx.truncate(0, 0)
    logits = ctx.forward_logits(0, text[:100], want_hidden=False)[0]
    want = log_softmax64(logits)[np.arange(100), text[1:]]
    got = []
    for c in range(0, 100, 37):  # (chunks that end inside a page)
        r = s.score([text[c:min(c + 37, 100)]], [text[c + 1:min(c + 37, 100) + 1]], top=4)
        got.append(r.logprob.double().cpu().numpy())
        assert (r.top_logprobs[:, 0] >= r.logprob - 1e-5).all() and (r.top_logprobs.diff(dim=1) <= 0).all()
    s.check()
    assert np.abs(np.concatenate(got) - want).max() < 0.25
    # in one chunk, and after a rejected draft: the same cache up to its blocks' exponents
    one = make()
    one.hidden([text[:20]])
    one.hidden([[1, 2, 3, 4, 5]])
    one.truncate([20])
    r = one.score([text[20:100]], [text[21:101]])
    one.check()
    assert np.abs(r.logprob.double().cpu().numpy() - want[20:]).max() < 0.25


def test_two_sequences_score_as_each_alone(models):
    ctx, make = models
    a, b = I.prompt_tokens(ctx.shape.vocab, 61, 3).tolist(), I.prompt_tokens(ctx.shape.vocab, 24, 4).tolist()
    both, alone = make(n_seqs=2), make(n_seqs=2)
    r = both.score([a[:60], b[:23]], [a[1:], b[1:]])
    one = alone.score([a[:60], []], [a[1:], []])
    two = alone.score([[], b[:23]], [[], b[1:]])
    both.check()
    alone.check()
    got, want = r.logprob.cpu().numpy(), np.concatenate([one.logprob.cpu().numpy(), two.logprob.cpu().numpy()])
    # (rows share tiles and splits differently: roundings of the 16-bit activations)
    assert np.abs(got - want).max() < (3e-2 if ctx.shape.bf16 else 1e-4)


def test_the_heads_gradient_lowers_the_loss(models):
    ctx, make = models
    text = I.prompt_tokens(ctx.shape.vocab, 41, 5).tolist()
    s = make()
    loss, grad = s.head_gradient([text[:40]], [text[1:]])
    s.truncate([0])
    s.head = s.head.float().sub(grad * (0.5 / grad.norm() ** 2)).to(s.type).clone()  # a step that linearly takes 0.5 off
    after, _ = s.head_gradient([text[:40]], [text[1:]])
    s.check()
    assert 0.2 < float(loss - after) < 0.8


def test_the_command_runs(capsys, monkeypatch):
    need_gpu()
    import sys

    from paper_2512_14681_gb300 import score

    monkeypatch.setattr(sys, "argv", ["score", "--shape", "tiny-f32", "--tokens", "50", "--chunk", "32"])
    score.main()
    out = capsys.readouterr().out
    assert "mean difference" in out and "head gradient" in out
