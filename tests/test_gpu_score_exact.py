"""The scoring path on fp32 decoders against the same layers in 64 bits.

Keys and values: what the cache holds is within half a code step of what a 64-bit forward over the same cached values
computes (e4m3: 2^-4 of a value, or 2^-10 of its block's unit 2^e), plus fp32's error of the layers before. Log
probabilities: attention in 64 bits over the values that the cache holds, so that rounding to 8 bits is on both sides; what
differs is fp32 arithmetic, some 2^-24 * sqrt(128 * layers) of numbers of size 1 to 10 in sums of up to 1,000 terms: 1e-3
is far above it and far below what one code or exponent in the wrong place makes of a token.
"""
import numpy as np
import pytest

from paper_2512_14681_gb300 import inputs as I
from tests.parity import need_gpu

pytestmark = pytest.mark.gpu


def forward64(torch, s, text, caches):
    """Log probabilities of every position's vocabulary, and each layer's rotated keys and values."""
    shape, hd = s.shape, s.shape.head_dim
    Hq, Hkv, n = shape.n_heads, shape.n_kv_heads, len(text)
    norm = lambda x, g: x / (x.square().mean(-1, keepdim=True) + shape.rms_eps).sqrt() * g.double()
    cs = s.rope[:n].double()
    c, d = cs[:, None, :, 0], cs[:, None, :, 1]

    def turn(x):
        a, b = x[..., :hd // 2], x[..., hd // 2:]
        return torch.cat([a * c - b * d, b * c + a * d], -1)

    late = torch.ones(n, n, device="cuda").triu(1).bool()
    x = s.embedding[torch.tensor(text, device="cuda")].double()
    kvs = []
    for w, (ck, cv) in zip(s.layers, caches):
        qkv = norm(x, w["n1"]) @ w["qkv"].double().T + (w["b"].double() if "b" in w else 0)
        q, k, v = (t.view(n, -1, hd) for t in qkv.split([Hq * hd, Hkv * hd, Hkv * hd], 1))
        kvs.append((turn(k), v))
        ck, cv = (t.double().repeat_interleave(Hq // Hkv, 1) for t in (ck, cv))
        p = torch.softmax((torch.einsum("rhd,khd->hrk", turn(q), ck) * hd ** -0.5).masked_fill(late, -float("inf")), -1)
        x = x + torch.einsum("hrk,khd->rhd", p, cv).reshape(n, -1) @ w["o"].double().T
        g, u = (norm(x, w["n2"]) @ w["gu"].double().T).chunk(2, 1)
        x = x + (g * torch.sigmoid(g) * u) @ w["down"].double().T
    return torch.log_softmax(norm(x, s.final_gain) @ s.head.double().T, -1), kvs


@pytest.mark.parametrize("shape", [I.TINY_F32, I.TINY_F32_BT], ids=lambda s: s.name)
def test_scores_against_64_bit_layers(shape):
    torch = need_gpu()
    from paper_2512_14681_gb300.jacobi import Context
    from paper_2512_14681_gb300.kv8 import Rows
    from paper_2512_14681_gb300.score import Scorer

    ctx = Context(shape, max_ctx=128, max_rows=128, logits_rows=128)
    ctx.init_random_weights(I.WEIGHT_SEED, I.WEIGHT_STD)
    s = Scorer(shape, lambda tid, n: ctx.get_weights(tid, 0, n), max_ctx=128)
    ctx.close()
    n = 90
    text = I.prompt_tokens(shape.vocab, n + 1, 8).tolist()
    # (one chunk: no block grows, and is rounded again, after a row has attended to it)
    got = s.score([text[:n]], [text[1:]]).logprob
    s.check()
    held = [c.read(Rows.of([n], [0])) for c in s.caches]
    lp, kvs = forward64(torch, s, text[:n], held)
    want = lp[torch.arange(n), torch.tensor(text[1:], device="cuda")]
    assert (got.double() - want).abs().max() < 1e-3
    for cache, mine, theirs in zip(s.caches, held, kvs):
        pages = cache.page_table[0, torch.arange(n, device="cuda") // 16].long()
        for e, a, b in zip((cache.k_exp, cache.v_exp), mine, theirs):
            unit = torch.exp2(e[pages].double())[..., None]
            assert ((a.double() - b).abs() <= torch.maximum(b.abs() * 2.0 ** -4, unit * 2.0 ** -10) + 1e-4).all()
