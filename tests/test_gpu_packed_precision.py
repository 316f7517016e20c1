"""How far packed attention in bf16 is from 64 bits, in the norm of a whole batch: no further than the roundings that it states.

The same formulas are computed in 64 bits twice, exactly and with each stated rounding put in: probabilities (relative to a row's largest) before P v,
probabilities and the scores' gradients before dv, dk and dq (for dq two terms in a text's first quarter and its first 512 rows), each
output; delta is exact, but for dq of rows with more than 128 keys, whose delta comes from `out` as it was given. For rows that tensor
copies cannot read nothing but the outputs is rounded. The distance of these two is what the kernels may have. The roundings of a batch
are at least 10^5 independent ones, so that their norm varies by less than 2%; sums in fp32 add below 10^-5 of a norm. 8% is allowed,
which each of these would pass in one of the batches: ds of dq as one term (by 19 to 43%), delta from the rounded `out` for rows of up to
128 keys (by 9 to 94%) or for dk (by 5 to 54%)."""
import math

import pytest

from tests.parity import need_gpu
from tests.test_gpu_packed import make, texts_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


def distances(torch, lens, q, k, v, d, scale, got, copies):
    """By output: (distance of the call's, distance that the roundings make), relative to the exact one's norm."""
    r = lambda x: x.to(torch.bfloat16).double()
    kept = r if copies else (lambda x: x)
    G = q.shape[1] // k.shape[1]
    sums = {name: [0.0, 0.0, 0.0] for name in ("out", "dq", "dk", "dv")}
    at = 0
    for n in lens:
        rows = slice(at, at + n)
        at += n
        if n == 0:
            continue
        Q, D = (x[rows].double().transpose(0, 1) for x in (q, d))
        K, V = (x[rows].double().transpose(0, 1).repeat_interleave(G, 0) for x in (k, v))
        s = (Q @ K.transpose(1, 2) * scale).masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -math.inf)
        e = torch.exp(s - s.amax(-1, keepdim=True))
        total = e.sum(-1, keepdim=True)
        p, dp = e / total, D @ V.transpose(1, 2)
        O = p @ V
        delta = (D * O).sum(-1, keepdim=True)
        ds = p * (dp - delta)
        i = torch.arange(n, device="cuda")[None, :, None]
        given = (D * got[0][rows].double().transpose(0, 1)).sum(-1, keepdim=True)
        ds_q = p * (dp - torch.where(i < 128, delta, given)) if copies else ds
        one = kept(ds_q)
        ds_q = torch.where(i < max(512, n // 4), one + kept(ds_q - one), one)
        group = lambda x: x.view(-1, G, n, q.shape[2]).sum(1)
        exact = (O, ds @ K * scale, group(ds.transpose(1, 2) @ Q) * scale, group(p.transpose(1, 2) @ D))
        near = (kept(e) @ V / total, ds_q @ K * scale, group(kept(ds).transpose(1, 2) @ Q) * scale, group(kept(p).transpose(1, 2) @ D))
        for name, x, y, z in zip(sums, exact, near, (got[0], *got[2:])):
            for a, b in enumerate((z[rows].double().transpose(0, 1) - x, r(y) - x, x)):
                sums[name][a] += (b * b).sum().item()
    return {name: (math.sqrt(a / c), math.sqrt(b / c)) for name, (a, b, c) in sums.items()}


BATCHES = [[2] * 40, [32, 17, 64, 8, 128, 33, 1, 100, 16, 31, 65, 2, 48, 127, 32, 90], [300] * 3, [1001, 512, 640], [2000]]


@pytest.mark.parametrize("copies", [True, False], ids=["copies", "odd"])
@pytest.mark.parametrize("heads", [(12, 2, 128, "bf16"), (28, 4, 128, "bf16"), (8, 8, 64, "bf16")], ids=lambda h: "%d-%d-%d-%s" % h)
@pytest.mark.parametrize("lens", BATCHES, ids=lambda v: "-".join(map(str, v[:4])))
def test_norms(torch, lens, heads, copies):
    from paper_2512_14681_gb300 import packed as P

    scale = heads[2] ** -0.5
    x, dtype = make(torch, heads, lens, seed=31)
    if not copies:  # rows at odd addresses and distances
        odd = []
        for t in x:
            flat = torch.empty(t.shape[0] * (t.shape[1] * t.shape[2] + 3) + 8, dtype=dtype, device="cuda")
            odd.append(flat.as_strided(t.shape, (t.shape[1] * t.shape[2] + 3, t.shape[2], 1), 1).copy_(t))
        x = odd
    q, k, v, d = x
    texts = texts_of(torch, lens)
    out, lse = P.attention(texts, q, k, v, scale, want_lse=True)
    got = (out, lse, *P.attention_grad(texts, q, k, v, out, lse, d, scale))
    P.check()
    for name, (off, by_rounding) in distances(torch, lens, q, k, v, d, scale, got, copies).items():
        print(f"{name} {off:.3e} {by_rounding:.3e}")
        assert off <= 1.08 * by_rounding, (name, off, by_rounding)


@pytest.mark.parametrize("heads", [(12, 2, 128, "f32"), (4, 2, 64, "f32")], ids=lambda h: "%d-%d-%d-%s" % h)
@pytest.mark.parametrize("lens", BATCHES, ids=lambda v: "-".join(map(str, v[:4])))
def test_norms_in_32_bits(torch, lens, heads):
    """A sum of m terms in fp32 is off by sqrt(m) u of its terms' norm where each addition's rounding has a sign of its own (u = 2^-24), and what a
    score is off by multiplies its probability. Scores, dp and delta are sums of head_dim terms, the outputs of n times the heads of a group
    at most: sqrt(head_dim) u of scores and sqrt(n G) u of the outputs. Scores of up to 6 times their norm in the rows that count make that six
    times as much in the exponent; the sum of both, doubled for delta, is allowed."""
    from paper_2512_14681_gb300 import packed as P

    scale = heads[2] ** -0.5
    (q, k, v, d), _ = make(torch, heads, lens, seed=32)
    texts = texts_of(torch, lens)
    out, lse = P.attention(texts, q, k, v, scale, want_lse=True)
    got = (out, lse, *P.attention_grad(texts, q, k, v, out, lse, d, scale))
    P.check()
    allowed = 2 * (6 * math.sqrt(heads[2]) + math.sqrt(max(lens) * heads[0] // heads[1])) * 2.0 ** -24
    for name, (off, _) in distances(torch, lens, q, k, v, d, scale, got, False).items():
        print(f"{name} {off:.3e} {allowed:.3e}")
        assert off <= allowed, (name, off, allowed)
