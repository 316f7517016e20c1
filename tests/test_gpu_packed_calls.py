"""Calls of packed attention that a user's tensors lead to."""
import math

import pytest

from tests.parity import need_gpu
from tests.test_gpu_packed import both, make, texts_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


@pytest.mark.parametrize("heads", [(7, 1, 128, "bf16"), (1, 1, 64, "bf16"), (1, 1, 128, "f32")], ids=lambda h: "%d-%d-%d-%s" % h)
def test_one_head_at_any_distance(torch, heads):
    """Where there is one head, its stride says nothing: [n][1][head_dim] as a view of [1][n][head_dim], and gradients into such views."""
    from paper_2512_14681_gb300 import packed as P

    lens, scale = [40, 3], heads[2] ** -0.5
    (q, k, v, d), dtype = make(torch, heads, lens, seed=30)
    texts = texts_of(torch, lens)
    want = both(torch, texts, lens, q, k, v, d, scale)
    turned = [x.contiguous() if x.shape[1] > 1 else x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v, d)]
    for x in turned:
        assert x.is_contiguous() and (x.shape[1] > 1 or x.stride(1) == 43 * heads[2])
    got = both(torch, texts, lens, *turned, scale)
    room = [torch.full((1, 43, heads[2]), math.nan, dtype=dtype, device="cuda").transpose(0, 1) if x.shape[1] == 1 else torch.empty_like(x) for x in turned[:3]]
    into = P.attention_grad(texts, *turned[:3], got[0], got[1], turned[3], scale, grads=room)
    for a, b, name in zip(got, want, ("out", "lse", "dq", "dk", "dv")):
        assert torch.equal(a, b), name
    for a, b in zip(into, got[2:]):
        assert torch.equal(a, b)
    P.check()
