"""Calls of the log probabilities and their gradient that go wrong easily: rows, streams, threads and devices that do not fit."""
import pytest

from tests.parity import need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


@pytest.mark.parametrize("kind", ["broadcast", "overlapping"])
def test_rows_that_share_memory_are_refused(torch, kind):
    from paper_2512_14681_gb300 import _lib as J
    from paper_2512_14681_gb300 import logprobs as L

    x, target = torch.randn(4, 500, device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda")
    bad = x[:1].expand(4, 500) if kind == "broadcast" else torch.randn(2000, device="cuda").as_strided((4, 500), (499, 1))
    r = L.token_logprobs(x, target)
    for call in (lambda: L.token_logprobs(bad, target, top=3), lambda: L.token_logprobs_grad(bad, target, r.row_stats, r.entropy, 1.0),
                 lambda: L.token_logprobs_grad(x, target, r.row_stats, r.entropy, 1.0, out=bad)):
        with pytest.raises(J.JfError, match="apart") as e:
            call()
        assert e.value.status == J.JF_EINVAL
    for stride in (0, 3, 10 ** 6):  # one row may have any
        one = L.token_logprobs(x.as_strided((1, 500), (stride, 1)), target[:1])
        assert torch.equal(one.logprob, r.logprob[:1])
    L.check()
