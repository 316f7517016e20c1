"""Calls of the policy loss and the log probabilities that are refused for their size."""
import pytest

from tests.parity import need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


def test_more_values_than_an_int_counts(torch):
    """A row of 2^32 + 5 values is no row of 5."""
    from paper_2512_14681_gb300 import _lib as J
    from paper_2512_14681_gb300 import logprobs as L

    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("takes 9 GB")
    z = torch.empty(1, (1 << 32) + 5, dtype=torch.bfloat16, device="cuda")
    z[0, :8] = 0.0
    t, x = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda")
    calls = [lambda: L.policy_loss(z, t, x[:1], x[:1], out=z), lambda: L.token_logprobs(z, t), lambda: L.token_logprobs_grad(z, t, x, None, 1.0, out=z)]
    for call in calls:
        with pytest.raises(J.JfError) as e:
            call()
        assert e.value.status == J.JF_EUNSUPPORTED
    del z
    torch.cuda.empty_cache()
