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


def test_a_captured_call_keeps_its_memory(torch):
    """Captured on a warmed-up stream; a larger eager call there, then fresh tensors: replays leave those alone."""
    from paper_2512_14681_gb300 import logprobs as L

    x, target = torch.randn(1, 100000, device="cuda"), torch.tensor([5], dtype=torch.int32, device="cuda")
    more = torch.randn(12, 150000, device="cuda")
    want, st = L.token_logprobs(x, target, top=2), torch.cuda.Stream()
    torch.cuda.synchronize()
    L.token_logprobs(x, target, top=2, stream=st)
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        got = L.token_logprobs(x, target, top=2)
    L.token_logprobs(more, target.repeat(12), top=64, stream=st)
    st.synchronize()
    with torch.cuda.stream(st):
        fresh = [torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda") for n in (512, 1 << 12, 1 << 17, 1 << 19) for _ in range(40)]
    torch.cuda.synchronize()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert all((t == 0x5A).all() for t in fresh)
    L.check()


def test_threads_on_one_stream(torch):
    """Calls of several threads, whose launches may come in any order."""
    import threading

    from paper_2512_14681_gb300 import logprobs as L

    x = [torch.randn(3, 60000, device="cuda") for _ in range(6)]
    target = torch.tensor([5, 50000, -1], dtype=torch.int32, device="cuda")
    want = [L.token_logprobs(v, target, top=9) for v in x]
    torch.cuda.synchronize()
    wrong = []

    def run(i):
        for _ in range(150):
            got = L.token_logprobs(x[i], target, top=9)
            if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                wrong.append(i)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(len(x))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
    L.check()


def test_check_takes_a_device_in_any_form(torch):
    from paper_2512_14681_gb300 import _lib as J
    from paper_2512_14681_gb300 import logprobs as L

    x, beyond = torch.randn(1, 50, device="cuda"), torch.tensor([50], dtype=torch.int32, device="cuda")
    for device in (None, "cuda", "cuda:0", torch.device("cuda"), torch.device("cuda", 0)):
        L.token_logprobs(x, beyond)
        with pytest.raises(J.JfError, match="vocabulary"):
            L.check(device)
        L.check(device)


def test_check_waits_for_every_stream(torch):
    from paper_2512_14681_gb300 import _lib as J
    from paper_2512_14681_gb300 import logprobs as L

    x, beyond = torch.randn(1, 50, device="cuda"), torch.tensor([50], dtype=torch.int32, device="cuda")
    L.token_logprobs(x, beyond)
    with pytest.raises(J.JfError):
        L.check()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        torch.cuda._sleep(200_000_000)
    L.token_logprobs(x, beyond, stream=st)
    with pytest.raises(J.JfError, match="vocabulary"):
        L.check()


def test_threads_share_the_first_error_word(torch, monkeypatch):
    """Threads whose first calls come together report into the word that check() reads."""
    import threading
    import time

    from paper_2512_14681_gb300 import logprobs as L

    zeros, device = torch.zeros, torch.device("cuda", torch.cuda.current_device())
    monkeypatch.setattr(L, "_err", {})
    monkeypatch.setattr(torch, "zeros", lambda *a, **k: (time.sleep(0.05), zeros(*a, **k))[1])
    got, start = [], threading.Barrier(8)

    def first():
        start.wait()
        got.append(L._error_word(device).data_ptr())

    threads = [threading.Thread(target=first) for _ in range(8)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert set(got) == {L._err[device].data_ptr()}


def test_check_clears_only_what_it_raised(torch, monkeypatch):
    """A report on another stream right after check() is not cleared with the one before, however late the clearing runs."""
    from paper_2512_14681_gb300 import _lib as J
    from paper_2512_14681_gb300 import logprobs as L

    x, beyond = torch.randn(1, 50, device="cuda"), torch.tensor([50], dtype=torch.int32, device="cuda")
    zero = torch.Tensor.zero_
    monkeypatch.setattr(torch.Tensor, "zero_", lambda t: (torch.cuda._sleep(100_000_000), zero(t))[1])
    st = torch.cuda.Stream()
    L.token_logprobs(x, beyond)
    with pytest.raises(J.JfError):
        L.check()
    L.token_logprobs(x, beyond, stream=st)
    with pytest.raises(J.JfError, match="vocabulary"):
        L.check()
    L.check()


def test_logits_that_require_a_gradient(torch):
    """Refused where autograd would record (a loss would get nothing through the result); by hand they get theirs."""
    from paper_2512_14681_gb300 import _lib as J
    from paper_2512_14681_gb300 import logprobs as L

    h, W = torch.randn(3, 16, device="cuda"), torch.randn(200, 16, device="cuda", requires_grad=True)
    target = torch.tensor([5, 199, 0], dtype=torch.int32, device="cuda")
    logits = h @ W.t()
    with pytest.raises(J.JfError, match="gradient") as e:
        L.token_logprobs(logits, target)
    assert e.value.status == J.JF_EUNSUPPORTED
    with torch.no_grad():
        r = L.token_logprobs(logits, target)
    assert torch.equal(r.logprob, L.token_logprobs(logits.detach(), target).logprob)
    logits.backward(L.token_logprobs_grad(logits.detach(), target, r.row_stats, r.entropy, -1.0))
    want, = torch.autograd.grad(-torch.log_softmax(h.double() @ W.double().t(), -1)[range(3), target.long()].sum(), W)
    # (a gradient of a logit is off by 2e-5 of |hot - p| <= 1 at most, a sum over 3 rows of them in fp32 by 2^-22 of its terms)
    assert ((W.grad - want).abs() <= 3e-5 * h.abs().sum(0)).all()
