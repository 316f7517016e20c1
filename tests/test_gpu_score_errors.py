"""What the device reports while tokens are scored reaches Scorer.check()."""
import pytest

from paper_2512_14681_gb300 import inputs as I
from tests.parity import need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def scorer():
    need_gpu()
    from paper_2512_14681_gb300.jacobi import Context
    from paper_2512_14681_gb300.score import Scorer

    ctx = Context(I.TINY_F32, max_ctx=64, max_rows=64, logits_rows=64)
    ctx.init_random_weights(I.WEIGHT_SEED, I.WEIGHT_STD)
    yield Scorer(I.TINY_F32, lambda tid, n: ctx.get_weights(tid, 0, n), max_ctx=64)
    ctx.close()


@pytest.mark.parametrize("code,status", [(1, "JF_ETIMEOUT"), (2, "JF_ETIMEOUT"), (3, "JF_ETIMEOUT"), (5, "JF_EDEVICE")])
@pytest.mark.parametrize("which", ["first", "last"])
def test_a_projection_that_reports_an_error(scorer, monkeypatch, code, status, which):
    """A projection's error word, filled in on the host in place of a kernel that fails."""
    from paper_2512_14681_gb300 import score
    from paper_2512_14681_gb300._lib import JfError

    calls, real = [], score.op_gemm

    def gemm(W, x):
        y, err, ws = real(W, x)
        calls.append(err)
        if (len(calls) == 1) == (which == "first") and (which == "first" or W is scorer.head):
            err.fill_(code)
        return y, err, ws

    monkeypatch.setattr(score, "op_gemm", gemm)
    scorer.truncate([0])
    scorer.score([[1, 2, 3]], [[2, 3, 4]])
    with pytest.raises(JfError, match=f"{status}.*projection"):
        scorer.check()
    monkeypatch.undo()
    scorer.truncate([0])
    scorer.score([[1, 2, 3]], [[2, 3, 4]])
    scorer.check()
