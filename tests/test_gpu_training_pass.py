"""Packed attention, the policy loss and their gradients in one pass, as a policy's update runs them, against 64-bit autograd.

A layer's attention and a head over rows of packed texts: x -> q, k, v -> attention -> + x -> logits -> loss of the next tokens. The
matrices of the projections are multiplied in the tests' own fp32, so that what is off is the operators': fp32 attention and loss are
held to the sum over the pass of what each may be off by, bf16 ones to the operators' own bounds at the values that they were given."""
import math

import pytest

from tests import packed_ref
from tests.packed_ref import U, inside
from tests.parity import need_gpu

pytestmark = pytest.mark.gpu
TERMS = dict(below=0.2, above=0.28, kl=0.05, eta=0.01)


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


class Pass:
    """Weights and a batch; step() goes forward and back through the operators, exact() in 64 bits through autograd."""

    def __init__(self, torch, lens, n_rows, dtype, Hq, Hkv, hd, vocab, seed=0):
        from paper_2512_14681_gb300 import packed as P

        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.torch, self.lens, self.heads, self.vocab, self.scale = torch, lens, (Hq, Hkv, hd), vocab, hd ** -0.5
        D = Hq * hd
        self.dtype = dtype
        self.x = r(n_rows, D).to(dtype)
        self.w_qkv = (r((Hq + 2 * Hkv) * hd, D) * D ** -0.5).to(dtype)
        self.w_head = (r(vocab, D) * D ** -0.5).to(dtype)
        self.targets = torch.randint(0, vocab, (n_rows,), generator=g, device="cuda").int()
        self.adv, self.weight = r(n_rows), torch.rand(n_rows, generator=g, device="cuda")
        self.old, self.ref = (-math.log(vocab) - 1 + r(n_rows) * 0.4 for _ in range(2))
        self.texts = P.Packed.of(lens, n_rows=n_rows, max_rows=max(lens))
        self.set(lens)

    def set(self, lens):
        torch = self.torch
        self.lens, self.n = lens, sum(lens)
        start = torch.tensor([0] + lens).cumsum(0).int()
        self.texts.row_start.copy_(start)
        self.targets[self.targets < 0] = 0
        self.targets[self.n:] = -1
        self.targets[(start[1:][torch.tensor(lens) > 0] - 1).long()] = -1  # a text's last token has no next one

    def step(self, wait=True):
        """Values of the pass on the current stream: (qkv, out, lse, logits, loss terms, grads)."""
        from paper_2512_14681_gb300 import logprobs as L
        from paper_2512_14681_gb300 import packed as P

        Hq, Hkv, hd = self.heads
        qkv = (self.x @ self.w_qkv.T).unflatten(1, (-1, hd))
        q, k, v = qkv.split([Hq, Hkv, Hkv], 1)
        out, lse = P.attention(self.texts, q, k, v, self.scale, want_lse=True)
        h = self.x + out.flatten(1)
        logits = h @ self.w_head.T
        terms = L.policy_loss(logits, self.targets, self.old, self.adv, weight=self.weight, ref_logprob=self.ref, below=TERMS["below"], above=TERMS["above"],
                              kl=TERMS["kl"], entropy=TERMS["eta"])
        d_h = terms.grad @ self.w_head
        d_qkv = self.torch.empty_like(qkv)
        P.attention_grad(self.texts, q, k, v, out, lse, d_h.unflatten(1, (-1, hd)), self.scale, grads=d_qkv.split([Hq, Hkv, Hkv], 1))
        d_x = d_h + d_qkv.flatten(1) @ self.w_qkv
        return dict(qkv=qkv, out=out, lse=lse, h=h, logits=logits, terms=terms, d_h=d_h, d_qkv=d_qkv, d_x=d_x, d_w=d_qkv.flatten(1).T @ self.x,
                    d_head=terms.grad.T @ h)

    def exact(self):
        torch = self.torch
        Hq, Hkv, hd = self.heads
        x, w, wh = (t.double().requires_grad_() for t in (self.x, self.w_qkv, self.w_head))
        q, k, v = (x @ w.T).unflatten(1, (-1, hd)).split([Hq, Hkv, Hkv], 1)
        rows, at = [], 0
        for n in self.lens:
            if n:
                Q = q[at:at + n].transpose(0, 1)
                K, V = (t[at:at + n].transpose(0, 1).repeat_interleave(Hq // Hkv, 0) for t in (k, v))
                s = (Q @ K.transpose(1, 2) * self.scale).masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -math.inf)
                rows.append((s.softmax(-1) @ V).transpose(0, 1).reshape(n, -1))
            at += n
        rows.append(x.new_zeros(x.shape[0] - at, Hq * hd))
        h = x + torch.cat(rows)
        logp = (h @ wh.T).log_softmax(-1)
        on = self.targets >= 0
        lp = logp.gather(1, self.targets.clamp(min=0).long()[:, None])[:, 0]
        A = self.adv.double()
        ratio = (lp - self.old.double()).exp()
        d = self.ref.double() - lp
        H = -(logp.exp() * logp).sum(-1)
        terms = -torch.minimum(ratio * A, ratio.clamp(1 - TERMS["below"], 1 + TERMS["above"]) * A) + TERMS["kl"] * (torch.expm1(d) - d) - TERMS["eta"] * H
        loss = torch.where(on, self.weight.double() * terms, 0.0)
        loss.sum().backward()
        return loss.detach(), x.grad, w.grad, wh.grad


def check():
    from paper_2512_14681_gb300 import logprobs as L
    from paper_2512_14681_gb300 import packed as P

    P.check()
    L.check()


@pytest.mark.parametrize("lens,rows", [([1], 1), ([40, 0, 1, 23], 70), ([200, 131], 331)], ids=["one", "some", "long"])
def test_a_pass_in_32_bits_against_autograd(torch, lens, rows):
    """Each value passes sums of at most N = max(width, vocab, rows) terms in fp32, five after one another in the forward pass and seven
    in the backward one: relative to the largest gradient, N u each by their worst case. Random signs stay below its root, 2 sqrt(N) u a
    stage; probabilities' slopes (scores up to 8, ratios up to e^2) multiply what came before by at most 16."""
    assert not torch.backends.cuda.matmul.allow_tf32
    p = Pass(torch, lens, rows, torch.float32, 8, 2, 64, 1003)
    got = p.step()
    check()
    loss, d_x, d_w, d_head = p.exact()
    N = 1003
    tol = 12 * 2 * math.sqrt(N) * U * 16
    for name, x, want in (("loss", got["terms"].loss, loss), ("d_x", got["d_x"], d_x), ("d_w", got["d_w"], d_w), ("d_head", got["d_head"], d_head)):
        off, top = (x.double() - want).abs().max().item(), want.abs().max().item()
        assert off <= tol * max(top, 1e-30), (name, off, top)
        assert top > 0 or rows == 1, name


@pytest.mark.parametrize("lens,rows", [([40, 0, 1, 23], 70), ([300, 131, 150], 600)], ids=["some", "long"])
def test_a_pass_in_bf16(torch, lens, rows):
    """Every operator within its own bounds at what the one before gave it."""
    from tests.test_gpu_policy import NAMES, reference

    p = Pass(torch, lens, rows, torch.bfloat16, 14, 2, 128, 2003)
    got = p.step()
    check()
    Hq, Hkv, hd = p.heads
    q, k, v = got["qkv"].split([Hq, Hkv, Hkv], 1)
    out, lse, t_out, t_lse = packed_ref.forward(torch, lens, 0, q, k, v, p.scale)
    inside(torch, got["out"], out, t_out, "out")
    inside(torch, got["lse"], lse, t_lse, "lse")
    s = dict(logits=got["logits"], targets=p.targets, old=p.old, ref=p.ref, adv=p.adv, weight=p.weight)
    want, bounds = reference(torch, s, TERMS["below"], TERMS["above"], TERMS["kl"], TERMS["eta"], 1.0)
    for x, w, b, name in zip(got["terms"], want, bounds, NAMES):
        inside(torch, x, w, b, name)
    want, bounds = packed_ref.backward(torch, lens, 0, q, k, v, got["d_h"].unflatten(1, (-1, hd)), p.scale, got["out"], got["lse"])
    for x, w, b, name in zip(got["d_qkv"].split([Hq, Hkv, Hkv], 1), want, bounds, ("dq", "dk", "dv")):
        inside(torch, x, w, b, name)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_a_captured_pass_follows_its_batch(torch, dtype):
    """Two graphs of the whole pass, replayed by turns with batches of other lengths, beside eager passes: the same bits."""
    passes = [Pass(torch, [90, 10, 60], 260, getattr(torch, dtype), 8, 2, 64, 1003, seed=i) for i in range(2)]
    for p in passes:
        p.texts = type(p.texts)(p.texts.row_start, 260, 200)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for p in passes:
            p.step()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for p in passes:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            kept = p.step()
        graphs.append((g, kept))
    for lens in ([90, 10, 60], [0, 200, 1], [1, 1, 1], [100, 100, 60]):
        for p in passes:
            p.set(lens)
        for g, _ in graphs:
            g.replay()
        for p, (_, kept) in zip(passes, graphs):
            now = p.step()
            for name in ("out", "lse", "logits", "d_qkv"):
                assert torch.equal(now[name], kept[name]), (lens, name)
            for a, b in zip(now["terms"], kept["terms"]):
                assert torch.equal(a, b)
            assert torch.equal(now["d_x"], kept["d_x"])
    check()
