"""Scoring tokens over an 8-bit cache: log probabilities of a given text (a draft's, a recorded trajectory's) with
entropy and top alternatives, decoder layers built from the library's single operators.

    python -m paper_2512_14681_gb300.score [--shape small-bf16] [--tokens 200] [--chunk 64] [--top 3]

One layer over a chunk of rows: projection (jf_op_gemm) -> keys and values appended to the layer's 8-bit pages, keys and
queries rotated on the way (Kv8Cache.append) -> attention over the pages (Kv8Cache.attention) -> output projection, MLP.
The last rows' logits go to token_logprobs. The command scores random tokens with the shape's random weights twice, over
the 8-bit cache and through a Context's 16-bit one, and prints how far the two are apart.
"""
from __future__ import annotations

import argparse

import numpy as np
import torch

from . import _lib as J
from . import inputs as I
from .jacobi import Context, op_gemm
from .kv8 import Kv8Cache, Rows, _take_error, rope_table
from .logprobs import TokenLogprobs, token_logprobs, token_logprobs_grad
from .logprobs import check as check_targets


WAIT_CODES = (1, 2, 3)  # of jf_op_gemm: a wait on a copy, a product or an accumulator ran out


class Scorer:
    """A decoder of `shape` (jf_model_config) whose sequences' keys and values are held in 8 bits. weights: id -> host
    fp32 array of a logical tensor, as Context.get_weights gives them."""

    def __init__(self, shape: I.ModelShape, weights, n_seqs: int = 1, max_ctx: int = 2048):
        self.shape, self.type = shape, torch.bfloat16 if shape.bf16 else torch.float32
        d, hd, Hq, Hkv = shape.d_model, shape.head_dim, shape.n_heads, shape.n_kv_heads
        t = lambda tid, rows, cols: torch.from_numpy(np.ascontiguousarray(weights(tid, rows * cols)).reshape(rows, cols)).to(self.type).cuda()
        gain = lambda tid: torch.from_numpy(np.ascontiguousarray(weights(tid, d))).cuda()
        self.embedding = t(0, shape.vocab, d)
        self.head = self.embedding if shape.tie_embeddings else t(1, shape.vocab, d)
        self.final_gain = gain(2)
        self.layers = []
        for l in range(shape.n_layers):
            o = 8 + 16 * l
            w = dict(n1=gain(o), qkv=torch.cat([t(o + 1, Hq * hd, d), t(o + 2, Hkv * hd, d), t(o + 3, Hkv * hd, d)]), o=t(o + 4, d, Hq * hd),
                     n2=gain(o + 5), gu=torch.cat([t(o + 6, shape.d_ff, d), t(o + 7, shape.d_ff, d)]), down=t(o + 8, d, shape.d_ff))
            if shape.qkv_bias:
                w["b"] = torch.cat([t(o + 9, 1, Hq * hd), t(o + 10, 1, Hkv * hd), t(o + 11, 1, Hkv * hd)], 1).float()
            self.layers.append(w)
        self.caches = [Kv8Cache.empty(n_seqs, max_ctx, Hkv, hd) for _ in self.layers]
        self.rope = rope_table(max_ctx, hd, shape.rope_theta)
        self.lens = [0] * n_seqs  # tokens that each sequence's pages hold
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")  # of the projections

    def _projection(self, W, x):
        y, err, _ = op_gemm(W, x)
        torch.maximum(self.err, err, out=self.err)
        return y

    def _norm(self, x, gain):
        return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + self.shape.rms_eps) * gain).to(self.type)

    def hidden(self, tokens, positions=None, mask=None):
        """Final hidden rows of the new tokens of every sequence (a list per sequence, appended at self.lens and kept:
        truncate() takes rejected ones back). positions, mask: as in Kv8Cache.append and .attention."""
        s = self.shape
        hd, Hq, Hkv = s.head_dim, s.n_heads, s.n_kv_heads
        rows = Rows.of([len(t) for t in tokens], self.lens)
        x = self.embedding[torch.tensor([t for seq in tokens for t in seq], device="cuda")].float()
        for w, cache in zip(self.layers, self.caches):
            qkv = self._projection(w["qkv"], self._norm(x, w["n1"]))
            if "b" in w:
                qkv = qkv + w["b"]
            q, k, v = qkv.split([Hq * hd, Hkv * hd, Hkv * hd], 1)
            q = cache.append(rows, k, v, q=q, rope=self.rope, positions=positions, q_dtype=self.type)
            att = cache.attention(rows, q, hd ** -0.5, mask=mask)
            x = x + self._projection(w["o"], att.view(-1, Hq * hd))
            g, u = self._projection(w["gu"], self._norm(x, w["n2"])).chunk(2, 1)
            x = x + self._projection(w["down"], (g * torch.sigmoid(g) * u).to(self.type))
        self.lens = [n + len(t) for n, t in zip(self.lens, tokens)]
        return self._norm(x, self.final_gain)

    def truncate(self, lens):
        self.lens = [min(a, b) for a, b in zip(self.lens, lens)]

    def score(self, tokens, targets, top: int = 0) -> TokenLogprobs:
        """Log probabilities of `targets` (the token after each new one; negative: none), rows of all sequences in order."""
        h = self.hidden(tokens)
        t = torch.tensor([t for seq in targets for t in seq], dtype=torch.int32, device="cuda")
        return token_logprobs(self._projection(self.head, h), t, top=top)

    def head_gradient(self, tokens, targets):
        """(mean negative log likelihood, its gradient by the head's matrix): one step of training the head on given
        tokens, as on the points of a recorded trajectory."""
        h = self.hidden(tokens)
        t = torch.tensor([t for seq in targets for t in seq], dtype=torch.int32, device="cuda")
        logits = self._projection(self.head, h)
        n = max(1, sum(t >= 0 for seq in targets for t in seq))
        r = token_logprobs(logits, t)
        d = token_logprobs_grad(logits, t, r.row_stats, None, -1.0 / n, out=logits)
        return -r.logprob.sum() / n, d.T @ h.float()

    def check(self):
        """Raise what the device has reported (synchronises)."""
        code = _take_error(self.err)
        if code:
            raise J.JfError(J.JF_ETIMEOUT if code in WAIT_CODES else J.JF_EDEVICE, f"a projection reported device code {code}")
        for c in self.caches:
            c.check()
        check_targets()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--shape", default="small-bf16", choices=[n for n in I.SHAPES if "2layer" in n or "small" in n or "tiny" in n])
    ap.add_argument("--tokens", type=int, default=200)
    ap.add_argument("--chunk", type=int, default=64, help="rows of one forward")
    ap.add_argument("--top", type=int, default=3)
    a = ap.parse_args()
    shape = I.SHAPES[a.shape]
    rows = max(a.chunk, 64)
    ctx = Context(shape, max_ctx=a.tokens + 16, max_rows=rows, logits_rows=rows)
    ctx.init_random_weights(I.WEIGHT_SEED, I.WEIGHT_STD)
    scorer = Scorer(shape, lambda tid, n: ctx.get_weights(tid, 0, n), max_ctx=a.tokens + 16)
    text = I.prompt_tokens(shape.vocab, a.tokens + 1).tolist()
    apart = []
    for c in range(0, a.tokens, a.chunk):
        new, targets = text[c:min(c + a.chunk, a.tokens)], text[c + 1:min(c + a.chunk, a.tokens) + 1]
        r = scorer.score([new], [targets], top=a.top)
        logits = torch.from_numpy(ctx.forward_logits(0, new, want_hidden=False)[0]).cuda()
        ctx.prefill(0, new)
        exact = token_logprobs(logits, torch.tensor(targets, dtype=torch.int32, device="cuda"))
        apart.append((r.logprob - exact.logprob).abs())
        print("tokens %4d-%4d: mean log probability %8.4f (16-bit cache %8.4f), entropy %.4f, apart by at most %.4f"
              % (c, c + len(new) - 1, r.logprob.mean(), exact.logprob.mean(), r.entropy.mean(), apart[-1].max()))
        if a.top:
            print("  after the last: " + ", ".join("%d (%.4f)" % (i, p) for i, p in zip(r.top_ids[-1].tolist(), r.top_logprobs[-1].tolist())))
    loss, grad = scorer.head_gradient([text[:8]], [text[1:9]])
    scorer.check()
    print("mean difference %.5f" % torch.cat(apart).mean())
    print("eight more tokens: loss %.4f, head gradient of norm %.4f" % (loss, grad.norm()))
    ctx.close()


if __name__ == "__main__":
    main()
