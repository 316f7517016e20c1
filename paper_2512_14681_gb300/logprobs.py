"""Log probabilities of given tokens with entropy and top alternatives, and their gradient (jf_op_token_logprobs*
of include/jf_ops.h), on the current stream or the one given as stream=: scores of a draft's or a trajectory's tokens, and the loss of training on them.

    r = token_logprobs(logits, targets, top=5)                                    # r.logprob, r.entropy, r.top_ids, ...
    d = token_logprobs_grad(logits, targets, r.row_stats, r.entropy, -1 / n)      # of the mean negative log likelihood
"""
from __future__ import annotations

import ctypes as C
import functools
from typing import NamedTuple

import torch

from . import _lib as J
from .kv8 import _checked, _dtype, _on_current, _on_stream, _raw_stream, _row_stride, _take_error, _want

_err = {}  # error word by device


class TokenLogprobs(NamedTuple):
    logprob: torch.Tensor        # [rows] log probability of the target (0 where it is negative)
    entropy: torch.Tensor        # [rows]
    lse: torch.Tensor            # [rows] log sum exp of the scaled logits
    row_stats: torch.Tensor      # [rows * 2], for the gradient
    top_ids: torch.Tensor | None       # int32 [rows][top], 0x7fffffff past the tokens that can occur
    top_logprobs: torch.Tensor | None  # [rows][top]


def _error_word(device):
    word = _err.get(device)
    if word is None:
        word = torch.zeros(1, dtype=torch.int32, device=device)
        torch.cuda.current_stream(device).synchronize()  # zero for every stream
        word = _err.setdefault(device, word)  # (the first of several threads')
    return word


def check(device=None):
    """Raise what the device has reported since the last check (waits for all of its streams), and clear it: a target
    beyond the vocabulary."""
    device = torch.device("cuda" if device is None else device)
    if device.index is None:
        device = torch.device(device.type, torch.cuda.current_device())
    word = _err.get(device)
    if word is None:
        return
    if _take_error(word):
        raise J.JfError(J.JF_EDEVICE, "a target was beyond the vocabulary")


@functools.lru_cache(maxsize=4096)
def _need(rows, vocab, top):
    n = C.c_size_t()
    _checked(J.load().jf_op_token_logprobs_workspace_bytes(rows, vocab, top, C.byref(n)), "jf_op_token_logprobs_workspace_bytes")
    return n.value


def _logits(t, name="logits"):
    _want(t.is_cuda and t.dim() == 2 and t.shape[1] >= 1 and (t.stride(1) == 1 or t.shape[1] == 1),
          "{}: CUDA [rows][vocab] with contiguous rows is wanted", name)
    return _row_stride(t, t.shape[1], name)


def _vector(t, rows, dtype, device, name):
    _want(t.device == device and t.dtype == dtype and t.is_contiguous() and t.numel() == rows,
          "{}: a contiguous {} tensor of {} elements on {} is wanted", name, dtype, rows, device)
    return t.data_ptr()


@_on_stream
def token_logprobs(logits, targets, top: int = 0, scale: float = 1.0) -> TokenLogprobs:
    """logits: CUDA [rows][vocab] (float32 or bfloat16, rows any distance apart but not one over the other); targets:
    int32 [rows]; scale: inverse temperature; top: alternatives listed per row (at most 64). No graph is recorded: logits
    that a loss goes back through are given as logits.detach(), and get token_logprobs_grad's result by logits.backward()."""
    if logits.requires_grad and torch.is_grad_enabled():
        raise J.JfError(J.JF_EUNSUPPORTED, "logits require a gradient, which is not recorded: detach() them, and see token_logprobs_grad")
    lib = J.load()
    ld, (rows, vocab), dev = _logits(logits), logits.shape, logits.device
    _on_current(dev)
    dtype = _dtype(logits.dtype)
    tp = _vector(targets, rows, torch.int32, dev, "targets")
    st = _raw_stream(dev)
    out = torch.empty(5 * rows, dtype=torch.float32, device=dev)
    logprob, entropy, lse, stats = torch.split_with_sizes(out, (rows, rows, rows, 2 * rows))
    ids = torch.empty(rows, top, dtype=torch.int32, device=dev) if top else None
    lps = torch.empty(rows, top, dtype=torch.float32, device=dev) if top else None
    need = _need(rows, vocab, top)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None  # the call's own, as in Kv8Cache.attention
    _checked(lib.jf_op_token_logprobs(dtype, logits.data_ptr(), ld, rows, vocab, scale, tp, logprob.data_ptr(), entropy.data_ptr(),
                                      lse.data_ptr(), stats.data_ptr(), top, ids.data_ptr() if top else None,
                                      lps.data_ptr() if top else None, ws.data_ptr() if ws is not None else None,
                                      ws.numel() if ws is not None else 0, _error_word(dev).data_ptr(), st),
             "jf_op_token_logprobs")
    return TokenLogprobs(logprob, entropy, lse, stats, ids, lps)


@_on_stream
def token_logprobs_grad(logits, targets, row_stats, entropy, grad_logprob, grad_entropy=None, scale: float = 1.0,
                        out=None):
    """Gradient of sum(grad_logprob * logprob + grad_entropy * entropy) by the logits, in their type. grad_logprob,
    grad_entropy: float32 [rows], a number, or None (0). out: where it goes (it may be `logits`)."""
    lib = J.load()
    ld, (rows, vocab), dev = _logits(logits), logits.shape, logits.device
    _on_current(dev)
    dtype = _dtype(logits.dtype)
    if out is None:
        out = torch.empty(rows, vocab, dtype=logits.dtype, device=dev)
    ld_out = _logits(out, "out")
    _want(out.dtype == logits.dtype and out.device == dev and out.shape == logits.shape, "out: like logits is wanted")

    def share(g, name):
        if g is None:
            return None, None
        if not isinstance(g, torch.Tensor):
            g = torch.full((rows,), float(g), dtype=torch.float32, device=dev)
        return g, _vector(g, rows, torch.float32, dev, name)

    gl, gl_p = share(grad_logprob, "grad_logprob")
    ge, ge_p = share(grad_entropy, "grad_entropy")
    ep = _vector(entropy, rows, torch.float32, dev, "entropy") if ge is not None else None
    _checked(lib.jf_op_token_logprobs_grad(dtype, logits.data_ptr(), ld, rows, vocab, scale,
                                           _vector(targets, rows, torch.int32, dev, "targets"),
                                           _vector(row_stats, 2 * rows, torch.float32, dev, "row_stats"), ep, gl_p, ge_p,
                                           out.data_ptr(), ld_out, _error_word(dev).data_ptr(), _raw_stream(dev)),
             "jf_op_token_logprobs_grad")
    return out
