"""Causal attention of packed texts and its backward pass (jf_op_packed_attention* of include/jf_ops.h): whole prompts,
trajectories or a training batch, one behind the other in the rows of one call and without a cache (attention over a
cache: kv8.py). Every call marshals arguments for one C entry point, on the current stream or the one given as stream=;
device memory comes from PyTorch. No graph is recorded for autograd: a loss goes back through attention() by
attention_grad().

    texts = Packed.of([512, 301, 1])                                    # 814 rows
    out, lse = attention(texts, q, k, v, 128 ** -0.5, want_lse=True)    # q [814][heads][128], k, v [814][kv heads][128]
    dq, dk, dv = attention_grad(texts, q, k, v, out, lse, d_out, 128 ** -0.5)
    check()                                                             # what the device reported (waits for it)
"""
from __future__ import annotations

import ctypes as C
import functools
from dataclasses import dataclass

import torch

from . import _lib as J
from .kv8 import _Fixed, _checked, _device_i32, _dtype, _on_current, _on_stream, _raw_stream, _take_error, _want, _zero_word

_err = {}  # error word by device


@dataclass(eq=False)
class Packed(_Fixed):
    """Texts of a batch (jf_packed): text b has rows row_start[b] .. row_start[b+1]-1 (an int32 CUDA tensor that the kernels
    read when they run), none of more than max_rows. Of n_rows rows those of no text get 0 (lse: -infinity)."""
    row_start: torch.Tensor
    n_rows: int
    max_rows: int

    _fixed = ("row_start", "n_rows", "max_rows")

    def __post_init__(self):
        _device_i32(self.row_start, 2, "row_start")
        self.c = J.Packed(self.row_start.data_ptr(), self.row_start.numel() - 1, self.n_rows, self.max_rows)
        _error_word(self.row_start.device)

    @classmethod
    def of(cls, lengths, n_rows=None, max_rows=None, device="cuda"):
        """From a host list of lengths; n_rows, max_rows: room for other lengths in row_start later (as many texts)."""
        start = [0]
        for n in lengths:
            start.append(start[-1] + n)
        n_rows = start[-1] if n_rows is None else n_rows
        return cls(torch.tensor(start, dtype=torch.int32, device=device), n_rows, min(n_rows, max(lengths, default=0) if max_rows is None else max_rows))


def _error_word(device):
    word = _err.get(device)
    if word is None:
        word = _err.setdefault(device, _zero_word(device))  # (the first of several threads')
    return word


def check(device=None):
    """Raise what the device has reported since the last check (waits for all of its streams), and clear it."""
    device = torch.device("cuda" if device is None else device)
    if device.index is None:
        device = torch.device(device.type, torch.cuda.current_device())
    word = _err.get(device)
    code = _take_error(word) if word is not None else 0
    if code:
        what = {4: "texts that do not lie one behind the other in the rows", 1: "a copy's wait ran out", 2: "a product's wait ran out"}
        raise J.JfError(J.JF_EDEVICE if code == 4 else J.JF_ETIMEOUT, what.get(code, f"device code {code}"))


@functools.lru_cache(maxsize=4096)
def _need(n_seqs, n_rows, max_rows, dtype, heads, kv_heads, head_dim, backward, device):
    n = C.c_size_t()
    t = J.Packed(16, n_seqs, n_rows, max_rows)  # (the address is not looked at)
    _checked(J.load().jf_op_packed_attention_workspace_bytes(C.byref(t), dtype, heads, kv_heads, head_dim, backward, C.byref(n)),
             "jf_op_packed_attention_workspace_bytes")
    return n.value


def _row_stride(shape, stride, n, name):
    """Of [n][heads][head_dim] values."""
    _want(len(shape) == 3 and shape[0] == n and stride[2] == 1 and (stride[1] == shape[2] or shape[1] == 1), "{}: [{}][heads][head_dim] with contiguous heads is wanted", name, n)
    width = shape[1] * shape[2]
    if n <= 1:
        return width  # (one row's stride may be anything)
    _want(stride[0] >= width, "{}: rows {} elements apart that are {} long (contiguous() gives them memory of their own)", name, stride[0], width)
    return stride[0]


@functools.lru_cache(maxsize=4096)
def _strides(n, q, q_stride, k, k_stride, v, v_stride):
    """Row strides of q, k, v, from shapes and strides alone."""
    lds = _row_stride(q, q_stride, n, "q"), _row_stride(k, k_stride, n, "k"), _row_stride(v, v_stride, n, "v")
    _want(k == v and k[2] == q[2], "q, k and v differ in head size, or k and v in heads")
    _want(k[1] > 0 and q[1] % k[1] == 0, "{} query heads over {} KV heads", q[1], k[1])
    return lds


def _alike(t, q, name):
    _want(t.dtype == q.dtype and t.device == q.device, "{}: of {} on {} is wanted", name, q.dtype, q.device)


def _arguments(texts, q, k, v):
    _want(q.is_cuda and texts.row_start.device == q.device, "q: a tensor on the texts' device is wanted")
    _on_current(q.device)
    if (q.requires_grad or k.requires_grad or v.requires_grad) and torch.is_grad_enabled():
        raise J.JfError(J.JF_EUNSUPPORTED, "q, k or v requires a gradient, which is not recorded: detach() them, and see attention_grad")
    _alike(k, q, "k")
    _alike(v, q, "v")
    n = texts.n_rows
    ld_q, ld_k, ld_v = _strides(n, q.shape, q.stride(), k.shape, k.stride(), v.shape, v.stride())
    _, heads, hd = q.shape
    kv_heads, dtype = k.shape[1], _dtype(q.dtype)
    return ((C.byref(texts.c), dtype, q.data_ptr(), ld_q, k.data_ptr(), ld_k, v.data_ptr(), ld_v, heads, kv_heads, hd),
            (texts.c.n_seqs, n, texts.max_rows, dtype, heads, kv_heads, hd))


@_on_stream
def attention(texts: Packed, q, k, v, scale: float, want_lse=False):
    """Causal attention of every text's rows over its own (jf_op_packed_attention): q [n_rows][heads][head_dim], k and v
    [n_rows][kv heads][head_dim], bfloat16 or float32, rows any distance apart. Returns out, or (out, lse)."""
    head, key = _arguments(texts, q, k, v)
    dev, n = q.device, _need(*key, 0, q.device.index)
    ws = torch.empty(n, dtype=torch.uint8, device=dev) if n else None  # the call's own, as in Kv8Cache.attention
    out = torch.empty(q.shape, dtype=q.dtype, device=dev)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=dev) if want_lse else None
    _checked(J.load().jf_op_packed_attention(*head, scale, out.data_ptr(), lse.data_ptr() if want_lse else None,
                                             ws.data_ptr() if n else None, n, _error_word(dev).data_ptr(), _raw_stream(dev)),
             "jf_op_packed_attention")
    return (out, lse) if want_lse else out


@_on_stream
def attention_grad(texts: Packed, q, k, v, out, lse, d_out, scale: float, grads=None):
    """(dq, dk, dv): gradients by q, k and v of a loss whose gradient by attention()'s out is d_out (jf_op_packed_attention_grad).
    grads: three tensors that they are written to (parts of one buffer's rows, for the projection's gradient); None: new ones."""
    head, key = _arguments(texts, q, k, v)
    dev, shape, n = q.device, q.shape, texts.n_rows
    _alike(out, q, "out")
    _alike(d_out, q, "d_out")
    ld_do = _row_stride(d_out.shape, d_out.stride(), n, "d_out")
    _want(out.shape == shape and d_out.shape == shape and out.is_contiguous(), "out, d_out: shaped like q (out contiguous) is wanted")
    _want(lse.shape == shape[:2] and lse.dtype == torch.float32 and lse.device == dev and lse.is_contiguous(),
          "lse: contiguous float32 [{}][{}] is wanted", n, shape[1])
    if grads is None:
        dtype, kv = q.dtype, k.shape
        dq, dk, dv = (torch.empty(shape, dtype=dtype, device=dev), torch.empty(kv, dtype=dtype, device=dev), torch.empty(kv, dtype=dtype, device=dev))
        ld_dq, ld_dk, ld_dv = shape[1] * shape[2], kv[1] * kv[2], kv[1] * kv[2]
    else:
        _want(len(grads) == 3 and all(g.shape == t.shape for g, t in zip(grads, (q, k, v))), "grads: shaped like q, k and v is wanted")
        dq, dk, dv = grads
        for g, name in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
            _alike(g, q, name)
        ld_dq, ld_dk, ld_dv = _strides(n, shape, dq.stride(), k.shape, dk.stride(), k.shape, dv.stride())
    need = _need(*key, 1, dev.index)
    ws = torch.empty(need, dtype=torch.uint8, device=dev)
    _checked(J.load().jf_op_packed_attention_grad(*head, scale, out.data_ptr(), lse.data_ptr(), d_out.data_ptr(), ld_do, dq.data_ptr(), ld_dq,
                                                  dk.data_ptr(), ld_dk, dv.data_ptr(), ld_dv, ws.data_ptr(), need,
                                                  _error_word(dev).data_ptr(), _raw_stream(dev)), "jf_op_packed_attention_grad")
    return dq, dk, dv
