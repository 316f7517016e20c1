"""A paged key/value cache held in 8 bits, and attention over it (jf_op_kv8_* of include/jf_ops.h).

A block of the cache (a page of 16 tokens, one KV head) holds e4m3 codes and one exponent: x ~ code * 2^e. append()
rotates and rounds new rows into it, attention() reads it, read() gives back the values that it stands for. Every
method marshals arguments and calls one C entry point, on the current stream or the one given as stream=; device
memory comes from PyTorch. No graph is recorded for autograd: results depend on their inputs' values only.

    cache = Kv8Cache.empty(n_seqs=1, max_ctx=4096, n_kv_heads=4, head_dim=128)
    rows = Rows.of(new=[32], lens=[1000])                 # 32 new tokens behind 1000 cached ones
    q = cache.append(rows, k, v, q=q, rope=rope_table(4096, 128, 1e6))
    out = cache.attention(rows, q, scale=128 ** -0.5)
    cache.check()                                         # what the device reported (waits for it)
"""
from __future__ import annotations

import ctypes as C
import functools
from dataclasses import dataclass

import torch

from . import _lib as J

PAGE = 16
DEVICE_CODES = {4: "an index was out of range (page table, lengths, positions)",
                7: "a value without a finite 8-bit form (NaN or infinite) was appended"}
_DTYPE = {torch.bfloat16: J.JF_BF16, torch.float32: J.JF_F32}


def _dtype(t):
    d = _DTYPE.get(t)
    if d is None:
        raise J.JfError(J.JF_EUNSUPPORTED, f"type {t}: bfloat16 or float32 is wanted")
    return d


def _checked(status: int, what: str):
    if status != J.JF_OK:
        raise J.JfError(status, what)


def _want(ok, what: str, *values):
    """A refusal, its message written only then."""
    if not ok:
        raise J.JfError(J.JF_EINVAL, what.format(*values))


def _raw_stream(device):
    return torch._C._cuda_getCurrentRawStream(device.index)


def _on_stream(call):
    """A call that takes stream=: entered, so that what the call allocates belongs to that stream too."""
    @functools.wraps(call)
    def wrapped(*args, stream=None, **kwargs):
        if stream is None:
            return call(*args, **kwargs)
        with torch.cuda.stream(stream):
            return call(*args, **kwargs)
    return wrapped


def _take_error(word) -> int:
    """The code in an error word, once all of its device's streams are done; the word is clear for each of them after."""
    torch.cuda.synchronize(word.device)
    code = int(word.item())
    if code:
        word.zero_()
        torch.cuda.current_stream(word.device).synchronize()  # (a later report must not be cleared with this one)
    return code


def _row_stride(t, width, name):
    """Elements from row to row of t, whose rows are `width` long and must not share memory (a broadcast row does)."""
    if t.shape[0] <= 1:
        return width  # (one row's stride may be anything)
    _want(t.stride(0) >= width, "{}: rows {} elements apart that are {} long (contiguous() gives them memory of their own)",
          name, t.stride(0), width)
    return t.stride(0)


_current_device = torch._C._cuda_getDevice


def _on_current(device):
    """Kernels are launched on the current device, in one of its streams."""
    _want(device.index == _current_device(), "tensors on {}, which is not the current device", device)


def _device_i32(t, n, name, device=None):
    _want(t.is_cuda and t.dtype == torch.int32 and t.is_contiguous() and t.numel() >= n,
          "{}: a contiguous int32 CUDA tensor of {} elements is wanted", name, n)
    _want(device is None or t.device == device, "{}: a tensor on {} is wanted", name, device)


def rope_table(n: int, head_dim: int, theta: float, device="cuda"):
    """(cos, sin) of positions 0 .. n-1, fp32 [n][head_dim / 2][2], frequency theta^(-2i/head_dim)."""
    freq = theta ** (-torch.arange(0, head_dim, 2, dtype=torch.float64, device=device) / head_dim)
    ang = torch.arange(n, dtype=torch.float64, device=device)[:, None] * freq
    return torch.stack([torch.cos(ang), torch.sin(ang)], -1).float().contiguous()


class _Fixed:
    """Attributes that are given once: calls go by the C structure that points into these tensors and would not follow."""
    _fixed = ()

    def __setattr__(self, name, value):
        _want(name not in self._fixed or self.__dict__.get(name, value) is value,
              "{} cannot be replaced (write into the tensor, or make another {})", name, type(self).__name__)
        super().__setattr__(name, value)


@dataclass(eq=False)
class Rows(_Fixed):
    """New rows of a batch (jf_kv8_rows): sequence b has rows row_start[b] .. row_start[b+1]-1 at slots len[b] ...
    Both are int32 CUDA tensors that the kernels read when they run."""
    row_start: torch.Tensor
    len: torch.Tensor
    n_rows: int
    max_rows: int

    _fixed = ("row_start", "len", "n_rows", "max_rows")

    def __post_init__(self):
        n_seqs = self.len.numel()
        _device_i32(self.row_start, n_seqs + 1, "row_start")
        _device_i32(self.len, n_seqs, "len", self.row_start.device)
        self.c = J.Kv8Rows(self.row_start.data_ptr(), self.len.data_ptr(), self.n_rows, self.max_rows)

    @classmethod
    def of(cls, new, lens, device="cuda"):
        """From host lists: rows per sequence, and the tokens that each holds before them."""
        start = [0]
        for n in new:
            start.append(start[-1] + n)
        i32 = dict(dtype=torch.int32, device=device)
        return cls(torch.tensor(start, **i32), torch.tensor(list(lens), **i32), start[-1], max(new) if len(new) else 0)


class Kv8Cache(_Fixed):
    """k, v: [n_pages][n_kv_heads][16][head_dim] codes (uint8 or float8_e4m3fn); k_exp, v_exp: int8
    [n_pages][n_kv_heads]; page_table: int32 [n_seqs][pages_per_seq]. All contiguous CUDA tensors on one device."""

    _fixed = ("k", "v", "k_exp", "v_exp", "page_table", "err")

    def __init__(self, k, v, k_exp, v_exp, page_table):
        for name, t in (("k", k), ("v", v)):
            _want(t.is_cuda and t.is_contiguous() and t.dim() == 4 and t.element_size() == 1 and t.shape[2] == PAGE,
                  "{}: contiguous 8-bit codes [pages][heads][16][head_dim] are wanted", name)
        for name, t in (("k_exp", k_exp), ("v_exp", v_exp)):
            _want(t.is_cuda and t.is_contiguous() and t.dtype == torch.int8 and t.shape == k.shape[:2],
                  "{}: contiguous int8 [pages][heads] is wanted", name)
        _want(k.shape == v.shape, "k and v differ in shape")
        _want(page_table.dim() == 2, "page_table: [sequences][pages] is wanted")
        _device_i32(page_table, page_table.numel(), "page_table")
        _want(len({t.device for t in (k, v, k_exp, v_exp, page_table)}) == 1, "the cache's tensors are on several devices")
        self.lib = J.load()
        self.k, self.v, self.k_exp, self.v_exp, self.page_table = k, v, k_exp, v_exp, page_table
        self.n_kv_heads, self.head_dim, self.device = k.shape[1], k.shape[3], k.device
        self.c = J.Kv8Cache(k.data_ptr(), v.data_ptr(), k_exp.data_ptr(), v_exp.data_ptr(), page_table.data_ptr(),
                            page_table.shape[0], k.shape[0], page_table.shape[1], k.shape[1], k.shape[3])
        self.err = torch.zeros(1, dtype=torch.int32, device=k.device)
        torch.cuda.current_stream(k.device).synchronize()  # zero for every stream
        self._need = {}

    @classmethod
    def empty(cls, n_seqs: int, max_ctx: int, n_kv_heads: int, head_dim: int, device="cuda"):
        """A cache with pages for max_ctx tokens of each sequence, handed out in order."""
        per_seq = (max_ctx + PAGE - 1) // PAGE
        pages = n_seqs * per_seq
        codes = lambda: torch.empty(pages, n_kv_heads, PAGE, head_dim, dtype=torch.uint8, device=device)
        exps = lambda: torch.empty(pages, n_kv_heads, dtype=torch.int8, device=device)
        return cls(codes(), codes(), exps(), exps(),
                   torch.arange(pages, dtype=torch.int32, device=device).view(n_seqs, per_seq))

    def _rows_of(self, t, heads, rows, name):
        """Row stride of [n_rows][heads * head_dim] (or [n_rows][heads][head_dim]) values."""
        width = heads * self.head_dim
        if t.dim() == 3:
            ok = t.shape[1:] == (heads, self.head_dim) and t.stride(2) == 1 and t.stride(1) == self.head_dim
        else:
            ok = t.dim() == 2 and t.shape[1] == width and t.stride(1) == 1
        _want(ok and t.shape[0] == rows.n_rows and t.device == self.device,
              "{}: [{}][{} x {}] with contiguous heads on {} is wanted", name, rows.n_rows, heads, self.head_dim, self.device)
        return _row_stride(t, width, name)

    def _batch(self, rows):
        _on_current(self.device)
        _want(rows.len.numel() == self.page_table.shape[0] and rows.len.device == self.device,
              "rows: as many sequences as the page table, on its device, are wanted")

    @_on_stream
    def append(self, rows: Rows, k, v, q=None, rope=None, positions=None, q_dtype=None):
        """Append the rows' keys and values (jf_op_kv8_append), rotated by `rope` at `positions` (None: their
        slots). With q: returns the rotated queries [n_rows][heads][head_dim] in q_dtype (None: q's type)."""
        self._batch(rows)
        ld_k, ld_v = self._rows_of(k, self.n_kv_heads, rows, "k"), self._rows_of(v, self.n_kv_heads, rows, "v")
        _want(k.dtype == v.dtype and (q is None or q.dtype == k.dtype), "q, k and v differ in type")
        heads = ld_q = 0
        q_out = None
        out_dtype = q_dtype or k.dtype
        if q is not None:
            width = q.shape[-1] if q.dim() == 2 else q.shape[1] * q.shape[2]
            _want(width % self.head_dim == 0, "q: whole heads are wanted")
            heads = width // self.head_dim
            ld_q = self._rows_of(q, heads, rows, "q")
            q_out = torch.empty(rows.n_rows, heads, self.head_dim, dtype=out_dtype, device=self.device)
        rope_len = 0
        if rope is not None:
            _want(rope.dtype == torch.float32 and rope.is_contiguous() and rope.shape[1:] == (self.head_dim // 2, 2) and
                  rope.device == self.device, "rope: contiguous float32 [positions][head_dim / 2][2] is wanted")
            rope_len = rope.shape[0]
        if positions is not None:
            _device_i32(positions, rows.n_rows, "positions", self.device)
        ptr = lambda t: t.data_ptr() if t is not None else None
        _checked(self.lib.jf_op_kv8_append(
            C.byref(self.c), C.byref(rows.c), _dtype(k.dtype), ptr(q), ld_q, k.data_ptr(), ld_k, v.data_ptr(), ld_v, heads,
            ptr(positions), ptr(rope), rope_len, _dtype(out_dtype), ptr(q_out), self.err.data_ptr(), _raw_stream(self.device)),
            "jf_op_kv8_append")
        return q_out

    @_on_stream
    def read(self, rows: Rows, dtype=torch.float32):
        """(k, v) values that the cache stands for at the rows' slots, [n_rows][n_kv_heads][head_dim]."""
        self._batch(rows)
        shape = (rows.n_rows, self.n_kv_heads, self.head_dim)
        k, v = (torch.empty(shape, dtype=dtype, device=self.device) for _ in range(2))
        _checked(self.lib.jf_op_kv8_read(C.byref(self.c), C.byref(rows.c), _dtype(dtype), k.data_ptr(), v.data_ptr(),
                                         self.err.data_ptr(), _raw_stream(self.device)), "jf_op_kv8_read")
        return k, v

    @_on_stream
    def attention(self, rows: Rows, q, scale: float, mask=None, want_lse=False):
        """Attention of the rows' queries [n_rows][heads][head_dim] over the cache (jf_op_kv8_attention); mask:
        int32 [n_rows][words] visibility bits among the sequence's new rows (None: causal). Returns out, or (out, lse)."""
        self._batch(rows)
        width = q.shape[-1] if q.dim() == 2 else q.shape[1] * q.shape[2]
        _want(width % self.head_dim == 0, "q: whole heads are wanted")
        heads = width // self.head_dim
        ld_q = self._rows_of(q, heads, rows, "q")
        dtype = _dtype(q.dtype)
        words = 0
        if mask is not None:
            _want(mask.dim() == 2, "mask: [rows][words] is wanted")
            words = mask.shape[1]
            _device_i32(mask, rows.n_rows * words, "mask", self.device)
        st = _raw_stream(self.device)
        key = (dtype, heads, rows.c.n_rows, rows.c.max_rows)
        need = self._need.get(key)
        if need is None:
            n = C.c_size_t()
            _checked(self.lib.jf_op_kv8_attention_workspace_bytes(C.byref(self.c), C.byref(rows.c), dtype, heads, C.byref(n)),
                     "jf_op_kv8_attention_workspace_bytes")
            need = self._need[key] = n.value
        # A workspace of the call's own: PyTorch's allocator hands its memory to the stream's next call, but not to another
        # stream, nor to a thread whose launches come between this call's two, nor (from a captured graph's pool) to anyone.
        ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        out = torch.empty(rows.n_rows, heads, self.head_dim, dtype=q.dtype, device=self.device)
        lse = torch.empty(rows.n_rows, heads, dtype=torch.float32, device=self.device) if want_lse else None
        _checked(self.lib.jf_op_kv8_attention(
            C.byref(self.c), C.byref(rows.c), dtype, q.data_ptr(), ld_q, heads, scale, mask.data_ptr() if mask is not None else None,
            words, out.data_ptr(), lse.data_ptr() if want_lse else None, ws.data_ptr(), ws.numel(), self.err.data_ptr(), st),
            "jf_op_kv8_attention")
        return (out, lse) if want_lse else out

    def check(self):
        """Raise what the device has reported since the last check (waits for all of its streams), and clear it."""
        code = _take_error(self.err)
        if code:
            raise J.JfError(J.JF_EDEVICE, DEVICE_CODES.get(code, f"device code {code}"))
