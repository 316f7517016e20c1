"""Layout and host-side refusals of the 8-bit cache's and the log probabilities' C entry points (no GPU: every call here
is refused before a launch)."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2512_14681_gb300 import _lib as J
from paper_2512_14681_gb300 import build as B


@pytest.fixture(scope="module")
def lib():
    B.build()
    return J.load()


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
def test_structs_match_the_header(tmp_path):
    structs = {"jf_kv8_cache": J.Kv8Cache, "jf_kv8_rows": J.Kv8Rows}
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "jf_ops.h"', "int main(void) {"]
    for name, py in structs.items():
        lines.append(f'  printf("{name} sizeof %zu\\n", sizeof({name}));')
        lines += [f'  printf("{name} {f} %zu\\n", offsetof({name}, {f}));' for f, _ in py._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(B.ROOT, "include"), str(src), "-o", str(exe)], check=True, capture_output=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n")
    got = {tuple(ln.split()[:2]): int(ln.split()[2]) for ln in out if ln.strip()}
    for name, py in structs.items():
        assert got[name, "sizeof"] == C.sizeof(py)
        for f, _ in py._fields_:
            assert got[name, f] == getattr(py, f).offset, (name, f)


def cache(**change):
    v = dict(k=256, v=256, k_exp=256, v_exp=256, page_table=256, n_seqs=2, n_pages=8, pages_per_seq=4, n_kv_heads=2, head_dim=64)
    v.update(change)
    return C.byref(J.Kv8Cache(*[v[f] for f, _ in J.Kv8Cache._fields_]))


def rows(**change):
    v = dict(row_start=256, len=256, n_rows=8, max_rows=5)
    v.update(change)
    return C.byref(J.Kv8Rows(*[v[f] for f, _ in J.Kv8Rows._fields_]))


BAD_CACHES = [(dict(k=None), J.JF_EINVAL), (dict(v=264), J.JF_EINVAL), (dict(k_exp=None), J.JF_EINVAL), (dict(page_table=None), J.JF_EINVAL),
              (dict(n_seqs=0), J.JF_EINVAL), (dict(n_pages=0), J.JF_EINVAL), (dict(pages_per_seq=0), J.JF_EINVAL),
              (dict(n_kv_heads=0), J.JF_EINVAL), (dict(head_dim=96), J.JF_EUNSUPPORTED), (dict(n_seqs=1025), J.JF_EUNSUPPORTED),
              (dict(pages_per_seq=(1 << 26) + 1), J.JF_EUNSUPPORTED)]
BAD_ROWS = [dict(row_start=None), dict(len=None), dict(n_rows=-1), dict(max_rows=0), dict(max_rows=9), dict(max_rows=-1)]


def append(lib, c, r, dtype=J.JF_BF16, q=None, ld_q=0, k=256, ld_k=128, v=256, ld_v=128, heads=0, rope=None, rope_len=0, out=J.JF_BF16,
           q_out=None, err=256):
    return lib.jf_op_kv8_append(c, r, dtype, q, ld_q, k, ld_k, v, ld_v, heads, None, rope, rope_len, out, q_out, err, None)


def attention(lib, c, r, dtype=J.JF_BF16, q=256, ld_q=256, heads=4, scale=1.0, mask=None, words=0, out=256, ws=256, nb=0, err=256):
    return lib.jf_op_kv8_attention(c, r, dtype, q, ld_q, heads, scale, mask, words, out, None, ws, nb, err, None)


def test_caches_and_rows_that_are_refused(lib):
    n = C.c_size_t()
    for c, r, want in [(cache(**b), rows(), s) for b, s in BAD_CACHES] + [(cache(), rows(**b), J.JF_EINVAL) for b in BAD_ROWS] + \
            [(None, rows(), J.JF_EINVAL), (cache(), None, J.JF_EINVAL)]:
        assert append(lib, c, r) == want
        assert attention(lib, c, r) == want
        assert lib.jf_op_kv8_read(c, r, J.JF_F32, 256, 256, 256, None) == want
        assert lib.jf_op_kv8_attention_workspace_bytes(c, r, J.JF_BF16, 4, C.byref(n)) == want


def test_arguments_of_append_and_read_that_are_refused(lib):
    for bad in (dict(dtype=2), dict(out=-1), dict(k=None), dict(v=None), dict(k=257), dict(ld_k=127), dict(ld_v=127), dict(err=None),
                dict(q=256, ld_q=256, heads=4), dict(q_out=256), dict(q=256, q_out=256, ld_q=255, heads=4),
                dict(q=256, q_out=256, ld_q=256, heads=3), dict(rope=256), dict(rope=260, rope_len=4), dict(dtype=J.JF_F32, k=258)):
        assert append(lib, cache(), rows(), **bad) == J.JF_EINVAL, bad
    assert append(lib, cache(), rows(n_rows=0, max_rows=0), k=None, v=None) == J.JF_OK
    for a in ((2, 256, 256, 256), (J.JF_F32, 258, 256, 256), (J.JF_F32, 256, 256, None)):
        assert lib.jf_op_kv8_read(cache(), rows(), *a, None) == J.JF_EINVAL
    assert lib.jf_op_kv8_read(cache(), rows(), J.JF_F32, None, None, 256, None) == J.JF_OK


def test_arguments_of_attention_that_are_refused(lib):
    for bad in (dict(dtype=5), dict(q=None), dict(out=None), dict(q=257), dict(out=258), dict(heads=0), dict(heads=3), dict(ld_q=255),
                dict(scale=float("nan")), dict(mask=256, words=0), dict(err=None), dict(ws=264), dict(dtype=J.JF_F32, out=260)):
        assert attention(lib, cache(), rows(), **bad) == J.JF_EINVAL, bad
    assert attention(lib, cache(), rows(n_rows=80, max_rows=65), mask=256, words=2) == J.JF_EINVAL
    assert attention(lib, cache(), rows(n_rows=0, max_rows=0), q=None, out=None) == J.JF_OK
    assert lib.jf_op_kv8_attention_workspace_bytes(cache(), rows(), J.JF_BF16, 4, None) == J.JF_EINVAL


def logprobs(lib, dtype=J.JF_F32, logits=256, ld=100, n=2, vocab=100, scale=1.0, targets=256, lp=256, top=0, ids=None, lps=None,
             ws=None, nb=0, err=256):
    return lib.jf_op_token_logprobs(dtype, logits, ld, n, vocab, scale, targets, lp, None, None, None, top, ids, lps, ws, nb, err, None)


def test_arguments_of_token_logprobs_that_are_refused(lib):
    for bad in (dict(dtype=3), dict(logits=None), dict(logits=258), dict(ld=99), dict(n=-1), dict(vocab=0), dict(scale=0.0),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(targets=None), dict(top=-1), dict(top=65, ids=256, lps=256),
                dict(top=3), dict(top=3, ids=256), dict(err=None)):
        assert logprobs(lib, **bad) == J.JF_EINVAL, bad
    assert logprobs(lib, n=0, logits=None) == J.JF_OK
    n = C.c_size_t()
    assert lib.jf_op_token_logprobs_workspace_bytes(1, 152064, 5, C.byref(n)) == J.JF_OK and n.value > 0
    assert logprobs(lib, n=1, vocab=152064, ld=152064, top=5, ids=256, lps=256, ws=256, nb=n.value - 1) == J.JF_ENOMEM
    assert logprobs(lib, n=1, vocab=152064, ld=152064, top=5, ids=256, lps=256, ws=264, nb=n.value) == J.JF_EINVAL
    for bad in ((-1, 10, 0), (1, 0, 0), (1, 10, 65), (1, 10, -1)):
        assert lib.jf_op_token_logprobs_workspace_bytes(*bad, C.byref(n)) == J.JF_EINVAL
    assert lib.jf_op_token_logprobs_workspace_bytes(1, 10, 0, None) == J.JF_EINVAL

    def grad(dtype=J.JF_F32, logits=256, ld=100, n=2, vocab=100, scale=1.0, targets=256, stats=256, h=256, g=256, gh=256, out=512,
             ld_out=100, err=256):
        return lib.jf_op_token_logprobs_grad(dtype, logits, ld, n, vocab, scale, targets, stats, h, g, gh, out, ld_out, err, None)

    for bad in (dict(dtype=9), dict(logits=None), dict(out=None), dict(out=514), dict(ld_out=99), dict(targets=None), dict(stats=None),
                dict(h=None), dict(scale=-1.0), dict(err=None), dict(out=256, ld_out=101)):
        assert grad(**bad) == J.JF_EINVAL, bad
    assert grad(n=0) == J.JF_OK
