"""Layouts and host-side refusals of packed attention's and the policy loss's C entry points (no GPU: every call here is
refused before a launch)."""
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
    structs = {"jf_packed": J.Packed, "jf_policy_terms": J.PolicyTerms}
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


def texts(row_start=256, n_seqs=2, n_rows=8, max_rows=5):
    return C.byref(J.Packed(row_start, n_seqs, n_rows, max_rows))


def attention(lib, t, dtype=J.JF_BF16, q=256, ld_q=256, k=256, ld_k=128, v=256, ld_v=128, heads=4, kv=2, hd=64, scale=1.0, out=1 << 24, lse=None, ws=256, nb=0,
              err=256):
    return lib.jf_op_packed_attention(t, dtype, q, ld_q, k, ld_k, v, ld_v, heads, kv, hd, scale, out, lse, ws, nb, err, None)


def grad(lib, t, dtype=J.JF_BF16, q=256, ld_q=256, k=256, ld_k=128, v=256, ld_v=128, heads=4, kv=2, hd=64, scale=1.0, out=256, lse=256, do=256,
         ld_do=256, dq=1 << 24, ld_dq=256, dk=2 << 24, ld_dk=128, dv=3 << 24, ld_dv=128, ws=256, nb=0, err=256):
    return lib.jf_op_packed_attention_grad(t, dtype, q, ld_q, k, ld_k, v, ld_v, heads, kv, hd, scale, out, lse, do, ld_do, dq, ld_dq, dk, ld_dk, dv, ld_dv,
                                           ws, nb, err, None)


def test_texts_and_shapes_that_are_refused(lib):
    n = C.c_size_t()
    cases = [(dict(t=None), J.JF_EINVAL)] + [(dict(t=texts(**b)), s) for b, s in (
        (dict(row_start=None), J.JF_EINVAL), (dict(n_seqs=0), J.JF_EINVAL), (dict(n_rows=-1), J.JF_EINVAL), (dict(max_rows=-1), J.JF_EINVAL),
        (dict(max_rows=9), J.JF_EINVAL), (dict(n_seqs=1025), J.JF_EUNSUPPORTED), (dict(n_rows=1 << 30, max_rows=1 << 30), J.JF_EUNSUPPORTED))]
    cases += [(dict(t=texts(), **b), s) for b, s in ((dict(dtype=2), J.JF_EINVAL), (dict(heads=0), J.JF_EINVAL), (dict(heads=3), J.JF_EINVAL), (dict(kv=0), J.JF_EINVAL),
                                                     (dict(hd=96), J.JF_EUNSUPPORTED), (dict(heads=258, kv=2), J.JF_EUNSUPPORTED), (dict(heads=65536, kv=65536), J.JF_EUNSUPPORTED))]
    for case, want in cases:
        case = {**dict(dtype=J.JF_BF16, heads=4, kv=2, hd=64), **case}
        t = case.pop("t")
        assert attention(lib, t, **case) == want, case
        assert grad(lib, t, **case) == want, case
        for back in (0, 1):
            assert lib.jf_op_packed_attention_workspace_bytes(t, case["dtype"], case["heads"], case["kv"], case["hd"], back, C.byref(n)) == want
    assert lib.jf_op_packed_attention_workspace_bytes(texts(), J.JF_F32, 4, 2, 64, 0, None) == J.JF_EINVAL


def test_arguments_that_are_refused(lib):
    both = [dict(q=None), dict(k=None), dict(v=None), dict(q=257), dict(ld_q=255), dict(ld_k=127), dict(ld_v=127), dict(out=None), dict(out=264),
            dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=-1.1e30), dict(err=None), dict(ws=264), dict(dtype=J.JF_F32, k=258)]
    for bad in both:
        assert attention(lib, texts(), **bad) == J.JF_EINVAL, bad
    for bad in both + [dict(lse=None), dict(do=None), dict(do=257), dict(ld_do=255), dict(dq=None), dict(dk=None), dict(dv=None), dict(ld_dq=255),
                       dict(ld_dk=127), dict(ld_dv=127), dict(dv=(1 << 24) + 1)]:
        assert grad(lib, texts(), **bad) == J.JF_EINVAL, bad
    assert attention(lib, texts(), lse=258) == J.JF_EINVAL and grad(lib, texts(), lse=258) == J.JF_EINVAL
    none = texts(n_rows=0, max_rows=0)
    assert attention(lib, none, q=None, out=None) == J.JF_OK and grad(lib, none, q=None, dk=None) == J.JF_OK
    assert grad(lib, texts(), dtype=J.JF_F32, nb=0) == J.JF_ENOMEM and grad(lib, texts(), dtype=J.JF_F32, ws=None, nb=1 << 20) == J.JF_ENOMEM


def test_outputs_that_share_memory_are_refused(lib):
    """Rows of 256, 128 and 128 bf16 values (512, 256 bytes), 8 of them. What is not refused here is so for its workspace of 0 bytes."""
    M, row = 1 << 24, 512
    grads, other = dict(dq=M, dk=2 * M, dv=3 * M), dict(q=M, k=M + 8 * row, v=M + 12 * row, out=M + 16 * row, lse=M + 24 * row, do=M + 32 * row)
    for name in grads:
        for by in (0, 7 * row, -16):
            for x in other:
                at = other[x] + (by if x != "lse" else 0)
                assert grad(lib, texts(), **{**other, "dq": 4 * M, "dk": 5 * M, "dv": 6 * M, name: at}) == J.JF_EINVAL, (name, x, by)
    assert grad(lib, texts(), **{**grads, "dk": M + 510}) == J.JF_EINVAL and grad(lib, texts(), **{**grads, "dv": 2 * M}) == J.JF_EINVAL
    fused = dict(ld_dq=512, ld_dk=512, ld_dv=512)  # dq, dk, dv as parts of one buffer's rows
    f32 = dict(dtype=J.JF_F32)
    assert grad(lib, texts(), dq=M, dk=M + 1024, dv=M + 1536, **fused, **f32) == J.JF_ENOMEM
    assert grad(lib, texts(), dq=M + 1024, dk=M, dv=M + 512, **fused, **f32) == J.JF_ENOMEM
    assert grad(lib, texts(), dq=M, dk=M + 1020, dv=M + 1536, **fused, **f32) == J.JF_EINVAL
    assert grad(lib, texts(), dq=M, dk=M + 1024, dv=M + 1540, **fused, **f32) == J.JF_EINVAL
    for out in (M, M + 256, M + 7 * row, M - 8 * row + 16):
        assert attention(lib, texts(), q=M, k=2 * M, v=3 * M, out=out) == J.JF_EINVAL
    assert attention(lib, texts(), q=M, k=2 * M, v=3 * M, out=4 * M, lse=4 * M + 64) == J.JF_EINVAL
    z = dict(logits=M, ld=100, n=3)
    for bad in (dict(g=M + 4), dict(g=M - 4), dict(g=M + 400), dict(g=M, ld_g=101), dict(ld=200, g=M + 396, ld_g=200), dict(ld=200, g=M + 404, ld_g=201)):
        assert policy(lib, **{**z, **bad}) == J.JF_EINVAL, bad


def policy(lib, terms=(0.2, 0.2, 0.0, 0.0), dtype=J.JF_F32, logits=256, ld=100, n=2, vocab=100, scale=1.0, targets=256, old=256, ref=256, adv=256, weight=None,
           g=1 << 24, ld_g=100, ws=256, nb=1 << 20, err=256):
    t = C.byref(J.PolicyTerms(*terms)) if terms else None
    return lib.jf_op_policy_loss(t, dtype, logits, ld, n, vocab, scale, targets, old, ref, adv, weight, 256, 256, 256, 256, 256, g, ld_g, ws, nb, err, None)


def test_arguments_of_the_policy_loss_that_are_refused(lib):
    nan, inf = float("nan"), float("inf")
    for bad in (dict(terms=None), dict(terms=(-0.1, 0, 0, 0)), dict(terms=(1.1, 0, 0, 0)), dict(terms=(nan, 0, 0, 0)), dict(terms=(0, -1, 0, 0)), dict(terms=(0, nan, 0, 0)),
                dict(terms=(0, 0, nan, 0)), dict(terms=(0, 0, 0, inf)), dict(terms=(0, 0, 0.1, 0), ref=None), dict(dtype=2), dict(logits=None), dict(logits=258),
                dict(ld=99), dict(n=-1), dict(vocab=0), dict(scale=0.0), dict(scale=nan), dict(targets=None), dict(adv=None), dict(g=(1 << 24) + 2), dict(ld_g=99),
                dict(g=256, ld=101), dict(ws=264), dict(err=None)):
        assert policy(lib, **bad) == J.JF_EINVAL, bad
    assert policy(lib, n=(1 << 30) + 1) == J.JF_EUNSUPPORTED
    n = C.c_size_t()
    assert lib.jf_op_policy_loss_workspace_bytes(J.JF_F32, 2, 100, C.byref(n)) == J.JF_OK
    if n.value:
        assert policy(lib, nb=n.value - 1) == J.JF_ENOMEM and policy(lib, ws=None) == J.JF_ENOMEM
    for bad in ((2, 1, 1), (0, -1, 1), (0, 1, 0)):
        assert lib.jf_op_policy_loss_workspace_bytes(*bad, C.byref(n)) == J.JF_EINVAL
    assert lib.jf_op_policy_loss_workspace_bytes(0, 1, 1, None) == J.JF_EINVAL
    assert policy(lib, n=0, logits=None) == J.JF_OK
