"""Limits of the policy loss's C entry point that the host checks (no GPU: every call here is refused before a launch)."""
import ctypes as C
import re

import pytest

from paper_2512_14681_gb300 import _lib as J
from paper_2512_14681_gb300 import build as B
from tests.test_more_ops_abi import policy


@pytest.fixture(scope="module")
def lib():
    B.build()
    return J.load()


def test_scales_that_masks_do_not_survive_are_refused(lib):
    """Logits that differ by more than 1e30 may count as that far apart: 1e30 * scale * log2 e has to pass the 126 up to which 2^-x is not 0.
    (No rows: what is not refused returns without a launch.)"""
    for scale in (9.9e-29, 1e-29, 1e-37, 1e-45, 0.0, -1.0, 1.1e30):
        assert policy(lib, n=0, scale=scale) == J.JF_EINVAL, scale
    for scale in (1.01e-28, 1e-20, 1.0, 0.99e30):
        assert policy(lib, n=0, scale=scale) == J.JF_OK, scale


@pytest.mark.parametrize("dtype,longest", [(J.JF_F32, 230400), (J.JF_BF16, 460800)], ids=["f32", "bf16"])
def test_rows_that_need_a_workspace(lib, dtype, longest):
    """Up to the length that the header names none is asked for; beyond, one that is missing or a byte too small is refused."""
    n, size = C.c_size_t(), 2 if dtype == J.JF_BF16 else 4
    for rows in (1, 2, 3, 200):
        for vocab in (1, 100, longest - 1, longest, longest + 16 // size - 1):
            assert lib.jf_op_policy_loss_workspace_bytes(dtype, rows, vocab, C.byref(n)) == J.JF_OK and n.value == 0, (rows, vocab)
    for rows in (1, 2, 200):
        for vocab in (longest + 16 // size, longest + 1000, 1 << 20):
            assert lib.jf_op_policy_loss_workspace_bytes(dtype, rows, vocab, C.byref(n)) == J.JF_OK and n.value >= rows * 24, (rows, vocab)
            z = dict(dtype=dtype, n=rows, vocab=vocab, ld=vocab, ld_g=vocab, g=1 << 40)
            assert policy(lib, nb=n.value - 1, **z) == J.JF_ENOMEM and policy(lib, nb=0, **z) == J.JF_ENOMEM and policy(lib, ws=None, **z) == J.JF_ENOMEM


def test_the_header_names_that_length():
    text = open(B.ROOT + "/include/jf_ops.h").read()
    fp32, bf16 = re.search(r"rows longer than a cluster's shared memory, ([0-9,]+) fp32 or ([0-9,]+) bf16 values", text).groups()
    assert (fp32, bf16) == ("230,400", "460,800")
