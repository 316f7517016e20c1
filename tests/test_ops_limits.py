"""Limits of the 8-bit cache's C entry points, refused before a launch (no GPU)."""
import ctypes as C

import pytest

from paper_2512_14681_gb300 import _lib as J
from paper_2512_14681_gb300 import build as B


@pytest.fixture(scope="module")
def lib():
    B.build()
    return J.load()


def test_more_kv_heads_than_a_grid_holds(lib):
    """Append's grid has a row of CTAs for each KV head's keys and one for its queries: 65,535 at most."""
    for heads, hd in ((32768, 64), (65535, 128), (1 << 20, 64)):
        c = C.byref(J.Kv8Cache(256, 256, 256, 256, 256, 2, 8, 4, heads, hd))
        r, n, ld = C.byref(J.Kv8Rows(256, 256, 8, 5)), C.c_size_t(), heads * hd
        assert lib.jf_op_kv8_append(c, r, J.JF_BF16, 256, ld, 256, ld, 256, ld, heads, None, None, 0, J.JF_BF16, 256, 256, None) == J.JF_EUNSUPPORTED
        assert lib.jf_op_kv8_append(c, r, J.JF_BF16, None, 0, 256, ld, 256, ld, 0, None, None, 0, J.JF_BF16, None, 256, None) == J.JF_EUNSUPPORTED
        assert lib.jf_op_kv8_read(c, r, J.JF_F32, 256, 256, 256, None) == J.JF_EUNSUPPORTED
        assert lib.jf_op_kv8_attention_workspace_bytes(c, r, J.JF_BF16, heads, C.byref(n)) == J.JF_EUNSUPPORTED
