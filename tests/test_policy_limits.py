"""Limits of the policy loss's C entry point that the host checks (no GPU: every call here is refused before a launch)."""
import pytest

from paper_2512_14681_gb300 import _lib as J
from paper_2512_14681_gb300 import build as B
from tests.test_more_ops_abi import policy


@pytest.fixture(scope="module")
def lib():
    B.build()
    return J.load()


def test_scales_that_masks_do_not_survive_are_refused(lib):
    """A logit of -infinity counts as -1e30 where products are taken: 1e30 * scale * log2 e has to pass the 126 below which 2^-x is not 0.
    (No rows: what is not refused returns without a launch.)"""
    for scale in (9.9e-29, 1e-29, 1e-37, 1e-45, 0.0, -1.0, 1.1e30):
        assert policy(lib, n=0, scale=scale) == J.JF_EINVAL, scale
    for scale in (1.01e-28, 1e-20, 1.0, 0.99e30):
        assert policy(lib, n=0, scale=scale) == J.JF_OK, scale
