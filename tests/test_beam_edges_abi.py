"""Host-side limits of the operators for many continuations of one prompt (no device needed)."""
import pytest

from test_beam_abi import reorder
from test_serve_abi import zq  # noqa: F401


@pytest.mark.parametrize("kw", [dict(free_capacity=1 << 30), dict(free_capacity=(1 << 31) - 1), dict(batch=16384, beams=32, max_pages=2048), dict(batch=1, beams=1, max_pages=1 << 30, page_size=1),
                                dict(batch=16384, beams=32, max_pages=1 << 20, page_size=1)])
def test_reorder_refuses_lists_whose_sums_pass_32_bits(zq, kw):  # noqa: F811
    assert reorder(zq, **kw) == zq.ERR_UNSUPPORTED and b"2^30" in zq.lib().zoqat_last_error()


@pytest.mark.parametrize("kw", [dict(free_capacity=(1 << 30) - 1), dict(batch=16384, beams=32, max_pages=2047), dict(batch=1, beams=1, max_pages=(1 << 30) - 1, page_size=1)])
def test_the_largest_lists_are_taken(zq, kw):  # noqa: F811
    assert reorder(zq, nbytes=0, **kw) == zq.ERR_WORKSPACE_SMALL        # (the check behind these)
