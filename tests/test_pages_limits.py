"""Sizes at the limits of a launch, refused on the host (no GPU work)."""
import pytest

from paper_2606_03928_amd import pages, vase
from tests.test_pages_abi import attn, cache


@pytest.mark.parametrize("T,code", [(1 << 24, vase.ERR_UNSUPPORTED), ((1 << 21) + 1, vase.ERR_UNSUPPORTED),
                                    (1 << 21, vase.ERR_UNSUPPORTED), ((1 << 21) - 1, vase.ERR_WORKSPACE)])
def test_attn_refuses_more_rows_than_the_joining_launch_takes(T, code):
    # a few tokens of 4 slots in a batch that is padded to T, the keys in ranges: 4 of its
    # 32 rows a token go to a workgroup of 256 threads, and 2^32 threads are too many
    lib = pages.load()
    assert attn(lib, cache(), T=T, max_new=1, wsb=0) == code
