"""Refusals of the KV memory's calls at the ends of their ranges: before anything is enqueued,
so that no GPU is needed and no pointer is read."""
import ctypes

import pytest

P = ctypes.c_void_p(1 << 20)
BIG = 1 << 40


@pytest.fixture(scope="module")
def M():
    from paper_2609_15359_gb300 import build
    build.build()
    from paper_2609_15359_gb300 import maps
    return maps


@pytest.mark.parametrize("R", [2**30 + 1, 2**31 - 1024, 2**31 - 1])
def test_block_tables_refuses_more_requests_than_it_can_count(M, R):
    """Places within the last tile of requests would pass 32 bits."""
    assert M.lib.maps_block_tables(R, 16, P, P, P, P, 8, P, 9, P, P, P, P, P, 5, P, P, BIG, None) == M.MAPS_E_INVALID
