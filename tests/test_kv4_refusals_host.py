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


def test_binding_refuses_block_tables_of_other_sizes(M):
    """Before anything is read: no GPU needed."""
    import torch
    good = dict(held=torch.zeros(4), want=torch.zeros(4), table=torch.zeros(4, 7), free_blocks=torch.zeros(9), n_free=torch.zeros(1),
                n_free_out=torch.zeros(1), got_out=torch.zeros(4), slot_off_out=torch.zeros(5), slots_out=torch.zeros(6),
                pos_out=torch.zeros(6), order=torch.zeros(4))
    ws = M.Workspace(device="cpu")
    with pytest.raises(TypeError):  # the sizes are right; host tensors are not
        M.maps_block_tables(16, **good, ws=ws)
    for name, n in (("want", 3), ("got_out", 3), ("slot_off_out", 4), ("order", 3), ("pos_out", 5), ("held", 5)):
        with pytest.raises(ValueError):
            M.maps_block_tables(16, **good | {name: torch.zeros(n)}, ws=ws)
    for table in (torch.zeros(3, 7), torch.zeros(28)):
        with pytest.raises(ValueError):
            M.maps_block_tables(16, **good | dict(table=table), ws=ws)
