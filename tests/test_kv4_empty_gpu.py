"""Calls of no tokens, whatever strides an empty tensor has."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_no_tokens():
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from paper_2609_15359_gb300 import maps as M
    ws = M.Workspace()
    none = torch.empty(0, device="cuda").bfloat16().as_strided((0, 2, 64), (1, 2, 7))
    slots = torch.empty(0, dtype=torch.int64, device="cuda")
    cache = torch.full(M.kv4_cache_shape(3, 2, 16, 64), 0xa5, dtype=torch.uint8, device="cuda")
    assert M.maps_kv4_append(none, none, slots, cache, 16, ws=ws) == 0
    assert M.maps_kv4_read(slots, cache, 16, none, none, ws=ws) == 0
    off, n = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    table = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    assert M.maps_kv4_attention(none, off, n, table, cache, 16, 0.1, none, ws=ws) == 0
    assert M.maps_check(ws) == 0 and (cache == 0xa5).all()
