"""Attention at the end of the range of lengths.  A unit or a step of tokens that begins
below the end of a request reaches past it, and its places are 32-bit numbers: the last
1,024 lengths below 2^31 would pass their range and are refused."""
import numpy as np
import pytest
import torch

import kv4_rows as R

pytestmark = pytest.mark.gpu

LAST = 2**31 - 1024


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from paper_2609_15359_gb300 import maps
    return maps


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n_q", [1, 200])
def test_the_longest_request(M, D, n_q):
    """2^31 - 1,024 tokens behind a table of blocks of 4,096 whose last one holds what the window shows."""
    rng = np.random.default_rng(D + n_q)
    S, Hq, H, window = 4096, 4, 2, 300
    held = window + n_q - 1
    k, v = (R.rounded(rng.normal(size=(held, H, D)).astype(np.float32), "fp16") for _ in range(2))
    q = R.rounded(rng.normal(size=(n_q, Hq, D)).astype(np.float32), "fp16")
    cache = torch.full(M.kv4_cache_shape(2, H, S, D), 0xff, dtype=torch.uint8, device="cuda")
    table = torch.zeros(1, 2**31 // S, dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    half = lambda x: torch.from_numpy(x).cuda().half()  # noqa: E731
    ws = M.Workspace()
    slots = S + (LAST - held + torch.arange(held, device="cuda")) % S
    assert M.maps_kv4_append(half(k), half(v), slots, cache, S, ws=ws) == 0
    out = torch.full((n_q, Hq, D), 77.0, dtype=torch.float16, device="cuda")
    lse = torch.zeros(n_q, Hq, device="cuda")
    off = torch.tensor([0, n_q], device="cuda")

    def status(n):
        assert M.maps_kv4_attention(half(q), off, torch.tensor([n], dtype=torch.int32, device="cuda"), table, cache, S, D ** -0.5,
                                    out, lse_out=lse, window=window, ws=ws) == 0
        return M.maps_check(ws)

    assert status(LAST) == 0
    e = R.expect("fp16", q, [0, n_q], [held], [k], [v], H, D ** -0.5, window=window)
    assert R.wrong(e, out.float().cpu().numpy(), lse.cpu().numpy()) is None
    for n in (LAST + 1, 2**31 - 97, 2**31 - 1):
        assert status(n) == M.MAPS_E_RANGE
    assert status(LAST) == 0


@pytest.mark.parametrize("n_q", [1, 300])
def test_more_work_than_a_call_can_count(M, n_q):
    """2^31 units and more are refused before any of them is begun: nothing is written."""
    S, B, D = 4096, 140, 64
    cache = torch.zeros(M.kv4_cache_shape(1, 1, S, D), dtype=torch.uint8, device="cuda")
    table = torch.zeros(B, 2**31 // S, dtype=torch.int32, device="cuda")
    q = torch.zeros(B * n_q, 1, D, dtype=torch.float16, device="cuda")
    out = torch.full_like(q, 7.0)
    ws = M.Workspace()
    off = torch.arange(B + 1, device="cuda") * n_q
    assert M.maps_kv4_attention(q, off, torch.full((B,), LAST, dtype=torch.int32, device="cuda"), table, cache, S, 0.1, out, ws=ws) == 0
    assert M.maps_check(ws) == M.MAPS_E_RANGE
    assert (out == 7).all()
