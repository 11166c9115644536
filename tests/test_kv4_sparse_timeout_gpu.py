"""The bounded waits of attention over lists: one block is never told that its copies have landed, so that every
warp of it runs into a limit, waits for what is under way and goes on to the joins, alone or in its cluster.  The
call ends with MAPS_E_TIMEOUT, the other rows and heads are right, and so is the next call."""
import numpy as np
import pytest
import torch

from test_kv4_sparse_gpu import M, attend_case  # noqa: F401

pytestmark = pytest.mark.gpu

CASES = [  # Hq, H, D, S, type, n_list, tokens of each row; the block, and the row and KV head that it has
    ((4, 1, 64, 16, "bf16", 12, [190, 192] * 300), 3, 3, 0), ((16, 1, 64, 16, "fp16", 20, [300, 320] * 300), 7, 7, 0),
    ((2, 1, 128, 32, "fp16", 9, [33, 288, 280] * 200), 1, 1, 0), ((4, 1, 256, 16, "bf16", 30, [480, 471] * 200), 0, 0, 0),
    ((4, 2, 128, 16, "bf16", 128, [2048, 2040, 1999]), 11, 0, 1), ((4, 2, 64, 16, "bf16", 128, [2048, 2040, 1999]), 32, 2, 0),
    ((8, 2, 256, 16, "fp16", 70, [1100, 1120]), 5, 0, 0), ((4, 2, 64, 64, "bf16", 2, [100, 3]), 0, 0, 0)]


def run_attend(M, case, args, ws):  # noqa: F811
    q, blocks, tokens, cache = args
    out, lse = torch.full_like(q, 77.0), torch.full(q.shape[:2], 77.0, device="cuda")
    assert M.maps_kv4_attention_blocks(q, blocks, tokens, cache, case[3], case[2] ** -0.5, out, lse_out=lse, ws=ws) == 0
    return out, lse


@pytest.mark.parametrize("tries", [100, 1000])
@pytest.mark.parametrize("case,block,row,head", CASES)
def test_waits_over_lists_run_out_and_the_next_call_is_right(M, case, block, row, head, tries):  # noqa: F811
    out, lse, args = attend_case(M, case)
    ws = M.Workspace()
    try:
        assert M.lib.maps_test_attention_withhold(block, tries) == 0
        got, got_lse = run_attend(M, case, args, ws)
        torch.cuda.synchronize()
    finally:
        assert M.lib.maps_test_attention_withhold(-1, 0) == 0
    assert M.maps_check(ws) == M.MAPS_E_TIMEOUT
    Hq, H = case[:2]
    others = np.ones((len(case[6]), Hq), bool)
    others[row, head * (Hq // H):(head + 1) * (Hq // H)] = False
    others = torch.from_numpy(others).cuda()
    assert torch.equal(got[others].view(torch.int16), out[others].view(torch.int16)) and torch.equal(got_lse[others], lse[others])
    got, got_lse = run_attend(M, case, args, ws)
    assert M.maps_check(ws) == 0
    assert torch.equal(got.view(torch.int16), out.view(torch.int16)) and torch.equal(got_lse, lse)
