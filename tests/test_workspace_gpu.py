"""Calls of the KV memory on another stream than the current one, with a workspace that is made, or
grows, while the current stream is busy, and with none."""
import numpy as np
import pytest
import torch

import kv4_rows as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from paper_2609_15359_gb300 import maps
    return maps


@pytest.mark.parametrize("kind", ["made while busy", "grows while busy", "large enough while busy", "none"])
@pytest.mark.parametrize("lens,n_q", [([900, 155, 3000], [1, 1, 1]), ([6100, 155], [701, 150])])
def test_attention_on_another_stream(M, kind, lens, n_q):
    rng = np.random.default_rng(len(lens))
    name, Hq, H, D = "bf16", 4, 2, 128
    k, v = (torch.randn(sum(lens), H, D, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(sum(n_q), Hq, D, device="cuda").bfloat16()
    nb = [-(-n // 16) for n in lens]
    table = torch.full((len(lens), max(nb)), -1, dtype=torch.int32)
    blocks, at, slots = torch.from_numpy(rng.permutation(sum(nb)).astype(np.int32)), 0, []
    for b, n in enumerate(lens):
        table[b, :nb[b]] = blocks[at:at + nb[b]]
        at += nb[b]
        j = torch.arange(n)
        slots.append(table[b, j // 16].long() * 16 + j % 16)
    table, slots = table.cuda(), torch.cat(slots).cuda()
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(n_q)])).cuda()
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    cache = torch.zeros(M.kv4_cache_shape(sum(nb), H, 16, D), dtype=torch.uint8, device="cuda")
    first = M.Workspace()
    assert M.maps_kv4_append(k, v, slots, cache, 16, ws=first) == 0
    args = (q, off, length, table, cache, 16, D ** -0.5)
    plain = torch.empty_like(q)
    assert M.maps_kv4_attention(*args, plain, ws=first) == 0
    assert M.maps_check(first) == 0
    split = np.cumsum(lens)[:-1]
    e = R.expect(name, q.float().cpu().numpy(), off.cpu().numpy(), lens, np.split(k.float().cpu().numpy(), split),
                 np.split(v.float().cpu().numpy(), split), H, D ** -0.5)
    assert R.wrong(e, plain.float().cpu().numpy()) is None
    side, out = torch.cuda.Stream(), torch.full_like(q, 3.0)
    need = M.lib.maps_kv4_attention_workspace_size(len(lens), sum(n_q), Hq, H, D)
    dirty = torch.full((3 * need,), 0xff, dtype=torch.uint8, device="cuda")
    big = torch.randn(8192, 8192, device="cuda").bfloat16()
    torch.cuda.synchronize()
    del dirty  # what the workspace's memory holds before it is zero-filled
    small = M.Workspace()
    for _ in range(20):
        big = big @ big * 1e-3  # some 15 ms of work on the current stream
    ws = {"made while busy": M.Workspace, "grows while busy": lambda: small,
          "large enough while busy": lambda: M.Workspace(need + 4096), "none": lambda: None}[kind]()
    assert M.maps_kv4_attention(*args, out, ws=ws, stream=side) == 0
    later = [torch.full((need,), 0xff, dtype=torch.uint8, device="cuda") for _ in range(4)]  # memory that was freed, if any was
    torch.cuda.synchronize()
    assert ws is None or M.maps_check(ws, side) == 0
    assert torch.equal(out, plain) and len(later) == 4


def test_an_error_of_the_first_call_outlives_growth(M):
    """Block tables report a bad length; append and attention then make the shared workspace grow."""
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    ws = M.Workspace()
    table, free, got = i32(0, 1, 2, 3).view(2, 2), i32(4, 5, 6, 7), i32(0, 0)
    off, slots = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    assert M.maps_block_tables(16, i32(5, -1), i32(6, 1), table, free, i32(4), i32(0), got, off, slots, ws=ws) == 0
    size = ws.nbytes
    q = torch.zeros(200, 4, 64, dtype=torch.bfloat16, device="cuda")
    cache = torch.zeros(M.kv4_cache_shape(8, 2, 16, 64), dtype=torch.uint8, device="cuda")
    assert M.maps_kv4_attention(q, torch.tensor([0, 100, 200], device="cuda"), i32(20, 20), table, cache, 16, 0.1, torch.empty_like(q),
                                ws=ws) == 0
    assert ws.nbytes > size
    assert M.maps_check(ws) == M.MAPS_E_RANGE and M.maps_check(ws) == 0
