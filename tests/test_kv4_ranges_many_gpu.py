"""Ranges of blocks for many requests: the first block that a request's tokens went to and those behind it are dealt out
apart, and in turns, so these are calls of every number of requests and heads where that could go wrong."""
import numpy as np
import pytest
import torch

from test_kv4_sparse_gpu import M, check_ranges, dev, filled, i32  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,H,D,S", [(1, 9, 64, 16), (303, 3, 64, 16), (305, 12, 64, 32), (609, 8, 128, 16), (1023, 1, 64, 16), (1024, 2, 64, 16), (1025, 1, 256, 16),
                                     (3000, 5, 64, 48), (80000, 1, 64, 16)])
@pytest.mark.parametrize("what", ["a token each", "mixed", "all"])
def test_block_ranges_of_many_requests(M, B, H, D, S, what):  # noqa: F811
    rng = np.random.default_rng(B + len(what))
    few = B > 10000
    lens = rng.integers(0, 20 if few else 3 * S, B)
    if what == "mixed":
        lens[rng.integers(0, B, 5)] = rng.integers(10 * S, 40 * S, 5)
        lens[-1] = 33 * S + 1
    held = None if what == "all" else np.maximum(lens - 1, 0)
    if what == "mixed":
        held = np.where(rng.random(B) < 0.1, rng.integers(0, 4 * S, B), held)  # of which some pass the length
        held[-1] = 1
    k, v, table, cache = filled(M, rng, lens, H, D, S)
    check_ranges(M, k, table, cache, [int(n) for n in lens], None if held is None else [int(n) for n in held], H, D, S)


@pytest.mark.parametrize("B,at", [(1, 0), (700, 0), (700, 699), (3000, 1024), (3000, 2999), (80000, 79999)])
@pytest.mark.parametrize("what", ["negative", "long", "first entry", "another entry", "held", "none"])
def test_block_ranges_of_many_requests_report_bad_data(M, B, at, what):  # noqa: F811
    P, S, H, D = 9, 16, 2, 64
    lens, held, table = np.full(B, 60), np.full(B, 30), np.tile(np.arange(4, dtype=np.int32), (B, 1))
    table[:, 0] = -1  # nobody looks at these
    if what == "negative":
        lens[at] = -1
    if what == "long":
        lens[at] = 65
    if what == "first entry":
        table[at, 1] = P
    if what == "another entry":
        table[at, 3] = -1
    if what == "held":
        held[at] = -1
    cache = torch.zeros(M.kv4_cache_shape(P, H, S, D), dtype=torch.uint8, device="cuda")
    codes, scale = torch.full((P, H, 2, D), 77, dtype=torch.int8, device="cuda"), torch.full((P, H), 77.0, device="cuda")
    ws = M.Workspace()
    assert M.maps_kv4_block_ranges(i32(held), i32(lens), dev(table), cache, S, codes, scale, ws=ws) == 0
    assert M.maps_check(ws) == (0 if what == "none" else M.MAPS_E_RANGE)
    touched = torch.zeros(P, dtype=torch.bool)
    touched[1:4] = B > 1 or what == "none"
    if B == 1 and what in ("first entry", "another entry"):
        touched[[2, 3] if what == "first entry" else [1, 2]] = True
    assert ((scale.cpu() == 0).all(1) == touched).all() and ((scale.cpu() == 77).all(1) == ~touched).all()
    assert ((codes.cpu() == 0).flatten(1).all(1) == touched).all()
