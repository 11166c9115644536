"""What the calls of sparse decoding report of bad data, wherever it stands, and what they leave as it is."""
import numpy as np
import pytest
import torch

import kv4_oracle as K
import kv4_rows as R
import kv4_sparse_oracle as O
from test_kv4_sparse_gpu import M, TYPES, dev, run_select, select_data  # noqa: F401

pytestmark = pytest.mark.gpu

# lengths, first, last, n_list, the entry of request 0 that is bad, whether it is used
ENTRIES = [
    ("fits", [40], 1, 1, 4, 1, True), ("fits, its last", [64], 0, 1, 4, 3, True), ("behind a row that fits", [40], 1, 1, 4, 3, False),
    ("first", [300], 2, 1, 6, 1, True), ("last", [300], 1, 2, 6, 17, True), ("behind the last", [300], 1, 2, 6, 19, False), ("scored", [300], 1, 2, 6, 9, True),
    ("first and last alone", [300], 2, 2, 4, 1, True), ("last and first alone", [300], 2, 2, 4, 18, True), ("between first and last alone", [300], 2, 2, 4, 9, False),
    ("one block", [1], 0, 1, 1, 0, True), ("first of a long row", [16 * 3000], 1, 2, 40, 0, True), ("last of a long row", [16 * 3000], 1, 2, 40, 2999, True)]


@pytest.mark.parametrize("bad", [-1, "behind", 0x7fffffff])
@pytest.mark.parametrize("case,rows", [(c, rows) for c in ENTRIES for rows in (1, 700) if rows == 1 or c[1][0] < 1000],  # many rows go to another form
                         ids=lambda x: x[0] if isinstance(x, tuple) else None)
def test_select_blocks_reports_every_entry_it_uses(M, case, bad, rows):  # noqa: F811
    _, lens, first, last, n_list, at, used = case
    c = (2, 1, 64, 16, "bf16", lens + [20] * (rows - 1), [1] * rows, first, last, n_list)
    q, table, codes, scale, off = select_data(c, np.random.default_rng(at))
    table = np.concatenate([table, np.full((rows, 2), -1, np.int32)], 1)  # nobody looks at these
    good = run_select(M, c, q, table, codes, scale, off)
    entry = table[0, at]
    table[0, at] = len(codes) if bad == "behind" else bad
    blocks, tokens = run_select(M, c, q, table, codes, scale, off, status=M.MAPS_E_RANGE if used else 0)
    assert np.array_equal(tokens, good[1]) and np.array_equal(blocks[1:], good[0][1:])
    if case[0] != "scored":  # whose score decides nothing: the list is the same but for the entry
        assert np.array_equal(blocks[0], np.where(good[0][0] == entry, table[0, at], good[0][0]) if used else good[0][0])
    want, _ = O.select(q, off, c[5], np.where(table < 0, 0, np.minimum(table, len(codes) - 1)), codes, scale, 16, first, last, n_list,
                       np.full(blocks.shape, -7), np.full(tokens.shape, -7))
    assert np.array_equal(want[1:], blocks[1:])


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("T,what", [(9, "pos"), (9, "axis"), (9, "both"), (4000, "both")])
def test_append_rotated_leaves_pairs_without_a_position(M, T, what, inter, kind):  # noqa: F811
    """Beside infinities, NaN and zeros of either sign: a pair that is not turned takes nothing from its partner."""
    rng = np.random.default_rng(T + inter)
    Hq, H, D, S, rot, n_pos = 3, 2, 128, 16, 96, 20
    F = rot // 2
    dt = TYPES[kind]
    x = [R.rounded(rng.normal(size=(T, h, D)).astype(np.float32), kind) for h in (Hq, H, H)]
    for y in x[:2]:
        for bad in (np.inf, -np.inf, np.nan, -0.0, 0.0):
            y[rng.random(y.shape) < 0.02] = bad
    angle = rng.uniform(0, 100, (n_pos, F))
    cos_sin = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
    pos = rng.integers(0, n_pos, (3, T)).astype(np.int32)
    axis = rng.integers(0, 3, F).astype(np.int32)
    axis[8:24] = 1  # lanes on one axis, and such as have several
    if what != "axis":
        pos[1, ::2], pos[2, 1::3] = -1, n_pos
    if what != "pos":
        axis[[3, 30, 31, F - 1]] = [3, -1, 8, 1 << 30]
    turned = []
    for y in x[:2]:
        z = O.rotate(y, np.clip(pos, 0, n_pos - 1), np.clip(axis, 0, 2), rot, inter, cos_sin)
        for f in range(F):
            p = pos[axis[f]] if 0 <= axis[f] < 3 else np.full(T, -1)
            lost = (p < 0) | (p >= n_pos)
            for c in ((2 * f, 2 * f + 1) if inter else (f, f + F)):
                z[lost, :, c] = y[lost, :, c]
        turned.append(z)
    n = T // S + 1
    cache = torch.zeros(M.kv4_cache_shape(n, H, S, D), dtype=torch.uint8, device="cuda")
    q, k, v = (torch.from_numpy(y).cuda().to(dt) for y in x)
    out, ws, slots = torch.empty_like(q), M.Workspace(), torch.arange(T, device="cuda")
    assert M.maps_kv4_append_rotated(q, k, v, dev(pos), dev(cos_sin), slots, cache, S, out, axis=dev(axis), interleaved=inter, ws=ws) == 0
    assert M.maps_check(ws) == M.MAPS_E_RANGE
    want, got = torch.from_numpy(turned[0]).to(dt), out.cpu()
    nan = want.isnan()
    assert torch.equal(got.isnan(), nan) and torch.equal(got[~nan].view(torch.int16), want[~nan].view(torch.int16))
    rows = [torch.empty(T, H, D, dtype=dt, device="cuda") for _ in range(2)]
    assert M.maps_kv4_read(slots, cache, S, *rows) == 0
    for y, z in zip(rows, (turned[1], x[2])):
        want = torch.from_numpy(K.held_as(z)).to(dt)
        assert torch.equal(y.cpu().isnan(), want.isnan()) and torch.equal(y.cpu().nan_to_num(), want.nan_to_num())
