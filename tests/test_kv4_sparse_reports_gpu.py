"""What the calls of sparse decoding report of bad data, wherever it stands, and what they leave as it is."""
import numpy as np
import pytest
import torch

import kv4_sparse_oracle as O
from test_kv4_sparse_gpu import M, run_select, select_data  # noqa: F401

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
