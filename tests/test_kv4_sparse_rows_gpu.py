"""Selected blocks where the form that takes a row changes: many rows of long tables, and tables so long that the rows
take their turns in the workspace."""
import numpy as np
import pytest

from test_kv4_sparse_gpu import M, check_select, select_data  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,H,D,kind", [(2, 2, 64, "bf16"), (6, 3, 128, "fp16"), (2, 1, 256, "bf16")])
@pytest.mark.parametrize("longest", [4094, 4095, 4096, 8190, 8191, 9000])  # a table has two blocks more
def test_select_blocks_of_many_rows_and_long_tables(M, longest, Hq, H, D, kind):  # noqa: F811
    rng = np.random.default_rng(longest + D)
    lens = np.concatenate([rng.integers(0, 800, 640 // H), [16 * longest, 16 * longest - 5, 16 * 2100, 16 * 4093, 16 * 257]])
    case = (Hq, H, D, 16, kind, [int(n) for n in rng.permutation(lens)], [1] * len(lens), 2, 1, 22)
    check_select(M, case, *select_data(case, rng))
    check_select(M, case, *select_data(case, rng, 40))


@pytest.mark.parametrize("Hq,H,D,kind,n_q", [(8, 8, 128, "bf16", [1]), (4, 2, 64, "fp16", [5]), (2, 2, 256, "bf16", [1, 1, 1]), (3, 1, 64, "bf16", [40])])
def test_select_blocks_of_few_rows_and_tables_longer_than_shared_memory(M, Hq, H, D, kind, n_q):  # noqa: F811
    """Every row and head has room of its own for its keys."""
    case = (Hq, H, D, 16, kind, [16 * (9000 + 700 * b) - 3 for b in range(len(n_q))], n_q, 1, 2, 90)
    check_select(M, case, *select_data(case, np.random.default_rng(H)))


@pytest.mark.parametrize("H,rows", [(1, 80), (3, 50)])
def test_select_blocks_of_rows_that_take_turns(M, H, rows):  # noqa: F811
    """Tables of 2^20 blocks: the workspace holds the keys of 2^26 / H rows and heads at a time."""
    most = 1 << 20
    n_q = [rows - 30, 30]
    case = (2 * H, H, 64, 16, "bf16", [16 * 9000 - 7, 16 * 300], n_q, 1, 2, 40)
    q, table, codes, scale, off = select_data(case, np.random.default_rng(rows))
    assert M.lib.maps_kv4_select_blocks_workspace_size(rows, H, most) < 4 * rows * H * most  # not all of them at once
    wide = np.full((2, most), -1, np.int32)
    wide[:, :table.shape[1]] = table
    check_select(M, case, q, wide, codes, scale, off)
