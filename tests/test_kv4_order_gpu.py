"""Block tables in an order that is no permutation: reported, and no block that is not free is handed
out, whatever the workspace held before."""
import numpy as np
import pytest
import torch

import kv4_oracle as K

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,cap", [(2, 2000), (64, 2000), (64, 5000), (1000, 20000), (1024, 600000), (3000, 60000), (20000, 400000), (20000, 600000)])
@pytest.mark.parametrize("what", ["twice", "outside"])
def test_an_order_that_leaves_a_request_out(R, cap, what):
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from paper_2609_15359_gb300 import maps as M
    rng = np.random.default_rng(R)
    S, mb = 16, 4
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()  # noqa: E731
    held = rng.integers(0, 30, R)
    want = held + rng.integers(1, 20, R)
    hb = -(-held // S)
    pool = 4 * R + 10
    perm = rng.permutation(pool).astype(np.int32)
    table = np.full((R, mb), -1, np.int32)
    table[np.arange(mb) < hb[:, None]] = perm[:hb.sum()]
    n_free = pool - int(hb.sum())
    free = np.concatenate([perm[hb.sum():], np.full(int(hb.sum()), -1, np.int32)])
    order = rng.permutation(R).astype(np.int32)
    left_out = int(order[0])
    bad = order.copy()
    bad[0] = order[R - 1] if what == "twice" else R
    ws = M.Workspace()
    st = {}

    def run(o):
        st.update(table=i32(table), n=i32([0]), got=i32(np.zeros(R)), off=torch.zeros(R + 1, dtype=torch.int64, device="cuda"),
                  slots=torch.full((cap,), -9, dtype=torch.int64, device="cuda"))
        assert M.maps_block_tables(S, i32(held), i32(want), st["table"], i32(free), i32([n_free]), st["n"], st["got"], st["off"], st["slots"],
                                   order=i32(o), ws=ws) == 0
        return M.maps_check(ws)

    ref = K.block_tables(S, held, want, table, free, n_free, order)
    for o, status in ((bad, M.MAPS_E_RANGE), (order, 0), (bad, M.MAPS_E_RANGE), (order, 0)):
        assert run(o) == status
        t, off, slots = st["table"].cpu().numpy(), st["off"].cpu().numpy(), st["slots"].cpu().numpy()
        if status == 0:
            assert np.array_equal(t, ref[0]) and np.array_equal(slots[:len(ref[5])], ref[5]) and int(st["n"]) == ref[2]
        else:
            assert np.array_equal(t[left_out], table[left_out]) and (slots[off[left_out]:off[left_out + 1]] == -1).all()
            used = t[t >= 0]
            assert len(np.unique(used)) == len(used)
