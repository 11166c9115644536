"""README's step on the KV memory, run as it stands, with a pool that is too small for one of
the requests: its new tokens have rows in the batch but no place in the cache."""
import os
import re

import numpy as np
import pytest
import torch

import kv4_rows as R

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_step_with_a_refused_request():
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from paper_2609_15359_gb300 import maps as M
    text = open(os.path.join(ROOT, "README.md")).read()
    code, = (c for c in re.findall(r"```python\n(.*?)```", text, re.S) if "maps_block_tables" in c)
    rng = np.random.default_rng(3)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    S, D, Hq, H, n_blocks = 16, 128, 32, 8, 12
    held = [20, 40, 30, 0]
    want = [21, 90, 31, 9]  # the second needs three blocks and comes last: two are left
    table = np.full((4, 6), -1, np.int32)
    table[0, :2], table[1, :3], table[2, :2] = [3, 9], [1, 0, 7], [11, 4]
    free = [2, 5, 6] + [-1] * 9
    T = sum(w - h for h, w in zip(held, want))
    old = [rng.normal(size=(n, 2, H, D)).astype(np.float32) for n in held]  # tokens of earlier steps
    new = rng.normal(size=(T, 2, H, D)).astype(np.float32)
    old, new = [R.K.bf16(x) for x in old], R.K.bf16(new)
    q = R.K.bf16(rng.normal(size=(T, Hq, D)).astype(np.float32))
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda().bfloat16()  # noqa: E731
    names = dict(M=M, torch=torch, n_blocks=n_blocks, held=i32(*held), want=i32(*want), table=torch.from_numpy(table).cuda(),
                 free_blocks=i32(*free), n_free=i32(3), n_free_out=i32(0), got=i32(0, 0, 0, 0), perm=i32(3, 0, 2, 1),
                 off=torch.zeros(5, dtype=torch.int64, device="cuda"), slots=torch.zeros(T, dtype=torch.int64, device="cuda"),
                 k=dev(new[:, 0]), v=dev(new[:, 1]), q=dev(q), out=torch.full((T, Hq, D), 7.0, device="cuda").bfloat16(), ws=M.Workspace())
    # what earlier steps wrote goes in as soon as the step has made its cache
    made, rest = code.split('device="cuda")\n', 1)
    exec(made + 'device="cuda")\n', names)
    for b, n in enumerate(held):
        j = np.arange(n)
        slots = torch.from_numpy(table[b, j // S].astype(np.int64) * S + j % S).cuda()
        assert M.maps_kv4_append(dev(old[b][:, 0]), dev(old[b][:, 1]), slots, names["cache"], S, ws=names["ws"]) == 0
    exec(rest, names)
    assert names["st"] == 0 and M.maps_check(names["ws"]) == 0
    assert names["got"].tolist() == [21, 40, 31, 9]
    off = names["off"].tolist()
    k, v, lens = [], [], []
    for b in range(4):
        refused = b == 1
        rows = np.concatenate([old[b], new[off[b]:off[b + 1]]]) if not refused else old[b][:0]
        k.append(rows[:, 0])
        v.append(rows[:, 1])
        lens.append(len(rows))
    e = R.expect("bf16", q, off, lens, k, v, H, D ** -0.5)
    out = names["out"].float().cpu().numpy()
    assert (out[off[1]:off[2]] == 0).all()  # refused: no key to see
    assert R.wrong(e, out) is None
