"""README's sparse step, run as it stands: with lists that hold every block it gives what attention over the
whole cache gives, to the bounds of kv4_rows.py."""
import os
import re

import numpy as np
import pytest
import torch

import kv4_rows as R
import kv4_sparse_oracle as O

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_sparse_step():
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from paper_2609_15359_gb300 import maps as M
    text = open(os.path.join(ROOT, "README.md")).read()
    code, = (c for c in re.findall(r"```python\n(.*?)```", text, re.S) if "maps_kv4_select_blocks" in c)
    rng = np.random.default_rng(4)
    S, D, Hq, H, lens = 16, 128, 32, 8, [900, 33, 1]
    nb = [-(-n // S) for n in lens]
    n_blocks = sum(nb) + 1
    perm = rng.permutation(n_blocks)
    table, at = np.full((3, max(nb)), -1, np.int32), 0
    for b in range(3):
        table[b, :nb[b]] = perm[at:at + nb[b]]
        at += nb[b]
    T = sum(lens)
    off = np.concatenate([[0], np.cumsum(lens)])
    pos = np.concatenate([np.arange(n) for n in lens]).astype(np.int32)
    req = np.repeat(np.arange(3), lens)
    angle = np.arange(900)[:, None] * 1e4 ** (-np.arange(64) / 64)
    turns = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
    q, k, v = (R.rounded(rng.normal(size=(T, h, D)).astype(np.float32), "bf16") for h in (Hq, H, H))
    dev = lambda x, t=None: torch.from_numpy(np.ascontiguousarray(x)).cuda().to(t or torch.from_numpy(np.ascontiguousarray(x)).dtype)  # noqa: E731
    b16 = torch.bfloat16
    names = dict(M=M, torch=torch, n_blocks=n_blocks, T=T, H=H, S=S, D=D, q=dev(q, b16), k=dev(k, b16), v=dev(v, b16), pos=dev(pos), cos_sin=dev(turns),
                 slots=dev(table[req, pos // S].astype(np.int64) * S + pos % S), held=dev(np.zeros(3, np.int32)), n=dev(np.array(lens, np.int32)),
                 table=dev(table), off=dev(off), cache=torch.zeros(M.kv4_cache_shape(n_blocks, H, S, D), dtype=torch.uint8, device="cuda"),
                 out=torch.zeros(T, Hq, D, dtype=b16, device="cuda"), ws=M.Workspace())
    for line in [x for x in code.strip().split("\n") if x]:
        exec(line, names)
        assert names.get("st", 0) == 0
    assert M.maps_check(names["ws"]) == 0
    tq = names["q"].float().cpu().numpy()
    assert np.array_equal(tq, torch.from_numpy(O.rotate(q, pos[None], None, D, False, turns)).bfloat16().float().numpy())
    lists, tokens = names["lists"].cpu().numpy(), names["tokens"].cpu().numpy()
    assert (tokens == (pos + 1)[:, None]).all()  # 57 blocks at most: all of them
    assert all((lists[i, :, :pos[i] // S + 1] == table[req[i], :pos[i] // S + 1]).all() for i in range(T))
    # the last rows of each request, against the keys as they are held
    tk = O.rotate(k, pos[None], None, D, False, turns)
    rows = [off[b + 1] - 1 for b in range(3)]
    group = Hq // H
    kk = [tk[off[b]:off[b + 1], h:h + 1] for b in range(3) for h in range(H)]
    vv = [v[off[b]:off[b + 1], h:h + 1] for b in range(3) for h in range(H)]
    e = R.expect("bf16", tq[rows].reshape(3 * H, group, D), np.arange(3 * H + 1), np.repeat(lens, H), kk, vv, 1, D ** -0.5)
    assert R.wrong(e, names["out"].float().cpu().numpy()[rows].reshape(3 * H, group, D)) is None
