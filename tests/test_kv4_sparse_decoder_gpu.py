"""The decoder example in its sparse form.  With lists as long as the longest request every query
attends over all blocks, so each step's outputs are those of attention in 64 bits over the turned keys
as the cache holds them; the tolerance is that of test_kv4_gpu.py.  With short lists it runs to its end."""
import os
import sys

import numpy as np
import pytest
import torch

import kv4_oracle as K
import kv4_sparse_oracle as O

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sparse", [20, 4])
def test_sparse_decoder_until_done(sparse):
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from kv4_decoder import M, Decoder
    rng = np.random.default_rng(1)
    R, blocks, S, D = 10, 40, 16, 128
    prompt, output = rng.integers(1, 200, R), rng.integers(1, 12, R)
    t = lambda x: torch.from_numpy(x.astype(np.int32)).cuda()  # noqa: E731
    d = Decoder(t(prompt), t(output), t(output * 2), blocks, heads=(8, 2), D=D, S=S, chunk=64, sparse=sparse)
    assert d.table.shape[1] <= 20
    keys, values = [[] for _ in range(R)], [[] for _ in range(R)]
    cos_sin = d.cos_sin.cpu().numpy()
    for step in range(400):
        if d.done():
            break
        r = d.step()
        assert M.maps_check(d.ws) == 0
        off, n, granted = (r[x].cpu().numpy() for x in ("off", "n", "granted"))
        pos = r["pos"].cpu().numpy()
        k = O.held_keys(O.rotate(r["k"].float().cpu().numpy(), pos[None], None, D, False, cos_sin))
        v = K.held_as(r["v"].float().cpu().numpy())
        for b in range(R):
            if granted[b]:
                keys[b].extend(k[off[b]:off[b + 1]])
                values[b].extend(v[off[b]:off[b + 1]])
                assert len(keys[b]) == n[b] and (pos[off[b]:off[b + 1]] == np.arange(n[b] - off[b + 1] + off[b], n[b])).all()
        out = r["out"].float().cpu().numpy()
        assert np.isfinite(out).all()
        if sparse < d.table.shape[1]:
            continue
        ref, _ = K.attention(r["q"].float().cpu().numpy(), off, n, [np.array(keys[b]).reshape(-1, 2, D) for b in range(R)],
                             [np.array(values[b]).reshape(-1, 2, D) for b in range(R)], 2, D ** -0.5)
        big = max(np.abs(v).max(), 15 * K.quantise(r["v"].float().cpu().numpy())[1].max(), 6.0)
        assert np.abs(out - ref).max() <= 4 * 2.0**-9 * big, step
    assert d.done()
