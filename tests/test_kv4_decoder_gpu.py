"""The decoder example: order, block tables, cache and attention together, until every
request is done, with a pool too small for all of them at once.  Every step's outputs
are compared with attention in 64 bits over what the cache holds by then, and no
block ever belongs to two requests.  The tolerance is that of test_kv4_gpu.py."""
import os
import sys

import numpy as np
import pytest
import torch

import kv4_oracle as K

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_decoder_until_done():
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from kv4_decoder import M, Decoder
    rng = np.random.default_rng(0)
    R, blocks, S = 12, 40, 16
    prompt, output = rng.integers(1, 200, R), rng.integers(1, 12, R)
    t = lambda x: torch.from_numpy(x.astype(np.int32)).cuda()  # noqa: E731
    d = Decoder(t(prompt), t(output), t(output * 2), blocks, heads=(8, 2), D=128, S=S, chunk=64)
    keys, values = [[] for _ in range(R)], [[] for _ in range(R)]
    queued = False
    for step in range(400):
        if d.done():
            break
        r = d.step()
        assert M.maps_check(d.ws) == 0
        off, n = r["off"].cpu().numpy(), r["n"].cpu().numpy()
        granted, slots = r["granted"].cpu().numpy(), r["slots"].cpu().numpy()
        queued |= bool((~d.admitted).any())
        assert (granted == (off[1:] > off[:-1])).all() and (slots >= 0).all()
        k, v = (K.held_as(r[x].float().cpu().numpy()) for x in "kv")
        for b in range(R):
            if granted[b]:
                keys[b].extend(k[off[b]:off[b + 1]])
                values[b].extend(v[off[b]:off[b + 1]])
                assert len(keys[b]) == n[b]
        table, held = d.table.cpu().numpy(), d.held.cpu().numpy()
        gone = d.returned.cpu().numpy()
        live = [table[b, :-(-int(held[b]) // S)] for b in range(R) if held[b] > 0 and not gone[b]]
        used = np.concatenate(live) if live else np.zeros(0, int)
        assert len(set(used.tolist())) == len(used) and int(d.n_free) + len(used) == blocks
        q = r["q"].float().cpu().numpy()
        ref, _ = K.attention(q, off, n, [np.array(keys[b]).reshape(-1, 2, 128) for b in range(R)],
                             [np.array(values[b]).reshape(-1, 2, 128) for b in range(R)], 2, 128 ** -0.5)
        big = max(np.abs(v).max(), 15 * K.quantise(r["v"].float().cpu().numpy())[1].max(), 6.0)
        assert np.abs(r["out"].float().cpu().numpy() - ref).max() <= 4 * 2.0**-9 * big, step
    assert d.done() and queued
