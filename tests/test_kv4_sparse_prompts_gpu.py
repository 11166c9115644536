"""The decoder example in its sparse form with lists shorter than the requests: prompts attend over all their keys, and
a request that decodes over its list, which leaves no row unwritten.  Both are compared with attention in 64 bits over
the keys as the cache holds them; the tolerance is that of test_kv4_gpu.py."""
import os
import sys

import numpy as np
import pytest
import torch

import kv4_oracle as K
import kv4_sparse_oracle as O

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_prompts_see_all_their_keys_and_decoding_requests_their_lists():
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from kv4_decoder import M, Decoder
    rng = np.random.default_rng(3)
    R, blocks, S, D, H, Hq = 8, 60, 16, 128, 2, 8
    prompt, output = rng.integers(60, 260, R), rng.integers(1, 14, R)
    prompt[0] = 65  # its last chunk is one token
    t = lambda x: torch.from_numpy(x.astype(np.int32)).cuda()  # noqa: E731
    d = Decoder(t(prompt), t(output), t(output * 2), blocks, heads=(Hq, H), D=D, S=S, chunk=64, sparse=3)
    keys, values = [[] for _ in range(R)], [[] for _ in range(R)]
    cos_sin = d.cos_sin.cpu().numpy()
    prompts_of_one, lists_short = 0, 0
    for step in range(400):
        if d.done():
            break
        before = d.held.cpu().numpy()
        r = d.step()
        assert M.maps_check(d.ws) == 0
        off, n, granted, pos = (r[x].cpu().numpy() for x in ("off", "n", "granted", "pos"))
        k = O.held_keys(O.rotate(r["k"].float().cpu().numpy(), pos[None], None, D, False, cos_sin))
        v = K.held_as(r["v"].float().cpu().numpy())
        q, out = r["q"].float().cpu().numpy(), r["out"].float().cpu().numpy()
        codes, scale, table = (x.cpu().numpy() for x in (d.codes, d.scale, d.table))
        blocks_of, tokens_of = O.select(q, off, n, table, codes, scale, S, 1, 2, 3, np.full((len(q), H, 3), -1), np.full((len(q), H), -1))
        assert np.isfinite(out).all()
        for b in range(R):
            if not granted[b]:
                continue
            keys[b].extend(k[off[b]:off[b + 1]])
            values[b].extend(v[off[b]:off[b + 1]])
            kk, vv = np.array(keys[b]).reshape(-1, H, D), np.array(values[b]).reshape(-1, H, D)
            big = max(np.abs(v).max(), 15 * K.quantise(r["v"].float().cpu().numpy())[1].max(), 6.0)
            if before[b] < prompt[b]:
                prompts_of_one += off[b + 1] - off[b] == 1
                ref, _ = K.attention(q[off[b]:off[b + 1]], [0, off[b + 1] - off[b]], [n[b]], [kk], [vv], H, D ** -0.5)
                assert np.abs(out[off[b]:off[b + 1]] - ref).max() <= 4 * 2.0**-9 * big, (step, b)
                continue
            i = off[b]
            assert off[b + 1] == i + 1
            for h in range(H):
                place = {int(x): j for j, x in enumerate(table[b, :-(-n[b] // S)])}
                at = np.concatenate([place[int(x)] * S + np.arange(S) for x in blocks_of[i, h] if x >= 0])[:tokens_of[i, h]]
                lists_short += len(at) < n[b]
                heads = slice(h * Hq // H, (h + 1) * Hq // H)
                ref, _ = K.attention(q[i:i + 1, heads], [0, 1], [len(at)], [kk[at][:, h:h + 1]], [vv[at][:, h:h + 1]], 1, D ** -0.5)
                assert np.abs(out[i, heads] - ref[0]).max() <= 4 * 2.0**-9 * big, (step, b, h)
    assert d.done() and prompts_of_one > 0 and lists_short > 0
