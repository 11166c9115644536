"""Attention with many queries where the running maximum keeps growing: every step of keys
scores far above the ones before, so that each step's scores are computed a second time
and the sums so far are brought to the new maximum.  Bounds: kv4_rows.py."""
import numpy as np
import pytest
import torch

import kv4_rows as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from paper_2609_15359_gb300 import maps
    return maps


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("D,Hq,H,rise,window", [(128, 8, 2, 0.12, 0), (64, 4, 4, 0.2, 0), (128, 4, 1, 0.5, 700), (64, 8, 1, 0.06, 0)])
def test_scores_that_keep_growing(M, name, D, Hq, H, rise, window):
    """Scores that rise by `rise` a token, 10 to 90 to a step of 128 keys."""
    rng = np.random.default_rng(D + Hq)
    lens, n_q = [6100, 700, 300], [2800 // Hq + 1, 300, 130]
    k, v = [], []
    along = rng.choice([-1.0, 1.0], (H, D))
    for n in lens:
        up = np.arange(n)[:, None, None] * rise / D ** 0.5
        k.append(R.rounded((along * up + 0.2 * rng.normal(size=(n, H, D))).astype(np.float32), name))
        v.append(R.rounded(rng.normal(size=(n, H, D)).astype(np.float32), name))
    T = sum(n_q)
    q = R.rounded((np.repeat(along, Hq // H, 0) + 0.2 * rng.normal(size=(T, Hq, D))).astype(np.float32), name)
    off = np.concatenate([[0], np.cumsum(n_q)])
    e = R.expect(name, q, off, lens, k, v, H, D ** -0.5, window=window)
    ws = M.Workspace()
    for _ in range(3):
        out, lse = R.run(M, rng, name, q, lens, n_q, k, v, D ** -0.5, window=window, ws=ws)
        assert R.wrong(e, out, lse) is None
