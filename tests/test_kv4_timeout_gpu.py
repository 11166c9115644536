"""The bounded waits of attention with many queries: one block is never told that its keys
are there, so that every warp of it runs into a limit.  The call ends with
MAPS_E_TIMEOUT, and the next one is right.  The four softmax warps of a tile
meet in a barrier without a limit of its own, so they have to leave together."""
import numpy as np
import pytest
import torch

import kv4_rows as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block,tries", [(0, 200), (77, 2000)])
@pytest.mark.parametrize("D", [64, 128])
def test_waits_run_out_and_the_next_call_is_right(D, block, tries):
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from paper_2609_15359_gb300 import maps as M
    rng = np.random.default_rng(D)
    Hq, H, lens, n_q = 4, 2, [3000, 6100, 500], [300, 701, 40]
    k, v = ([rng.normal(size=(n, H, D)).astype(np.float16).astype(np.float32) for n in lens] for _ in range(2))
    q = rng.normal(size=(sum(n_q), Hq, D)).astype(np.float16).astype(np.float32)
    off = np.concatenate([[0], np.cumsum(n_q)])
    try:
        assert M.lib.maps_test_attention_withhold(block, tries) == 0
        R.run(M, rng, "fp16", q, lens, n_q, k, v, D ** -0.5, status=M.MAPS_E_TIMEOUT)
    finally:
        assert M.lib.maps_test_attention_withhold(-1, 0) == 0
    out, lse = R.run(M, rng, "fp16", q, lens, n_q, k, v, D ** -0.5)
    assert R.wrong(R.expect("fp16", q, off, lens, k, v, H, D ** -0.5), out, lse) is None
