"""Rows held as NaN.  A value held as NaN makes the outputs of the queries that see it NaN, and
nothing else: lse has no value in it.  A key held as NaN makes both NaN.  The same with few
queries, with many, and for a request beside others.  Bounds: kv4_rows.py."""
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
@pytest.mark.parametrize("D,Hq,H,window", [(128, 4, 2, 0), (64, 8, 2, 0), (128, 8, 1, 90), (256, 4, 2, 0)])
@pytest.mark.parametrize("lens,n_q", [([300, 40], [3, 1]), ([300, 6100, 40], [200, 701, 40]), ([20011], [1])])
def test_values_and_keys_held_as_nan(M, name, D, Hq, H, window, lens, n_q):
    rng = np.random.default_rng(D + Hq + len(lens))
    k, v = ([R.rounded(rng.normal(size=(n, H, D)).astype(np.float32), name) for n in lens] for _ in range(2))
    for b, n in enumerate(lens):
        m = n_q[b]
        v[b][n - m // 2 - 1, 0, 5] = np.nan      # seen by half of the queries of one KV head
        v[b][max(0, n - m - 100), H - 1, 0] = np.inf  # by all of another's, or by those that its window reaches
        if b == 0:
            k[b][n - 1, H - 1, D - 1] = np.nan   # by the last query alone
    q = R.rounded(rng.normal(size=(sum(n_q), Hq, D)).astype(np.float32), name)
    e = R.expect(name, q, np.concatenate([[0], np.cumsum(n_q)]), lens, k, v, H, D ** -0.5, window=window)
    assert H * len(lens) == 1 or (np.isnan(e["out"]).any(-1) & np.isfinite(e["lse"])).any()
    out, lse = R.run(M, rng, name, q, lens, n_q, k, v, D ** -0.5, window=window)
    assert R.wrong(e, out, lse) is None
    out2, _ = R.run(M, rng, name, q, lens, n_q, k, v, D ** -0.5, window=window, with_lse=False)
    assert np.array_equal(out, out2, equal_nan=True)
