"""Attention over the 4-bit cache held to a bound for every output, every row and every lse.
test_kv4_rows_host.py shows what the bounds reject in each of these cases."""
import numpy as np
import pytest
import torch

import kv4_cases as C
import kv4_rows as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("name", C.CASES)
def test_rows(name, kind):
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from paper_2609_15359_gb300 import maps as M
    c = C.CASES[name]
    rng, q, k, v = C.data(name, kind)
    _, e = C.expect(name, kind, q, k, v)
    out, lse = R.run(M, rng, kind, q, c["lens"], c["n_q"], k, v, c["D"] ** -0.5, c["S"], c["causal"], c["window"])
    assert R.wrong(e, out, lse) is None


@pytest.mark.parametrize("seed", range(12))
def test_rows_of_random_calls(seed):
    """Random heads, lengths, queries, windows, block sizes and types, some of them with one request of much work."""
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from paper_2609_15359_gb300 import maps as M
    rng = np.random.default_rng(seed)
    for _ in range(6):
        kind = str(rng.choice(["bf16", "fp16"]))
        H, group, D = int(rng.integers(1, 4)), int(rng.choice([1, 2, 3, 5, 8])), int(rng.choice([64, 128, 256]))
        B, most = int(rng.integers(1, 12)), int(rng.choice([20, 200, 1500]))
        lens = rng.integers(0, most, B)
        n_q = np.ones(B, int) if rng.random() < 0.3 else rng.integers(0, int(rng.choice([4, 12, 90, 300])), B)
        if rng.random() < 0.4:
            lens[0], n_q[0] = 6100, 2800 // (H * group) + 1
        if n_q.sum() == 0 or lens.sum() == 0:
            continue
        causal, window, S = bool(rng.random() < 0.8), int(rng.choice([0, 0, 1, 40, 500])), int(rng.choice([16, 32, 48, 64]))
        k = [R.rounded(rng.normal(size=(n, H, D)).astype(np.float32), kind) for n in lens]
        v = [R.rounded((rng.normal(size=(n, H, D)) * 2.0 ** rng.uniform(-6, 6, (n, H, 1))).astype(np.float32), kind) for n in lens]
        q = R.rounded((rng.choice([0.5, 1, 3]) * rng.normal(size=(n_q.sum(), H * group, D))).astype(np.float32), kind)
        e = R.expect(kind, q, np.concatenate([[0], np.cumsum(n_q)]), lens, k, v, H, D ** -0.5, causal, window)
        out, lse = R.run(M, rng, kind, q, lens, n_q, k, v, D ** -0.5, S, causal, window)
        assert R.wrong(e, out, lse) is None, (kind, H, group, D, lens, n_q, causal, window, S)
