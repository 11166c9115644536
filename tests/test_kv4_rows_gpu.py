"""Attention over the 4-bit cache held to a bound for every output, every row and every lse.
test_kv4_rows_host.py shows what the bounds reject in each of these cases."""
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
