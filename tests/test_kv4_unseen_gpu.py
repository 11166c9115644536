"""Places of a request that no query sees, ahead of a window, hold whatever they hold: scales and zeros
that are infinite or NaN there, as memory that was never written may have them, do not matter.
Bounds: kv4_rows.py."""
import numpy as np
import pytest
import torch

import kv4_rows as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [0x7f80, 0xff80, 0x7fc0, 0x7f7f])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,m,window", [(6100, 701, 100), (2117, 3, 70), (3000, 1, 1)])
def test_what_lies_ahead_of_the_window(D, n, m, window, bits):
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from paper_2609_15359_gb300 import maps as M
    rng = np.random.default_rng(n + D)
    Hq, H, S, name = 4, 2, 16, "bf16"
    k, v = (R.rounded(rng.normal(size=(n, H, D)).astype(np.float32), name) for _ in range(2))
    q = R.rounded(rng.normal(size=(m, Hq, D)).astype(np.float32), name)
    blocks = -(-n // S)
    table = torch.from_numpy(rng.permutation(blocks).astype(np.int32)).cuda()[None]
    j = torch.arange(n, device="cuda")
    slots = table[0, j // S].long() * S + j % S
    cache = torch.full(M.kv4_cache_shape(blocks, H, S, D), 0xff, dtype=torch.uint8, device="cuda")
    dev = lambda x: torch.from_numpy(x).cuda().bfloat16()  # noqa: E731
    ws = M.Workspace()
    assert M.maps_kv4_append(dev(k), dev(v), slots, cache, S, ws=ws) == 0
    unseen = max(0, n - m - window + 1)
    at = j[:unseen]
    words = cache.view(torch.int16).view(blocks, H, -1)[:, :, 8 * D:].view(blocks, H, 2, 16, 2)  # of K and V, {scale, zero} of each token
    value = torch.tensor(bits if bits < 0x8000 else bits - 0x10000, dtype=torch.int16, device="cuda")
    for h in range(H):
        for which in range(2):
            words[table[0, at // S].long(), h, which, at % S] = value
    out = torch.full((m, Hq, D), 77.0, device="cuda").bfloat16()
    lse = torch.zeros(m, Hq, device="cuda")
    assert M.maps_kv4_attention(dev(q), torch.tensor([0, m], device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda"), table, cache, S,
                                D ** -0.5, out, lse_out=lse, window=window, ws=ws) == 0
    assert M.maps_check(ws) == 0
    e = R.expect(name, q, [0, m], [n], [k], [v], H, D ** -0.5, window=window)
    assert R.wrong(e, out.float().cpu().numpy(), lse.cpu().numpy()) is None
