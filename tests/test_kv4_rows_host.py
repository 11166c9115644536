"""What the row-wise bounds reject, in every case that they are used on: outputs of zeros, a part of
the keys left out or given other tokens' values, rows of another head, and lse a little off.
The right outputs, rounded to their type, pass."""
import numpy as np
import pytest

import kv4_cases as C
import kv4_rows as R


def spoilt(name, q, k, v, off, how):
    """(rows, head, outputs) of one query head and the longest request with a part of its keys, about what one
    multiprocessor has of a call, left out or with the values of the tokens 16 places on."""
    c = C.CASES[name]
    b = int(np.argmax(c["lens"]))
    n, rows = c["lens"][b], np.arange(off[b], off[b + 1])
    # seen by every row, and near the end of what the first one sees
    first = n - len(rows) if c["causal"] else n - 1
    width = max(48, n // 152)
    a = max(0, first + 1 - width - 16) // 16 * 16
    at = n - len(rows) + np.arange(len(rows))[:, None]
    j = np.arange(n)
    seen = (j <= at if c["causal"] else np.ones((len(rows), n), bool)) & ((j > at - c["window"]) if c["window"] else True)
    w = q[rows, 0].astype(np.float64) @ R.held(k[b][:, 0])[0].T * c["D"] ** -0.5
    w = np.where(seen, w, -np.inf)
    p = np.exp(w - w.max(1, keepdims=True))
    values = R.held(v[b][:, 0])[0].copy()
    if how == "left out":
        p[:, a:a + width] = 0
    else:
        values[a:a + width] = np.roll(values, -16, 0)[a:a + width]
    return rows, 0, p @ values / p.sum(1, keepdims=True)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("name", C.CASES)
def test_what_is_rejected(name, kind):
    _, q, k, v = C.data(name, kind)
    off, e = C.expect(name, kind, q, k, v)
    right = R.rounded(e["out"].astype(np.float32), kind).astype(np.float64)
    assert R.wrong(e, right, e["lse"].astype(np.float32)) is None
    live = np.isfinite(e["lse"]).all(1)
    # every row that sees a key rejects zeros, not just one of them
    norm = np.linalg.norm(e["out"][live], axis=-1)
    assert (norm > e["norm"][live]).all()
    assert R.wrong(e, np.zeros_like(right)) is not None
    for how in ("left out", "other tokens"):
        rows, x, out = spoilt(name, q, k, v, off, how)
        bad = right.copy()
        bad[rows, x] = R.rounded(out.astype(np.float32), kind)
        assert R.wrong(e, bad) is not None, how
    bad = right.copy()
    bad[:, [0, -1]] = bad[:, [-1, 0]]
    assert R.wrong(e, bad) is not None
    lse = e["lse"] + np.where(np.isfinite(e["lse"]), 3e-3, 0)
    assert R.wrong(e, right, lse) is not None
    assert (e["lse_tol"][live] < 3e-3).all()
