"""Attention over lists held to what attention behind block tables is held to: values of very different
magnitudes, rows of one value, and rows held as NaN (test_kv4_magnitudes_gpu.py, test_kv4_nan_gpu.py),
with every query's list naming the blocks that it sees; scales of any sign."""
import numpy as np
import pytest
import torch

import kv4_rows as R
import test_kv4_magnitudes_gpu as G
import test_kv4_nan_gpu as N

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from paper_2609_15359_gb300 import maps
    return maps


def run_lists(M, rng, name, q, lens, n_q, k, v, scale, S=16, causal=True, window=0, with_lse=True, ws=None, status=0):
    """As kv4_rows.run, through lists: a row's list names its request's blocks, and its tokens end where the row stands."""
    assert causal and not window
    dt = dict(bf16=torch.bfloat16, fp16=torch.float16)[name]
    dev = lambda x, t=None: torch.from_numpy(np.ascontiguousarray(x)).cuda().to(t or torch.from_numpy(np.ascontiguousarray(x)).dtype)  # noqa: E731
    H, D = k[0].shape[1:]
    T, Hq, _ = q.shape
    nb = [-(-int(n) // S) for n in lens]
    perm = rng.permutation(sum(nb) + 2)
    lists, tokens, slots, at = np.full((T, H, max(nb)), -1, np.int32), np.zeros((T, H), np.int32), [], 0
    row = 0
    for b, n in enumerate(lens):
        mine = perm[at:at + nb[b]]
        at += nb[b]
        j = np.arange(int(n))
        slots.append(mine[j // S].astype(np.int64) * S + j % S)
        for x in range(n_q[b]):
            lists[row, :, :nb[b]] = mine
            tokens[row] = max(0, n - n_q[b] + x + 1)
            row += 1
    cache = torch.full(M.kv4_cache_shape(len(perm), H, S, D), 0xff, dtype=torch.uint8, device="cuda")
    assert M.maps_kv4_append(dev(np.concatenate(k), dt), dev(np.concatenate(v), dt), dev(np.concatenate(slots)), cache, S) == 0
    qd = dev(q, dt)
    out = torch.full_like(qd, 77.0)
    lse = torch.full((T, Hq), 77.0, device="cuda") if with_lse else None
    ws = ws or M.Workspace()
    assert M.maps_kv4_attention_blocks(qd, dev(lists), dev(tokens), cache, S, scale, out, lse_out=lse, ws=ws) == 0
    assert M.maps_check(ws) == status
    return out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64) if with_lse else None


@pytest.fixture(autouse=True)
def through_lists(monkeypatch):
    monkeypatch.setattr(R, "run", run_lists)


@pytest.mark.parametrize("name,loud", [("bf16", 14), ("bf16", 24), ("bf16", 60), ("fp16", 14), ("fp16", 24)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("where", ["early", "everywhere", "last"])
def test_loud_rows_of_no_weight(M, name, loud, D, where):
    G.test_loud_rows_of_no_weight(M, "few", name, loud, D, where)


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("steps", [-0.02, 0.002, 0.02])
def test_values_that_grow_or_shrink(M, name, D, steps):
    G.test_values_that_grow_or_shrink(M, "few", name, D, steps)


@pytest.mark.parametrize("name,nats,size", [("bf16", 16, 1.0), ("bf16", 24, 1.0), ("fp16", 12, 4096.0)])
@pytest.mark.parametrize("D", [64, 128])
def test_a_silent_row_that_all_look_at(M, name, D, nats, size):
    G.test_a_silent_row_that_all_look_at(M, "few", name, D, nats, size)


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nats", [10, 13, 16, 18])
def test_a_flat_tail_behind_one_row(M, name, D, nats):
    G.test_a_flat_tail_behind_one_row(M, "few", name, D, nats)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power", [0, 60, 126])
@pytest.mark.parametrize("share", [1.0, 0.2])
def test_rows_of_one_value(M, D, power, share):
    G.test_rows_of_one_value(M, "few", D, power, share)


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("D,Hq,H", [(128, 4, 2), (64, 8, 2), (256, 4, 2), (128, 16, 1)])
@pytest.mark.parametrize("lens,n_q", [([300, 40], [3, 1]), ([20011], [1])])
def test_values_and_keys_held_as_nan(M, name, D, Hq, H, lens, n_q):
    N.test_values_and_keys_held_as_nan(M, name, D, Hq, H, 0, lens, n_q)


@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-30, -3.0, 1e4])
@pytest.mark.parametrize("D,Hq", [(64, 5), (128, 16), (256, 3)])
def test_scales_of_any_sign_and_size(M, scale, D, Hq):
    rng = np.random.default_rng(D)
    lens = [500, 33, 1]
    k, v = ([R.rounded(rng.normal(size=(n, 1, D)).astype(np.float32), "bf16") for n in lens] for _ in range(2))
    q = R.rounded(rng.normal(size=(3, Hq, D)).astype(np.float32), "bf16")
    e = R.expect("bf16", q, np.arange(4), lens, k, v, 1, np.float32(scale))
    assert R.wrong(e, *run_lists(M, rng, "bf16", q, lens, [1] * 3, k, v, scale)) is None


@pytest.mark.parametrize("power", [-120, -60, 60, 100])
def test_queries_of_any_size(M, power):
    """With the scale to match, so that scores are a few nats."""
    rng = np.random.default_rng(3)
    lens = [300, 77]
    k, v = ([R.rounded(rng.normal(size=(n, 2, 128)).astype(np.float32), "bf16") for n in lens] for _ in range(2))
    q = R.rounded((rng.normal(size=(2, 8, 128)) * 2.0**power).astype(np.float32), "bf16")
    scale = float(np.float32(0.1 * 2.0**-power))
    e = R.expect("bf16", q, np.arange(3), lens, k, v, 2, scale)
    assert R.wrong(e, *run_lists(M, rng, "bf16", q, lens, [1] * 2, k, v, scale)) is None
