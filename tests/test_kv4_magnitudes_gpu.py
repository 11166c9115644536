"""Attention over values of very different magnitudes.  What a row's output is off by is bounded by
the terms of that row (kv4_rows.py): value rows that are far larger count for nothing
where their weight does, or where the row does not see them, and a row that every
query looks at counts for nothing where its value is zero."""
import numpy as np
import pytest
import torch

import kv4_rows as R

pytestmark = pytest.mark.gpu

FORMS = {"few": ([700, 300, 130], [3, 1, 2]), "many": ([6100, 700, 300], [701, 300, 130])}
HQ, H = 4, 2


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from paper_2609_15359_gb300 import maps
    return maps


def inputs(rng, name, D, form, size=2.0**-10):
    """Queries along a direction, keys of a few nats about it, values of one size; the direction to raise or lower keys by."""
    lens, n_q = FORMS[form]
    along = rng.choice([-1.0, 1.0], (H, D))
    k = [0.6 * rng.normal(size=(n, H, D)) for n in lens]
    v = [size * rng.normal(size=(n, H, D)) for n in lens]
    q = np.repeat(along, HQ // H, 0) + 0.3 * rng.normal(size=(sum(n_q), HQ, D))
    return lens, n_q, k, v, R.rounded(q.astype(np.float32), name), along / D ** 0.5


def compare(M, rng, name, D, lens, n_q, k, v, q, centre=0):
    k, v = ([R.rounded(x.astype(np.float32), name) for x in y] for y in (k, v))
    e = R.expect(name, q, np.concatenate([[0], np.cumsum(n_q)]), lens, k, v, H, D ** -0.5, centre=centre)
    assert np.isfinite(e["out"]).all()
    out, lse = R.run(M, rng, name, q, lens, n_q, k, v, D ** -0.5)
    assert R.wrong(e, out, lse) is None


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("name,loud", [("bf16", 14), ("bf16", 24), ("bf16", 60), ("fp16", 14), ("fp16", 24)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("where", ["early", "everywhere", "last"])
def test_loud_rows_of_no_weight(M, form, name, loud, D, where):
    """Value rows 2^loud times the others, under weights e^-60 of theirs (early, everywhere), or seen by the last query alone."""
    rng = np.random.default_rng(loud + D)
    lens, n_q, k, v, q, along = inputs(rng, name, D, form)
    for b, n in enumerate(lens):
        at = {"early": [64], "everywhere": np.arange(20, n - 20, 50), "last": [n - 1]}[where]
        v[b][at] *= 2.0**loud
        v[b][at] = np.clip(v[b][at], -6e4, 6e4) if name == "fp16" else v[b][at]
        if where != "last":
            k[b][at] = -60 * along + 0.05 * rng.normal(size=(len(at), H, D))
    compare(M, rng, name, D, lens, n_q, k, v, q)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("steps", [-0.002, 0.002, -0.02, 0.02])
def test_values_that_grow_or_shrink(M, form, name, D, steps):
    """Powers of two a token, over at most 2^24, or 2^60 for bfloat16."""
    rng = np.random.default_rng(D)
    lens, n_q, k, v, q, _ = inputs(rng, name, D, form, 1.0)
    for b, n in enumerate(lens):
        power = np.minimum(abs(steps) * np.arange(n), 60 if name == "bf16" else 24)
        power = power if steps > 0 else power[::-1]
        v[b] *= 2.0 ** (power - power.max() / 2)[:, None, None]
    compare(M, rng, name, D, lens, n_q, k, v, q)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("name,nats,size", [("bf16", 8, 1.0), ("bf16", 16, 1.0), ("bf16", 24, 1.0), ("fp16", 8, 1.0), ("fp16", 12, 4096.0)])
@pytest.mark.parametrize("D", [64, 128])
def test_a_silent_row_that_all_look_at(M, form, name, D, nats, size):
    """Values large enough for half outputs to be normal numbers."""
    rng = np.random.default_rng(nats)
    lens, n_q, k, v, q, along = inputs(rng, name, D, form, size)
    for b in range(len(lens)):
        k[b][0] = nats * along
        v[b][0] = 0.0
    compare(M, rng, name, D, lens, n_q, k, v, q)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nats", [10, 12, 13, 14, 15, 16, 18])
def test_a_flat_tail_behind_one_row(M, form, name, D, nats):
    """One key outweighs each of the others by e^nats, and its value is zero but in one channel: the
    others' weights, all alike, are all that the other channels are made of.  (Few queries: as many
    requests as it takes for one warp to have most of a request; for half outputs the row is one whose
    zeros are held as the code in the middle.)"""
    rng = np.random.default_rng(nats)
    lens, n_q = ([300] * 800, [1] * 800) if form == "few" else FORMS[form]
    along = rng.choice([-1.0, 1.0], (H, D))
    k = [np.zeros((n, H, D)) for n in lens]
    v = [1 + 0.25 * rng.normal(size=(n, H, D)) for n in lens]
    q = R.rounded(np.repeat(np.repeat(along, HQ // H, 0)[None], sum(n_q), 0).astype(np.float32), name)
    for b in range(len(lens)):
        k[b][0] = nats * along / D ** 0.5
        v[b][0] = 0.0
        v[b][0, :, 7] = 4.0
        if form == "few" and name == "fp16":
            v[b][0, :, 7], v[b][0, :, 8] = 3.5, -4.0
    compare(M, rng, name, D, lens, n_q, k, v, q, centre=8 if form == "few" and name == "fp16" else 0)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power", [0, 40, 60, 100, 126])
@pytest.mark.parametrize("share", [1.0, 0.2])
def test_rows_of_one_value(M, form, D, power, share):
    """Value rows whose channels are all alike, up to the end of bfloat16's range: their step is zero, and the value comes
    in with the zero point alone.  All rows, or a fifth of them among others of their size."""
    rng = np.random.default_rng(power + D)
    lens, n_q, k, v, q, _ = inputs(rng, "bf16", D, form, 0.25)
    for b, n in enumerate(lens):
        alike = rng.random(n) < share
        v[b][alike] = rng.uniform(-1.9, 1.9, (alike.sum(), H, 1))
        v[b] *= 2.0**power
    compare(M, rng, "bf16", D, lens, n_q, k, v, q)
