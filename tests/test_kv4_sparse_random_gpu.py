"""Random calls of sparse decoding's exact operators: sizes, layouts and lengths over their whole ranges, with the longest
tables among them.  Lists, ranges, turned queries and the cache's bytes are compared bit for bit."""
import math
import random

import numpy as np
import pytest

import test_kv4_sparse_gpu as G
from test_kv4_sparse_gpu import M  # noqa: F401

pytestmark = pytest.mark.gpu


def spread(r, a, b):
    return int(round(math.exp(r.uniform(math.log(a), math.log(b)))))


@pytest.mark.parametrize("seed", range(12))
def test_random_selections(M, seed):  # noqa: F811
    r = random.Random(seed)
    for _ in range(25):
        H, D, S, group = r.choice([1, 1, 2, 3, 4, 8]), r.choice([64, 128, 256]), r.choice([16, 16, 16, 32, 48, 64, 256]), r.choice([1, 2, 3, 4, 5, 7, 8, 16, 20])
        B, most, room = r.choice([1, 1, 2, 3, 7, 30, spread(r, 1, 700)]), spread(r, 1, r.choice([300, 4000, 14000])), 40000
        lens = []
        for _ in range(B):
            nb = r.choice([most, r.randint(0, most), r.randint(0, min(most, 40))])
            if nb > 300:  # a limited number of blocks in all
                nb = min(nb, room)
                room -= nb
            lens.append(max(0, nb * S - r.randint(0, S - 1)))
        n_q = [r.choice([1, 1, 1, 0, r.randint(1, 5)]) for _ in range(B)]
        n_q[0] = max(n_q[0], 1)
        first, last = r.choice([0, 1, 2, r.randint(0, 30)]), r.choice([1, 2, r.randint(1, 30)])
        case = (group * H, H, D, S, r.choice(["bf16", "fp16"]), lens, n_q, first, last, first + last + r.choice([0, 1, 5, spread(r, 1, 3000), spread(r, 1, 100)]))
        data = G.select_data(case, np.random.default_rng(r.randrange(1 << 30)), r.choice([None, None, 1, 2, 3]))
        G.check_select(M, case, *data, lay_q=r.choice([None, "odd", "gaps"]))


@pytest.mark.parametrize("seed", range(6))
def test_random_ranges(M, seed):  # noqa: F811
    r = random.Random(seed)
    for _ in range(12):
        H, D, S, B = r.choice([1, 2, 3, 5, 8, 9, 17]), r.choice([64, 128, 256]), r.choice([16, 16, 32, 48, 64, 512]), r.choice([1, 2, 5, spread(r, 1, 1500)])
        most = max(1, min(spread(r, 1, 6000), 50000 // (B * H)))
        lens = [r.choice([0, 1, r.randint(0, most), most]) for _ in range(B)]
        held = r.choice([None, [max(0, n - r.choice([0, 1, 1, r.randint(0, 40)])) for n in lens], [r.randint(0, 2 * most) for _ in lens]])
        k, v, table, cache = G.filled(M, np.random.default_rng(r.randrange(1 << 30)), lens, H, D, S, scale=r.choice([1.0, 1e-3, 1e4]))
        G.check_ranges(M, k, table, cache, lens, held, H, D, S)


@pytest.mark.parametrize("seed", range(6))
def test_random_turns(M, seed):  # noqa: F811
    r = random.Random(seed)
    for _ in range(25):
        D, H, T, axes = r.choice([64, 128, 256]), r.choice([1, 2, 3, 5, 8]), spread(r, 1, r.choice([90, 90, 9000])), r.choice([1, 1, 2, 3, 4, 8])
        rot = r.choice([0, 16, 32, 48, D // 2, D - 16, D, D])
        G.test_append_rotated(M, (T, r.choice([0, H, 2 * H, 5 * H, 7]), H, D, r.choice([16, 32, 48, 64, 4096]), r.choice(["bf16", "fp16"]), axes if rot else 1, rot,
                                  r.random() < 0.5, r.choice(["plain", "fused", "gaps", "odd"]), r.choice([0, 0.1, 0.5, 1])))
