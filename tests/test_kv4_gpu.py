"""Block tables, the 4-bit KV cache and attention over it on the GPU.

Whole numbers and the cache's bytes equal the oracle's.  Attention is compared
with 64 bits on the values that the cache holds.  Its tolerance is derived: with
u the unit roundoff of the 16-bit type (2^-9 bfloat16, 2^-12 half), the weights,
the values and the output are each rounded at most once to 16 bits, and a value
is its zero plus up to 15 steps, so an output is off by at most about
3u max(|v|, 15 scale); 4u leaves room for the 32-bit sums.  The log-sum of the
weights comes from sums in 32 bits alone, of codes that may carry an offset of
1,024: 2^-21 sm_scale 1,024 max(scale) max(sum |q|) bounds that, besides 1e-5 of its
own size and of 1."""
import numpy as np
import pytest
import torch

import kv4_oracle as K

pytestmark = pytest.mark.gpu

TYPES = {"bf16": (torch.bfloat16, 2.0**-9), "fp16": (torch.float16, 2.0**-12)}


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from paper_2609_15359_gb300 import maps
    return maps


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


# ------------------------------------------------------------------ block tables
def tables_case(rng, R, S, max_blocks, free_share, steps=3000):
    held = rng.integers(0, min(max_blocks * S, steps) + 1, R)
    kind = rng.random(R)
    want = np.where(kind < 0.2, rng.integers(0, held + 1),
                    np.where(kind < 0.6, np.minimum(held + 1, max_blocks * S),
                             np.minimum(held + rng.integers(0, steps, R), max_blocks * S)))
    hb, wb = -(-held // S), -(-want // S)
    need, back = np.maximum(wb - hb, 0).sum(), np.maximum(hb - wb, 0).sum()
    n_free = max(0, int(need * free_share) - int(back))
    pool = int(hb.sum()) + n_free + 1
    perm = rng.permutation(pool)
    table = np.full((R, max_blocks), -7, np.int32)
    at = 0
    for r in range(R):
        table[r, :hb[r]] = perm[at:at + hb[r]]
        at += hb[r]
    free = np.full(pool, -1, np.int32)
    free[:n_free] = perm[at:at + n_free]
    return held.astype(np.int32), want.astype(np.int32), table, free, n_free, rng.permutation(R).astype(np.int32)


def run_tables(M, S, held, want, table, free, n_free, order, cap, ws=None, with_pos=True):
    R = len(held)
    t, f = dev(table), dev(free)
    out = dict(n=torch.full((1,), -9, dtype=torch.int32, device="cuda"),
               got=torch.full((max(R, 1),), -9, dtype=torch.int32, device="cuda")[:R],
               off=torch.full((R + 1,), -9, dtype=torch.int64, device="cuda"),
               slots=torch.full((cap,), -9, dtype=torch.int64, device="cuda"),
               pos=torch.full((cap,), -9, dtype=torch.int32, device="cuda"))
    ws = ws or M.Workspace()
    args = (S, dev(held), dev(want), t, f, dev(np.array([n_free], np.int32)), out["n"], out["got"], out["off"],
            out["slots"], out["pos"] if with_pos else None)
    for _ in range(2):  # a second call on the same lengths and stack gives the same
        assert M.maps_block_tables(*args, order=None if order is None else dev(order), ws=ws) == 0
    st = M.maps_check(ws)
    return st, t.cpu().numpy(), f.cpu().numpy(), {k: v.cpu().numpy() for k, v in out.items()}


@pytest.mark.parametrize("R,S,max_blocks,share,ordered", [
    (1, 16, 4, 2.0, False), (2, 1, 40, 1.0, True), (7, 3, 900, 0.5, True), (31, 16, 300, 1.0, True),
    (33, 16, 300, 0.0, True), (300, 64, 60, 0.7, True), (1024, 16, 200, 1.0, False),
    (1025, 7, 500, 0.3, True), (3001, 16, 190, 0.95, True), (9000, 128, 24, 0.99, True)])
def test_block_tables(M, R, S, max_blocks, share, ordered):
    rng = np.random.default_rng(R * 31 + S)
    held, want, table, free, n_free, order = tables_case(rng, R, S, max_blocks, share)
    order = order if ordered else None
    ref = K.block_tables(S, held, want, table, free, n_free, order)
    cap = len(ref[5])
    st, t, f, o = run_tables(M, S, held, want, table, free, n_free, order, cap)
    assert st == 0
    assert np.array_equal(t, ref[0]) and np.array_equal(f, ref[1]) and o["n"][0] == ref[2]
    assert np.array_equal(o["got"], ref[3]) and np.array_equal(o["off"], ref[4])
    assert np.array_equal(o["slots"], ref[5]) and np.array_equal(o["pos"], ref[6])
    st, t, f, o = run_tables(M, S, held, want, table, free, n_free, order, cap + 300, with_pos=False)
    assert st == 0 and np.array_equal(o["slots"][:cap], ref[5]) and (o["slots"][cap:] == -9).all()
    assert (o["pos"] == -9).all()


def test_block_tables_long_rows(M):
    """One request of a million tokens among idle ones, and its release."""
    S, mb = 16, 70000
    held, want = np.array([0, 5, 0], np.int32), np.array([1 << 20, 5, 0], np.int32)
    table = np.full((3, mb), -1, np.int32)
    table[1, 0] = 9
    free = np.arange(100000, 100000 + 66000, dtype=np.int32)
    ref = K.block_tables(S, held, want, table, free, 66000)
    st, t, f, o = run_tables(M, S, held, want, table, free, 66000, None, 1 << 20)
    assert st == 0 and np.array_equal(t, ref[0]) and np.array_equal(o["slots"], ref[5])
    free2 = f.copy()
    ref2 = K.block_tables(S, want, np.array([0, 5, 0], np.int32), t, free2, ref[2])
    st, t2, f2, o = run_tables(M, S, want, np.array([0, 5, 0], np.int32), t, free2, ref[2], None, 0)
    assert st == 0 and o["n"][0] == 66000 and np.array_equal(f2, ref2[1])


def test_block_tables_no_requests(M):
    st, _, _, o = run_tables(M, 16, np.zeros(0, np.int32), np.zeros(0, np.int32), np.zeros((0, 4), np.int32),
                             np.arange(3, dtype=np.int32), 3, None, 0)
    assert st == 0 and o["n"][0] == 3 and o["off"].tolist() == [0]


@pytest.mark.parametrize("what", ["negative", "long", "order", "cap", "n_free", "pool"])
def test_block_tables_reports_bad_data(M, what):
    S, table, free = 4, np.full((3, 4), 2, np.int32), np.arange(6, dtype=np.int32)
    held, want, order = np.array([3, 4, 0], np.int32), np.array([4, 9, 1], np.int32), np.arange(3, dtype=np.int32)
    n_free, cap = 6, 7
    if what == "negative":
        want[1] = -1
    if what == "long":
        want[1] = 17
    if what == "order":
        order[2] = 3
    if what == "cap":
        cap = 6
    if what == "n_free":
        n_free = 7
    if what == "pool":
        want[0], n_free = 0, 6  # a returned block, and no room for it
    ws = M.Workspace()
    assert run_tables(M, S, held, want, table, free, n_free, order, cap, ws=ws)[0] == M.MAPS_E_RANGE
    good = (np.array([3, 4, 0], np.int32), np.array([4, 9, 1], np.int32))
    ref = K.block_tables(S, *good, table, free, 5)
    st, t, _, o = run_tables(M, S, *good, table, free, 5, None, 7, ws=ws)
    assert st == 0 and np.array_equal(t, ref[0]) and np.array_equal(o["slots"], ref[5])


# ------------------------------------------------------------------ the cache
def laid_out(x, how):
    """x [T, H, D] in one of the layouts that programs have it in."""
    T, H, D = x.shape
    if how == "dense":
        return x.contiguous()
    if how == "fused":  # beside other heads
        big = torch.empty(T, 3 * H + 1, D, dtype=x.dtype, device=x.device)
        return big[:, H:2 * H].copy_(x)
    if how == "heads first":
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    big = torch.empty(T * (H * D + 3) + 1, dtype=x.dtype, device=x.device)  # odd base and row stride
    return big[1:].as_strided((T, H, D), (H * D + 3, D, 1)).copy_(x)


LAYOUTS = ["dense", "fused", "heads first", "odd"]


def rounded(x, name):
    """x as the 16-bit type, as float32."""
    if name == "bf16":
        return K.bf16(x)
    return x.astype(np.float16).astype(np.float32)


@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("T,H,D,S", [(1, 1, 64, 16), (5, 3, 128, 16), (33, 2, 256, 48), (50, 1, 128, 64)])
def test_append_and_read(M, name, how, T, H, D, S):
    rng = np.random.default_rng(T + D)
    dt = TYPES[name][0]
    n = -(-T // S) + 2
    k, v = (rounded(rng.normal(size=(T, H, D)).astype(np.float32) * 10.0 ** rng.integers(-3, 3, (T, H, 1)), name)
            for _ in range(2))
    if T > 4:
        k[1], v[2] = 0.75, 0.0  # constant rows
        k[3, 0, 5], v[4, 0, D - 1], v[4, 0, 0] = np.nan, np.inf, -np.inf
    slots = rng.permutation(n * S)[:T].astype(np.int64)
    if T > 8:
        slots[[0, 7]] = -1
    ref = np.full((n, H, K.record_bytes(S, D)), 0xA5, np.uint8)
    cache = dev(ref)
    for i in range(T):
        for h in range(H):
            if slots[i] >= 0:
                K.put(ref, S, D, int(slots[i]), h, k[i, h], v[i, h])
    ws = M.Workspace()
    assert M.maps_kv4_append(laid_out(dev(k, dt), how), laid_out(dev(v, dt), how), dev(slots), cache, S, ws=ws) == 0
    assert M.maps_check(ws) == 0
    got = cache.cpu().numpy()
    par = lambda c: c.reshape(n, H, S // 16, -1)[..., 16 * D:].copy().view("<u2")  # noqa: E731
    nan_got, nan_ref = (par(got) & 0x7fff) > 0x7f80, (par(ref) & 0x7fff) > 0x7f80
    assert np.array_equal(nan_got, nan_ref)  # any NaN will do
    assert np.array_equal(np.where(nan_got, 0, par(got)), np.where(nan_ref, 0, par(ref)))
    codes = lambda c: c.reshape(n, H, S // 16, -1)[..., :16 * D]  # noqa: E731
    assert np.array_equal(codes(got), codes(ref))
    ko, vo = (laid_out(torch.full((T, H, D), 9.0, dtype=dt, device="cuda"), how) for _ in range(2))
    assert M.maps_kv4_read(dev(slots), cache, S, ko, vo, ws=ws) == 0
    assert M.maps_check(ws) == 0
    for y, x in ((ko, k), (vo, v)):
        want = np.where((slots >= 0)[:, None, None], rounded(K.held_as(x), name), 0)
        assert np.array_equal(y.float().cpu().numpy(), want, equal_nan=True)


def test_append_consecutive_tokens(M):
    """Prompts as they come: runs of consecutive slots over blocks, from any place in one."""
    rng = np.random.default_rng(5)
    for T, H, D, S, start in ((200, 3, 128, 16, 0), (333, 2, 64, 32, 7), (100, 5, 256, 16, 15)):
        n = T // S + 3
        blocks = rng.permutation(n)
        p = np.arange(start, start + T)
        slots = (blocks[p // S] * S + p % S).astype(np.int64)
        k, v = (rounded(rng.normal(size=(T, H, D)).astype(np.float32), "bf16") for _ in range(2))
        cache = torch.zeros(M.kv4_cache_shape(n, H, S, D), dtype=torch.uint8, device="cuda")
        ws = M.Workspace()
        assert M.maps_kv4_append(dev(k, torch.bfloat16), dev(v, torch.bfloat16), dev(slots), cache, S, ws=ws) == 0
        assert M.maps_check(ws) == 0
        ref = np.zeros(tuple(cache.shape), np.uint8)
        for i in range(0, T, 7):
            K.put(ref, S, D, int(slots[i]), H - 1, k[i, H - 1], v[i, H - 1])
        ko, vo = (torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        assert M.maps_kv4_read(dev(slots), cache, S, ko, vo, ws=ws) == 0
        assert np.array_equal(ko.float().cpu().numpy(), K.bf16(K.held_as(k)))
        assert np.array_equal(vo.float().cpu().numpy(), K.bf16(K.held_as(v)))
        one = torch.zeros_like(cache)  # the same rows, one token a call
        for i in range(0, T, 7):
            assert M.maps_kv4_append(dev(k[i:i + 1], torch.bfloat16), dev(v[i:i + 1], torch.bfloat16),
                                     dev(slots[i:i + 1]), one, S, ws=ws) == 0
        assert np.array_equal(one.cpu().numpy()[:, H - 1], ref[:, H - 1])


@pytest.mark.parametrize("how", ["dense", "fused", "odd"])
@pytest.mark.parametrize("T,H,D,S,name", [(20000, 2, 128, 16, "bf16"), (9001, 5, 64, 48, "fp16"), (5003, 8, 256, 32, "bf16"),
                                          (40001, 1, 128, 64, "fp16")])
def test_many_rows_equal_few(M, T, H, D, S, name, how):
    """One call of many tokens writes and reads what calls of a few do: runs of every length and phase,
    slots out of order, skipped and non-finite tokens."""
    rng = np.random.default_rng(T)
    dt = TYPES[name][0]
    n = T // S + 40
    slots = np.full(T, -1, np.int64)
    free = rng.permutation(n)
    i = used = 0
    while i < T and used + 9 < n:  # a run over whole blocks, from any place in the first, then a gap
        run = int(min(T - i, rng.choice([1, 3, 15, 16, 17, 33, 200, 1000])))
        start = int(rng.integers(0, S)) if rng.random() < 0.5 else 0
        need = -(-(start + run) // S)
        if used + need > n:
            break
        p = np.arange(start, start + run)
        slots[i:i + run] = free[used:used + need][p // S] * S + p % S
        used += need
        i += run + int(rng.integers(0, 3))
    k, v = (torch.randn(T, H, D, device="cuda").to(dt) for _ in range(2))
    k[rng.integers(0, T, 9)] = 0.5
    v[rng.integers(0, T, 9), 0, 3] = float("nan")
    k[rng.integers(0, T, 9), H - 1, D - 1] = float("inf")
    k, v, at = laid_out(k, how), laid_out(v, how), dev(slots)
    ws = M.Workspace()
    shape = M.kv4_cache_shape(n, H, S, D)
    one, parts = (torch.full(shape, 0xA5, dtype=torch.uint8, device="cuda") for _ in range(2))
    assert M.maps_kv4_append(k, v, at, one, S, ws=ws) == 0
    for a in range(0, T, 997):
        assert M.maps_kv4_append(k[a:a + 997], v[a:a + 997], at[a:a + 997], parts, S, ws=ws) == 0
    assert torch.equal(one, parts)
    outs = [[laid_out(torch.full((T, H, D), 9.0, dtype=dt, device="cuda"), how) for _ in range(2)] for _ in range(2)]
    assert M.maps_kv4_read(at, one, S, *outs[0], ws=ws) == 0
    for a in range(0, T, 997):
        assert M.maps_kv4_read(at[a:a + 997], one, S, outs[1][0][a:a + 997], outs[1][1][a:a + 997], ws=ws) == 0
    assert M.maps_check(ws) == 0
    for x, y in zip(*outs):
        assert torch.equal(torch.nan_to_num(x, nan=123.0), torch.nan_to_num(y, nan=123.0))


def test_append_reports_slots_past_the_cache(M):
    k = torch.randn(3, 1, 64, device="cuda").half()
    cache = torch.zeros(M.kv4_cache_shape(2, 1, 16, 64), dtype=torch.uint8, device="cuda")
    ws = M.Workspace()
    slots = torch.tensor([0, 32, 1 << 50], device="cuda")
    assert M.maps_kv4_append(k, k, slots, cache, 16, ws=ws) == 0
    assert M.maps_check(ws) == M.MAPS_E_RANGE
    out = torch.full_like(k, 7), torch.full_like(k, 7)
    assert M.maps_kv4_read(slots, cache, 16, *out, ws=ws) == 0
    assert M.maps_check(ws) == M.MAPS_E_RANGE
    assert (out[0][1:] == 0).all() and (out[0][0] != 0).any()


# ------------------------------------------------------------------ attention
def fill(M, rng, lens, H, D, S, name, ws, spare=3, at_end=False, n_blocks=None, spread=1.0):
    """A cache of random keys and values behind block tables; every place that holds no token is NaN."""
    dt = TYPES[name][0]
    nb = [-(-int(n) // S) for n in lens]
    used = sum(nb)
    P = n_blocks or used + spare
    perm = rng.permutation(used) + (P - used if at_end else 0) if n_blocks else rng.permutation(P)[:used]
    table = np.full((len(lens), max(max(nb, default=0), 1) + 1), -1, np.int32)
    slots, at = [], 0
    for b, n in enumerate(lens):
        table[b, :nb[b]] = perm[at:at + nb[b]]
        at += nb[b]
        j = np.arange(n)
        slots.append(table[b, j // S].astype(np.int64) * S + j % S)
    slots = np.concatenate(slots).astype(np.int64) if lens else np.zeros(0, np.int64)
    T = len(slots)
    k = rounded((rng.normal(size=(T, H, D)) * (0.3 + rng.random((H, D))) + rng.normal(size=(H, D)) * spread).astype(np.float32), name)
    v = rounded((rng.normal(size=(T, H, D)) * 10.0 ** rng.uniform(-1, 1, (T, H, 1))).astype(np.float32), name)
    if n_blocks:
        cache = torch.empty(M.kv4_cache_shape(P, H, S, D), dtype=torch.uint8, device="cuda")
        cache[torch.from_numpy(perm).cuda().long()] = 0xff
    else:
        cache = torch.full(M.kv4_cache_shape(P, H, S, D), 0xff, dtype=torch.uint8, device="cuda")
    if T:
        assert M.maps_kv4_append(dev(k, dt), dev(v, dt), dev(slots), cache, S, ws=ws) == 0
    cut = np.cumsum([0] + [int(n) for n in lens])
    hk, hv = K.held_as(k), K.held_as(v)
    top = max(float(K.quantise(x)[1].max()) if T else 0.0 for x in (k, v))
    return cache, table, [hk[a:b] for a, b in zip(cut, cut[1:])], [hv[a:b] for a, b in zip(cut, cut[1:])], top


def check(M, rng, lens, n_q, Hq, H, D, S, name, causal=True, window=0, how="dense", stream=None, scale=None, gain=1.0, **kw):
    ws = M.Workspace()
    dt, u = TYPES[name]
    cache, table, k, v, top = fill(M, rng, lens, H, D, S, name, ws, **kw)
    off = np.concatenate([[0], np.cumsum(n_q)]).astype(np.int64)
    T = int(off[-1]) + 2  # two rows that no request has
    q = rounded((rng.normal(size=(T, Hq, D)) * gain).astype(np.float32), name)
    q_dev = laid_out(dev(q, dt), how)
    out = laid_out(torch.full((T, Hq, D), 77.0, dtype=dt, device="cuda"), how)
    lse = torch.full((T, Hq), 77.0, dtype=torch.float32, device="cuda")
    scale = D ** -0.5 if scale is None else scale
    args = (q_dev, dev(off), dev(np.asarray(lens, np.int32)), dev(table), cache, S, scale)
    torch.cuda.synchronize()
    st = M.maps_kv4_attention(*args, out, lse_out=lse, causal=causal, window=window, ws=ws, stream=stream)
    assert st == 0
    assert M.maps_check(ws, stream) == 0
    ref, ref_lse = K.attention(q, off, lens, k, v, H, scale, causal, window)
    o, l = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    assert (o[-2:] == 77).all() and (l[-2:] == 77).all()
    o, l, ref, ref_lse = o[:-2], l[:-2], ref[:-2], ref_lse[:-2]
    empty = np.isneginf(ref_lse)
    assert np.array_equal(empty, np.isneginf(l)) and (o[empty] == 0).all()
    big = max([15 * top] + [float(np.abs(x).max()) for x in v if x.size])
    err = np.abs(o - ref).max(initial=0)
    assert err <= 4 * u * big, (err, 4 * u * big)
    lim = 2.0**-21 * abs(scale) * 1024 * top * np.abs(q).sum(-1).max(initial=0) + 1e-5 * (1 + np.abs(ref_lse[~empty]))
    off_by = np.abs(l[~empty] - ref_lse[~empty])
    assert (off_by <= lim).all(), off_by.max()
    again = torch.full_like(out, 5.0)
    assert M.maps_kv4_attention(*args, again, causal=causal, window=window, ws=ws, stream=stream) == 0
    assert M.maps_check(ws, stream) == 0
    assert np.array_equal(again[:-2].float().cpu().numpy().astype(np.float64), o)  # the same bits, with and without lse


LENS = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 1000, 0, 31]


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("Hq,H,D,S", [(4, 4, 64, 16), (8, 2, 128, 16), (8, 1, 128, 32), (10, 2, 128, 48),
                                      (7, 1, 64, 64), (16, 1, 256, 16), (6, 2, 256, 32), (24, 1, 128, 16),
                                      (3, 3, 128, 128)])
def test_decode(M, name, Hq, H, D, S):
    check(M, np.random.default_rng(Hq * D + S), LENS, [1] * len(LENS), Hq, H, D, S, name)


@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("name", ["bf16", "fp16"])
def test_decode_layouts(M, name, how):
    check(M, np.random.default_rng(1), [5, 40, 200], [1, 1, 1], 8, 2, 128, 16, name, how=how)
    check(M, np.random.default_rng(1), [50, 400], [3, 40], 4, 2, 64, 16, name, how=how)


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("window", [0, 1, 16, 100])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("Hq,H,D", [(4, 1, 128), (6, 2, 64), (2, 2, 256)])
def test_several_queries(M, name, causal, window, Hq, H, D):
    """Drafted tokens and chunks, more queries than tokens, requests without a query."""
    lens = [0, 1, 2, 5, 20, 64, 90, 257, 700, 33, 400]
    n_q = [3, 1, 5, 5, 2, 8, 0, 5, 9, 33, 130]
    check(M, np.random.default_rng(Hq + window), lens, n_q, Hq, H, D, 16, name, causal=causal, window=window)


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("Hq,H,D,S,causal,window", [
    (8, 2, 128, 16, True, 0), (4, 4, 128, 32, True, 0), (8, 1, 64, 16, True, 0), (3, 1, 128, 48, False, 0),
    (4, 2, 64, 64, True, 200), (2, 1, 256, 16, True, 0), (8, 1, 128, 16, True, 77), (5, 1, 64, 16, False, 300)])
def test_chunks(M, name, Hq, H, D, S, causal, window):
    lens = [513, 700, 128, 1100, 65, 0, 300]
    n_q = [513, 200, 128, 257, 65, 40, 1]
    check(M, np.random.default_rng(Hq * 7 + D), lens, n_q, Hq, H, D, S, name, causal=causal, window=window)


@pytest.mark.parametrize("Hq,H,D,name", [(8, 1, 128, "bf16"), (2, 2, 64, "fp16"), (16, 2, 256, "bf16")])
def test_one_long_request(M, Hq, H, D, name):
    check(M, np.random.default_rng(2), [20011], [1], Hq, H, D, 16, name)
    check(M, np.random.default_rng(3), [20011, 3], [4, 2], Hq, H, D, 64, name, window=15000)


@pytest.mark.parametrize("Hq,D,n,name", [(8, 128, 100003, "bf16"), (16, 128, 120001, "fp16"), (16, 256, 60001, "bf16"), (4, 64, 180007, "fp16")])
def test_one_head_over_the_whole_device(M, Hq, D, n, name):
    """One KV head's keys lie with every multiprocessor: more parts to join than shared memory takes at once."""
    check(M, np.random.default_rng(11), [n], [1], Hq, 1, D, 64, name)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,H", [(1, 1), (4, 2)])
def test_rows_about_where_forms_and_tiles_end(M, Hq, H, D):
    n_q = [96, 97, 127, 128, 129, 255, 256, 257, 385, 48, 49, 64, 65, 1, 0]
    lens = [90, 97, 140, 128, 700, 100, 256, 300, 385, 48, 500, 64, 66, 1, 20]
    check(M, np.random.default_rng(12), lens, n_q, Hq, H, D, 32, "bf16")
    check(M, np.random.default_rng(13), lens, n_q, Hq, H, D, 16, "fp16", window=33)


def test_many_short_requests(M):
    rng = np.random.default_rng(4)
    lens = rng.integers(0, 50, 2500).tolist()
    check(M, rng, lens, [1] * len(lens), 4, 1, 64, 16, "bf16")
    lens = rng.integers(0, 20, 6000).tolist()
    check(M, rng, lens, rng.integers(0, 3, 6000), 2, 1, 64, 16, "fp16")


@pytest.mark.parametrize("gain,scale", [(30.0, None), (1.0, 0.0), (1.0, -0.1), (1e-4, 1.0), (200.0, 1.0)])
def test_peaked_and_flat_weights(M, gain, scale):
    """Weights that sit on one key, all equal, negative scale, scores of several hundred."""
    for name in ("bf16", "fp16"):
        check(M, np.random.default_rng(6), [300, 1, 77], [1, 1, 1], 8, 2, 128, 16, name, gain=gain, scale=scale)
        check(M, np.random.default_rng(6), [300, 260], [200, 256], 4, 2, 64, 16, name, gain=gain, scale=scale)


def test_nan_rows_reach_only_who_sees_them(M):
    """A key held as NaN: queries ahead of it are untouched, those behind it are NaN."""
    rng = np.random.default_rng(8)
    for n_q in (3, 200):
        T = 300
        k = torch.randn(T, 1, 128, device="cuda").bfloat16()
        v = torch.randn(T, 1, 128, device="cuda").bfloat16()
        k[T - 2] = float("nan")
        cache = torch.zeros(M.kv4_cache_shape(20, 1, 16, 128), dtype=torch.uint8, device="cuda")
        table = dev(rng.permutation(20)[None].astype(np.int32))
        p = torch.arange(T, device="cuda")
        slots = table[0, p // 16].long() * 16 + p % 16
        ws = M.Workspace()
        assert M.maps_kv4_append(k, v, slots, cache, 16, ws=ws) == 0
        q = torch.randn(n_q, 4, 128, device="cuda").bfloat16()
        out = torch.zeros_like(q)
        assert M.maps_kv4_attention(q, dev(np.array([0, n_q])), dev(np.array([T], np.int32)), table, cache, 16, 0.09,
                                    out, ws=ws) == 0
        assert M.maps_check(ws) == 0
        assert torch.isfinite(out[:-2]).all() and torch.isnan(out[-2:]).all()


def test_offsets_past_32_bits(M):
    """Blocks at the end of a cache of more than 4 GiB."""
    rng = np.random.default_rng(9)
    for lens, n_q in (([300, 40], [1, 2]), ([300], [200])):
        check(M, rng, lens, n_q, 4, 2, 128, 16, "bf16", n_blocks=1_200_000, at_end=True)


def test_another_stream(M):
    s = torch.cuda.Stream()
    for n_q in ([1, 1], [2, 150]):
        check(M, np.random.default_rng(10), [900, 155], n_q, 8, 2, 128, 16, "bf16", stream=s)


@pytest.mark.parametrize("n_q", [1, 100])
def test_bad_tables_and_lengths_are_reported(M, n_q):
    rng = np.random.default_rng(11)
    ws = M.Workspace()
    cache, table, _, _, _ = fill(M, rng, [100, 100], 1, 128, 16, "bf16", ws)
    q = torch.randn(2 * n_q, 4, 128, device="cuda").bfloat16()
    out = torch.zeros_like(q)
    off = dev(np.array([0, n_q, 2 * n_q]))

    def status(table, lens):
        assert M.maps_kv4_attention(q, off, dev(np.array(lens, np.int32)), dev(table), cache, 16, 0.1, out, ws=ws) == 0
        return M.maps_check(ws)

    assert status(table, [100, 100]) == 0
    for wrong in (-1, cache.shape[0], 2**31 - 1, -2**31):
        t = table.copy()
        t[1, 3] = wrong
        assert status(t, [100, 100]) == M.MAPS_E_RANGE
        assert status(t, [100, 48]) == 0  # the entry is not used
    assert status(table, [100, -1]) == M.MAPS_E_RANGE
    assert status(table, [table.shape[1] * 16 + 1, 100]) == M.MAPS_E_RANGE
    assert status(table, [100, 100]) == 0


def heavy(Hq):
    """A request's tokens and queries that take a call past the work up to which one form serves all its requests."""
    return 6100, 2800 // Hq + 1


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("Hq,H,D,S,causal,window", [
    (8, 2, 128, 16, True, 0), (4, 4, 128, 32, True, 0), (8, 1, 64, 16, True, 0), (3, 1, 128, 48, False, 0),
    (4, 2, 64, 64, True, 200), (8, 1, 128, 16, True, 77), (5, 1, 64, 16, False, 300), (6, 3, 64, 16, True, 1)])
def test_chunks_of_much_work(M, name, Hq, H, D, S, causal, window):
    n, m = heavy(Hq)
    lens = [513, 700, 128, n, 1100, 65, 0, 300, 0, 1, 2, 20, 64, 90, 257]
    n_q = [513, 200, 128, m, 257, 65, 40, 1, 130, 99, 100, 97, 200, 0, 33]
    check(M, np.random.default_rng(Hq * 11 + D), lens, n_q, Hq, H, D, S, name, causal=causal, window=window)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,H", [(1, 1), (4, 2)])
def test_rows_about_where_forms_end_in_much_work(M, Hq, H, D):
    n, m = heavy(Hq)
    n_q = [96, 97, 127, 128, 129, m, 255, 256, 257, 385, 48, 49, 64, 65, 1, 0]
    lens = [90, 97, 140, 128, 700, n, 100, 256, 300, 385, 48, 500, 64, 66, 1, 20]
    check(M, np.random.default_rng(14), lens, n_q, Hq, H, D, 32, "bf16", how="odd")
    check(M, np.random.default_rng(15), lens, n_q, Hq, H, D, 16, "fp16", window=33)


@pytest.mark.parametrize("gain,scale", [(30.0, None), (1.0, 0.0), (1.0, -0.1), (1e-4, 1.0), (200.0, 1.0)])
def test_peaked_and_flat_weights_of_much_work(M, gain, scale):
    n, m = heavy(4)
    for name in ("bf16", "fp16"):
        check(M, np.random.default_rng(16), [300, n, 260], [200, m, 256], 4, 2, 64, 16, name, gain=gain, scale=scale)


def test_many_short_requests_beside_much_work(M):
    rng = np.random.default_rng(17)
    n, m = heavy(2)
    lens = rng.integers(0, 40, 2300).tolist() + [n]
    check(M, rng, lens, np.append(rng.integers(0, 3, 2300), m), 2, 1, 64, 16, "fp16")


def test_nan_keys_in_much_work(M):
    rng = np.random.default_rng(18)
    T, n_q = 21500, 200
    k = torch.randn(T, 1, 128, device="cuda").bfloat16()
    v = torch.randn(T, 1, 128, device="cuda").bfloat16()
    k[T - 2] = float("nan")
    blocks = T // 16 + 1
    cache = torch.zeros(M.kv4_cache_shape(blocks, 1, 16, 128), dtype=torch.uint8, device="cuda")
    table = dev(rng.permutation(blocks)[None].astype(np.int32))
    p = torch.arange(T, device="cuda")
    ws = M.Workspace()
    assert M.maps_kv4_append(k, v, table[0, p // 16].long() * 16 + p % 16, cache, 16, ws=ws) == 0
    q = torch.randn(n_q, 4, 128, device="cuda").bfloat16()
    out = torch.zeros_like(q)
    args = (q, dev(np.array([0, n_q])), dev(np.array([T], np.int32)))
    assert M.maps_kv4_attention(*args, table, cache, 16, 0.09, out, ws=ws) == 0
    assert M.maps_check(ws) == 0
    assert torch.isfinite(out[:-2]).all() and torch.isnan(out[-2:]).all()
    for wrong in (-1, blocks, 2**31 - 1, -2**31):
        t = table.clone()
        t[0, 900] = wrong
        assert M.maps_kv4_attention(*args, t, cache, 16, 0.09, out, ws=ws) == 0
        assert M.maps_check(ws) == M.MAPS_E_RANGE


def test_sweep(M):
    """Random shapes, types, lengths, windows and layouts."""
    rng = np.random.default_rng(12)
    for _ in range(60):
        H, group = int(rng.integers(1, 4)), int(rng.choice([1, 2, 3, 4, 7, 8, 12]))
        B = int(rng.integers(1, 9))
        most = int(rng.choice([20, 200, 1500]))
        lens = rng.integers(0, most, B)
        n_q = np.ones(B, int) if rng.random() < 0.4 else rng.integers(0, int(rng.choice([4, 12, 90, 300])), B)
        check(M, rng, lens.tolist(), n_q.tolist(), group * H, H, int(rng.choice([64, 128, 256])),
              int(rng.choice([16, 32, 48, 64])), str(rng.choice(["bf16", "fp16"])), causal=bool(rng.random() < 0.8),
              window=int(rng.choice([0, 0, 1, 40, 500])), how=str(rng.choice(LAYOUTS)))
