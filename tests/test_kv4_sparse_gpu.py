"""Sparse decoding on the 4-bit cache on the GPU: keys and queries turned on the way, ranges of
blocks, selected blocks and attention over them.

Turned queries, the cache's bytes, ranges and lists are compared bit for bit: the definitions leave
no choice.  Attention over lists is held to the row-wise bounds of kv4_rows.py, each row and KV
head being a request of its own there."""
import numpy as np
import pytest
import torch

import kv4_oracle as K
import kv4_rows as R
import kv4_sparse_oracle as O

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from paper_2609_15359_gb300 import maps
    return maps


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def i32(x):
    return dev(np.asarray(x, np.int32))


# ------------------------------------------------------------------ rotary positions on the way into the cache
ROTATE = [  # T, Hq, H, D, S, type, axes, rot, interleaved, layout, share of tokens without a slot
    (1, 1, 1, 64, 16, "bf16", 1, 64, False, "plain", 0), (1, 32, 8, 128, 16, "bf16", 1, 128, False, "fused", 0),
    (3, 5, 5, 128, 32, "fp16", 1, 128, True, "plain", 0.3), (17, 6, 2, 64, 48, "fp16", 3, 32, True, "fused", 0.2),
    (33, 0, 3, 256, 16, "bf16", 2, 256, False, "plain", 0), (40, 16, 1, 256, 64, "fp16", 4, 240, False, "odd", 0.1),
    (19, 3, 3, 64, 16, "bf16", 3, 48, False, "odd", 0.1), (21, 4, 2, 128, 16, "bf16", 8, 112, True, "odd", 0),
    (50, 7, 1, 128, 4096, "bf16", 3, 96, False, "gaps", 0), (64, 2, 2, 64, 16, "fp16", 1, 0, False, "plain", 0.1),
    (700, 8, 4, 128, 16, "bf16", 3, 128, False, "fused", 0.02), (3001, 10, 5, 64, 32, "fp16", 3, 64, True, "plain", 0.1),
    (5003, 4, 4, 128, 16, "bf16", 1, 128, False, "odd", 0), (6000, 3, 3, 256, 16, "bf16", 2, 16, True, "fused", 0),
    (9000, 6, 6, 64, 64, "bf16", 1, 32, False, "plain", 0), (7001, 3, 3, 256, 16, "bf16", 4, 256, False, "fused", 0.01),
    (6600, 6, 3, 256, 32, "fp16", 2, 240, True, "odd", 0.1)]


def lay(x, layout, dtype):
    """x on the device in a layout: its own, among others' rows, or off 16-byte boundaries."""
    T, h, D = x.shape
    if layout == "gaps":
        whole = torch.zeros(T, h + 2, D + 8, dtype=dtype, device="cuda")
        view = whole[:, 1:h + 1, 8:]
    elif layout == "odd":
        whole = torch.zeros(T, h, D + 5, dtype=dtype, device="cuda")
        view = whole[..., 3:3 + D]
    else:
        return dev(x, dtype)
    return view.copy_(dev(x, dtype))


def rotate_case(T, Hq, H, D, S, kind, axes, rot, inter, layout, skip, seed=0):
    rng = np.random.default_rng(T * 7 + D + rot + seed)
    x = [R.rounded((rng.normal(size=(T, h, D)) * 2.0 ** rng.integers(-3, 4, (T, h, 1))).astype(np.float32), kind) for h in (Hq, H, H)]
    n_pos = int(rng.integers(1, 500))
    angle = rng.uniform(0, 1e4, (n_pos, rot // 2))
    cos_sin = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
    pos = rng.integers(0, n_pos, (axes, T)).astype(np.int32)
    axis = None if axes == 1 else rng.integers(0, axes, rot // 2) if inter else np.arange(rot // 2) * axes // max(rot // 2, 1)
    n = -(-T // S) + 3
    at = rng.permutation(n * S)[:T] if T < 1000 else (rng.permutation(n)[:, None] * S + np.arange(S)).reshape(-1)[S // 2:][:T]
    slots = np.where(rng.random(T) < skip, -1, at).astype(np.int64)
    return x, cos_sin, pos, axis, slots, n


@pytest.mark.parametrize("case", ROTATE, ids=lambda c: "-".join(map(str, c)))
def test_append_rotated(M, case):
    T, Hq, H, D, S, kind, axes, rot, inter, layout, skip = case
    (q, k, v), cos_sin, pos, axis, slots, n = rotate_case(*case)
    dt = TYPES[kind]
    if layout == "fused":
        qkv = dev(np.concatenate([q, k, v], 1), dt)
        dq, dk, dv = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    else:
        dq, dk, dv = (lay(x, layout, dt) for x in (q, k, v))
    cache = torch.full(M.kv4_cache_shape(n, H, S, D), 0xab, dtype=torch.uint8, device="cuda")
    ref = cache.cpu().numpy()
    turned = O.rotate(k, pos, axis, rot, inter, cos_sin)
    for i in range(T if T <= 100 else 0):
        for h in range(H):
            if slots[i] >= 0:
                K.put(ref, S, D, int(slots[i]), h, turned[i, h], v[i, h])
    out = torch.full((T, Hq, D), 7.0, dtype=dt, device="cuda") if Hq else None
    args = (dk, dv, dev(pos), dev(cos_sin), dev(slots), cache, S)
    kw = dict(axis=None if axis is None else i32(axis), interleaved=inter, ws=M.Workspace())
    assert M.maps_kv4_append_rotated(dq if Hq else None, *args, out, **kw) == 0
    assert M.maps_check(kw["ws"]) == 0
    expect = O.rotate(q, pos, axis, rot, inter, cos_sin)
    if Hq:
        assert torch.equal(out.cpu(), torch.from_numpy(expect).to(dt))
    if T <= 100:
        assert np.array_equal(cache.cpu().numpy(), ref)
    else:
        # the same keys, values of the one and turned keys as 32 bits of the other, through what a slot reads back as
        rows = [torch.empty(T, H, D, dtype=dt, device="cuda") for _ in range(2)]
        assert M.maps_kv4_read(dev(slots), cache, S, *rows) == 0
        for y, x in zip(rows, (turned, v)):
            want = torch.from_numpy(np.where((slots >= 0)[:, None, None], K.held_as(x), 0)).to(dt)
            assert torch.equal(y.cpu(), want)
        left = np.ones(n * S, bool)
        left[slots[slots >= 0]] = False
        old = torch.empty(int(left.sum()), H, D, dtype=dt, device="cuda")
        new = torch.empty_like(old)
        fresh = torch.full_like(cache, 0xab)
        at = dev(np.flatnonzero(left).astype(np.int64))
        assert M.maps_kv4_read(at, cache, S, new, torch.empty_like(new)) == 0 and M.maps_kv4_read(at, fresh, S, old, torch.empty_like(old)) == 0
        assert torch.equal(old.view(torch.int16), new.view(torch.int16))
    if Hq:  # in place, over again with the same result in the cache
        before = cache.clone()
        assert M.maps_kv4_append_rotated(dq, *args, dq, **kw) == 0 and M.maps_check(kw["ws"]) == 0
        assert torch.equal(dq.cpu(), torch.from_numpy(expect).to(dt)) and torch.equal(before, cache)


def test_append_rotated_of_no_channels_is_append(M):
    rng = np.random.default_rng(5)
    T, H, D, S = 300, 2, 128, 16
    k, v = (dev(rng.normal(size=(T, H, D)).astype(np.float32), torch.bfloat16) for _ in range(2))
    k[5, 1, 3], v[7, 0, 0] = float("inf"), float("nan")
    slots = dev(rng.permutation(400 * S)[:T].astype(np.int64))
    a, b = (torch.zeros(M.kv4_cache_shape(400, H, S, D), dtype=torch.uint8, device="cuda") for _ in range(2))
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert M.maps_kv4_append(k, v, slots, a, S) == 0
    assert M.maps_kv4_append_rotated(None, k, v, torch.zeros(1, T, dtype=torch.int32, device="cuda"), torch.zeros(9, 0, device="cuda"),
                                     slots, b, S, None, axis=none) == 0
    assert torch.equal(a, b)


@pytest.mark.parametrize("T", [20, 5000])
@pytest.mark.parametrize("inter", [False, True])
def test_append_rotated_of_values_that_are_no_numbers(M, T, inter):
    """A turned row with an infinity or NaN is held as NaN; what its queries become follows the arithmetic."""
    rng = np.random.default_rng(T)
    H, D, S, rot = 2, 64, 16, 32
    x = [R.rounded(rng.normal(size=(T, H, D)).astype(np.float32), "bf16") for _ in range(3)]
    for i, bad in enumerate((np.inf, -np.inf, np.nan, 3e38)):
        for y in x:
            y[i + 1, 1, 5 + 9 * i] = bad
            y[i + 7, 0, 40] = bad
    cos_sin = np.concatenate([np.cos(np.arange(90.0).reshape(-1, 1) + np.zeros(16)), np.sin(np.arange(90.0).reshape(-1, 1) + np.zeros(16))], 1).astype(np.float32)
    pos = rng.integers(0, 90, (1, T)).astype(np.int32)
    n = T // S + 1
    cache = torch.zeros(M.kv4_cache_shape(n, H, S, D), dtype=torch.uint8, device="cuda")
    slots = np.arange(T, dtype=np.int64)
    q, k, v = (dev(y, torch.bfloat16) for y in x)
    out = torch.empty_like(q)
    assert M.maps_kv4_append_rotated(q, k, v, dev(pos), dev(cos_sin), dev(slots), cache, S, out, interleaved=inter) == 0
    turned = O.rotate(x[1], pos, None, rot, inter, cos_sin)
    want = O.rotate(x[0], pos, None, rot, inter, cos_sin)
    got = out.float().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    assert np.array_equal(got[ok], torch.from_numpy(want).bfloat16().float().numpy()[ok])
    ref = np.zeros(cache.shape, np.uint8)
    for i in range(20):
        for h in range(H):
            K.put(ref, S, D, i, h, turned[i, h], x[2][i, h])
    rows = [torch.empty(20, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    assert M.maps_kv4_read(dev(slots[:20]), cache, S, *rows[:2]) == 0 and M.maps_kv4_read(dev(slots[:20]), dev(ref), S, *rows[2:]) == 0
    for a, b in ((0, 2), (1, 3)):
        a, b = rows[a].float().cpu().numpy(), rows[b].float().cpu().numpy()
        assert np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(a[~np.isnan(a)], b[~np.isnan(b)])


@pytest.mark.parametrize("what", ["pos", "negative", "axis", "slot"])
@pytest.mark.parametrize("T", [9, 5000])
def test_append_rotated_reports_bad_data(M, what, T):
    H, D, S = 1, 64, 16
    k = torch.ones(T, H, D, dtype=torch.bfloat16, device="cuda")
    pos, axis = torch.zeros(2, T, dtype=torch.int32, device="cuda"), torch.zeros(32, dtype=torch.int32, device="cuda")
    slots = torch.arange(T, device="cuda")
    if what == "pos":
        pos[1, 3], axis[31] = 10, 1
    if what == "negative":
        pos[0, T - 1] = -1
    if what == "axis":
        axis[7] = 2
    if what == "slot":
        slots[2] = 1 << 40
    cache = torch.zeros(M.kv4_cache_shape(T // S + 1, H, S, D), dtype=torch.uint8, device="cuda")
    ws = M.Workspace()
    q = torch.ones(T, 2, D, dtype=torch.bfloat16, device="cuda")
    assert M.maps_kv4_append_rotated(q, k, k, pos, torch.ones(10, 64, device="cuda"), slots, cache, S, torch.empty_like(q), axis=axis, ws=ws) == 0
    assert M.maps_check(ws) == M.MAPS_E_RANGE and M.maps_check(ws) == 0


# ------------------------------------------------------------------ ranges
def filled(M, rng, lens, H, D, S, spare=2, scale=1.0):
    """(keys, values per request, table, cache) with the cache's unused places NaN."""
    lens = np.asarray(lens)
    nb = -(-lens // S)
    P = int(nb.sum()) + spare
    perm = rng.permutation(P).astype(np.int32)
    table = np.full((len(lens), max(int(nb.max(initial=0)), 1) + 1), -1, np.int32)
    k, v, slots, at = [], [], [], 0
    bias, size = rng.normal(size=(H, D)) * 2, rng.uniform(0.3, 1.5, (H, D))
    for b, n in enumerate(lens):
        table[b, :nb[b]] = perm[at:at + nb[b]]
        at += nb[b]
        j = np.arange(n)
        slots.append(table[b, j // S].astype(np.int64) * S + j % S)
        k.append(K.bf16(((rng.normal(size=(n, H, D)) * size + bias) * scale).astype(np.float32)))
        v.append(K.bf16(rng.normal(size=(n, H, D)).astype(np.float32)))
    cache = torch.full(M.kv4_cache_shape(P, H, S, D), 0xff, dtype=torch.uint8, device="cuda")
    write(M, np.concatenate(k), np.concatenate(v), np.concatenate(slots), cache, S)
    return k, v, table, cache


def write(M, k, v, slots, cache, S):
    assert M.maps_kv4_append(dev(k, torch.bfloat16), dev(v, torch.bfloat16), dev(slots), cache, S) == 0


RANGES = [  # lengths, tokens held before, H, D, S
    ([1], [0], 1, 64, 16), ([1], None, 2, 128, 16), ([15, 16, 17, 0, 33], [0, 15, 16, 0, 33], 3, 128, 16), ([5, 40, 64], [4, 39, 70], 1, 256, 32),
    ([100, 0, 3, 47, 48, 49], None, 2, 64, 48), ([70, 200], [65, 64], 5, 128, 64), ([5000], None, 1, 64, 4096), ([4100, 4095], [4099, 4094], 2, 128, 4096),
    ([900, 33, 1500, 16], [0, 5, 700, 17], 8, 128, 16), ([3000] * 3 + [1] * 300, [0] * 3 + [0] * 300, 2, 64, 16)]


def check_ranges(M, k, table, cache, lens, held, H, D, S, ws=None):
    P = cache.shape[0]
    codes, scale = torch.full((P, H, 2, D), 77, dtype=torch.int8, device="cuda"), torch.full((P, H), 77.0, device="cuda")
    ws = ws or M.Workspace()
    args = (None if held is None else i32(held), i32(lens), dev(table), cache, S)
    assert M.maps_kv4_block_ranges(*args, codes, scale, ws=ws) == 0 and M.maps_check(ws) == 0
    want_c, want_s = np.full(codes.shape, 77), np.full((P, H), 77, np.float32)
    for b, n in enumerate(lens):
        for j in range(min(held[b], n) // S if held is not None else 0, -(-n // S)):
            for h in range(H):
                want_c[table[b, j], h], want_s[table[b, j], h] = O.range_of(O.held_keys(k[b][j * S:(j + 1) * S, h]))
    assert np.array_equal(scale.cpu().numpy(), want_s, equal_nan=True)
    assert np.array_equal(codes.cpu().numpy(), want_c)
    return codes, scale


@pytest.mark.parametrize("case", range(len(RANGES)))
def test_block_ranges(M, case):
    lens, held, H, D, S = RANGES[case]
    rng = np.random.default_rng(case)
    k, v, table, cache = filled(M, rng, lens, H, D, S)
    check_ranges(M, k, table, cache, lens, held, H, D, S)


@pytest.mark.parametrize("scale", [0.0, 1e-38, 3e-37, 1e-30, 1e30, 1e38])
def test_block_ranges_of_any_size(M, scale):
    rng = np.random.default_rng(8)
    lens = [100, 33, 16]
    k, v, table, cache = filled(M, rng, lens, 2, 128, 16, scale=scale)
    check_ranges(M, k, table, cache, lens, None, 2, 128, 16)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_block_ranges_of_rows_that_differ(M, D):
    """Rows far apart in size and offset, of one value, and such as are held as NaN."""
    rng = np.random.default_rng(D)
    S, lens, H = 32, [32, 64, 50, 96], 2
    k, v, table, cache = filled(M, rng, lens, H, D, S)
    k[0][:] = K.bf16((rng.normal(size=k[0].shape) * 2.0 ** rng.integers(-60, 60, (32, H, 1))).astype(np.float32))
    k[1][:] = K.bf16((1000 + rng.normal(size=k[1].shape) * 2.0 ** rng.integers(-20, 3, (64, H, 1))).astype(np.float32))
    k[2][:] = K.bf16(rng.normal(size=(50, H, 1)).astype(np.float32))  # a row has one value
    k[3][40, 1, D - 1] = np.nan
    k[3][70, 0, 0] = np.inf
    for b, n in enumerate(lens):
        j = np.arange(n)
        write(M, k[b], v[b], table[b, j // S].astype(np.int64) * S + j % S, cache, S)
    check_ranges(M, k, table, cache, lens, None, H, D, S)


@pytest.mark.parametrize("what", ["negative", "long", "table", "held"])
def test_block_ranges_report_bad_data(M, what):
    rng = np.random.default_rng(1)
    k, v, table, cache = filled(M, rng, [40, 20], 1, 64, 16)
    lens, held = [40, 20], [0, 0]
    if what == "negative":
        lens[1] = -1
    if what == "long":
        lens[0] = table.shape[1] * 16 + 1
    if what == "table":
        table[0, 1] = cache.shape[0]
    if what == "held":
        held[0] = -5
    codes, scale = torch.zeros(cache.shape[0], 1, 2, 64, dtype=torch.int8, device="cuda"), torch.zeros(cache.shape[0], 1, device="cuda")
    ws = M.Workspace()
    assert M.maps_kv4_block_ranges(i32(held), i32(lens), dev(table), cache, 16, codes, scale, ws=ws) == 0
    assert M.maps_check(ws) == M.MAPS_E_RANGE and M.maps_check(ws) == 0


# ------------------------------------------------------------------ selection
SELECT = [  # Hq, H, D, S, type, lengths, queries, first, last, n_list
    (1, 1, 64, 16, "bf16", [1], [1], 0, 1, 1), (4, 2, 128, 16, "bf16", [100], [1], 1, 2, 4), (32, 8, 128, 16, "bf16", [3000, 0, 64, 65, 17], [1] * 5, 1, 2, 5),
    (5, 5, 64, 32, "fp16", [700, 31, 33], [5, 3, 1], 0, 1, 7), (16, 1, 256, 16, "bf16", [5000], [1], 2, 2, 40), (7, 1, 128, 64, "fp16", [9000, 4000], [1, 9], 3, 1, 4),
    (6, 2, 64, 16, "bf16", [2, 300, 0, 90], [5, 40, 3, 0], 1, 1, 9), (8, 4, 128, 48, "bf16", [20000, 1], [2, 1], 1, 2, 200), (3, 1, 64, 16, "fp16", [70000], [1], 0, 2, 513),
    (2, 1, 64, 16, "bf16", [16 * 300] * 40, [1] * 40, 1, 1, 33), (2, 2, 128, 16, "bf16", [257 * 16 + 3], [1], 1, 1, 255)]


def select_data(case, rng, levels=None):
    Hq, H, D, S, kind, lens, n_q, first, last, n_list = case
    lens = np.asarray(lens)
    nb = -(-lens // S)
    P = int(nb.sum()) + 3
    perm = rng.permutation(P).astype(np.int32)
    table = np.full((len(lens), max(int(nb.max()), 1) + 2), -1, np.int32)
    at = 0
    for b in range(len(lens)):
        table[b, :nb[b]] = perm[at:at + nb[b]]
        at += nb[b]
    codes = np.sort(rng.integers(-127, 128, (P, H, 2, D)), axis=2).astype(np.int8)
    scale = K.bf16(rng.uniform(0.01, 0.02, (P, H)).astype(np.float32))
    if levels:  # many blocks alike
        same = rng.integers(0, levels, P)
        codes, scale = codes[same], scale[same]
    T = int(np.sum(n_q))
    q = R.rounded(rng.normal(size=(T, Hq, D)).astype(np.float32), kind)
    return q, table, codes, scale, np.concatenate([[0], np.cumsum(n_q)])


def run_select(M, case, q, table, codes, scale, off, status=0, ws=None, lay_q=None, stream=None):
    Hq, H, D, S, kind, lens, n_q, first, last, n_list = case
    T = len(q)
    blocks, tokens = torch.full((T, H, n_list), -7, dtype=torch.int32, device="cuda"), torch.full((T, H), -7, dtype=torch.int32, device="cuda")
    ws = ws or M.Workspace()
    assert M.maps_kv4_select_blocks(lay(q, lay_q, TYPES[kind]), dev(off.astype(np.int64)), i32(lens), dev(table), dev(codes), dev(scale), S, first, last,
                                    blocks, tokens, ws=ws) == 0
    assert M.maps_check(ws) == status
    return blocks.cpu().numpy(), tokens.cpu().numpy()


def check_select(M, case, q, table, codes, scale, off, **kw):
    Hq, H, D, S, kind, lens, n_q, first, last, n_list = case
    blocks, tokens = run_select(M, case, q, table, codes, scale, off, **kw)
    T = len(q)
    want, want_t = O.select(q, off, lens, table, codes, scale, S, first, last, n_list, np.full((T, H, n_list), -7), np.full((T, H), -7))
    assert np.array_equal(tokens, want_t)
    assert np.array_equal(blocks, want)


@pytest.mark.parametrize("case", range(len(SELECT)))
def test_select_blocks(M, case):
    rng = np.random.default_rng(100 + case)
    check_select(M, SELECT[case], *select_data(SELECT[case], rng))
    check_select(M, SELECT[case], *select_data(SELECT[case], rng), lay_q="odd")


@pytest.mark.parametrize("Hq,H,D,kind", [(2, 2, 64, "bf16"), (12, 2, 128, "fp16"), (14, 2, 256, "bf16")])
def test_select_blocks_of_many_rows(M, Hq, H, D, kind):
    """So many that few threads take each: rows of every length that these handle in a way of its own."""
    rng = np.random.default_rng(D)
    lens = np.concatenate([rng.integers(0, 3000, 300), [16 * 21, 16 * 149, 16 * 150, 16 * 278, 16 * 279, 16 * 534, 16 * 535, 16 * 2070, 16 * 2071, 16 * 4000]])
    case = (Hq, H, D, 16, kind, list(rng.permutation(lens)), [1] * len(lens), 2, 1, 22)
    check_select(M, case, *select_data(case, rng))
    check_select(M, case, *select_data(case, rng, 40))


@pytest.mark.parametrize("D,kind", [(128, "bf16"), (256, "fp16")])
def test_select_blocks_of_long_rows(M, D, kind):
    """A cluster's blocks share a row, whose last blocks are few or none for some of them."""
    for n in (2049, 4100, 8193, 9001):
        case = (6, 1, D, 16, kind, [16 * n - 3, 16 * 40], [1, 2], 1, 2, 127)
        check_select(M, case, *select_data(case, np.random.default_rng(n)))


@pytest.mark.parametrize("levels", [1, 2, 3, 50])
def test_select_blocks_of_equal_scores(M, levels):
    """Ties go to the earlier blocks, in rows that one pass of the threads covers and in longer ones."""
    for lens in ([400 * 16 - 5, 77 * 16], [900 * 16], [3000 * 16, 1200 * 16]):
        case = (4, 2, 64, 16, "bf16", lens, [1] * len(lens), 1, 2, 61)
        check_select(M, case, *select_data(case, np.random.default_rng(levels), levels))


def test_select_blocks_of_scales_and_queries_that_are_no_numbers(M):
    case = (4, 2, 128, 16, "bf16", [3000, 3000, 3000, 3000, 3000], [1] * 5, 1, 1, 30)
    rng = np.random.default_rng(2)
    q, table, codes, scale, off = select_data(case, rng)
    scale[rng.random(scale.shape) < 0.1] = np.nan  # fewer than n_list of them, and
    scale[table[1, :150]] = np.nan                 # more
    scale[rng.random(scale.shape) < 0.1] = 0
    q[2], q[3, 0, 5], q[4, 3, 9] = 0, np.nan, np.inf
    check_select(M, case, q, table, codes, scale, off)


@pytest.mark.parametrize("size", [1e-40, 1e-37, 1e-20, 1e20, 3e38])
def test_select_blocks_for_queries_of_any_size(M, size):
    case = (8, 1, 64, 16, "bf16", [2000, 1999], [1, 1], 0, 1, 20)
    q, table, codes, scale, off = select_data(case, np.random.default_rng(3))
    check_select(M, case, K.bf16(np.clip(q * size, -3.3e38, 3.3e38).astype(np.float32)), table, codes, scale, off)


def test_select_blocks_of_signed_scores_of_any_size(M):
    case = (2, 1, 64, 16, "bf16", [5000, 4000], [1, 1], 0, 1, 100)
    rng = np.random.default_rng(4)
    q, table, codes, scale, off = select_data(case, rng)
    scale *= (2.0 ** rng.integers(-100, 100, scale.shape)).astype(np.float32)
    check_select(M, case, q, table, codes, scale, off)


def test_select_blocks_of_rows_longer_than_shared_memory(M):
    case = (2, 1, 64, 16, "bf16", [16 * 40000 - 9, 16 * 9], [1, 1], 1, 2, 700)
    check_select(M, case, *select_data(case, np.random.default_rng(6)))


def test_select_blocks_leaves_rows_of_no_request(M):
    case = (4, 2, 64, 16, "bf16", [300, 200, 500], [1] * 3, 1, 1, 4)
    q, table, codes, scale, off = select_data(case, np.random.default_rng(7))
    q = np.concatenate([q, q, q])
    off = np.array([2, 3, 3, 5])
    blocks, tokens = run_select(M, case, q, table, codes, scale, off)
    for rows in (slice(0, 2), slice(5, 9)):
        assert (blocks[rows] == -7).all() and (tokens[rows] == -7).all()
    want, want_t = O.select(q, off, case[5], table, codes, scale, 16, 1, 1, 4, np.full(blocks.shape, -7), np.full(tokens.shape, -7))
    assert np.array_equal(blocks, want) and np.array_equal(tokens, want_t)


@pytest.mark.parametrize("B", [255, 256, 257, 70000])
def test_select_blocks_of_many_requests(M, B):
    """The request of a row is found among any number, with empty ones between."""
    rng = np.random.default_rng(B)
    n_q = (rng.random(B) < (0.6 if B < 1000 else 0.01)).astype(int) * rng.integers(1, 3, B)
    case = (1, 1, 64, 16, "bf16", list(rng.integers(0, 200, B)), list(n_q), 1, 1, 5)
    check_select(M, case, *select_data(case, rng))


@pytest.mark.parametrize("what", ["negative", "long", "offsets", "table"])
def test_select_blocks_report_bad_data(M, what):
    case = (4, 2, 64, 16, "bf16", [300, 400], [1, 1], 1, 1, 4)
    q, table, codes, scale, off = select_data(case, np.random.default_rng(9))
    if what == "negative":
        case[5][1] = -1
    if what == "long":
        case[5][0] = table.shape[1] * 16 + 1
    if what == "offsets":
        off[2] = 3
    if what == "table":
        table[0, 5] = len(codes)
    run_select(M, case, q, table, codes, scale, off, status=M.MAPS_E_RANGE)


# ------------------------------------------------------------------ attention over lists
ATTEND = [  # Hq, H, D, S, type, n_list, tokens of each row (the same for its heads, or drawn below them)
    (1, 1, 64, 16, "bf16", 1, [1, 0, 16, 5]), (4, 1, 128, 16, "fp16", 7, [100, 112, 97, 1, 0, 33]), (8, 2, 128, 32, "bf16", 40, [1280, 1249, 3, 0, 640]),
    (32, 8, 128, 16, "bf16", 64, [1024] * 9), (20, 4, 64, 64, "fp16", 33, [2100, 2112, 0, 64, 65]), (16, 1, 256, 32, "bf16", 60, [1900, 31]),
    (24, 1, 128, 16, "bf16", 30, [470, 480]), (5, 5, 256, 16, "fp16", 9, [140] * 7), (16, 2, 64, 48, "bf16", 20, [950, 1]), (2, 1, 128, 4096, "bf16", 2, [8000, 4097, 7]),
    (3, 3, 64, 16, "bf16", 3, list(range(48)) * 20), (8, 8, 128, 16, "bf16", 4, [64, 50] * 200), (4, 1, 128, 64, "bf16", 1000, [64000])]


def attend_case(M, case, seed=0, lay_q=None, with_lse=True, ws=None, patch=None, status=0, distinct=True):
    Hq, H, D, S, kind, n_list, tokens = case
    rng = np.random.default_rng(seed + D + n_list)
    T, group = len(tokens), Hq // H
    n = np.repeat(np.asarray(tokens)[:, None], H, 1)
    n[::2, 1:] = rng.integers(0, np.maximum(n[::2, 1:], 0) + 1)  # heads of a row may differ
    P = min(2 * n_list + 5, 3000)
    k = R.rounded((rng.normal(size=(P * S, H, D)) + rng.normal(size=(H, D))).astype(np.float32), kind)
    v = R.rounded((rng.normal(size=(P * S, H, D)) * 2.0 ** rng.uniform(-1, 1, (P * S, H, 1))).astype(np.float32), kind)
    ids = np.stack([[rng.permutation(P)[:n_list] if distinct else rng.integers(0, P, n_list) for _ in range(H)] for _ in range(T)]).astype(np.int32)
    q = R.rounded((2 * rng.normal(size=(T, Hq, D))).astype(np.float32), kind)
    dt = TYPES[kind]
    cache = torch.full(M.kv4_cache_shape(P, H, S, D), 0xff, dtype=torch.uint8, device="cuda")
    assert M.maps_kv4_append(dev(k, dt), dev(v, dt), dev(np.arange(P * S)), cache, S) == 0
    unused = np.arange(n_list) >= -(-np.maximum(n, 0) // S)[..., None]
    given = np.where(unused, rng.choice([-1, P, 1 << 30], ids.shape), ids).astype(np.int32)  # nobody looks at these
    if patch:
        patch(given, n)
    dq = lay(q, lay_q, dt)
    out = lay(np.full(q.shape, 77.0, np.float32), lay_q, dt)
    lse = torch.full((T, Hq), 77.0, device="cuda") if with_lse else None
    ws = ws or M.Workspace()
    assert M.maps_kv4_attention_blocks(dq, dev(given), i32(n), cache, S, D ** -0.5, out, lse_out=lse, ws=ws) == 0
    assert M.maps_check(ws) == status
    if status:
        return None
    kk, vv, lens = [], [], []
    for i in range(T):
        for h in range(H):
            m = max(int(n[i, h]), 0)
            at = (ids[i, h, :, None].astype(np.int64) * S + np.arange(S)).reshape(-1)[:m]
            kk.append(k[at][:, h:h + 1])
            vv.append(v[at][:, h:h + 1])
            lens.append(m)
    e = R.expect(kind, q.reshape(T * H, group, D), np.arange(T * H + 1), lens, kk, vv, 1, D ** -0.5)
    e["has"] = (n >= 0).reshape(-1)
    o = out.float().cpu().numpy().reshape(T * H, group, D)
    l = lse.cpu().numpy().reshape(T * H, group) if with_lse else None
    assert R.wrong(e, o, l) is None
    assert (o[~e["has"]] == 77).all() and (l is None or (l[~e["has"]] == 77).all())
    return out, lse, (dq, dev(given), i32(n), cache)


@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_attention_blocks(M, case):
    attend_case(M, ATTEND[case])


@pytest.mark.parametrize("case", [1, 2, 5])
def test_attention_blocks_of_other_strides_and_no_lse(M, case):
    attend_case(M, ATTEND[case], seed=1, lay_q="odd", with_lse=False)
    attend_case(M, ATTEND[case], seed=2, lay_q="gaps")


def test_attention_blocks_named_twice(M):
    attend_case(M, ATTEND[2], distinct=False)


@pytest.mark.parametrize("case", [2, 5, 10])
def test_attention_blocks_leaves_rows_of_negative_tokens(M, case):
    def patch(given, n):
        n[1], n[-1, 0] = -1, -5
        given[1] = 1 << 30
    attend_case(M, ATTEND[case], patch=patch)


def test_attention_blocks_of_no_row_with_tokens(M):
    def patch(given, n):
        n[:] = -1
    attend_case(M, ATTEND[2], patch=patch)
    def zero(given, n):
        n[:] = 0
    attend_case(M, ATTEND[2], patch=zero)


@pytest.mark.parametrize("what", ["many", "block", "negative block"])
def test_attention_blocks_report_bad_data(M, what):
    def patch(given, n):
        if what == "many":
            n[0, 0] = ATTEND[2][5] * 32 + 1
        else:
            given[0, 0, 0] = -1 if what == "negative block" else 1 << 30
    attend_case(M, ATTEND[2], patch=patch, status=M.MAPS_E_RANGE)


def test_attention_over_all_blocks_is_attention(M):
    """Lists of all blocks in their order: what the dense call gives, to both calls' bounds."""
    rng = np.random.default_rng(0)
    Hq, H, D, S, lens = 8, 2, 128, 16, [700, 33, 0, 1500]
    k, v, table, cache = filled(M, rng, lens, H, D, S)
    q = K.bf16((2 * rng.normal(size=(4, Hq, D))).astype(np.float32))
    L = table.shape[1]
    lists = np.repeat(table[:, None], H, 1)
    out, lse = torch.empty(4, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(4, Hq, device="cuda")
    assert M.maps_kv4_attention_blocks(dev(q, torch.bfloat16), dev(lists), i32(np.repeat(np.array(lens)[:, None], H, 1)), cache, S, D ** -0.5, out, lse_out=lse) == 0
    e = R.expect("bf16", q, np.arange(5), lens, k, v, H, D ** -0.5)
    assert R.wrong(e, out.float().cpu().numpy(), lse.cpu().numpy()) is None
    dense, dense_lse = torch.empty_like(out), torch.empty_like(lse)
    assert M.maps_kv4_attention(dev(q, torch.bfloat16), dev(np.arange(5)), i32(lens), dev(table), cache, S, D ** -0.5, dense, lse_out=dense_lse) == 0
    assert R.wrong(e, dense.float().cpu().numpy(), dense_lse.cpu().numpy()) is None
