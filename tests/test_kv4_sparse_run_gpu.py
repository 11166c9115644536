"""The sparse-decoding calls together, as a decoder uses them: block tables, keys turned on their way
into the cache, ranges of the blocks that tokens went to, lists, attention over them; step by
step, on other streams and in graphs.  Lists and ranges are compared bit for bit, attention with the
row-wise bounds of kv4_rows.py."""
import numpy as np
import pytest
import torch

import kv4_oracle as K
import kv4_rows as R
import kv4_sparse_oracle as O

pytestmark = pytest.mark.gpu


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


class Step:
    """One decoder's memory and a step over it."""

    def __init__(self, M, R_, Hq, H, D, S, n_list, pool, most, kind="bf16", seed=0):
        self.M, self.R, self.Hq, self.H, self.D, self.S, self.n_list, self.kind = M, R_, Hq, H, D, S, n_list, kind
        self.dt = dict(bf16=torch.bfloat16, fp16=torch.float16)[kind]
        self.rng = np.random.default_rng(seed)
        self.cache = torch.full(M.kv4_cache_shape(pool, H, S, D), 0xff, dtype=torch.uint8, device="cuda")
        self.codes = torch.full(M.kv4_range_shape(pool, H, D), 77, dtype=torch.int8, device="cuda")
        self.scale = torch.full((pool, H), float("nan"), device="cuda")
        self.table = torch.full((R_, most), -1, dtype=torch.int32, device="cuda")
        self.free, self.n_free = torch.arange(pool, dtype=torch.int32, device="cuda"), i32([pool])
        self.held = np.zeros(R_, np.int64)
        angle = np.arange(most * S)[:, None] * 1e4 ** (-np.arange(D // 2) / (D // 2))
        self.turns = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
        self.keys = [np.zeros((0, H, D), np.float32) for _ in range(R_)]  # as they were given to the cache, turned
        self.values = [np.zeros((0, H, D), np.float32) for _ in range(R_)]
        self.ws = M.Workspace()

    def rows(self, T, heads, size=1.0):
        return R.rounded((self.rng.normal(size=(T, heads, self.D)) * size).astype(np.float32), self.kind)

    def step(self, want, first=1, last=2):
        M, S = self.M, self.S
        want = np.asarray(want)
        T = int(np.maximum(want - self.held, 0).sum())
        got, off = i32(np.zeros(self.R)), torch.zeros(self.R + 1, dtype=torch.int64, device="cuda")
        slots, pos, n_free = torch.zeros(T, dtype=torch.int64, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda"), i32([0])
        held = i32(self.held)
        assert M.maps_block_tables(S, held, i32(want), self.table, self.free, self.n_free, n_free, got, off, slots, pos_out=pos, ws=self.ws) == 0
        q, k, v = self.rows(T, self.Hq, 2.0), self.rows(T, self.H) + 0, self.rows(T, self.H)
        dq, dk, dv = (dev(x, self.dt) for x in (q, k, v))
        assert M.maps_kv4_append_rotated(dq, dk, dv, pos, dev(self.turns), slots, self.cache, S, dq, ws=self.ws) == 0
        assert M.maps_kv4_block_ranges(held, got, self.table, self.cache, S, self.codes, self.scale, ws=self.ws) == 0
        blocks = torch.full((T, self.H, self.n_list), -5, dtype=torch.int32, device="cuda")
        tokens = torch.full((T, self.H), -5, dtype=torch.int32, device="cuda")
        assert M.maps_kv4_select_blocks(dq, off, got, self.table, self.codes, self.scale, S, first, last, blocks, tokens, ws=self.ws) == 0
        out, lse = torch.full((T, self.Hq, self.D), 7.0, dtype=self.dt, device="cuda"), torch.full((T, self.Hq), 7.0, device="cuda")
        assert M.maps_kv4_attention_blocks(dq, blocks, tokens, self.cache, S, self.D ** -0.5, out, lse_out=lse, ws=self.ws) == 0
        assert M.maps_check(self.ws) == 0
        self.n_free = n_free
        # ---- the same by definition
        p = pos.cpu().numpy()[None]
        turned_q = torch.from_numpy(O.rotate(q, p, None, self.D, False, self.turns)).to(self.dt)
        assert torch.equal(dq.cpu(), turned_q)
        tk = O.rotate(k, p, None, self.D, False, self.turns)
        at, lens, table = off.cpu().numpy(), got.cpu().numpy(), self.table.cpu().numpy()
        assert np.array_equal(lens, want)
        codes, scale = self.codes.cpu().numpy(), self.scale.cpu().numpy()
        for b in range(self.R):
            self.keys[b] = np.concatenate([self.keys[b], tk[at[b]:at[b + 1]]])[:want[b]]
            self.values[b] = np.concatenate([self.values[b], v[at[b]:at[b + 1]]])[:want[b]]
            for j in range(-(-int(want[b]) // S)):
                for h in range(self.H):
                    c, s = O.range_of(O.held_keys(self.keys[b][j * S:(j + 1) * S, h]))
                    assert np.array_equal(codes[table[b, j], h], c) and scale[table[b, j], h] == s
        wb, wt = O.select(turned_q.float().numpy(), at, lens, table, codes, scale, S, first, last, self.n_list,
                          np.full(blocks.shape, -5), np.full(tokens.shape, -5))
        assert np.array_equal(blocks.cpu().numpy(), wb) and np.array_equal(tokens.cpu().numpy(), wt)
        where = {int(table[b, j]): (b, j) for b in range(self.R) for j in range(-(-int(want[b]) // S))}
        kk, vv, n = [], [], []
        for i in range(T):
            for h in range(self.H):
                m = int(wt[i, h])
                rows = [np.arange(where[int(x)][1] * S, where[int(x)][1] * S + S) for x in wb[i, h] if x >= 0]
                rows = np.concatenate(rows)[:m] if rows else np.zeros(0, int)
                b = where[int(wb[i, h, 0])][0] if m else 0
                kk.append(self.keys[b][rows][:, h:h + 1])
                vv.append(self.values[b][rows][:, h:h + 1])
                n.append(m)
        group = self.Hq // self.H
        e = R.expect(self.kind, turned_q.float().numpy().reshape(T * self.H, group, self.D), np.arange(T * self.H + 1), n, kk, vv, 1, self.D ** -0.5)
        assert R.wrong(e, out.float().cpu().numpy().reshape(T * self.H, group, self.D), lse.cpu().numpy().reshape(T * self.H, group)) is None
        self.held = want


@pytest.mark.parametrize("Hq,H,D,S,kind", [(8, 2, 64, 16, "bf16"), (6, 2, 128, 32, "fp16"), (4, 1, 256, 16, "bf16")])
def test_decoding_step_by_step(M, Hq, H, D, S, kind):
    """A prompt each, then tokens, drafts of which some are taken back, a request that ends and one that comes."""
    d = Step(M, 4, Hq, H, D, S, n_list=6, pool=120, most=30, kind=kind)
    want = np.array([150, 33, 0, 290])
    d.step(want)
    for n in range(5):
        want = want + np.array([1, 1, 0, 4])
        d.step(want)
        want = want - np.array([0, 0, 0, 3])  # drafts not accepted
        d.step(want)
    want = np.array([want[0] + 1, 0, 77, want[3] + 1])  # the second is done, the third begins
    d.step(want)
    d.step(want + np.array([1, 0, 1, 1]))


def state(M, seed, T=6, Hq=8, H=2, D=128, S=16, n_list=9, n=500):
    """Inputs of a step whose cache is filled: everything that the four calls read and write."""
    rng = np.random.default_rng(seed)
    nb = -(-n // S)
    P = T * nb + 2
    table = rng.permutation(P)[:T * nb].reshape(T, nb).astype(np.int32)
    f = lambda *s: dev(rng.normal(size=s).astype(np.float32), torch.bfloat16)  # noqa: E731
    s = dict(S=S, cache=torch.full(M.kv4_cache_shape(P, H, S, D), 0xff, dtype=torch.uint8, device="cuda"), table=dev(table),
             codes=torch.zeros(M.kv4_range_shape(P, H, D), dtype=torch.int8, device="cuda"), scale=torch.zeros(P, H, device="cuda"),
             off=dev(np.arange(T + 1)), held=i32(np.full(T, n - 1)), n=i32(np.full(T, n)), q=f(T, Hq, D), k=f(T, H, D), v=f(T, H, D),
             pos=i32(np.full((1, T), n - 1)), turns=dev(rng.normal(size=(n, D)).astype(np.float32)),
             slots=dev(table[:, -1].astype(np.int64) * S + (n - 1) % S), q_out=f(T, Hq, D), blocks=i32(np.zeros((T, H, n_list))),
             tokens=i32(np.zeros((T, H))), out=f(T, Hq, D), lse=torch.zeros(T, Hq, device="cuda"))
    j = np.arange(n - 1)
    old = (table[:, j // S].astype(np.int64) * S + j % S).reshape(-1)
    assert M.maps_kv4_append(f(len(old), H, D), f(len(old), H, D), dev(old), s["cache"], S) == 0
    assert M.maps_kv4_block_ranges(None, s["held"], s["table"], s["cache"], S, s["codes"], s["scale"]) == 0
    return s


def run(M, s, ws=None, stream=None):
    kw = dict(ws=ws, stream=stream)
    st = [M.maps_kv4_append_rotated(s["q"], s["k"], s["v"], s["pos"], s["turns"], s["slots"], s["cache"], s["S"], s["q_out"], **kw),
          M.maps_kv4_block_ranges(s["held"], s["n"], s["table"], s["cache"], s["S"], s["codes"], s["scale"], **kw),
          M.maps_kv4_select_blocks(s["q_out"], s["off"], s["n"], s["table"], s["codes"], s["scale"], s["S"], 1, 2, s["blocks"], s["tokens"], **kw),
          M.maps_kv4_attention_blocks(s["q_out"], s["blocks"], s["tokens"], s["cache"], s["S"], 0.1, s["out"], lse_out=s["lse"], **kw)]
    assert st == [0] * 4


WRITTEN = ("cache", "codes", "scale", "q_out", "blocks", "tokens", "out", "lse")


def results(s):
    return {x: s[x].clone() for x in WRITTEN}


def same(a, b):
    return [x for x in WRITTEN if not torch.equal(a[x].view(torch.uint8), b[x].view(torch.uint8))]


@pytest.mark.parametrize("T,n", [(1, 20000), (6, 500), (40, 900), (300, 400)])
def test_repeated_calls_give_the_same_bits(M, T, n):
    """Whatever the split: clusters of blocks, one block, few threads for many rows."""
    s, ws = state(M, 1, T=T, n=n), M.Workspace()
    run(M, s, ws)
    first = results(s)
    for _ in range(20):
        for x in ("out", "lse", "blocks", "tokens", "q_out"):
            s[x].zero_()
        run(M, s, ws)
        assert not same(first, results(s))
    assert M.maps_check(ws) == 0


def test_graphs_replayed_on_new_inputs(M):
    """Two captured graphs that share a workspace, one after the other, on inputs that change in place."""
    a, b, ws = state(M, 2), state(M, 3, T=40, n=700), M.Workspace()
    run(M, a, ws), run(M, b, ws)  # what a first call sets up
    side = torch.cuda.Stream()
    graphs = []
    side.wait_stream(torch.cuda.current_stream())
    for s in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            run(M, s, ws)
        graphs.append(g)
    for seed in (7, 8):
        for s, g, T in ((a, graphs[0], 6), (b, graphs[1], 40)):
            new = state(M, seed, T=T, n=500 if T == 6 else 700)
            for x in s:
                if x != "S":
                    s[x].copy_(new[x])
            eager = {k: v if k == "S" else v.clone() for k, v in s.items()}
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            run(M, eager, M.Workspace())
            assert not same(results(eager), results(s))
    assert M.maps_check(ws) == 0


def test_two_streams_at_once(M):
    """Each with a workspace of its own, named or none; the calls of one stream do not wait for the other's."""
    states = [state(M, 10 + x, T=5 + 30 * x, n=600) for x in range(2)]
    copies = [{k: v if k == "S" else v.clone() for k, v in s.items()} for s in states]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for n in range(5):
        for x in range(2):
            if n % 2:
                run(M, states[x], stream=streams[x])
            else:
                with torch.cuda.stream(streams[x]):
                    run(M, states[x])
    torch.cuda.synchronize()
    for s, c in zip(states, copies):
        run(M, c)
        assert not same(results(s), results(c))


def test_a_padded_batch(M):
    """Rows behind the last request: lists of -1 tokens that were set once leave them out of every call's work."""
    s = state(M, 4)
    pad = 5
    more = {x: torch.cat([s[x], torch.full((pad, *s[x].shape[1:]), 3, dtype=s[x].dtype, device="cuda")]) for x in ("q", "q_out", "blocks", "out", "lse")}
    more["tokens"] = torch.cat([s["tokens"], i32(np.full((pad, 2), -1))])
    run(M, s)
    want = results(s)
    p = s | more
    p["slots"] = torch.cat([s["slots"], dev(np.full(pad, -1))])
    p["pos"] = torch.cat([s["pos"], i32(np.zeros((1, pad)))], 1)
    p["k"], p["v"] = (torch.cat([s[x], torch.full((pad, 2, 128), float("nan"), dtype=torch.bfloat16, device="cuda")]) for x in "kv")
    run(M, p)
    for x in ("q_out", "blocks", "tokens", "out", "lse"):
        assert torch.equal(p[x][:6], want[x])
    assert (p["blocks"][6:] == 3).all() and (p["tokens"][6:] == -1).all() and (p["out"][6:] == 3).all() and (p["lse"][6:] == 3).all()


def test_empty_calls(M):
    s = state(M, 5)
    z = {x: s[x][:0] for x in ("q", "k", "v", "slots", "q_out", "blocks", "tokens", "out", "lse", "held", "n", "table")}
    z["pos"], z["off"] = s["pos"][:, :0].contiguous(), s["off"][:1]
    before = {x: s[x].clone() for x in ("cache", "codes", "scale")}
    run(M, s | z)
    assert all(torch.equal(before[x], s[x]) for x in before)


def test_a_call_without_cache_blocks_reports_what_points_there(M):
    s = state(M, 6)
    none = dict(cache=s["cache"][:0], codes=s["codes"][:0], scale=s["scale"][:0])
    ws = M.Workspace()
    for call in (lambda x: M.maps_kv4_append_rotated(x["q"], x["k"], x["v"], x["pos"], x["turns"], x["slots"], x["cache"], 16, x["q_out"], ws=ws),
                 lambda x: M.maps_kv4_block_ranges(x["held"], x["n"], x["table"], x["cache"], 16, x["codes"], x["scale"], ws=ws),
                 lambda x: M.maps_kv4_select_blocks(x["q"], x["off"], x["n"], x["table"], x["codes"], x["scale"], 16, 1, 2, x["blocks"], x["tokens"], ws=ws),
                 lambda x: M.maps_kv4_attention_blocks(x["q"], x["blocks"], x["tokens"] + 5, x["cache"], 16, 0.1, x["out"], ws=ws)):
        assert call(s | none) == 0 and M.maps_check(ws) == M.MAPS_E_RANGE


def test_long_offsets(M):
    """A cache, its ranges and the strides of queries past 2^31 bytes and elements: the last blocks are the ones in use."""
    free, _ = torch.cuda.mem_get_info()
    H, D, S, Hq = 8, 256, 64, 8
    P = (1 << 31) // (S // 16 * (16 * D + 128) * H) * 5  # 10 GB
    cache = torch.empty(M.kv4_cache_shape(P, H, S, D), dtype=torch.uint8, device="cuda")
    codes, scale = torch.empty(M.kv4_range_shape(P, H, D), dtype=torch.int8, device="cuda"), torch.empty(P, H, device="cuda")
    rng = np.random.default_rng(0)
    n, T = 700, 3
    nb = -(-n // S)
    table = np.sort(rng.permutation(P // 5)[:T * nb]).reshape(T, nb).astype(np.int32) + P // 5 * 4 - 1
    j = np.arange(n)
    slots = dev((table[:, j // S].astype(np.int64) * S + j % S).reshape(-1))
    k, v = (R.rounded(rng.normal(size=(T * n, H, D)).astype(np.float32), "bf16") for _ in range(2))
    row = (1 << 31) // T + 64  # elements between the queries' rows
    room = torch.zeros(2 * row + Hq * D, dtype=torch.bfloat16, device="cuda")
    q = R.rounded((2 * rng.normal(size=(T, Hq, D))).astype(np.float32), "bf16")
    dq = room.as_strided((T, Hq, D), (row, D, 1)).copy_(dev(q, torch.bfloat16))
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert M.maps_kv4_append_rotated(None, dev(k, torch.bfloat16), dev(v, torch.bfloat16), i32(np.zeros((1, T * n))), torch.zeros(1, 0, device="cuda"), slots,
                                     cache, S, None, axis=none) == 0
    lens = i32([n] * T)
    assert M.maps_kv4_block_ranges(None, lens, dev(table), cache, S, codes, scale) == 0
    for i in (0, T - 1):
        for b in (0, nb - 1):
            for h in (0, H - 1):
                c, x = O.range_of(O.held_keys(k[i * n + b * S:min(n, b * S + S) + i * n if b == nb - 1 else i * n + b * S + S, h][:min(S, n - b * S)]))
                assert np.array_equal(codes[table[i, b], h].cpu().numpy(), c) and float(scale[table[i, b], h]) == x
    L = 5
    blocks, tokens = i32(np.zeros((T, H, L))), i32(np.zeros((T, H)))
    assert M.maps_kv4_select_blocks(dq, dev(np.arange(T + 1)), lens, dev(table), codes, scale, S, 1, 1, blocks, tokens) == 0
    used = np.unique(table)
    small = {int(x): y for y, x in enumerate(used)}
    c, s = codes[dev(used.astype(np.int64))].cpu().numpy(), scale[dev(used.astype(np.int64))].cpu().numpy()
    wb, wt = O.select(q, np.arange(T + 1), [n] * T, np.vectorize(small.get)(table), c, s, S, 1, 1, L, np.zeros((T, H, L), int), np.zeros((T, H), int))
    got = np.vectorize(small.get)(blocks.cpu().numpy())
    assert np.array_equal(got, wb) and np.array_equal(tokens.cpu().numpy(), wt)
    out = torch.zeros(T, Hq, D, dtype=torch.bfloat16, device="cuda")
    assert M.maps_kv4_attention_blocks(dq, blocks, tokens, cache, S, D ** -0.5, out) == 0
    kk, vv = [], []
    for i in range(T):
        for h in range(H):
            rows = np.concatenate([np.flatnonzero(table[i] == used[x])[0] * S + np.arange(S) for x in wb[i, h]])[:wt[i, h]] + i * n
            kk.append(k[rows][:, h:h + 1])
            vv.append(v[rows][:, h:h + 1])
    e = R.expect("bf16", q.reshape(T * H, 1, D), np.arange(T * H + 1), [len(x) for x in kk], kk, vv, 1, D ** -0.5)
    assert R.wrong(e, out.float().cpu().numpy().reshape(T * H, 1, D)) is None
