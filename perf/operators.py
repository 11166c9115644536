"""Measured cases of the decoder-side operators: block tables, the 4-bit KV cache, attention over it.

Each case is one call (for the cache's write: one write and one read-back) on data
made from a seed.  Where `own` is true, run() makes the framework's calls; where it
is false, it computes the same results with elementary torch operations in 32 bits.
exact() gives the results of the definitions in 64 bits.

The 4-bit cache's layout, as the framework documents it: cache[block][kv head] is a
record of S/16 groups; a group holds 16 tokens as

  8*D bytes   K codes, token by token, two channels a byte (the even one in the low half);
  8*D bytes   V codes, in units of 16 bits that hold 4 neighbouring channels of one token;
  128 bytes   16 x (K scale, K zero), then 16 x (V scale, V zero), all bfloat16.

With D/8 channels to each g, B = min(D/32, 4) and channel = g*(D/8) + 4*(a*B + b) + r,
token = 8h + 2t + parity, the V unit of (h, a, g, t, b, parity) is at 16-bit index
((((h*A + a)*8 + g)*4 + t)*B + b)*2 + parity.  A value is scale*code + zero.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# --------------------------------------------------------------------------- cases
def listed():
    return [
        # one decode step of a small decoder: 64 running requests take a token each
        dict(name="tables_decode", op="tables", R=64, S=16, most=8192, new=0.0, gone=0.0, prompt=2048, enough=1.0, lens=1),
        # 4,096 requests with prompts of 64 to 8,192 tokens: an eighth has finished, an eighth is
        # admitted in the scheduler's order, the others take a token; the pool runs short
        dict(name="tables_admit", op="tables", R=4096, S=16, most=65536, new=0.125, gone=0.125, prompt=8192, enough=0.9, lens=2),
        # one decode step's keys and values of 512 requests
        dict(name="append_decode", op="append", T=512, H=8, D=128, S=16, dtype="bf16", skip=0.0, fused=True),
        # odd head count and token count, half precision, some tokens without a slot
        dict(name="append_odd", op="append", T=3001, H=5, D=64, S=32, dtype="fp16", skip=0.1, fused=False),
        # a whole prefill batch of 65,536 tokens
        dict(name="append_prefill", op="append", T=65536, H=8, D=128, S=16, dtype="bf16", skip=0.0, fused=True),
        # a single request of up to 2,048 tokens: the latency of one token
        dict(name="attn_one", op="attn", B=1, low=1024, high=2048, n_q=1, Hq=32, H=8, D=128, S=16, dtype="bf16", window=0, causal=True, holes=0.0, lens=3),
        # a decoder's 64 residents, prompts up to 2,048 tokens and what they have generated, a few places idle
        dict(name="attn_decode", op="attn", B=64, low=33, high=4096, n_q=1, Hq=32, H=8, D=128, S=16, dtype="bf16", window=0, causal=True, holes=0.05, lens=4),
        # a decoder filled to half a million tokens, prompts up to 8,192 tokens
        dict(name="attn_decode_full", op="attn", B=128, low=64, high=8192, n_q=1, Hq=32, H=8, D=128, S=16, dtype="bf16", window=0, causal=True, holes=0.0, lens=5),
        # few requests with very long contexts, five query heads to a KV head, half precision
        dict(name="attn_long", op="attn", B=3, low=40001, high=131071, n_q=1, Hq=20, H=4, D=64, S=64, dtype="fp16", window=0, causal=True, holes=0.0, lens=6),
        # one KV head of 256 channels for sixteen query heads
        dict(name="attn_mqa", op="attn", B=31, low=200, high=16384, n_q=1, Hq=16, H=1, D=256, S=32, dtype="bf16", window=0, causal=True, holes=0.0, lens=7),
        # four drafted tokens and the last accepted one, sliding window
        dict(name="attn_drafts", op="attn", B=48, low=5, high=4096, n_q=5, Hq=16, H=4, D=128, S=32, dtype="bf16", window=1024, causal=True, holes=0.0, lens=8),
        # chunks of prompts, up to 1,024 new tokens each, behind what is cached already
        dict(name="attn_chunk", op="attn", B=6, low=1500, high=9000, n_q=1024, Hq=32, H=8, D=128, S=16, dtype="bf16", window=0, causal=True, holes=0.0, lens=9),
    ]


def draw(rng):
    def spread(a, b):
        return min(b, max(a, int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))))

    op = rng.choice(["tables", "append", "attn", "attn", "attn"])
    S = rng.choice([16, 16, 32, 64])
    lens = rng.randrange(1 << 20)
    if op == "tables":
        R = spread(1, 16384)
        return dict(op=op, R=R, S=S, most=max(64, min(65536, (1 << 24) // R * S)), new=rng.choice([0.0, 0.1, 0.3]),
                    gone=rng.choice([0.0, 0.1]), prompt=spread(32, 8192 if R <= 4096 else 1024), enough=rng.choice([0.5, 0.95, 1.0]), lens=lens)
    H, D, dtype = rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128, 128, 256]), rng.choice(["bf16", "bf16", "fp16"])
    if op == "append":
        return dict(op=op, T=spread(1, 65536 * 1024 // (H * D)), H=H, D=D, S=S, dtype=dtype, skip=rng.choice([0.0, 0.1]), fused=rng.random() < 0.5)
    group = rng.choice([1, 2, 3, 4, 5, 7, 8, 16])
    kind = rng.choice(["decode", "decode", "drafts", "chunk"])
    n_q = 1 if kind == "decode" else rng.randint(2, 9) if kind == "drafts" else spread(16, 1024)
    high = spread(n_q + 1, 131072 if kind == "decode" else 32768 if kind == "drafts" else 8192)
    c = dict(op=op, B=spread(1, 256), low=max(1, high // rng.choice([1, 4, 50])), high=high, n_q=n_q, Hq=group * H, H=H, D=D, S=S, dtype=dtype,
             window=rng.choice([0, 0, 0, 128, 1024]), causal=rng.random() < 0.9, holes=rng.choice([0.0, 0.1]), lens=lens)
    while c["B"] > 1 and (c["B"] * c["high"] * H * D > 1 << 29 or c["B"] * c["high"] * c["n_q"] * c["Hq"] * D > 3 << 35):
        c["B"] = (c["B"] + 1) // 2
    while c["high"] * c["n_q"] * c["Hq"] * D > 3 << 35:
        c["n_q"] = (c["n_q"] + 1) // 2
    return c


# --------------------------------------------------------------------------- lengths, the same for every seed but for their order
def table_lengths(c):
    r = np.random.default_rng(c["lens"])
    R = c["R"]
    held = np.minimum(r.integers(min(32, c["prompt"]), c["prompt"] + 1, R) + r.lognormal(5.5, 1.0, R).astype(np.int64), c["most"] - 1)
    want = held + 1
    kind = r.random(R)
    want[kind < c["gone"]] = 0
    new = kind > 1 - c["new"]
    held[new], want[new] = 0, np.minimum(held[new], c["most"])
    return held, want


def attn_lengths(c):
    r = np.random.default_rng(c["lens"])
    n = r.integers(c["low"], c["high"] + 1, c["B"])
    n_q = np.full(c["B"], c["n_q"]) if c["n_q"] <= 16 else r.integers(max(1, c["n_q"] // 3), c["n_q"] + 1, c["B"])
    n = np.maximum(n, n_q)
    hole = r.random(c["B"]) < c["holes"]
    hole[0] = False
    n[hole] = 0
    return n, n_q


def blocks(n, S):
    return -(-n // S)


def record_bytes(c):
    return c["S"] // 16 * (16 * c["D"] + 128)


# --------------------------------------------------------------------------- the 4-bit form, in elementary operations
def quantise(x):
    """Codes (uint8) and bfloat16 (scale, zero) of rows of the last axis; arithmetic in 32 bits."""
    x = x.float()
    low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    third = torch.full((), 1 / 15, dtype=torch.float32, device=x.device)
    scale, zero = ((high - low) * third).bfloat16(), low.bfloat16()
    bad = ~torch.isfinite(low + high) & (~torch.isfinite(low) | ~torch.isfinite(high))
    scale, zero = torch.where(bad, math.nan, scale), torch.where(bad, math.nan, zero)
    s = scale.float()
    inv = torch.where(s >= 2.0**-126, torch.ones_like(s) / s, torch.zeros_like(s))
    codes = torch.round((x - zero.float()) * inv).clamp(0, 15)
    return torch.where(bad, 0.0, codes).to(torch.uint8), scale, zero


def pack(kc, ks, kz, vc, vs, vz):
    """Records [blocks, H, record] of codes [blocks, H, S, D] and parameters [blocks, H, S, 1]."""
    P, H, S, D = kc.shape
    G, B = S // 16, min(D // 32, 4)
    A = D // 32 // B
    k = kc.view(P, H, G, 16, D // 2, 2)
    k = (k[..., 0] | k[..., 1] << 4).view(P, H, G, 8 * D)
    v = vc.view(P, H, G, 2, 4, 2, 8, A, B, 2, 2).permute(0, 1, 2, 3, 7, 6, 4, 8, 5, 9, 10)
    v = (v[..., 0] | v[..., 1] << 4).reshape(P, H, G, 8 * D)
    par = torch.stack([torch.cat([ks, kz], -1).view(P, H, G, 16, 2), torch.cat([vs, vz], -1).view(P, H, G, 16, 2)], 3)
    return torch.cat([k, v, par.contiguous().view(torch.uint8).view(P, H, G, 128)], -1).view(P, H, -1)


def unpack(rec, D):
    """Float K and V [..., S, D] of records [..., record]."""
    lead, G = rec.shape[:-1], rec.shape[-1] // (16 * D + 128)
    B = min(D // 32, 4)
    A = D // 32 // B
    rec = rec.view(*lead, G, 16 * D + 128)
    par = rec[..., 16 * D:].contiguous().view(torch.bfloat16).view(*lead, G, 2, 16, 2).float()
    n = len(lead)

    def halves(x):
        return torch.stack([x & 15, x >> 4], -1)

    k = halves(rec[..., : 8 * D].reshape(*lead, G, 16, D // 2)).view(*lead, G, 16, D).float()
    v = halves(rec[..., 8 * D : 16 * D].reshape(*lead, G, 2, A, 8, 4, B, 2, 2))
    v = v.permute(*range(n + 1), n + 1, n + 4, n + 6, n + 3, n + 2, n + 5, n + 7, n + 8).reshape(*lead, G, 16, D).float()
    k = k * par[..., 0, :, 0:1] + par[..., 0, :, 1:2]
    v = v * par[..., 1, :, 0:1] + par[..., 1, :, 1:2]
    return k.reshape(*lead, G * 16, D), v.reshape(*lead, G * 16, D)


# --------------------------------------------------------------------------- inputs
def ints(x, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda", dtype)


def keys_values(g, rows, D):
    """Keys with channels of their own scale and offset, as they come out of a projection, and plain values."""
    H = rows[-1]
    k = torch.randn(*rows, D, device="cuda", generator=g)
    k *= 0.5 + torch.rand(H, D, device="cuda", generator=g)
    k += torch.randn(H, D, device="cuda", generator=g)
    return k, torch.randn(*rows, D, device="cuda", generator=g) * 0.7


def prepare_tables(c, seed):
    r = np.random.default_rng(seed)
    held, want = table_lengths(c)
    at = r.permutation(c["R"])
    held, want = held[at], want[at]
    S, R = c["S"], c["R"]
    hb, wb = blocks(held, S), blocks(want, S)
    grow, back = np.maximum(wb - hb, 0).sum(), np.maximum(hb - wb, 0).sum()
    n_free = max(0, int(math.ceil(grow * c["enough"])) - int(back)) + (5 if c["enough"] >= 1 else 0)
    pool = int(hb.sum()) + n_free + 3
    perm = r.permutation(pool)
    table = np.full((R, blocks(c["most"], S)), -1, np.int32)
    rep = np.repeat(np.arange(R), hb)
    table[rep, np.arange(hb.sum()) - np.repeat(np.cumsum(hb) - hb, hb)] = perm[: hb.sum()]
    free = np.full(pool, -1, np.int32)
    free[:n_free] = perm[hb.sum() : hb.sum() + n_free]
    T = int(np.maximum(want - held, 0).sum())
    st = dict(c=c, held=ints(held), want=ints(want), order=ints(r.permutation(R)), table=ints(table), free=ints(free), n_free=ints([n_free]))
    st.update(n_free_out=torch.zeros(1, dtype=torch.int32, device="cuda"), got=torch.zeros(R, dtype=torch.int32, device="cuda"),
              off=torch.zeros(R + 1, dtype=torch.int64, device="cuda"), slots=torch.zeros(T, dtype=torch.int64, device="cuda"),
              pos=torch.zeros(T, dtype=torch.int32, device="cuda"))
    return st


def prepare_append(c, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    T, H, D, S, dt = c["T"], c["H"], c["D"], c["S"], DTYPES[c["dtype"]]
    k, v = keys_values(g, (T, H), D)
    if c["fused"]:  # keys and values as they lie in the output of one projection, behind two query heads to each KV head
        qkv = torch.empty(T, 4 * H, D, device="cuda", dtype=dt)
        k, v = qkv[:, 2 * H : 3 * H].copy_(k), qkv[:, 3 * H :].copy_(v)
    else:
        k, v = k.to(dt), v.to(dt)
    n = blocks(T, S) + 3
    slots = torch.randperm(n * S, device="cuda", generator=g)[:T] if T <= 4096 else \
        (torch.randperm(n, device="cuda", generator=g)[:, None] * S + torch.arange(S, device="cuda")).view(-1)[:T].contiguous()
    slots = torch.where(torch.rand(T, device="cuda", generator=g) < c["skip"], -1, slots)
    return dict(c=c, k=k, v=v, slots=slots, cache=torch.zeros(n, H, record_bytes(c), dtype=torch.uint8, device="cuda"),
                k_out=torch.empty(T, H, D, dtype=dt, device="cuda"), v_out=torch.empty(T, H, D, dtype=dt, device="cuda"))


def prepare_attn(c, seed):
    r, g = np.random.default_rng(seed), torch.Generator("cuda").manual_seed(seed)
    n, n_q = attn_lengths(c)
    at = r.permutation(c["B"])
    n, n_q = n[at], n_q[at]
    S, H, D, dt = c["S"], c["H"], c["D"], DTYPES[c["dtype"]]
    nb = blocks(n, S)
    P = int(nb.sum()) + 1
    perm = r.permutation(P)[: P - 1]
    most = blocks(max(c["high"], c["n_q"]), S)
    table = np.full((c["B"], most), -1, np.int32)
    rep = np.repeat(np.arange(c["B"]), nb)
    within = np.arange(P - 1) - np.repeat(np.cumsum(nb) - nb, nb)
    table[rep, within] = perm
    used = np.zeros(P, np.int64)  # tokens of each block that hold one; the others hold whatever was there
    used[perm] = np.minimum(S, n[rep] - within * S)
    stale = torch.arange(S, device="cuda") >= ints(used, torch.int64)[:, None]
    cache = torch.empty(P, H, record_bytes(c), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 27) // (H * S * D))
    for a in range(0, P, step):
        k, v = keys_values(g, (min(step, P - a), S, H), D)
        kc, ks, kz = quantise(k.transpose(1, 2).contiguous())
        vc, vs, vz = quantise(v.transpose(1, 2).contiguous())
        old = stale[a : a + step][:, None, :, None]
        cache[a : a + step] = pack(kc, torch.where(old, math.nan, ks), kz, vc, torch.where(old, math.nan, vs), torch.where(old, math.inf, vz))
    T = int(n_q.sum())
    q = torch.randn(T, c["Hq"], D, device="cuda", generator=g).to(dt)
    off = np.concatenate([[0], np.cumsum(n_q)])
    return dict(c=c, q=q, off=ints(off, torch.int64), n=ints(n), table=ints(table), cache=cache, most_q=int(n_q.max()), most_n=int(n.max()),
                out=torch.empty_like(q), lse=torch.empty(T, c["Hq"], dtype=torch.float32, device="cuda"))


def prepare(case, seed):
    st = {"tables": prepare_tables, "append": prepare_append, "attn": prepare_attn}[case["op"]](case, seed)
    st["kept"] = {}  # what a program keeps between calls: the framework's workspace
    return st


# --------------------------------------------------------------------------- plain forms
def ramp(counts):
    """For counts [n]: the owner of each of the sum(counts) elements, and its place within it."""
    rep = torch.repeat_interleave(torch.arange(counts.numel(), device="cuda"), counts)
    return rep, torch.arange(rep.numel(), device="cuda") - (counts.cumsum(0) - counts)[rep]


def plain_tables(s):
    S, held, want = s["c"]["S"], s["held"].long(), s["want"].long()
    hb, wb = (held + S - 1) // S, (want + S - 1) // S
    grow, back = (wb - hb).clamp(min=0), (hb - wb).clamp(min=0)
    table, free, n_free = s["table"].clone(), s["free"].clone(), s["n_free"].long()
    rep, i = ramp(back)
    free[n_free + torch.arange(rep.numel(), device="cuda")] = table[rep, wb[rep] + i]
    N, order = n_free + back.sum(), s["order"].long()
    upto = grow[order].cumsum(0)
    granted, before = torch.empty_like(grow, dtype=torch.bool), torch.empty_like(grow)
    granted[order] = (grow[order] == 0) | (upto <= N)
    before[order] = upto - grow[order]
    take = torch.where(granted, grow, 0)
    rep, i = ramp(take)
    table[rep, hb[rep] + i] = free[N - 1 - before[rep] - i]
    add = (want - held).clamp(min=0)
    off = torch.cat([add.new_zeros(1), add.cumsum(0)])
    rep, i = ramp(add)
    pos = held[rep] + i
    slots = torch.where(granted[rep], table[rep, torch.where(granted[rep], pos // S, 0)].long() * S + pos % S, -1)
    return dict(table=table, free=free, n_free=(N - take.sum()).int(), got=torch.where((want < held) | granted, want, held).int(),
                off=off, slots=slots, pos=pos.int())


def plain_append(s):
    out = {}
    there = (s["slots"] >= 0)[:, None, None]
    kc, ks, kz = quantise(s["k"])
    vc, vs, vz = quantise(s["v"])
    out["k"] = torch.where(there, kc.float() * ks.float() + kz.float(), 0.0).to(s["k"].dtype)
    out["v"] = torch.where(there, vc.float() * vs.float() + vz.float(), 0.0).to(s["v"].dtype)
    return out


def plain_attn(s):
    c, q, n = s["c"], s["q"], s["n"].long()
    H, D, S = c["H"], c["D"], c["S"]
    n_q = s["off"].diff()
    group, Q, L = c["Hq"] // H, s["most_q"], blocks(s["most_n"], S) * S
    k, v = unpack(s["cache"][s["table"][:, : L // S].clamp(min=0).long()], D)  # [B, L/S, H, S, D]
    k, v = k.transpose(1, 2).reshape(-1, H, L, D), v.transpose(1, 2).reshape(-1, H, L, D)
    at = torch.arange(L, device="cuda")
    v = torch.where((at < n[:, None])[:, None, :, None], v, 0.0)
    i = torch.arange(Q, device="cuda")
    row = (s["off"][:-1, None] + i).clamp(max=q.shape[0] - 1)
    x = q[row].float().view(-1, Q, H, group, D).permute(0, 2, 3, 1, 4).reshape(-1, H, group * Q, D)
    w = (x @ k.transpose(2, 3)).view(-1, H, group, Q, L) / math.sqrt(D)
    pos = (n - n_q)[:, None, None] + i[:, None]  # [B, Q, 1]
    seen = (at < n[:, None, None]) & (pos >= 0)
    if c["causal"]:
        seen = seen & (at <= pos)
    if c["window"]:
        seen = seen & (at > pos - c["window"])
    w = torch.where(seen[:, None, None], w, -math.inf)
    m = w.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(w - m)
    total = p.sum(-1, keepdim=True)
    o = (p.view(-1, H, group * Q, L) @ v).view(-1, H, group, Q, D) / torch.where(total == 0, 1.0, total)
    lse = (m + total.log())[..., 0]
    rep, j = ramp(n_q)
    return dict(out=o.permute(0, 3, 1, 2, 4)[rep, j].reshape(-1, c["Hq"], D).to(q.dtype), lse=lse.permute(0, 3, 1, 2)[rep, j].reshape(-1, c["Hq"]))


# --------------------------------------------------------------------------- the framework's calls
def framework(s):
    if "M" not in s["kept"]:
        from paper_2609_15359_gb300 import maps as M

        s["kept"].update(M=M, ws=M.Workspace())
    return s["kept"]["M"], s["kept"]["ws"]


def done(status):
    if status:
        raise RuntimeError("status %d" % status)


def own_tables(s):
    M, ws = framework(s)
    done(M.maps_block_tables(s["c"]["S"], s["held"], s["want"], s["table"], s["free"], s["n_free"], s["n_free_out"], s["got"], s["off"],
                             s["slots"], s["pos"], order=s["order"], ws=ws))
    return dict(table=s["table"], free=s["free"], n_free=s["n_free_out"], got=s["got"], off=s["off"], slots=s["slots"], pos=s["pos"])


def own_append(s):
    M, ws = framework(s)
    done(M.maps_kv4_append(s["k"], s["v"], s["slots"], s["cache"], s["c"]["S"], ws=ws))
    done(M.maps_kv4_read(s["slots"], s["cache"], s["c"]["S"], s["k_out"], s["v_out"], ws=ws))
    return dict(k=s["k_out"], v=s["v_out"])


def own_attn(s):
    M, ws = framework(s)
    c = s["c"]
    done(M.maps_kv4_attention(s["q"], s["off"], s["n"], s["table"], s["cache"], c["S"], 1 / math.sqrt(c["D"]), s["out"], lse_out=s["lse"],
                              causal=c["causal"], window=c["window"], ws=ws))
    return dict(out=s["out"], lse=s["lse"])


def run(state):
    if own:
        return {"tables": own_tables, "append": own_append, "attn": own_attn}[state["c"]["op"]](state)
    return {"tables": plain_tables, "append": plain_append, "attn": plain_attn}[state["c"]["op"]](state)


# --------------------------------------------------------------------------- what a pass cannot do without
def spans(c):
    """(tokens read, pairs of query and key) summed over the requests."""
    n, n_q = attn_lengths(c)
    tokens = pairs = 0
    for a, b in zip(n.tolist(), n_q.tolist()):
        pos = np.arange(a - b, a)
        last = np.minimum(pos, a - 1) if c["causal"] else np.full(b, a - 1)
        first = np.maximum(pos - c["window"] + 1, 0) if c["window"] else np.zeros(b, np.int64)
        keys = np.where(pos >= 0, np.maximum(last - first + 1, 0), 0)
        pairs += int(keys.sum())
        live = keys > 0
        if live.any():
            tokens += int(last[live].max() - first[live].min() + 1)
    return tokens, pairs


def work(case):
    c = case
    if c["op"] == "tables":
        held, want = table_lengths(c)
        hb, wb = blocks(held, c["S"]), blocks(want, c["S"])
        T = int(np.maximum(want - held, 0).sum())
        # lengths and order in, lengths and offsets out, each moved block read and written, slots and positions out
        return {"bytes": 24 * c["R"] + 8 * int(np.abs(wb - hb).sum()) + 12 * T, "flops": 0}
    if c["op"] == "append":
        rows = c["T"] * c["H"]
        # keys and values in, codes and parameters out and in again, values out
        return {"bytes": rows * (4 * c["D"] + 2 * (c["D"] + 8) + 4 * c["D"]) + 16 * c["T"], "flops": 12 * rows * c["D"]}
    tokens, pairs = spans(c)
    _, n_q = attn_lengths(c)
    T = int(n_q.sum())
    return {"bytes": tokens * c["H"] * (c["D"] + 8) + 4 * blocks(tokens, c["S"]) + T * c["Hq"] * (4 * c["D"] + 4), "flops": 4 * pairs * c["Hq"] * c["D"]}


# --------------------------------------------------------------------------- the definitions in 64 bits
def exact_row(x):
    """What a row is held as: 16 evenly spaced levels between its extremes, the step and the lowest in bfloat16."""
    low, high = x.min(-1).values, x.max(-1).values
    step, zero = ((high - low) / 15).bfloat16().double()[..., None], low.bfloat16().double()[..., None]
    code = torch.round((x - zero) / torch.where(step > 0, step, 1.0)).clamp(0, 15)
    return zero + step * code


def exact_append(s):
    gone = (s["slots"] < 0).nonzero()[:, 0]
    k, v = exact_row(s["k"].double()), exact_row(s["v"].double())
    k[gone], v[gone] = 0, 0
    return dict(k=k, v=v)


def exact_tokens(s, b, n):
    """K and V [n, H, D] of request b in 64 bits, by the place of each code."""
    c = s["c"]
    H, D, S = c["H"], c["D"], c["S"]
    B = min(D // 32, 4)
    A = D // 32 // B
    j = torch.arange(n, device="cuda")
    rec = s["cache"][s["table"][b].long()[j // S]]  # [n, H, record]
    at = j % S // 16 * (16 * D + 128)
    tok = j % 16
    ch = torch.arange(D, device="cuda")

    def byte(index):  # [n, D] -> [n, H, D]
        return torch.gather(rec, 2, index[:, None].expand(n, H, index.shape[1])).long()

    kc = byte(at[:, None] + tok[:, None] * (D // 2) + ch // 2) >> (ch % 2 * 4) & 15
    gg, w, r = ch // (D // 8), ch % (D // 8) // 4, ch % 4
    h, t, parity = tok[:, None] // 8, tok[:, None] % 8 // 2, tok[:, None] % 2
    unit = ((((h * A + w // B) * 8 + gg) * 4 + t) * B + w % B) * 2 + parity
    vc = byte(at[:, None] + 8 * D + unit * 2 + r // 2) >> (r % 2 * 4) & 15

    def param(which):  # 0: K scale, 1: K zero, 2: V scale, 3: V zero; the 16 bits as the high half of a float
        p = (at + 16 * D + which // 2 * 64 + tok * 4 + which % 2 * 2)[:, None]
        bits = byte(p) << 16 | byte(p + 1) << 24
        return torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int().view(torch.float32).double()

    return kc * param(0) + param(1), vc * param(2) + param(3)


def exact_attn(s):
    c = s["c"]
    off, lens = s["off"].tolist(), s["n"].tolist()
    group = c["Hq"] // c["H"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        lo, hi = off[b], off[b + 1]
        if n == 0 or hi == lo:
            continue
        k, v = exact_tokens(s, b, n)
        key = torch.arange(n, device="cuda")
        pos = torch.arange(hi - lo, device="cuda")[:, None] + n - (hi - lo)
        hide = pos < 0
        if c["causal"]:
            hide = hide | (key > pos)
        if c["window"]:
            hide = hide | (key <= pos - c["window"])
        hide = hide.expand(hi - lo, n)
        for h in range(c["Hq"]):
            w = (s["q"][lo:hi, h].double() @ k[:, h // group].T) * c["D"] ** -0.5
            w = w.masked_fill(hide, -math.inf)
            lse[lo:hi, h] = torch.logsumexp(w, -1)
            out[lo:hi, h] = torch.nan_to_num(torch.softmax(w, -1), nan=0.0) @ v[:, h // group]
    return dict(out=out, lse=lse)


def exact(case, seed):
    if case["op"] == "tables":
        return None  # whole numbers
    s = prepare(case, seed)
    return exact_append(s) if case["op"] == "append" else exact_attn(s)
