"""Measured cases of sparse decoding on the 4-bit KV cache: keys rotated to their positions as
they are appended, ranges of the keys of each cache block, the blocks that a cheap score selects
for each query, and attention over those blocks alone.

Each case is one call (for the append: one call and one read-back of what the cache holds; for
the ranges: one call and the values that its 8-bit codes stand for) on data made from a seed.
Where `own` is true, run() makes the framework's calls; where it is false, it computes the same
results with elementary torch operations in 32 bits.  exact() gives the results of the
definitions in 64 bits.

The 4-bit cache's layout, as the framework documents it: cache[block][kv head] is a record of
S/16 groups; a group holds 16 tokens as

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
        # one decode step of 512 requests: queries, keys and values of one token each, out of one projection
        dict(name="rotate_decode", op="rotate", T=512, Hq=32, H=8, D=128, S=16, dtype="bf16", axes=1, rot=128, inter=False, skip=0.0, fused=True, reach=131072),
        # images among text: three axes, a part of the channels, neighbouring pairs, odd counts, some tokens without a slot
        dict(name="rotate_odd", op="rotate", T=3001, Hq=15, H=5, D=64, S=32, dtype="fp16", axes=3, rot=32, inter=True, skip=0.1, fused=False, reach=32768),
        # a whole prefill batch of 65,536 tokens with three axes
        dict(name="rotate_prefill", op="rotate", T=65536, Hq=32, H=8, D=128, S=16, dtype="bf16", axes=3, rot=128, inter=False, skip=0.0, fused=True, reach=32768),
        # one decode step of 512 requests: the block that each new token went to
        dict(name="ranges_decode", op="ranges", B=512, low=64, high=8192, new=1, H=8, D=128, S=16, lens=1),
        # prompts that have just been filled in
        dict(name="ranges_prefill", op="ranges", B=48, low=1500, high=8192, new=0, H=8, D=128, S=16, lens=2),
        # a single request with a very long context: the latency of one token
        dict(name="select_one", op="select", B=1, low=100000, high=131072, n_q=1, Hq=32, H=8, D=128, S=16, dtype="bf16", n_list=128, first=1, last=2, holes=0.0, lens=3),
        # a decoder filled to half a million tokens, a few places idle
        dict(name="select_decode", op="select", B=128, low=64, high=8192, n_q=1, Hq=32, H=8, D=128, S=16, dtype="bf16", n_list=64, first=1, last=2, holes=0.05, lens=4),
        # drafted tokens behind long contexts, large blocks, five query heads to a KV head, half precision
        dict(name="select_drafts", op="select", B=7, low=3001, high=65536, n_q=5, Hq=20, H=4, D=64, S=64, dtype="fp16", n_list=33, first=0, last=1, holes=0.0, lens=5),
        # a single query over 2,048 selected tokens: the latency of one token
        dict(name="attend_one", op="attend", B=1, n_q=1, Hq=32, H=8, D=128, S=16, dtype="bf16", n_list=128, short=0.0, lens=6),
        # a decode step over 2,048 selected tokens each, an eighth of the requests shorter than that or idle
        dict(name="attend_decode", op="attend", B=128, n_q=1, Hq=32, H=8, D=128, S=16, dtype="bf16", n_list=128, short=0.125, lens=7),
        # drafted tokens that select much the same large blocks, five query heads to a KV head, half precision
        dict(name="attend_drafts", op="attend", B=48, n_q=5, Hq=20, H=4, D=64, S=64, dtype="fp16", n_list=33, short=0.1, lens=8),
        # one KV head of 256 channels for sixteen query heads
        dict(name="attend_mqa", op="attend", B=31, n_q=1, Hq=16, H=1, D=256, S=32, dtype="bf16", n_list=125, short=0.0, lens=9),
    ]


def draw(rng):
    def spread(a, b):
        return min(b, max(a, int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))))

    op = rng.choice(["rotate", "ranges", "select", "select", "attend", "attend"])
    H, D, S, dtype = rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128, 128, 256]), rng.choice([16, 16, 32, 64]), rng.choice(["bf16", "bf16", "fp16"])
    group, lens = rng.choice([1, 2, 3, 4, 5, 7, 8, 16]), rng.randrange(1 << 20)
    if op == "rotate":
        return dict(op=op, T=spread(1, 65536 * 48 * 128 // ((group + 2) * H * D)) if rng.random() < 0.7 else spread(1, 4096), Hq=group * H, H=H, D=D, S=S,
                    dtype=dtype, axes=rng.choice([1, 1, 2, 3, 4]), rot=rng.choice([D, D, D // 2, 32, D - 16]), inter=rng.random() < 0.4,
                    skip=rng.choice([0.0, 0.1]), fused=rng.random() < 0.5, reach=spread(1024, 131072))
    if op == "ranges":
        high = spread(1, 65536)
        c = dict(op=op, B=spread(1, 1024), low=max(1, high // rng.choice([1, 4, 50])), high=high, new=rng.choice([0, 1, 1, 5, spread(16, 1024)]), H=H, D=D, S=S, lens=lens)
        while c["B"] > 1 and c["B"] * min(c["high"], c["new"] + S if c["new"] else c["high"]) * H * D > 1 << 28:
            c["B"] = (c["B"] + 1) // 2
        return c
    n_q = rng.choice([1, 1, 1, rng.randint(2, 9), spread(16, 256)])
    if op == "select":
        high = spread(n_q + 1, 131072)
        c = dict(op=op, B=spread(1, 512), low=max(1, high // rng.choice([1, 4, 50])), high=high, n_q=n_q, Hq=group * H, H=H, D=D, S=S, dtype=dtype,
                 n_list=spread(4, 512), first=rng.choice([0, 1, 2]), last=rng.choice([1, 2]), holes=rng.choice([0.0, 0.1]), lens=lens)
        while c["B"] > 1 and c["B"] * n_q * blocks(high, S) * H * D > 1 << 26:
            c["B"] = (c["B"] + 1) // 2
        while c["n_q"] * blocks(high, S) * H * D > 1 << 26:
            c["n_q"] = (c["n_q"] + 1) // 2
        return c
    c = dict(op=op, B=spread(1, 512), n_q=n_q, Hq=group * H, H=H, D=D, S=S, dtype=dtype, n_list=spread(1, 512), short=rng.choice([0.0, 0.1, 0.5]), lens=lens)
    while c["B"] > 1 and c["B"] * n_q * c["n_list"] * S * H * D > 1 << 28:
        c["B"] = (c["B"] + 1) // 2
    while c["n_q"] * c["n_list"] * S * H * D > 1 << 28:
        c["n_q"], c["n_list"] = (c["n_q"] + 1) // 2, (c["n_list"] + 1) // 2
    return c


# --------------------------------------------------------------------------- lengths and lists, the same for every seed but for their order
def lengths(c):
    r = np.random.default_rng(c["lens"])
    n = np.maximum(r.integers(c["low"], c["high"] + 1, c["B"]), c.get("n_q", 1))
    hole = r.random(c["B"]) < c.get("holes", 0.0)
    hole[0] = False
    n[hole] = 0
    return n


def lists(c):
    """(blocks [T, H, n_list] numbered from 0, tokens [T, H]): the rows of a request choose among the same few blocks more than they take."""
    r = np.random.default_rng(c["lens"])
    B, m, H, L, S = c["B"], c["n_q"], c["H"], c["n_list"], c["S"]
    among = L if m == 1 else L + L // 4 + 1
    pick = r.random((B, m, H, among)).argsort(-1)[..., :L]
    pick.sort(-1)
    ids = (pick + (np.arange(B)[:, None, None, None] * H + np.arange(H)[:, None]) * among).reshape(B * m, H, L)
    tokens = (L - 1) * S + r.integers(1, S + 1, B)
    few = r.random(B) < c["short"]
    few[0] = False
    tokens[few] = r.integers(0, L * S, B)[few] * (r.random(B) < 0.7)[few]
    return ids, np.repeat(np.repeat(tokens, m)[:, None], H, 1)


def blocks(n, S):
    return -(-n // S)


def record_bytes(c):
    return c["S"] // 16 * (16 * c["D"] + 128)


# --------------------------------------------------------------------------- the 4-bit form and the ranges, in elementary operations
def const(x, like):
    return torch.full((), x, dtype=torch.float32, device=like.device)


def quantise(x):
    """Codes (uint8) and bfloat16 (scale, zero) of rows of the last axis; arithmetic in 32 bits."""
    x = x.float()
    low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    scale, zero = ((high - low) * const(1 / 15, x)).bfloat16(), low.bfloat16()
    bad = ~torch.isfinite(low) | ~torch.isfinite(high) | ~torch.isfinite(high - low)
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


def halves(x):
    return torch.stack([x & 15, x >> 4], -1)


def unpack_keys(rec, D):
    """Float K [..., S, D] of records [..., record]."""
    lead, G = rec.shape[:-1], rec.shape[-1] // (16 * D + 128)
    rec = rec.view(*lead, G, 16 * D + 128)
    par = rec[..., 16 * D : 16 * D + 64].contiguous().view(torch.bfloat16).view(*lead, G, 16, 2).float()
    k = halves(rec[..., : 8 * D].reshape(*lead, G, 16, D // 2)).view(*lead, G, 16, D).float()
    return (k * par[..., 0:1] + par[..., 1:2]).reshape(*lead, G * 16, D)


def unpack_values(rec, D):
    lead, G = rec.shape[:-1], rec.shape[-1] // (16 * D + 128)
    B = min(D // 32, 4)
    A = D // 32 // B
    n = len(lead)
    rec = rec.view(*lead, G, 16 * D + 128)
    par = rec[..., 16 * D + 64 :].contiguous().view(torch.bfloat16).view(*lead, G, 16, 2).float()
    v = halves(rec[..., 8 * D : 16 * D].reshape(*lead, G, 2, A, 8, 4, B, 2, 2))
    v = v.permute(*range(n + 1), n + 1, n + 4, n + 6, n + 3, n + 2, n + 5, n + 7, n + 8).reshape(*lead, G, 16, D).float()
    return (v * par[..., 0:1] + par[..., 1:2]).reshape(*lead, G * 16, D)


def eighths(low, high):
    """Codes (-127 .. 127, as float32) [..., 2, D] and scale [...] that hold the range of each channel, rounded outward: the scale is the
    least bfloat16 number 127 times which is no less than any end; 64 bits where an end may lie on a border."""
    most = torch.maximum(low.abs(), high.abs()).amax(-1, keepdim=True)
    bad = ~torch.isfinite(most)
    scale = torch.where(bad, 0.0, most / 127).bfloat16()
    scale = torch.where(scale.double() * 127 < most, (scale.view(torch.int16) + 1).view(torch.bfloat16), scale).double()
    scale = torch.where(scale >= 2.0**-126, scale, 0.0)
    unit = torch.where(scale > 0, scale, math.inf)
    codes = torch.stack([torch.floor(low / unit), torch.ceil(high / unit)], -2)
    return torch.where(bad[..., None], 0.0, codes).float(), torch.where(bad, math.nan, scale)[..., 0].float()


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


def fill_cache(g, c, used):
    """A cache of len(used) blocks whose first used[i] places hold a token; the others hold what is no number."""
    H, D, S, P = c["H"], c["D"], c["S"], len(used)
    stale = torch.arange(S, device="cuda") >= ints(used, torch.int64)[:, None]
    cache = torch.empty(P, H, record_bytes(c), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 27) // (H * S * D))
    for a in range(0, P, step):
        k, v = keys_values(g, (min(step, P - a), S, H), D)
        kc, ks, kz = quantise(k.transpose(1, 2).contiguous())
        vc, vs, vz = quantise(v.transpose(1, 2).contiguous())
        old = stale[a : a + step][:, None, :, None]
        cache[a : a + step] = pack(kc, torch.where(old, math.nan, ks), kz, vc, torch.where(old, math.nan, vs), torch.where(old, math.inf, vz))
    return cache


def prepare_rotate(c, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    T, Hq, H, D, S, dt, P, F = c["T"], c["Hq"], c["H"], c["D"], c["S"], DTYPES[c["dtype"]], c["reach"], c["rot"] // 2
    k, v = keys_values(g, (T, H), D)
    q = torch.randn(T, Hq, D, device="cuda", generator=g)
    if c["fused"]:  # as they lie in the output of one projection
        qkv = torch.empty(T, Hq + 2 * H, D, device="cuda", dtype=dt)
        q, k, v = qkv[:, :Hq].copy_(q), qkv[:, Hq : Hq + H].copy_(k), qkv[:, Hq + H :].copy_(v)
    else:
        q, k, v = q.to(dt), k.to(dt), v.to(dt)
    angle = torch.arange(P, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(F, device="cuda", dtype=torch.float64) / F)
    pos = torch.randint(0, P, (c["axes"], T), device="cuda", generator=g, dtype=torch.int32)
    axis = torch.arange(F, device="cuda", dtype=torch.int32) * c["axes"] // F if not c["inter"] else torch.arange(F, device="cuda", dtype=torch.int32) % c["axes"]
    n = blocks(T, S) + 3
    slots = torch.randperm(n * S, device="cuda", generator=g)[:T] if T <= 4096 else \
        (torch.randperm(n, device="cuda", generator=g)[:, None] * S + torch.arange(S, device="cuda")).view(-1)[:T].contiguous()
    slots = torch.where(torch.rand(T, device="cuda", generator=g) < c["skip"], -1, slots)
    return dict(c=c, q=q, k=k, v=v, pos=pos, axis=axis, cos_sin=torch.cat([angle.cos(), angle.sin()], 1).float(), slots=slots,
                cache=torch.zeros(n, H, record_bytes(c), dtype=torch.uint8, device="cuda"), q_out=torch.empty(T, Hq, D, dtype=dt, device="cuda"),
                k_out=torch.empty(T, H, D, dtype=dt, device="cuda"), v_out=torch.empty(T, H, D, dtype=dt, device="cuda"))


def prepare_ranges(c, seed):
    r, g = np.random.default_rng(seed), torch.Generator("cuda").manual_seed(seed)
    n = lengths(c)[r.permutation(c["B"])]
    held = np.maximum(n - c["new"], 0) if c["new"] else np.zeros_like(n)
    S = c["S"]
    first, nb = held // S, blocks(n, S)
    P = int((nb - first).sum()) + 3
    perm = r.permutation(P)[: P - 3]
    rep = np.repeat(np.arange(c["B"]), nb - first)
    at = np.arange(P - 3) - np.repeat(np.cumsum(nb - first) - (nb - first), nb - first) + first[rep]
    table = np.full((c["B"], blocks(c["high"], S)), -1, np.int32)  # the blocks before those are not looked at
    table[rep, at] = perm
    used = np.zeros(P, np.int64)
    used[perm] = np.minimum(S, n[rep] - at * S)
    return dict(c=c, cache=fill_cache(g, c, used), table=ints(table), held=ints(held), n=ints(n), most=int((nb - first).max()),
                codes=torch.zeros(P, c["H"], 2, c["D"], dtype=torch.int8, device="cuda"), scale=torch.zeros(P, c["H"], dtype=torch.float32, device="cuda"))


def prepare_select(c, seed):
    r, g = np.random.default_rng(seed), torch.Generator("cuda").manual_seed(seed)
    B, H, D, S, m = c["B"], c["H"], c["D"], c["S"], c["n_q"]
    n = lengths(c)[r.permutation(B)]
    nb = blocks(n, S)
    P = int(nb.sum()) + 1
    perm = r.permutation(P)[: P - 1]
    table = np.full((B, blocks(c["high"], S)), -1, np.int32)
    rep = np.repeat(np.arange(B), nb)
    table[rep, np.arange(P - 1) - np.repeat(np.cumsum(nb) - nb, nb)] = perm
    codes, scale = torch.empty(P, H, 2, D, dtype=torch.int8, device="cuda"), torch.empty(P, H, dtype=torch.float32, device="cuda")
    step = max(1, (1 << 27) // (H * S * D))
    for a in range(0, P, step):
        p = min(step, P - a)
        k, _ = keys_values(g, (p, S, H), D)
        k += 0.5 * torch.randn(p, 1, H, D, device="cuda", generator=g)  # neighbouring tokens are alike
        x, y = eighths(k.amin(1), k.amax(1))
        codes[a : a + p], scale[a : a + p] = x.to(torch.int8), y
    T = B * m
    q = torch.randn(T, c["Hq"], D, device="cuda", generator=g).to(DTYPES[c["dtype"]])
    return dict(c=c, q=q, off=ints(np.arange(B + 1) * m, torch.int64), n=ints(n), table=ints(table), codes=codes, scale=scale, most=int(nb.max()),
                blocks=torch.full((T, H, c["n_list"]), -1, dtype=torch.int32, device="cuda"), tokens=torch.zeros(T, H, dtype=torch.int32, device="cuda"))


def prepare_attend(c, seed):
    r, g = np.random.default_rng(seed), torch.Generator("cuda").manual_seed(seed)
    ids, tokens = lists(c)
    at = (r.permutation(c["B"])[:, None] * c["n_q"] + np.arange(c["n_q"])).reshape(-1)
    ids, tokens = ids[at], tokens[at]
    P = int(ids.max()) + 2
    ids = r.permutation(P).astype(np.int32)[ids]
    ids[np.arange(c["n_list"]) >= blocks(tokens, c["S"])[..., None]] = -1
    T, dt = ids.shape[0], DTYPES[c["dtype"]]
    q = torch.randn(T, c["Hq"], c["D"], device="cuda", generator=g).to(dt)
    return dict(c=c, q=q, blocks=ints(ids), tokens=ints(tokens), cache=fill_cache(g, c, np.full(P, c["S"])), out=torch.empty_like(q),
                lse=torch.empty(T, c["Hq"], dtype=torch.float32, device="cuda"))


def prepare(case, seed):
    st = {"rotate": prepare_rotate, "ranges": prepare_ranges, "select": prepare_select, "attend": prepare_attend}[case["op"]](case, seed)
    st["kept"] = {}  # what a program keeps between calls: the framework's workspace
    return st


# --------------------------------------------------------------------------- plain forms
def rotate(x, c, cos, sin):
    """x [T, heads, D] float32 with the first rot channels turned by the angles whose cosines and sines are [T, 1, rot/2]."""
    F = c["rot"] // 2
    if c["inter"]:
        a, b = x[..., 0 : 2 * F : 2], x[..., 1 : 2 * F : 2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :F], x[..., F : 2 * F]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., 2 * F :]], -1)


def plain_rotate(s):
    c, F, dt = s["c"], s["c"]["rot"] // 2, s["q"].dtype
    row = s["pos"][s["axis"].long()].T.long()  # [T, rot/2]
    f = torch.arange(F, device="cuda")
    cos, sin = s["cos_sin"][row, f][:, None], s["cos_sin"][row, F + f][:, None]
    there = (s["slots"] >= 0)[:, None, None]
    kc, ks, kz = quantise(rotate(s["k"].float(), c, cos, sin))
    vc, vs, vz = quantise(s["v"])
    return dict(q=rotate(s["q"].float(), c, cos, sin).to(dt), k=torch.where(there, kc.float() * ks.float() + kz.float(), 0.0).to(dt),
                v=torch.where(there, vc.float() * vs.float() + vz.float(), 0.0).to(dt))


def plain_ranges(s):
    c, n, S = s["c"], s["n"].long(), s["c"]["S"]
    j = s["held"].long()[:, None] // S + torch.arange(s["most"], device="cuda")  # [B, most]
    b, i = ((j < (n[:, None] + S - 1) // S)).nonzero(as_tuple=True)
    j = j[b, i]
    block = s["table"][b, j].long()
    k = unpack_keys(s["cache"][block], c["D"])  # [blocks, H, S, D]
    there = (torch.arange(S, device="cuda") < (n[b] - j * S)[:, None])[:, None, :, None]
    codes, scale = eighths(torch.where(there, k, math.inf).amin(2), torch.where(there, k, -math.inf).amax(2))
    codes_out, scale_out = s["codes"].float(), s["scale"].clone()
    codes_out[block], scale_out[block] = codes, scale
    return codes_out * scale_out[..., None, None]


def plain_select(s):
    c, n, T, m = s["c"], s["n"].long(), s["q"].shape[0], s["most"]
    H, D, S, L = c["H"], c["D"], c["S"], c["n_list"]
    i = torch.arange(T, device="cuda")
    b = torch.searchsorted(s["off"], i, right=True) - 1
    seen = (n[b] - s["off"][b + 1] + i + 1).clamp(min=0)  # keys that a row sees
    nb = (seen + S - 1) // S
    q = s["q"].double().view(T, H, -1, D)
    w = torch.stack([q.clamp(max=0).sum(2), q.clamp(min=0).sum(2)], 2).float()  # [T, H, 2, D], beside the lowest and the highest
    step = w.abs().amax((2, 3), keepdim=True) * const(1 / 127, w)
    inv = torch.where(step >= 2.0**-126, torch.ones_like(step) / step, torch.zeros_like(step))
    w = torch.round(w * inv).clamp(-127, 127)
    w = torch.where(torch.isfinite(step), w, math.nan)
    table = s["table"][:, :m].clamp(min=0).long()
    mine = s["codes"][table].float().permute(0, 2, 1, 3, 4).reshape(-1, H, m, 2 * D)  # [B, H, m, 2D]
    score = (mine[b] @ w.view(T, H, 2 * D, 1))[..., 0] * s["scale"][table].transpose(1, 2)[b]  # whole numbers below 2^24, exact in any order
    j = torch.arange(m, device="cuda")
    there, always = j < nb[:, None], (j < c["first"]) | (j >= nb[:, None] - c["last"])
    rank = torch.where(always & there, 2, torch.where(there, 1, 0))[:, None].expand(T, H, m)
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices
    order = order.gather(2, torch.sort(rank.gather(2, order), dim=-1, descending=True, stable=True).indices)
    count = torch.clamp(nb, max=L)
    take = torch.where(torch.arange(m, device="cuda") < count[:, None, None], order, m)[..., :L].sort(-1).values
    ids = torch.where(take < m, s["table"][:, :m][b][:, None].expand(T, H, m).gather(2, take.clamp(max=m - 1)), -1)
    out = s["blocks"].clone().fill_(-1)
    out[..., : ids.shape[2]] = ids
    tokens = torch.where(count > 0, (count - 1) * S + seen - (nb - 1) * S, 0)
    return dict(blocks=out, tokens=tokens[:, None].expand(T, H).int())


def plain_attend(s):
    c, q, n = s["c"], s["q"], s["tokens"][..., None, None]
    T, H, D = q.shape[0], c["H"], c["D"]
    rec = s["cache"][s["blocks"].clamp(min=0).long(), torch.arange(H, device="cuda")[:, None]]  # [T, H, n_list, record]
    at = torch.arange(c["n_list"] * c["S"], device="cuda")
    w = q.float().view(T, H, -1, D) @ unpack_keys(rec, D).view(T, H, -1, D).transpose(2, 3) / math.sqrt(D)
    w = torch.where(at < n, w, -math.inf)
    v = torch.where(at[:, None] < n, unpack_values(rec, D).view(T, H, -1, D), 0.0)
    m = w.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(w - m)
    total = p.sum(-1, keepdim=True)
    o = (p @ v) / torch.where(total == 0, 1.0, total)
    return dict(out=o.reshape(q.shape).to(q.dtype), lse=(m + total.log()).reshape(T, -1))


# --------------------------------------------------------------------------- the framework's calls
def framework(s):
    if "M" not in s["kept"]:
        from paper_2609_15359_gb300 import maps as M

        s["kept"].update(M=M, ws=M.Workspace())
    return s["kept"]["M"], s["kept"]["ws"]


def done(status):
    if status:
        raise RuntimeError("status %d" % status)


def own_rotate(s):
    M, ws = framework(s)
    c = s["c"]
    done(M.maps_kv4_append_rotated(s["q"], s["k"], s["v"], s["pos"], s["cos_sin"], s["slots"], s["cache"], c["S"], s["q_out"], axis=s["axis"],
                                   interleaved=c["inter"], ws=ws))
    done(M.maps_kv4_read(s["slots"], s["cache"], c["S"], s["k_out"], s["v_out"], ws=ws))
    return dict(q=s["q_out"], k=s["k_out"], v=s["v_out"])


def own_ranges(s):
    M, ws = framework(s)
    done(M.maps_kv4_block_ranges(s["held"], s["n"], s["table"], s["cache"], s["c"]["S"], s["codes"], s["scale"], ws=ws))
    return s["codes"] * s["scale"][..., None, None]


def own_select(s):
    M, ws = framework(s)
    c = s["c"]
    done(M.maps_kv4_select_blocks(s["q"], s["off"], s["n"], s["table"], s["codes"], s["scale"], c["S"], c["first"], c["last"], s["blocks"], s["tokens"], ws=ws))
    return dict(blocks=s["blocks"], tokens=s["tokens"])


def own_attend(s):
    M, ws = framework(s)
    c = s["c"]
    done(M.maps_kv4_attention_blocks(s["q"], s["blocks"], s["tokens"], s["cache"], c["S"], 1 / math.sqrt(c["D"]), s["out"], lse_out=s["lse"], ws=ws))
    return dict(out=s["out"], lse=s["lse"])


def run(state):
    if own:
        return {"rotate": own_rotate, "ranges": own_ranges, "select": own_select, "attend": own_attend}[state["c"]["op"]](state)
    return {"rotate": plain_rotate, "ranges": plain_ranges, "select": plain_select, "attend": plain_attend}[state["c"]["op"]](state)


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    H, D, S = c["H"], c["D"], c["S"]
    if c["op"] == "rotate":
        T, rows = c["T"], c["T"] * H
        # queries in and out, keys and values in, codes and parameters out and in again, values out; angles, positions and slots
        return {"bytes": 4 * T * c["Hq"] * D + rows * (4 * D + 2 * (D + 8) + 4 * D) + min(T * c["axes"], c["reach"]) * 4 * c["rot"] + T * (4 * c["axes"] + 16),
                "flops": 3 * T * (c["Hq"] + H) * c["rot"] + 12 * rows * D}
    if c["op"] == "ranges":
        n = lengths(c)
        held = np.maximum(n - c["new"], 0) if c["new"] else np.zeros_like(n)
        touched = int((blocks(n, S) - held // S).sum())
        # codes and parameters of the keys in, codes and scales out and in again, their values out
        return {"bytes": int((n - held // S * S).sum()) * H * (D // 2 + 4) + touched * (4 + H * (2 * (2 * D + 4) + 8 * D)), "flops": 4 * int((n - held // S * S).sum()) * H * D}
    if c["op"] == "select":
        nb = int(blocks(lengths(c), S).sum())
        T = c["B"] * c["n_q"]
        return {"bytes": nb * (4 + H * (2 * D + 4)) + T * (2 * c["Hq"] * D + 4 * H * (c["n_list"] + 1)), "flops": 4 * nb * c["n_q"] * H * D}
    ids, tokens = lists(c)
    T, j = ids.shape[0], np.arange(c["n_list"])
    there = np.clip(tokens[..., None] - j * S, 0, S)  # tokens of each entry that count
    most = np.zeros(int(ids.max()) + 1, np.int64)
    np.maximum.at(most, ids.reshape(-1), there.reshape(-1))
    return {"bytes": int(most.sum()) * (D + 8) + 4 * int((there > 0).sum()) + T * (c["Hq"] * (4 * D + 4) + 4 * H), "flops": 4 * int(tokens.sum()) * c["Hq"] // H * D}


# --------------------------------------------------------------------------- the definitions in 64 bits
def exact_row(x):
    """What a row is held as: 16 evenly spaced levels between its extremes, the step and the lowest in bfloat16."""
    low, high = x.min(-1).values, x.max(-1).values
    step, zero = ((high - low) / 15).bfloat16().double()[..., None], low.bfloat16().double()[..., None]
    code = torch.round((x - zero) / torch.where(step > 0, step, 1.0)).clamp(0, 15)
    return zero + step * code


def exact_rotate(s):
    """Each pair as a complex number, times that of its angle."""
    c, F = s["c"], s["c"]["rot"] // 2
    T = c["T"]
    turn = torch.empty(T, F, dtype=torch.complex128, device="cuda")
    for f, a in enumerate(s["axis"].tolist()):
        row = s["cos_sin"][s["pos"][a].long()].double()
        turn[:, f] = torch.complex(row[:, f], row[:, F + f])

    def turned(x):
        y = x.double()
        at = [slice(0, 2 * F, 2), slice(1, 2 * F, 2)] if c["inter"] else [slice(0, F), slice(F, 2 * F)]
        z = torch.complex(y[..., at[0]].contiguous(), y[..., at[1]].contiguous()) * turn[:, None]
        y = y.clone()
        y[..., at[0]], y[..., at[1]] = z.real, z.imag
        return y

    gone = (s["slots"] < 0).nonzero()[:, 0]
    k, v = exact_row(turned(s["k"])), exact_row(s["v"].double())
    k[gone], v[gone] = 0, 0
    return dict(q=turned(s["q"]), k=k, v=v)


def key_code(rec, at, tok, D):
    """K [n, H, D] of tokens `tok` of the groups that begin at byte `at` of the records rec [n, H, record], in 64 bits, by the place of each code."""
    n, H, _ = rec.shape
    ch = torch.arange(D, device="cuda")

    def byte(index):
        return torch.gather(rec, 2, index[:, None].expand(n, H, index.shape[1])).long()

    code = byte(at[:, None] + tok[:, None] * (D // 2) + ch // 2) >> (ch % 2 * 4) & 15
    return code * param(byte, at, tok, D, 0) + param(byte, at, tok, D, 1)


def value_code(rec, at, tok, D):
    n, H, _ = rec.shape
    B = min(D // 32, 4)
    A = D // 32 // B
    ch = torch.arange(D, device="cuda")

    def byte(index):
        return torch.gather(rec, 2, index[:, None].expand(n, H, index.shape[1])).long()

    g, w, r = ch // (D // 8), ch % (D // 8) // 4, ch % 4
    h, t, parity = tok[:, None] // 8, tok[:, None] % 8 // 2, tok[:, None] % 2
    unit = ((((h * A + w // B) * 8 + g) * 4 + t) * B + w % B) * 2 + parity
    code = byte(at[:, None] + 8 * D + unit * 2 + r // 2) >> (r % 2 * 4) & 15
    return code * param(byte, at, tok, D, 2) + param(byte, at, tok, D, 3)


def param(byte, at, tok, D, which):
    """0: K scale, 1: K zero, 2: V scale, 3: V zero; the 16 bits as the high half of a float."""
    p = (at + 16 * D + which // 2 * 64 + tok * 4 + which % 2 * 2)[:, None]
    bits = byte(p) << 16 | byte(p + 1) << 24
    return torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int().view(torch.float32).double()


def exact_ranges(s):
    c = s["c"]
    S, D, H = c["S"], c["D"], c["H"]
    out = torch.zeros(*s["codes"].shape, dtype=torch.float64, device="cuda")
    block, count = [], []
    for b, (a, n) in enumerate(zip(s["held"].tolist(), s["n"].tolist())):
        row = s["table"][b].tolist()
        for j in range(a // S, blocks(n, S)):
            block.append(row[j])
            count.append(min(S, n - j * S))
    block, count = ints(block, torch.int64), ints(count, torch.int64)
    for part in torch.arange(len(block), device="cuda").split(1024):
        rec, low, high = s["cache"][block[part]], None, None
        for t in range(S):
            here = t < count[part]
            k = key_code(rec, torch.full_like(part, t // 16 * (16 * D + 128)), torch.full_like(part, t % 16), D).float().double()  # what is held has 32 bits
            low = k if low is None else torch.where(here[:, None, None], torch.minimum(low, k), low)
            high = k if high is None else torch.where(here[:, None, None], torch.maximum(high, k), high)
        part_of, two = torch.frexp(torch.maximum(low.abs(), high.abs()).amax(-1, keepdim=True) / 127)
        step = torch.ceil(part_of * 256) * (two.long() - 8 + 1023 << 52).view(torch.float64)  # 8 significant bits, upwards; the power of two by its bits
        out[block[part]] = torch.stack([(low / step).floor(), (high / step).ceil()], 2) * step[..., None, :]
    return out


def exact_attend(s):
    c = s["c"]
    S, D, H = c["S"], c["D"], c["H"]
    group = c["Hq"] // H
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for i, row in enumerate(s["tokens"].tolist()):
        for h, n in enumerate(row):
            if n == 0:
                continue
            j = torch.arange(n, device="cuda")
            rec = s["cache"][s["blocks"][i, h].long()[j // S], h][:, None]
            at, tok = j % S // 16 * (16 * D + 128), j % 16
            k, v = key_code(rec, at, tok, D)[:, 0], value_code(rec, at, tok, D)[:, 0]
            x = slice(h * group, (h + 1) * group)
            w = s["q"][i, x].double() @ k.T * D**-0.5
            lse[i, x] = torch.logsumexp(w, -1)
            out[i, x] = torch.softmax(w, -1) @ v
    return dict(out=out, lse=lse)


def exact(case, seed):
    if case["op"] == "select":
        return None  # whole numbers
    if case["op"] == "attend" and case["B"] * case["n_q"] * case["H"] > 8192:
        return None  # a pair of row and head at a time
    s = prepare(case, seed)
    return {"rotate": exact_rotate, "ranges": exact_ranges, "attend": exact_attend}[case["op"]](s)
