"""Attention over the 4-bit cache held to bounds of its own for every row.

With s c + z a held value (c its code, s and z in bfloat16), p a row's softmax weights
and A = sum_j p_j (s_j c_j + |z_j|), the magnitude of what is summed, the calls may round

  - the output once, to the 16-bit type (u, half a step: 2^-8 bfloat16, 2^-11 half);
  - a weight and a value once each to 11 bits: 2^-11 of each term, twice;
  - a score in 32 bits: sums of D/16 products of 16 channels and a few operations
    more, each 2^-23 of the magnitude summed; it enters the weights as it is;
  - sums over keys in 32 bits: 2^-23 of A for each product of 16 keys;
  - weights too small for 11 bits, by 2^-32 of the largest term each.

An element is held to the worst case of these.  A row's error as a vector is held to
the same but for the roundings to 11 bits, which are independent of one another:
4 times 2^-11 of the root of the summed squares of the terms, which is all that
they can be where one key counts, and five deviations where many do.
Test infrastructure only."""
import numpy as np

import kv4_oracle as K

U = {"bf16": 2.0**-8, "fp16": 2.0**-11}


def held(x, centre=0):
    """(values, magnitudes, rows held as NaN) of rows in 64 bits; what is held as NaN counts as 0.
    centre: what the codes are taken about; the few-query form takes half outputs' values about 8, so that
    s |c - 8| + |z + 8 s| is what is summed there."""
    c, s, z = K.quantise(x)
    bad = np.isnan(s[..., 0])
    s, z = (np.where(bad[..., None], 0, y).astype(np.float64) for y in (s, z))
    return s * c + z, s * np.abs(c - float(centre)) + np.abs(z + centre * s), bad


def expect(name, q, off, lens, k, v, Hkv, scale, causal=True, window=0, centre=0, run=None):
    """out, lse and what they may be off by, in 64 bits.  q [T, Hq, D]; k, v: per request [n, Hkv, D] as given to the cache.
    run: the most keys that are summed one after another where that is known, and not more than 164 parts of
    such sums are joined; with it a row's error as a vector takes the scores' roundings as independent too."""
    T, Hq, D = q.shape
    e = dict(out=np.zeros((T, Hq, D)), lse=np.full((T, Hq), -np.inf), tol=np.zeros((T, Hq, D)),
             norm=np.zeros((T, Hq)), lse_tol=np.zeros((T, Hq)), has=np.zeros(T, bool))
    group, u = Hq // Hkv, U[name]
    for b in range(len(lens)):
        lo, hi, n = int(off[b]), int(off[b + 1]), int(lens[b])
        e["has"][lo:hi] = True
        if n == 0 or hi == lo:
            continue
        j = np.arange(n)
        at = n - (hi - lo) + np.arange(hi - lo)[:, None]
        seen = np.broadcast_to(at >= 0, (hi - lo, n)).copy()
        if causal:
            seen &= j <= at
        if window:
            seen &= j > at - window
        live = seen.any(1)
        seen = seen[live]
        keys = seen.sum(1)
        rows = np.arange(lo, hi)[live]
        if len(rows) == 0:
            continue
        for h in range(Hkv):
            kv, ka, kbad = held(k[b][:, h])
            vv, va, vbad = held(v[b][:, h], centre)
            for x in range(h * group, (h + 1) * group):
                qx = q[rows, x].astype(np.float64)
                w = np.where(seen, qx @ kv.T * scale, -np.inf)
                size = np.where(seen, np.abs(qx) @ ka.T * abs(scale), 0).max(1)
                score = (D / 16 + 8) * 2.0**-23 * size
                m = w.max(1, keepdims=True)
                p = np.exp(w - m)
                total = p.sum(1, keepdims=True)
                p /= total
                out, A = p @ vv, p @ va
                spread = np.sqrt((p * p) @ (va * va))
                most = (p * va.max(1)).max(1)
                sums = (keys / 16 + 64 if run is None else np.minimum(keys, run) / 16 + 64 + 164) * 2.0**-23
                rest = ((2 * score + sums)[:, None] * A + (keys * 2.0**-32 * most)[:, None])
                e["out"][rows, x] = np.where((seen & (kbad | vbad)).any(1)[:, None], np.nan, out)
                e["tol"][rows, x] = u * np.abs(out) + 2.0**-10 * (1 + 2.0**-9) * A + rest
                eleven = 4 * 2.0**-11
                if run is not None:
                    eleven, rest = eleven + 8 * score, sums[:, None] * A + (keys * 2.0**-32 * most)[:, None]
                e["norm"][rows, x] = (u * np.linalg.norm(out, axis=1) + eleven * np.linalg.norm(spread, axis=1) +
                                      np.linalg.norm(rest, axis=1))
                lse = (m + np.log(total))[:, 0]
                e["lse"][rows, x] = np.where((seen & kbad).any(1), np.nan, lse)
                e["lse_tol"][rows, x] = 2 * score + (keys / 128 + 64) * 2.0**-23 + 2.0**-21 * (2 + np.abs(lse))
    return e


def wrong(e, out, lse=None):
    """What is wrong with the rows that requests have, or None."""
    has = e["has"]
    ref, out = e["out"][has], np.asarray(out, np.float64)[has]
    nan = np.isnan(ref)
    if not np.array_equal(nan, np.isnan(out)):
        return f"{np.isnan(out).sum()} values are NaN, {nan.sum()} are to be"
    err = np.where(nan, 0, np.abs(out - np.where(nan, out, ref)))
    over = (err > e["tol"][has]).sum()
    norm = np.sqrt((err * err).sum(-1))
    rows = (norm > e["norm"][has]).sum()
    if over or rows:
        at = np.unravel_index(np.argmax(norm - e["norm"][has]), norm.shape)
        return f"{over} values and {rows} rows are off; row {at} by {norm[at]}, {e['norm'][has][at]} allowed"
    if lse is not None:
        r, l = e["lse"][has], np.asarray(lse, np.float64)[has]
        if not (np.array_equal(np.isnan(r), np.isnan(l)) and np.array_equal(np.isneginf(r), np.isneginf(l))):
            return f"lse: {np.isnan(l).sum()} NaN and {np.isneginf(l).sum()} empty, {np.isnan(r).sum()} and {np.isneginf(r).sum()} are to be"
        ok = np.isfinite(r)
        off = np.abs(l[ok] - r[ok]) - e["lse_tol"][has][ok]
        if (off > 0).any():
            return f"lse: {(off > 0).sum()} are off, one by {off.max()} more than allowed"
    return None


def rounded(x, name):
    """x as the 16-bit type, as float32."""
    return K.bf16(x) if name == "bf16" else np.asarray(x, np.float32).astype(np.float16).astype(np.float32)


def run(M, rng, name, q, lens, n_q, k, v, scale, S=16, causal=True, window=0, with_lse=True, ws=None,
        status=0):
    """Writes k, v to the slots of a cache whose other places are NaN, and attends: (out, lse) as float64."""
    import torch
    dt = dict(bf16=torch.bfloat16, fp16=torch.float16)[name]
    dev = lambda x, t=None: torch.from_numpy(np.ascontiguousarray(x)).cuda().to(t) if t else torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    H, D = k[0].shape[1:]
    nb = [-(-int(n) // S) for n in lens]
    perm = rng.permutation(sum(nb) + 2)
    table = np.full((len(lens), max(nb) + 1), -1, np.int32)
    slots, at = [], 0
    for b, n in enumerate(lens):
        table[b, :nb[b]] = perm[at:at + nb[b]]
        at += nb[b]
        j = np.arange(int(n))
        slots.append(table[b, j // S].astype(np.int64) * S + j % S)
    cache = torch.full(M.kv4_cache_shape(len(perm), H, S, D), 0xff, dtype=torch.uint8, device="cuda")
    ws = ws or M.Workspace()
    assert M.maps_kv4_append(dev(np.concatenate(k), dt), dev(np.concatenate(v), dt), dev(np.concatenate(slots)), cache, S, ws=ws) == 0
    off = np.concatenate([[0], np.cumsum(n_q)]).astype(np.int64)
    qd = dev(q, dt)
    out = torch.full_like(qd, 77.0)
    lse = torch.full(q.shape[:2], 77.0, dtype=torch.float32, device="cuda") if with_lse else None
    assert M.maps_kv4_attention(qd, dev(off), dev(np.asarray(lens, np.int32)), dev(table), cache, S, scale, out, lse_out=lse,
                                causal=causal, window=window, ws=ws) == 0
    assert M.maps_check(ws) == status
    return out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64) if with_lse else None
