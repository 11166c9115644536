"""Plain restatement of the block tables, the 4-bit KV cache and the attention
over it, request by request and token by token, from their definitions
(include/maps.h).  Attention is in 64 bits.  Test infrastructure only."""
import numpy as np


def block_tables(S, held, want, table, free, n_free, order=None):
    """(table, free, n_free_out, got, off, slots, pos), taking and returning block by block."""
    R = len(held)
    table, stack = table.copy(), list(free[:n_free])
    stack_copy = free.copy()
    for r in range(R):
        if want[r] < held[r]:
            for i in range(-(-int(want[r]) // S), -(-int(held[r]) // S)):
                stack_copy[len(stack)] = table[r, i]
                stack.append(table[r, i])
    got, asked, N = np.array(want, np.int32), 0, len(stack)
    granted = np.ones(R, bool)
    for r in (range(R) if order is None else order):
        if want[r] < held[r]:
            continue
        hb, wb = -(-int(held[r]) // S), -(-int(want[r]) // S)
        asked += wb - hb
        if wb > hb and asked > N:
            granted[r], got[r] = False, held[r]
            continue
        for i in range(hb, wb):
            table[r, i] = stack.pop()
    off, slots, pos = np.zeros(R + 1, np.int64), [], []
    for r in range(R):
        off[r + 1] = off[r] + max(0, int(want[r]) - int(held[r]))
        for p in range(int(held[r]), int(want[r])):
            pos.append(p)
            slots.append(int(table[r, p // S]) * S + p % S if granted[r] else -1)
    return (table, stack_copy, len(stack), got, off, np.array(slots, np.int64),
            np.array(pos, np.int32))


def bf16(x):
    """Nearest bfloat16 (ties to even) of finite float32 values, as float32."""
    b = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    b = (b + 0x7fff + ((b >> 16) & 1)) & 0xffff0000
    return b.astype(np.uint32).view(np.float32)


def quantise(x):
    """codes (uint8), scale, zero (float32) of rows of the last axis."""
    x = np.asarray(x, np.float32)
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        low, high = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
        spread = high - low
        bad = ~np.isfinite(x).all(-1, keepdims=True) | ~np.isfinite(spread)
        spread, low = np.where(bad, 0, spread), np.where(bad, 0, low)
        scale, zero = bf16(spread * np.float32(1 / 15)), bf16(low)
        inv = np.where(scale >= np.float32(2.0**-126), np.float32(1) / scale, np.float32(0))
        codes = np.clip(np.rint((x - zero) * inv), 0, 15)
    nan = np.float32(np.nan)
    return (np.where(bad, 0, codes).astype(np.uint8), np.where(bad, nan, scale).astype(np.float32),
            np.where(bad, nan, zero).astype(np.float32))


def held_as(x):
    """The float32 values that rows are held as."""
    c, s, z = quantise(x)
    return (s.astype(np.float64) * c + z).astype(np.float32)


def record_bytes(S, D):
    return S // 16 * (16 * D + 128)


def put(cache, S, D, slot, h, k, v):
    """Writes one token's rows k, v [D] of head h at a slot of cache [blocks, H, record] (uint8)."""
    rec, w = cache[slot // S, h], slot % S
    base, tau = w // 16 * (16 * D + 128), w % 16
    B = min(D // 32, 4)
    A = D // 32 // B
    for which, row in enumerate((k, v)):
        c, s, z = quantise(row)
        for d in range(D):
            if which == 0:
                byte, shift = base + tau * (D // 2) + d // 2, 4 * (d % 2)
            else:
                g, rest = divmod(d, D // 8)
                word, r = divmod(rest, 4)
                unit = ((((tau // 8 * A + word // B) * 8 + g) * 4 + tau % 8 // 2) * B + word % B) * 2 + tau % 2
                byte, shift = base + 8 * D + 2 * unit + r // 2, 4 * (r % 2)
            rec[byte] = (rec[byte] & (0xf0 >> shift)) | (int(c[d]) << shift)
        par = np.array([s[0], z[0]], np.float32).view(np.uint32) >> 16
        at = base + 16 * D + 64 * which + 4 * tau
        rec[at:at + 4] = par.astype("<u2").view(np.uint8)


def attention(q, off, lens, k, v, Hkv, scale, causal=True, window=0):
    """out [T, Hq, D], lse [T, Hq] in 64 bits.  k, v: per request [n, Hkv, D]."""
    T, Hq, D = q.shape
    out, lse = np.zeros((T, Hq, D)), np.full((T, Hq), -np.inf)
    group = Hq // Hkv
    for b in range(len(lens)):
        lo, hi, n = int(off[b]), int(off[b + 1]), int(lens[b])
        if n == 0 or hi == lo:
            continue
        j = np.arange(n)
        p = n - (hi - lo) + np.arange(hi - lo)[:, None]
        seen = np.broadcast_to(p >= 0, (hi - lo, n)).copy()
        if causal:
            seen &= j <= p
        if window:
            seen &= j > p - window
        for x in range(Hq):
            kk, vv = k[b][:, x // group].astype(np.float64), v[b][:, x // group].astype(np.float64)
            w = q[lo:hi, x].astype(np.float64) @ kk.T * scale
            w[~seen] = -np.inf
            live = seen.any(1)
            m = w[live].max(1, keepdims=True)
            e = np.exp(w[live] - m)
            total = e.sum(1, keepdims=True)
            out[lo:hi, x][live] = e @ vv / total
            lse[lo:hi, x][live] = (m + np.log(total))[:, 0]
    return out, lse
