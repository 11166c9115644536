"""Plain restatement of rotary positions on the way into the 4-bit cache, of the blocks' ranges
and of the blocks that a score selects, row by row from their definitions (include/maps.h).
Everything here is exact: 32-bit steps where the definition rounds, whole numbers, 64 bits
elsewhere.  Test infrastructure only."""
import numpy as np

import kv4_oracle as K


def rotate(x, pos, axis, rot, interleaved, cos_sin):
    """x [T, heads, D] float32 turned by the tokens' positions pos [axes, T]: every product and sum in 32 bits."""
    y, F = x.astype(np.float32).copy(), rot // 2
    for f in range(F):
        p = pos[0 if axis is None else axis[f]]
        c, s = (cos_sin[p, at].astype(np.float32)[:, None] for at in (f, F + f))
        a, b = (2 * f, 2 * f + 1) if interleaved else (f, f + F)
        with np.errstate(all="ignore"):
            y[..., a] = x[..., a] * c - x[..., b] * s
            y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def range_of(keys):
    """(codes [2, D] int, scale) of the keys [n, D] of a block and head, float32 as they are held."""
    D = keys.shape[1]
    if not np.isfinite(keys).all():
        return np.zeros((2, D), int), np.float32(np.nan)
    low, high = keys.min(0).astype(np.float64), keys.max(0).astype(np.float64)
    most = max(np.abs(low).max(), np.abs(high).max()) / 127
    if most == 0:
        return np.zeros((2, D), int), np.float32(0)
    grid = 2.0 ** max(np.frexp(most)[1] - 8, -133)  # of bfloat16 numbers of that size
    scale = np.ceil(most / grid) * grid
    if scale * 127 < most * 127:  # most / 127 was rounded down to a number of the grid
        scale += grid
    if scale < 2.0**-126:
        return np.zeros((2, D), int), np.float32(0)
    return np.stack([np.floor(low / scale), np.ceil(high / scale)]).astype(int), np.float32(scale)


def weights(q):
    """(N, P) as whole numbers of the query heads q [group, D] of one KV head, or None where they are no numbers."""
    q = q.astype(np.float64)
    with np.errstate(all="ignore"):
        w = np.stack([np.minimum(q, 0).sum(0), np.maximum(q, 0).sum(0)]).astype(np.float32)
        step = np.abs(w).max() * np.float32(1 / 127)
        if not np.isfinite(step):
            return None
        inv = np.float32(1) / step if step >= np.float32(2.0**-126) else np.float32(0)
        return np.clip(np.rint(w * inv), -127, 127).astype(int)


def scores(w, codes, scale):
    """float32 scores of blocks: codes [n, 2, D], scale [n]."""
    if w is None:
        return np.full(len(scale), np.nan, np.float32)
    with np.errstate(all="ignore"):
        return (codes.astype(int) * w).sum((1, 2)).astype(np.float32) * scale.astype(np.float32)


def select(q, off, lens, table, codes, scale, S, first, last, n_list, blocks, tokens):
    """blocks and tokens updated for the rows that requests have."""
    T, Hq, D = q.shape
    H = codes.shape[1]
    blocks, tokens = blocks.copy(), tokens.copy()
    for b in range(len(lens)):
        for i in range(int(off[b]), int(off[b + 1])):
            seen = int(lens[b]) - (int(off[b + 1]) - i) + 1 if lens[b] else 0
            blocks[i], tokens[i] = -1, 0
            if seen <= 0:
                continue
            nb = -(-seen // S)
            for h in range(H):
                take = np.arange(nb)
                if nb > n_list:
                    w = weights(q[i, h * (Hq // H):(h + 1) * (Hq // H)])
                    x = scores(w, codes[table[b, :nb], h], scale[table[b, :nb], h])
                    j = np.arange(nb)
                    always = (j < first) | (j >= nb - last)
                    order = np.lexsort((j, -np.where(np.isnan(x), 0, x), ~np.isnan(x), ~always))
                    take = np.sort(order[:n_list])
                blocks[i, h, :len(take)] = table[b, take]
                tokens[i, h] = (len(take) - 1) * S + seen - (nb - 1) * S
    return blocks, tokens


def held_keys(k):
    return K.held_as(k)
