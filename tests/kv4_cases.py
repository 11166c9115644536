"""Cases of attention over the 4-bit cache that tests hold to row-wise bounds (kv4_rows.py), with the
data that those bounds are shown to be sharp on.  Test infrastructure only."""
import numpy as np

import kv4_rows as R

LENS = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 1000, 0, 31]


def case(Hq, H, D, S, lens, n_q=None, causal=True, window=0):
    return dict(Hq=Hq, H=H, D=D, S=S, lens=list(lens), n_q=list(n_q or [1] * len(lens)), causal=causal, window=window)


def much(Hq):
    """A request whose work takes a call to the form for many queries."""
    return 6100, 2800 // Hq + 1


CASES = {
    # one token a request
    "decode 64": case(4, 4, 64, 16, LENS), "decode 128": case(8, 2, 128, 48, LENS), "decode 128 wide": case(24, 1, 128, 16, LENS),
    "decode 256": case(16, 1, 256, 32, LENS),
    # one KV head's keys with every multiprocessor
    "device 128": case(8, 1, 128, 64, [100003]), "device 128 sixteen": case(16, 1, 128, 64, [60001]),
    "device 256": case(16, 1, 256, 64, [30001]), "device 64": case(4, 1, 64, 64, [180007]),
    "long 128": case(8, 1, 128, 16, [20011]), "long 256": case(16, 2, 256, 64, [20011, 3], [4, 2], window=15000),
    # drafted tokens and small chunks
    "drafts": case(16, 4, 128, 32, [5, 64, 700, 1500, 2000], [5] * 5, window=1024),
    "several": case(6, 2, 64, 16, [0, 1, 2, 5, 20, 64, 90, 257, 700, 33, 400], [3, 1, 5, 5, 2, 8, 0, 5, 9, 33, 130]),
    "chunks 256": case(2, 1, 256, 16, [513, 700, 128, 0, 300], [100, 200, 128, 40, 1]),
    # many queries
    "chunks 128": case(8, 2, 128, 16, [513, 6100, 128, 700, 65, 0, 300], [300, much(8)[1], 128, 257, 65, 40, 1]),
    "chunks 64": case(8, 1, 64, 16, [513, 6100, 90], [200, much(8)[1], 33]),
    "chunks window": case(4, 2, 64, 64, [6100, 300, 1100], [much(4)[1], 130, 257], window=200),
    "chunks both ways": case(3, 1, 128, 48, [6100, 1], [much(3)[1], 99], causal=False),
}


def data(name, kind):
    """(rng, q, k, v) of a case: scores of two nats' spread, values of one or two in magnitude."""
    c = CASES[name]
    rng = np.random.default_rng(len(name) * 1000 + c["D"])
    k = [R.rounded(rng.normal(size=(n, c["H"], c["D"])).astype(np.float32), kind) for n in c["lens"]]
    v = [R.rounded((rng.normal(size=(n, c["H"], c["D"])) * 2.0 ** rng.uniform(-1, 1, (n, c["H"], 1))).astype(np.float32), kind)
         for n in c["lens"]]
    q = R.rounded((2 * rng.normal(size=(sum(c["n_q"]), c["Hq"], c["D"]))).astype(np.float32), kind)
    return rng, q, k, v


def expect(name, kind, q, k, v):
    c = CASES[name]
    off = np.concatenate([[0], np.cumsum(c["n_q"])])
    # few queries: equal runs for at least 152 x 8 warps, of units of up to 96 keys, two of which may be cut; many: a request at most
    units = sum(n * c["H"] * -(-m * c["Hq"] // (8 * c["H"])) for n, m in zip(c["lens"], c["n_q"]))
    run = max(c["lens"]) if max(c["n_q"]) > 96 else units / 1216 + 192
    return off, R.expect(kind, q, off, c["lens"], k, v, c["H"], c["D"] ** -0.5, c["causal"], c["window"], run=run)
