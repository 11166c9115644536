"""The block tables' and the 4-bit cache's oracle on worked examples, sizes that
the library answers on the host, and the refusals of each call: they come
before anything is enqueued, so no GPU is needed and none of the pointers is
read."""
import ctypes

import numpy as np
import pytest

import kv4_oracle as K


@pytest.fixture(scope="module")
def M():
    from paper_2609_15359_gb300 import build
    build.build()
    from paper_2609_15359_gb300 import maps
    return maps


def test_block_tables_worked_example():
    # blocks of 4; request 0 finishes (returns 7, 8), 1 takes a token in its block, 2 opens a
    # block, 3 wants three blocks and is last in the order: two are left for it, so it is refused
    table = np.array([[7, 8, -1], [5, -1, -1], [3, -1, -1], [-1, -1, -1]], np.int32)
    free = np.array([1, -1, -1, -1], np.int32)
    t, f, n, got, off, slots, pos = K.block_tables(4, [6, 2, 4, 0], [0, 3, 5, 9], table, free, 1,
                                                   order=[2, 0, 1, 3])
    assert t.tolist() == [[7, 8, -1], [5, -1, -1], [3, 8, -1], [-1, -1, -1]]
    assert f.tolist() == [1, 7, 8, -1] and n == 2
    assert got.tolist() == [0, 3, 5, 0] and off.tolist() == [0, 0, 1, 2, 11]
    assert slots.tolist() == [22, 32] + [-1] * 9
    assert pos.tolist() == [2, 4] + list(range(9))


def test_quantise_worked_examples():
    c, s, z = K.quantise(np.arange(16, dtype=np.float32) - 3)
    assert c.tolist() == list(range(16)) and s[0] == 1 and z[0] == -3
    c, s, z = K.quantise(np.full(64, 2.5, np.float32))
    assert not c.any() and s[0] == 0 and z[0] == 2.5
    for bad in (np.nan, np.inf, -np.inf):
        x = np.ones(64, np.float32)
        x[5] = bad
        assert np.isnan(K.held_as(x)).all()
    x = np.random.default_rng(0).normal(size=(50, 128)).astype(np.float32)
    step = K.quantise(x)[1]
    # half a step, and the rounding of the step (15 codes of it) and of the lowest level
    assert (np.abs(K.held_as(x) - x) <= step * (0.5 + 15 * 2.0**-8) + np.abs(x).max() * 2.0**-8).all()


@pytest.mark.parametrize("D", [64, 128, 256])
def test_v_units_are_a_permutation(D):
    """Every byte of a group is written by exactly the codes the layout gives it."""
    cache = np.zeros((1, 1, K.record_bytes(16, D)), np.uint8)
    row = (np.arange(D) % 16).astype(np.float32)
    row[0], row[1] = 0, 15
    for tau in range(16):
        K.put(cache, 16, D, tau, 0, np.full(D, 1, np.float32), row)
    count = np.bincount(np.concatenate([cache[0, 0, 8 * D:16 * D] & 15, cache[0, 0, 8 * D:16 * D] >> 4]),
                        minlength=16)
    assert (count == 16 * np.bincount(row.astype(int), minlength=16)).all()


def test_sizes(M):
    for S in (16, 32, 48, 64, 4096):
        for D in (64, 128, 256):
            assert M.lib.maps_kv4_record_bytes(S, D) == K.record_bytes(S, D)
    for S, D in ((0, 128), (8, 128), (24, 128), (8192, 128), (16, 32), (16, 96), (16, 512), (-16, 64)):
        assert M.lib.maps_kv4_record_bytes(S, D) == 0
    assert M.lib.maps_kv4_workspace_size() >= 256
    assert M.lib.maps_block_tables_workspace_size(0) >= 256
    assert M.lib.maps_block_tables_workspace_size(1000) >= 8000
    assert M.lib.maps_kv4_attention_workspace_size(8, 8, 8, 8, 128) >= 256


# any address will do: a refused call reads nothing
P = ctypes.c_void_p(1 << 20)
BIG = 1 << 34


def tables(M, **kw):
    a = dict(R=4, S=16, held=P, want=P, order=P, table=P, max_blocks=8, free=P, pool=9, n_free=P,
             n_free_out=P, got=P, off=P, slots=P, cap=5, pos=P, ws=P, ws_bytes=BIG, stream=None) | kw
    return M.lib.maps_block_tables(*a.values())


@pytest.mark.parametrize("bad", [dict(R=-1), dict(S=0), dict(max_blocks=-1), dict(pool=-1), dict(cap=-1),
                                 dict(held=None), dict(want=None), dict(table=None), dict(free=None),
                                 dict(n_free=None), dict(n_free_out=None), dict(got=None), dict(off=None),
                                 dict(slots=None), dict(ws=None), dict(ws=ctypes.c_void_p(8))])
def test_block_tables_refuses(M, bad):
    assert tables(M, **bad) == M.MAPS_E_INVALID


def test_block_tables_refuses_a_small_workspace(M):
    assert tables(M, ws_bytes=256) == M.MAPS_E_WORKSPACE


def append(M, **kw):
    a = dict(dtype=0, T=4, H=2, D=128, S=16, k=P, kr=256, kh=128, v=P, vr=256, vh=128, slots=P, cache=P,
             n_blocks=3, ws=P, ws_bytes=256, stream=None) | kw
    return M.lib.maps_kv4_append(*a.values())


def read(M, **kw):
    a = dict(dtype=0, T=4, H=2, D=128, S=16, slots=P, cache=P, n_blocks=3, k=P, kr=256, kh=128, v=P, vr=256,
             vh=128, ws=P, ws_bytes=256, stream=None) | kw
    return M.lib.maps_kv4_read(*a.values())


ROWS_BAD = [dict(dtype=2), dict(dtype=-1), dict(T=-1), dict(T=1 << 30), dict(H=0), dict(D=96), dict(S=8),
            dict(S=24), dict(k=None), dict(v=None), dict(slots=None), dict(cache=None), dict(n_blocks=-1),
            dict(cache=ctypes.c_void_p((1 << 20) + 8)), dict(k=ctypes.c_void_p((1 << 20) + 1)), dict(ws=None)]


@pytest.mark.parametrize("bad", ROWS_BAD)
@pytest.mark.parametrize("call", [append, read])
def test_cache_rows_refuse(M, call, bad):
    assert call(M, **bad) == M.MAPS_E_INVALID


@pytest.mark.parametrize("call", [append, read])
def test_cache_rows_small_workspace_and_no_tokens(M, call):
    assert call(M, ws_bytes=128) == M.MAPS_E_WORKSPACE
    assert call(M, T=0, k=None, v=None, slots=None) == M.MAPS_OK  # nothing to enqueue


def attention(M, **kw):
    a = dict(dtype=0, B=2, T=3, Hq=8, Hkv=2, D=128, S=16, q=P, qr=1024, qh=128, off=P, n=P, table=P,
             max_blocks=4, cache=P, n_blocks=9, scale=0.1, causal=1, window=0, out=P, outr=1024, outh=128,
             lse=None, ws=P, ws_bytes=BIG, stream=None) | kw
    return M.lib.maps_kv4_attention(*a.values())


@pytest.mark.parametrize("bad", [dict(dtype=7), dict(B=-1), dict(T=-1), dict(T=(1 << 30) + 1), dict(Hq=7),
                                 dict(Hq=0), dict(Hkv=0), dict(Hkv=-2), dict(D=100), dict(S=20),
                                 dict(max_blocks=-1), dict(n_blocks=-1), dict(window=-1),
                                 dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None),
                                 dict(off=None), dict(n=None), dict(table=None), dict(cache=None),
                                 dict(out=None), dict(ws=None), dict(causal=2),
                                 dict(cache=ctypes.c_void_p((1 << 20) + 8)),
                                 dict(q=ctypes.c_void_p((1 << 20) + 1)),
                                 dict(lse=ctypes.c_void_p((1 << 20) + 2))])
def test_attention_refuses(M, bad):
    assert attention(M, **bad) == M.MAPS_E_INVALID


def test_attention_small_workspace_and_nothing_to_do(M):
    assert attention(M, ws_bytes=128) == M.MAPS_E_WORKSPACE
    assert attention(M, T=0) == M.MAPS_OK
    assert attention(M, B=0) == M.MAPS_OK


def test_binding_refuses_other_types_and_shapes(M):
    import torch
    with pytest.raises(ValueError):
        M.kv4_cache_shape(4, 2, 16, 100)
    assert M.kv4_cache_shape(4, 2, 32, 64) == (4, 2, 2 * 1152)
    with pytest.raises(TypeError):  # host tensors
        M.maps_kv4_append(torch.zeros(1, 1, 64, dtype=torch.bfloat16), torch.zeros(1, 1, 64, dtype=torch.bfloat16),
                          torch.zeros(1, dtype=torch.int64), torch.zeros(1, 1, 1152, dtype=torch.uint8), 16,
                          ws=M.Workspace(device="cpu"))
    with pytest.raises(TypeError):
        M._dtype(torch.zeros(1))
