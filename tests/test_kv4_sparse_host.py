"""Refusals of the sparse-decoding calls, before anything is enqueued: no GPU is needed and no pointer
is read.  Worked examples of their oracle."""
import ctypes

import numpy as np
import pytest
import torch

import kv4_oracle as K
import kv4_sparse_oracle as O

P = 1 << 20  # an aligned address that nobody reads
BIG = 1 << 40


@pytest.fixture(scope="module")
def M():
    from paper_2609_15359_gb300 import build
    build.build()
    from paper_2609_15359_gb300 import maps
    return maps


def rotated(M, **kw):
    a = dict(dtype=0, T=5, Hq=8, H=2, D=128, S=16, q=P, qr=1024, qh=128, k=P, kr=256, kh=128, v=P, vr=256, vh=128, axes=3, pos=P, axis=P, rot=128,
             inter=0, cos_sin=P, n_pos=9, slots=P, cache=P, n_blocks=4, q_out=P, or_=1024, oh=128, ws=P, ws_bytes=BIG, stream=None) | kw
    return M.lib.maps_kv4_append_rotated(*a.values())


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(T=-1), dict(H=0), dict(H=65536), dict(Hq=-1), dict(Hq=65536), dict(D=96), dict(S=24), dict(S=8192), dict(T=1 << 30), dict(n_blocks=-1),
    dict(axes=0), dict(axes=9), dict(rot=-16), dict(rot=144), dict(rot=8), dict(rot=100), dict(inter=2), dict(n_pos=-1), dict(q=None), dict(q_out=None),
    dict(k=None), dict(v=None), dict(slots=None), dict(cache=None), dict(cache=P + 8), dict(pos=None), dict(pos=P + 2), dict(axis=P + 2), dict(cos_sin=None),
    dict(cos_sin=P + 8), dict(q=P + 1), dict(q_out=P + 1), dict(k=P + 1), dict(v=P + 1), dict(ws=None), dict(ws=P + 16)], ids=str)
def test_append_rotated_refuses(M, bad):
    assert rotated(M, **bad) == M.MAPS_E_INVALID


def ranges(M, **kw):
    a = dict(B=3, H=2, D=128, S=16, held=P, kv_len=P, table=P, max_blocks=7, cache=P, n_blocks=9, codes=P, scale=P, ws=P, ws_bytes=BIG, stream=None) | kw
    return M.lib.maps_kv4_block_ranges(*a.values())


@pytest.mark.parametrize("bad", [
    dict(B=-1), dict(B=(1 << 30) + 1), dict(H=0), dict(H=65536), dict(D=32), dict(S=0), dict(S=100), dict(max_blocks=-1), dict(max_blocks=1 << 31),
    dict(n_blocks=-1), dict(kv_len=None), dict(table=None), dict(cache=None), dict(codes=None), dict(scale=None), dict(cache=P + 4), dict(codes=P + 8),
    dict(scale=P + 2), dict(held=P + 1), dict(kv_len=P + 2), dict(table=P + 2), dict(ws=None)], ids=str)
def test_block_ranges_refuse(M, bad):
    assert ranges(M, **bad) == M.MAPS_E_INVALID


def select(M, **kw):
    a = dict(dtype=1, B=3, T=4, Hq=8, H=2, D=128, S=16, q=P, qr=1024, qh=128, off=P, kv_len=P, table=P, max_blocks=70, codes=P, scale=P, n_blocks=9,
             first=1, last=2, n_list=8, blocks=P, tokens=P, ws=P, ws_bytes=BIG, stream=None) | kw
    return M.lib.maps_kv4_select_blocks(*a.values())


@pytest.mark.parametrize("bad", [
    dict(dtype=-1), dict(B=-1), dict(T=-1), dict(T=(1 << 30) + 1), dict(T=1 << 30, H=4), dict(H=0), dict(Hq=1), dict(Hq=9), dict(Hq=65536), dict(D=80),
    dict(S=17), dict(max_blocks=-1), dict(max_blocks=1 << 31), dict(n_blocks=-1), dict(first=-1), dict(last=0), dict(n_list=0), dict(n_list=2), dict(first=7),
    dict(first=0x7fffffff), dict(last=0x7fffffff), dict(n_list=(1 << 20) + 1), dict(n_list=1 << 20, S=4096), dict(q=None), dict(off=None), dict(kv_len=None),
    dict(table=None), dict(codes=None), dict(scale=None), dict(blocks=None), dict(tokens=None), dict(q=P + 1), dict(codes=P + 8), dict(off=P + 4),
    dict(blocks=P + 2), dict(ws=None)], ids=str)
def test_select_blocks_refuses(M, bad):
    assert select(M, **bad) == M.MAPS_E_INVALID


def attend(M, **kw):
    a = dict(dtype=0, T=4, Hq=8, H=2, D=128, S=16, q=P, qr=1024, qh=128, blocks=P, tokens=P, n_list=8, cache=P, n_blocks=9, scale=0.1, out=P, or_=1024, oh=128,
             lse=P, ws=P, ws_bytes=BIG, stream=None) | kw
    return M.lib.maps_kv4_attention_blocks(*a.values())


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(T=-1), dict(T=(1 << 30) + 1), dict(T=1 << 29), dict(H=0), dict(Hq=1), dict(Hq=7), dict(Hq=65536), dict(D=192), dict(S=15), dict(n_list=0),
    dict(n_list=(1 << 20) + 1), dict(n_list=1 << 20, S=2048), dict(n_blocks=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(out=None),
    dict(blocks=None), dict(tokens=None), dict(cache=None), dict(cache=P + 8), dict(q=P + 1), dict(out=P + 1), dict(lse=P + 2), dict(blocks=P + 1),
    dict(tokens=P + 2), dict(ws=None), dict(ws=P + 128)], ids=str)
def test_attention_blocks_refuses(M, bad):
    assert attend(M, **bad) == M.MAPS_E_INVALID


def test_small_workspaces_and_nothing_to_do(M):
    for call in (rotated, ranges, select, attend):
        assert call(M, ws_bytes=255) == M.MAPS_E_WORKSPACE
    need = M.lib.maps_kv4_select_blocks_workspace_size(4, 2, 1 << 20)
    assert need >= 4 * 2 * (1 << 20) * 4 and select(M, max_blocks=1 << 20, ws_bytes=need - 1) == M.MAPS_E_WORKSPACE
    assert M.lib.maps_kv4_select_blocks_workspace_size(512, 8, 8192) == 256
    assert rotated(M, T=0) == 0 and ranges(M, B=0) == 0 and select(M, T=0) == 0 and select(M, B=0) == 0 and attend(M, T=0) == 0


def test_binding_refuses_other_types_and_shapes(M):
    """Sizes come first, then tensors that are not on the GPU."""
    z, i = torch.zeros, lambda *s: torch.zeros(*s, dtype=torch.int32)
    ws = M.Workspace(device="cpu")
    h = lambda *s: z(*s, dtype=torch.bfloat16)  # noqa: E731
    cache = z(M.kv4_cache_shape(9, 2, 16, 128), dtype=torch.uint8)
    assert M.kv4_range_shape(9, 2, 128) == (9, 2, 2, 128)
    good = dict(q=h(5, 8, 128), k=h(5, 2, 128), v=h(5, 2, 128), pos=i(3, 5), cos_sin=z(7, 64), slots=z(5, dtype=torch.int64), cache=cache, S=16,
                q_out=h(5, 8, 128), axis=i(32))
    with pytest.raises(TypeError):
        M.maps_kv4_append_rotated(**good, ws=ws)
    for bad in (dict(v=h(5, 2, 64)), dict(slots=z(4)), dict(q=None), dict(q_out=None), dict(q_out=h(5, 4, 128)), dict(q=h(4, 8, 128), q_out=h(4, 8, 128)),
                dict(q=h(5, 8, 64), q_out=h(5, 8, 64)), dict(pos=i(3, 4)), dict(pos=i(4)), dict(axis=i(31)), dict(cos_sin=z(7))):
        with pytest.raises(ValueError):
            M.maps_kv4_append_rotated(**good | bad, ws=ws)
    good = dict(held=i(3), kv_len=i(3), table=i(3, 4), cache=cache, S=16, codes=z(9, 2, 2, 128, dtype=torch.int8), scale=z(9, 2))
    with pytest.raises(TypeError):
        M.maps_kv4_block_ranges(**good, ws=ws)
    for bad in (dict(held=i(2)), dict(table=i(2, 4)), dict(table=i(12))):
        with pytest.raises(ValueError):
            M.maps_kv4_block_ranges(**good | bad, ws=ws)
    good = dict(q=h(5, 8, 128), qo_off=z(4, dtype=torch.int64), kv_len=i(3), table=i(3, 4), codes=z(9, 2, 2, 128, dtype=torch.int8), scale=z(9, 2), S=16, first=1,
                last=1, blocks_out=i(5, 2, 4), tokens_out=i(5, 2))
    with pytest.raises(TypeError):
        M.maps_kv4_select_blocks(**good, ws=ws)
    for bad in (dict(qo_off=z(3)), dict(table=i(4, 4)), dict(codes=z(9, 2, 2, 64)), dict(blocks_out=i(5, 8)), dict(blocks_out=i(5, 3, 4)), dict(tokens_out=i(5, 3))):
        with pytest.raises(ValueError):
            M.maps_kv4_select_blocks(**good | bad, ws=ws)
    good = dict(q=h(5, 8, 128), blocks=i(5, 2, 4), tokens=i(5, 2), cache=cache, S=16, sm_scale=1.0, out=h(5, 8, 128), lse_out=z(5, 8))
    with pytest.raises(TypeError):
        M.maps_kv4_attention_blocks(**good, ws=ws)
    for bad in (dict(out=h(5, 4, 128)), dict(blocks=i(5, 8)), dict(blocks=i(5, 3, 4)), dict(tokens=i(2, 5)), dict(lse_out=z(5, 4))):
        with pytest.raises(ValueError):
            M.maps_kv4_attention_blocks(**good | bad, ws=ws)


def test_rotation_worked_example():
    x = np.arange(16, dtype=np.float32).reshape(1, 1, 16)
    quarter = np.concatenate([np.zeros((2, 4)), np.ones((2, 4))], 1).astype(np.float32)  # a quarter turn
    y = O.rotate(x, np.array([[1]]), None, 8, False, quarter)
    assert y[0, 0].tolist() == [-4, -5, -6, -7, 0, 1, 2, 3] + list(range(8, 16))
    y = O.rotate(x, np.array([[1]]), None, 8, True, quarter)
    assert y[0, 0].tolist() == [-1, 0, -3, 2, -5, 4, -7, 6] + list(range(8, 16))
    none = np.concatenate([np.ones((1, 4)), np.zeros((1, 4))], 1).astype(np.float32)
    both = np.concatenate([none, quarter])
    y = O.rotate(x, np.array([[0], [1]]), [0, 1, 0, 0], 8, False, both)  # the second pair alone
    assert y[0, 0].tolist() == [0, -5, 2, 3, 4, 1, 6, 7] + list(range(8, 16))


def test_range_worked_examples():
    codes, scale = O.range_of(np.array([[1, -127], [3, 50]], np.float32))
    assert scale == 1 and codes.tolist() == [[1, -127], [3, 50]]
    codes, scale = O.range_of(np.array([[0.5, -130]], np.float32))
    assert scale == np.float32(1 + 2.0**-7 * 4) and codes.tolist() == [[0, -127], [1, -126]]  # 130 / 127 is 1.0236: 1.03125
    assert O.range_of(np.array([[0.0, 0.0]], np.float32))[1] == 0
    assert np.isnan(O.range_of(np.array([[np.inf, 0]], np.float32))[1])
    rng = np.random.default_rng(0)
    for size in 2.0 ** rng.uniform(-125, 120, 200):
        k = (rng.normal(size=(7, 5)) * size).astype(np.float32)
        codes, scale = O.range_of(k)
        low, high = codes * np.float64(scale)
        if scale == 0:  # the header's exception
            assert np.abs(k).max() < 2.0**-119 and not codes.any()
            continue
        assert (low <= k).all() and (k <= high).all()
        assert np.abs(codes).max() in (126, 127)  # a scale is at most 1 + 2^-7 times what it has to be
        assert K.bf16(np.array([scale]))[0] == scale


def test_selection_worked_example():
    # five blocks of 16, first and last always, of the others the one that scores highest; ties to the earlier
    codes = np.zeros((6, 1, 2, 64), np.int8)
    codes[:, 0, 1, 0] = [1, 5, 9, 9, 2, 0]
    table = np.array([[4, 3, 2, 1, 0, -1]])
    q = np.zeros((1, 1, 64), np.float32)
    q[0, 0, 0] = 2
    none = np.full((1, 1, 3), -7), np.full((1, 1), -7)
    blocks, tokens = O.select(q, [0, 1], [70], table, codes, np.ones((6, 1), np.float32), 16, 1, 1, 3, *none)
    assert blocks.tolist() == [[[4, 3, 0]]] and tokens.tolist() == [[2 * 16 + 6]]
    blocks, tokens = O.select(-q, [0, 1], [70], table, codes, np.ones((6, 1), np.float32), 16, 0, 1, 2, none[0][..., :2], none[1])
    assert blocks.tolist() == [[[4, 0]]]  # the lowest ends are all 0
    blocks, tokens = O.select(q, [0, 1], [30], table, codes, np.ones((6, 1), np.float32), 16, 1, 1, 3, *none)
    assert blocks.tolist() == [[[4, 3, -1]]] and tokens.tolist() == [[30]]
