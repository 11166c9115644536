"""The binding's native marshalling: it is there, its calls give what those through Python's give, and what
it does not expect it leaves to Python, which refuses the same things with the same errors."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    from paper_2609_15359_gb300 import maps
    assert maps._fast is not None and maps._fast.torch_version == torch.__version__
    return maps


T, Hq, H, D, S, P, L = 21, 8, 2, 64, 16, 12, 3


def arguments(M, seed=0):
    """Of every call, by name, with room for what it writes."""
    g = torch.Generator("cuda").manual_seed(seed)
    f = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()  # noqa: E731
    i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = torch.zeros(M.kv4_cache_shape(P, H, S, D), dtype=torch.uint8, device="cuda")
    slots = torch.arange(T, device="cuda")
    codes = torch.randint(-127, 128, M.kv4_range_shape(P, H, D), device="cuda", generator=g, dtype=torch.int32).to(torch.int8)
    scale = torch.rand(P, H, device="cuda", generator=g)
    table = torch.arange(P, dtype=torch.int32, device="cuda").view(2, 6)
    lists = torch.randint(0, P, (T, H, L), device="cuda", generator=g, dtype=torch.int32)
    off = torch.tensor([0, 10, T], device="cuda")
    return dict(
        append=dict(k=f(T, H, D), v=f(T, H, D), slots=slots, cache=cache.clone(), S=S),
        read=dict(slots=slots, cache=torch.randint(0, 60, cache.shape, device="cuda", generator=g).to(torch.uint8), S=S, k_out=f(T, H, D), v_out=f(T, H, D)),
        append_rotated=dict(q=f(T, Hq, D), k=f(T, H, D), v=f(T, H, D), pos=i([list(range(T))] * 2), cos_sin=torch.randn(T, 32, device="cuda", generator=g),
                            slots=slots, cache=cache.clone(), S=S, q_out=f(T, Hq, D), axis=i([0, 1] * 8), interleaved=True),
        block_ranges=dict(held=i([0, 3]), kv_len=i([70, 40]), table=table, cache=torch.randint(0, 60, cache.shape, device="cuda", generator=g).to(torch.uint8), S=S,
                          codes=codes.clone(), scale=scale.clone()),
        select_blocks=dict(q=f(T, Hq, D), qo_off=off, kv_len=i([90, 80]), table=table, codes=codes, scale=scale, S=S, first=1, last=1,
                           blocks_out=torch.zeros_like(lists), tokens_out=i([[0] * H] * T)),
        attention_blocks=dict(q=f(T, Hq, D), blocks=lists, tokens=i([[40] * H] * T), cache=torch.randint(0, 60, cache.shape, device="cuda", generator=g).to(torch.uint8),
                              S=S, sm_scale=0.125, out=f(T, Hq, D), lse_out=torch.zeros(T, Hq, device="cuda")))


CALLS = ("append", "read", "append_rotated", "block_ranges", "select_blocks", "attention_blocks")


def variants(M, call, kw):
    """Other forms that are as good: strided rows, None where that may be."""
    yield dict(kw)
    for x in ("k", "v", "q", "out", "k_out", "q_out"):
        if x in kw:
            wide = torch.zeros(*kw[x].shape[:2], D + 5, dtype=kw[x].dtype, device="cuda")
            wide[..., 2:D + 2] = kw[x]
            yield kw | {x: wide[..., 2:D + 2]}
    for x in ("axis", "held", "lse_out"):
        if x in kw:
            yield kw | {x: None}
    if call == "append_rotated":
        yield kw | dict(q=None, q_out=None)
        yield kw | dict(pos=kw["pos"][0].contiguous(), axis=None)
        yield {x: kw[x].half() if x in ("q", "k", "v", "q_out") else kw[x] for x in kw}


@pytest.mark.parametrize("call", CALLS)
def test_native_and_python_marshalling_agree(M, call, monkeypatch):
    native = M._fast
    seen = []

    class Watched:
        def __getattr__(self, name):
            def go(*a):
                seen.append(getattr(native, name)(*a))
                return seen[-1]
            return go
    for kw in variants(M, call, arguments(M)[call]):
        got = []
        for path in (Watched(), None):
            mine = {x: v.clone() if isinstance(v, torch.Tensor) and v.is_contiguous() else v for x, v in kw.items()}
            monkeypatch.setattr(M, "_fast", path)
            ws = M.Workspace()
            assert getattr(M, "maps_kv4_" + call)(**mine, ws=ws) == 0 and M.maps_check(ws) == 0
            got.append({x: v.clone() for x, v in mine.items() if isinstance(v, torch.Tensor)})
        for x in got[0]:
            assert torch.equal(got[0][x].contiguous().view(torch.uint8), got[1][x].contiguous().view(torch.uint8)), x
    assert seen and all(st == 0 for st in seen)  # none of them was left to Python


def spoilt(x, v):
    """Arguments of another place, type, size or order; some sizes are as good (a cache of fewer blocks)."""
    if isinstance(v, torch.Tensor):
        yield v.cpu()
        yield v.double()
        if v.dim() > 1 and v.shape[0] > 1:
            yield v[: v.shape[0] - 1]
        if v.dim() > 1:
            yield v.transpose(0, v.dim() - 1)
        if v.dim() == 1 and v.numel() > 1:
            yield v[:1]
    yield "no"


@pytest.mark.parametrize("call", CALLS)
def test_what_is_not_expected_is_refused_as_in_python(M, call, monkeypatch):
    kw = arguments(M)[call]
    native = M._fast
    for x in kw:
        for bad in spoilt(x, kw[x]):
            errors = []
            for path in (native, None):
                monkeypatch.setattr(M, "_fast", path)
                try:
                    errors.append(getattr(M, "maps_kv4_" + call)(**kw | {x: bad}, ws=M.Workspace()))
                except Exception as e:  # noqa: BLE001
                    errors.append(type(e))
            assert errors[0] == errors[1], (x, errors)
            if isinstance(kw[x], torch.Tensor) and not (isinstance(bad, torch.Tensor) and bad.is_cuda and bad.dtype == kw[x].dtype):
                assert isinstance(errors[0], type), (x, errors)


def test_native_functions_return_none_for_anything_else(M):
    for call in CALLS:
        f = getattr(M._fast, call)
        good = list(arguments(M)[call].values())
        assert f() is None and f(*good) is None and f(*[None] * 16) is None and f(*[1 << 70] * 14) is None and f(*["x"] * 9) is None
        ws = M.Workspace()
        assert f(*good, ws.address, ws.nbytes, 0, 0) is None  # one too many
        assert f(*good, ws.address, 1.5, 0) is None


def test_status_and_workspace_errors_pass_through(M):
    kw = arguments(M)["attention_blocks"]
    assert M._fast.attention_blocks(*kw.values(), M.Workspace().address, 255, 0) == M.MAPS_E_WORKSPACE
    assert M.maps_kv4_attention_blocks(**kw | dict(sm_scale=float("nan")), ws=M.Workspace()) == M.MAPS_E_INVALID
    assert M.maps_kv4_select_blocks(**arguments(M)["select_blocks"] | dict(last=0), ws=M.Workspace()) == M.MAPS_E_INVALID
    # a row of keys longer than shared memory takes a workspace that grows
    table = torch.zeros(2, 10000, dtype=torch.int32, device="cuda")
    ws = M.Workspace()
    assert M.maps_kv4_select_blocks(**arguments(M)["select_blocks"] | dict(table=table), ws=ws) == 0 and M.maps_check(ws) == 0
    assert ws.nbytes >= T * H * 10000 * 4
