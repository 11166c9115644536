"""The binding's native marshalling without a GPU: a process of its own gives it functions that stand in for the
library's, and CUDA tensors of addresses that nobody reads.  A tensor that has no memory (a lane of torch.vmap) is
left to Python, whichever argument it is."""
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = """
import ctypes, sys
import torch
from paper_2609_15359_gb300 import _marshal as m

i64, i32 = ctypes.c_int64, ctypes.c_int32
calls = []
bytes_of = ctypes.CFUNCTYPE(ctypes.c_size_t, i32, i32)(lambda S, D: S // 16 * (16 * D + 128))
size_of = ctypes.CFUNCTYPE(ctypes.c_size_t, i64, i32, i64)(lambda T, H, n: 256)
run = ctypes.CFUNCTYPE(ctypes.c_int)(lambda: calls.append(1) or 0)  # looks at none of its arguments
at = lambda f: ctypes.cast(f, ctypes.c_void_p).value
m.bind(at(bytes_of), at(run), at(run), at(run), at(run), at(size_of), at(run), at(run))


def z(*shape, t=torch.bfloat16):
    plain = torch.empty(shape, dtype=t, device="meta")
    storage = torch._C._construct_storage_from_data_pointer(1 << 20, torch.device("cuda", 0), plain.numel() * plain.element_size())
    return torch._C._construct_CUDA_Tensor_From_Storage_And_Metadata(
        dict(size=shape, stride=plain.stride(), storage_offset=0, dtype=t, device=torch.device("cuda", 0)), storage)


T, Hq, H, D, S, P, L = 5, 4, 2, 64, 16, 9, 3
number, long = torch.int32, torch.int64
codes, scale, cache = z(P, H, 2, D, t=torch.int8), z(P, H, t=torch.float32), z(P, H, 1152, t=torch.uint8)
slots = z(T, t=long)
call = sys.argv[1]
args = dict(
    append=dict(k=z(T, H, D), v=z(T, H, D), slots=slots, cache=cache, S=S),
    read=dict(slots=slots, cache=cache, S=S, k_out=z(T, H, D), v_out=z(T, H, D)),
    append_rotated=dict(q=z(T, Hq, D), k=z(T, H, D), v=z(T, H, D), pos=z(2, T, t=number), cos_sin=z(7, 32, t=torch.float32), slots=slots, cache=cache, S=S,
                        q_out=z(T, Hq, D), axis=z(16, t=number), interleaved=False),
    block_ranges=dict(held=z(3, t=number), kv_len=z(3, t=number), table=z(3, 4, t=number), cache=cache, S=S, codes=codes, scale=scale),
    select_blocks=dict(q=z(T, Hq, D), qo_off=z(4, t=long), kv_len=z(3, t=number), table=z(3, 4, t=number), codes=codes, scale=scale, S=S, first=1, last=1,
                       blocks_out=z(T, H, L, t=number), tokens_out=z(T, H, t=number)),
    attention_blocks=dict(q=z(T, Hq, D), blocks=z(T, H, L, t=number), tokens=z(T, H, t=number), cache=cache, S=S, sm_scale=0.1, out=z(T, Hq, D),
                          lse_out=z(T, Hq, t=torch.float32)))[call]
go = lambda a: getattr(m, call)(*a.values(), 1 << 20, 256, 0)
assert go(args) == 0 and calls == [1]
for name in args:
    if not isinstance(args[name], torch.Tensor):
        continue
    print(name, flush=True)

    def without(lane):
        assert type(lane) is torch.Tensor and lane.is_cuda and lane.shape == args[name].shape
        assert go(args | {name: lane}) is None
        return 0

    torch.vmap(without, out_dims=None)(z(1, *args[name].shape, t=args[name].dtype))
    assert sum(range(1000)) == 499500 and calls == [1]
print("as expected")
"""


@pytest.mark.parametrize("call", ("append", "read", "append_rotated", "block_ranges", "select_blocks", "attention_blocks"))
def test_tensors_without_memory_are_left_to_python(call):
    from paper_2609_15359_gb300 import build
    build.build()
    pytest.importorskip("paper_2609_15359_gb300._marshal", exc_type=ImportError)  # needs PyTorch's headers
    for f in ("_construct_storage_from_data_pointer", "_construct_CUDA_Tensor_From_Storage_And_Metadata"):
        if not hasattr(torch._C, f):
            pytest.skip(f"this PyTorch has no {f}")
    r = subprocess.run([sys.executable, "-c", SCRIPT, call], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.endswith("as expected\n"), (r.returncode, r.stdout, r.stderr[-2000:])
