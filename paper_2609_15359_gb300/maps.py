"""Thin Python binding of the MAPS C ABI (``include/maps.h``).

Argument marshalling only: every function passes torch tensors' device
pointers and the current CUDA stream to the function of the same name in
``libmaps.so`` and returns its status.  Every step of the computation runs in
the library's CUDA kernels; there is no CPU path.  Importing this module
loads the library and fails loudly when it is missing.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

MAPS_OK = 0
MAPS_E_INVALID = -1
MAPS_E_RANGE = -2
MAPS_E_UNBOUNDED = -3
MAPS_E_TIMEOUT = -4
MAPS_E_CUDA = -5
MAPS_E_WORKSPACE = -6

BF16, F16 = 0, 1

MODE_SNAPSHOT = 0
MODE_SEQUENTIAL = 1
MODE_ALG1_SNAPSHOT = 2
MODE_ALG1_SEQUENTIAL = 3

STATUS_NAMES = {0: "MAPS_OK", -1: "MAPS_E_INVALID", -2: "MAPS_E_RANGE",
                -3: "MAPS_E_UNBOUNDED", -4: "MAPS_E_TIMEOUT", -5: "MAPS_E_CUDA",
                -6: "MAPS_E_WORKSPACE"}

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmaps.so")


class StreamCfg(ctypes.Structure):
    """``maps_stream_cfg`` of include/maps.h."""
    _fields_ = [("N", ctypes.c_int64), ("D", ctypes.c_int32), ("H", ctypes.c_int32),
                ("cap", ctypes.c_int32), ("batch", ctypes.c_int32), ("window", ctypes.c_int32),
                ("alpha_ppm", ctypes.c_uint32), ("max_wait", ctypes.c_int32),
                ("dispatch_policy", ctypes.c_int32), ("local_order", ctypes.c_int32),
                ("accounting", ctypes.c_int32), ("per_step", ctypes.c_int32),
                ("beta", ctypes.c_int32)]


# maps_stream_cfg policy fields
STREAM_MAPS, STREAM_MC, STREAM_RR, STREAM_LR = 0, 1, 2, 3
STREAM_SJF, STREAM_FCFS = 0, 1
STREAM_OCCUPANCY, STREAM_STAGED, STREAM_HELD = 0, 1, 2


class RRCfg(ctypes.Structure):
    """``maps_rr_cfg`` of include/maps.h."""
    _fields_ = [("n_req", ctypes.c_int64), ("N", ctypes.c_int32), ("C", ctypes.c_int32),
                ("t_tok_us", ctypes.c_int32), ("theta_ppm", ctypes.c_uint32)]


class MapsError(RuntimeError):
    def __init__(self, status: int, what: str = ""):
        super().__init__(f"{what}: {STATUS_NAMES.get(status, status)}")
        self.status = status


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with paper_2609_15359_gb300.build.build() "
            "(nvcc, sm_103a). There is no CPU fallback.")
    lib = ctypes.CDLL(LIB_PATH)
    i32, i64, u32, sz, vp, f32 = (ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32,
                                  ctypes.c_size_t, ctypes.c_void_p, ctypes.c_float)
    sigs = {
        "maps_version": ([], ctypes.c_int),
        "maps_last_cuda_error": ([], ctypes.c_int),
        "maps_check": ([vp, vp], ctypes.c_int),
        "maps_set_dispatch_events": ([vp, vp], ctypes.c_int),
        "maps_test_withhold_lookback": ([i32, u32], ctypes.c_int),
        "maps_test_absent_block": ([i32], ctypes.c_int),
        "maps_test_calibrate_absent_block": ([i32, u32], ctypes.c_int),
        "maps_test_attention_withhold": ([i32, u32], ctypes.c_int),
        "maps_calibrate_workspace_size": ([i64, i64], sz),
        "maps_calibrate": ([vp, vp, i64, u32, vp, i64, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "maps_project_occupancy_workspace_size": ([i32, i32, i64], sz),
        "maps_project_occupancy": ([i32, i32, vp, i64, vp, vp, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "maps_dispatch_workspace_size": ([i32, i32, i32, i64], sz),
        "maps_dispatch": ([i32, i32, i32, i32, vp, vp, vp, vp, vp, i64, vp, vp, vp, i64, vp, vp,
                           vp, vp, vp, sz, vp], ctypes.c_int),
        "maps_order_local_workspace_size": ([i64, i32], sz),
        "maps_order_local": ([i64, i32, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp], ctypes.c_int),
        "maps_order_local_static": ([i64, i32, vp, vp, vp, vp, i32, vp, vp, vp, vp], ctypes.c_int),
        "maps_rr_pressure_workspace_size": ([ctypes.POINTER(RRCfg), i64], sz),
        "maps_rr_pressure": ([ctypes.POINTER(RRCfg), i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp],
                             ctypes.c_int),
        "maps_stream_workspace_size": ([ctypes.POINTER(StreamCfg)], sz),
        "maps_stream_run": ([ctypes.POINTER(StreamCfg), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz,
                             vp],
                            ctypes.c_int),
        "maps_block_tables_workspace_size": ([i32], sz),
        "maps_block_tables": ([i32, i32, vp, vp, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp, i64, vp,
                               vp, sz, vp], ctypes.c_int),
        "maps_kv4_record_bytes": ([i32, i32], sz),
        "maps_kv4_workspace_size": ([], sz),
        "maps_kv4_append": ([i32, i64, i32, i32, i32, vp, i64, i64, vp, i64, i64, vp, vp, i64, vp,
                             sz, vp], ctypes.c_int),
        "maps_kv4_read": ([i32, i64, i32, i32, i32, vp, vp, i64, vp, i64, i64, vp, i64, i64, vp,
                           sz, vp], ctypes.c_int),
        "maps_kv4_attention_workspace_size": ([i32, i64, i32, i32, i32], sz),
        "maps_kv4_attention": ([i32, i32, i64, i32, i32, i32, i32, vp, i64, i64, vp, vp, vp, i64,
                                vp, i64, f32, i32, i32, vp, i64, i64, vp, vp, sz, vp],
                               ctypes.c_int),
    }
    for name, (args, res) in sigs.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    return lib


lib = _load()
EXPORTS = ("maps_version", "maps_last_cuda_error", "maps_check", "maps_set_dispatch_events",
           "maps_test_withhold_lookback", "maps_test_absent_block",
           "maps_test_calibrate_absent_block", "maps_test_attention_withhold",
           "maps_calibrate_workspace_size", "maps_calibrate",
           "maps_project_occupancy_workspace_size", "maps_project_occupancy",
           "maps_dispatch_workspace_size", "maps_dispatch",
           "maps_order_local_workspace_size", "maps_order_local", "maps_order_local_static",
           "maps_stream_workspace_size", "maps_stream_run",
           "maps_rr_pressure_workspace_size", "maps_rr_pressure",
           "maps_block_tables_workspace_size", "maps_block_tables", "maps_kv4_record_bytes",
           "maps_kv4_workspace_size", "maps_kv4_append", "maps_kv4_read",
           "maps_kv4_attention_workspace_size", "maps_kv4_attention")


# The handle of the current stream without a stream object, which costs 3.2 us, a third of a call.  PyTorch promises
# this function to nobody, so where it is missing the object has to do.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _ptr(t, dtype=None) -> int | None:
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("expected a CUDA tensor")
    if dtype is not None and t.dtype is not dtype:
        raise TypeError(f"expected {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise TypeError("expected a contiguous tensor")
    return t.data_ptr()


class Workspace:
    """Zero-filled device scratch owned by the caller, grown on demand.

    It is allocated and zero-filled on the stream of the call that needs it (the
    current one where it is made beforehand).  A call on another stream first waits
    for that, and the memory is not handed out again before that stream is done.
    Growing keeps the status word, so maps_check still reads what earlier calls
    recorded; a call without a workspace has nobody to read its data errors."""

    def __init__(self, nbytes: int = 0, device=None, stream=None):
        self.device = torch.device("cuda") if device is None else torch.device(device)
        self.on_gpu = self.device.type == "cuda"
        self._take(max(int(nbytes), 256), stream)

    def _take(self, nbytes: int, stream=None) -> None:
        on = _stream(stream) if self.on_gpu else None
        if on is not None and on != _stream(None):
            with torch.cuda.stream(stream):
                return self._take(nbytes)
        old = getattr(self, "_buf", None)
        if old is not None and on not in self.known:
            self._meet(stream)
        self.filled, self.known = None, {on}  # the zero-fill, and the streams that are behind it
        self.buf = torch.zeros(nbytes, dtype=torch.uint8, device=self.device)
        if old is not None:
            self._buf[:4].copy_(old[:4])
        if self.on_gpu and not torch.cuda.is_current_stream_capturing():
            self.filled = torch.cuda.Event()
            self.filled.record(torch.cuda.current_stream(self.device))

    @property
    def buf(self):
        return self._buf

    @buf.setter
    def buf(self, buf) -> None:
        self._buf, self.ptr, self.nbytes = buf, ctypes.c_void_p(buf.data_ptr()), buf.numel()

    def _meet(self, stream) -> None:
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        with torch.cuda.stream(s):
            # what was queued before a capture began is done by the time that its graph runs
            if self.filled is not None and not torch.cuda.is_current_stream_capturing():
                s.wait_event(self.filled)
        self._buf.record_stream(s)
        self.known.add(s.cuda_stream)

    def ensure(self, nbytes: int, stream=None) -> "Workspace":
        """At least `nbytes`, to be used by work on `stream` (the current one)."""
        if nbytes > self.nbytes:
            self._take(int(nbytes), stream)
        elif self.on_gpu and _stream(stream) not in self.known:
            self._meet(stream)
        return self


def _scratch(ws: Workspace | None, nbytes: int, stream):
    """The workspace of a call that needs `nbytes`, and its stream's handle."""
    if ws is None:
        ws = Workspace(nbytes, stream=stream)
    on = _stream(stream) if ws.on_gpu else None
    if nbytes > ws.nbytes or on not in ws.known:
        ws.ensure(nbytes, stream)
    return ws, on


@functools.lru_cache(maxsize=4096)
def _need(device: int | None, query: str, *sizes: int) -> int:
    """A size query: it depends on the sizes alone, or on the multiprocessors of `device` too."""
    return getattr(lib, query)(*sizes)


def maps_check(ws: Workspace, stream=None) -> int:
    return lib.maps_check(ws.ptr, _stream(stream))


def maps_set_dispatch_events(before=None, after=None) -> int:
    """Benchmarking aid: torch.cuda.Event objects that later SNAPSHOT
    maps_dispatch calls of this thread record around their scoring kernel
    (None, None turns it off).  The events must already exist on the device:
    record each once first."""
    h = lambda e: None if e is None else ctypes.c_void_p(e.cuda_event)  # noqa: E731
    return lib.maps_set_dispatch_events(h(before), h(after))


def maps_calibrate(true_len, pred_len, alpha_ppm: int, query_pred=None, bound_out=None,
                   q_dev_out=None, q_host: bool = False, ws: Workspace | None = None,
                   stream=None):
    """Returns (status, q) where q is the host quantile when ``q_host``."""
    n = true_len.numel()
    m = 0 if query_pred is None else query_pred.numel()
    ws, on = _scratch(ws, lib.maps_calibrate_workspace_size(n, m), stream)
    qh = ctypes.c_int32(0)
    st = lib.maps_calibrate(_ptr(true_len, torch.int32), _ptr(pred_len, torch.int32), n,
                            int(alpha_ppm), _ptr(query_pred, torch.int32), m,
                            _ptr(bound_out, torch.int32), _ptr(q_dev_out, torch.int32),
                            ctypes.byref(qh) if q_host else None, ws.ptr, ws.nbytes,
                            on)
    return st, (int(qh.value) if q_host else None)


def kmax_shape(D: int, H: int) -> tuple[int, int]:
    """Shape of the 16-step summary of K (uint32 values, stored as int32)."""
    return D, (H + 15) // 16


def maps_project_occupancy(D: int, H: int, res_off, prompt, gen, bound, K_out, kmax_out=None,
                           ws: Workspace | None = None, stream=None) -> int:
    R = prompt.numel()
    ws, on = _scratch(ws, lib.maps_project_occupancy_workspace_size(D, H, R), stream)
    return lib.maps_project_occupancy(D, H, _ptr(res_off, torch.int64), R,
                                      _ptr(prompt, torch.int32), _ptr(gen, torch.int32),
                                      _ptr(bound, torch.int32), _ptr(K_out, torch.int32),
                                      _ptr(kmax_out, torch.int32), ws.ptr, ws.nbytes,
                                      on)


def maps_dispatch(mode: int, D: int, H: int, S: int, K, cap, Q, cand_prompt, cand_bound,
                  choice_out, headroom_out=None, res_off=None, prompt=None, gen=None,
                  bound=None, kmax=None, ws: Workspace | None = None, stream=None) -> int:
    J = cand_prompt.numel()
    R = 0 if prompt is None else prompt.numel()
    ws, on = _scratch(ws, lib.maps_dispatch_workspace_size(mode, D, H, J), stream)
    return lib.maps_dispatch(mode, D, H, S, _ptr(K, torch.int32), _ptr(kmax, torch.int32),
                             _ptr(cap, torch.int32),
                             _ptr(Q, torch.int32), _ptr(res_off, torch.int64), R,
                             _ptr(prompt, torch.int32), _ptr(gen, torch.int32),
                             _ptr(bound, torch.int32), J, _ptr(cand_prompt, torch.int32),
                             _ptr(cand_bound, torch.int32), _ptr(choice_out, torch.int32),
                             _ptr(headroom_out, torch.int64), ws.ptr, ws.nbytes,
                             on)


def maps_order_local(D: int, dec, bound, wait, arrival, max_wait: int, perm_out, seg_off_out,
                     ws: Workspace | None = None, stream=None) -> int:
    N = dec.numel()
    ws, on = _scratch(ws, lib.maps_order_local_workspace_size(N, D), stream)
    return lib.maps_order_local(N, D, _ptr(dec, torch.int32), _ptr(bound, torch.int32),
                                _ptr(wait, torch.int32), _ptr(arrival, torch.int32),
                                int(max_wait), _ptr(perm_out, torch.int32),
                                _ptr(seg_off_out, torch.int64), ws.ptr, ws.nbytes,
                                on)


def maps_order_local_static(D: int, dec, bound, wait, arrival, max_wait: int, perm_out,
                            seg_off_out, sync_status: bool = True, stream=None) -> int:
    """maps_order_local with the library's fixed scratch array: no workspace,
    no allocation.  N <= 65,536 and D <= 4,096."""
    N = dec.numel()
    st = ctypes.c_int32(0)
    return lib.maps_order_local_static(N, D, _ptr(dec, torch.int32), _ptr(bound, torch.int32),
                                       _ptr(wait, torch.int32), _ptr(arrival, torch.int32),
                                       int(max_wait), _ptr(perm_out, torch.int32),
                                       _ptr(seg_off_out, torch.int64),
                                       ctypes.byref(st) if sync_status else None,
                                       _stream(stream))


def stream_cfg(N: int, D: int, H: int, cap: int, batch: int, window: int, alpha_ppm: int,
               max_wait: int, dispatch_policy: int = STREAM_MAPS, local_order: int = STREAM_SJF,
               accounting: int = STREAM_OCCUPANCY, per_step: int = 0,
               beta: int = -1) -> StreamCfg:
    return StreamCfg(int(N), int(D), int(H), int(cap), int(batch), int(window), int(alpha_ppm),
                     int(max_wait), int(dispatch_policy), int(local_order), int(accounting),
                     int(per_step), int(beta))


def maps_stream_run(cfg: StreamCfg, arrival_ms, prompt, true_len, pred, choice_out, q_out,
                    stats_out, dec_stats_out=None, ws: Workspace | None = None,
                    stream=None, pred_delay=None) -> int:
    """The whole streaming loop on the device; returns the full status.
    dec_stats_out: optional [D][4] int64 per-decoder statistics; pred_delay:
    [N] int32 prediction delays (required when cfg.beta >= 0)."""
    ws, on = _scratch(ws, lib.maps_stream_workspace_size(ctypes.byref(cfg)), stream)
    return lib.maps_stream_run(ctypes.byref(cfg), _ptr(arrival_ms, torch.int64),
                               _ptr(prompt, torch.int32), _ptr(true_len, torch.int32),
                               _ptr(pred, torch.int32), _ptr(pred_delay, torch.int32),
                               _ptr(choice_out, torch.int32),
                               _ptr(q_out, torch.int32), _ptr(stats_out, torch.int64),
                               _ptr(dec_stats_out, torch.int64), ws.ptr, ws.nbytes,
                               on)


def maps_rr_pressure(N: int, C: int, t_tok_us: int, theta_ppm: int, arrival_us, prompt, out_len,
                     admit_out, done_out, stats_out, t_sim_out, ws: Workspace | None = None,
                     stream=None) -> int:
    """The App. A round-robin simulation of n_real realisations at once.
    arrival_us [n_real][n_req] int64, prompt / out_len [n_real][n_req] int32;
    outputs admit / done [n_real][n_req] int64, stats [n_real][N][6] int64,
    t_sim [n_real] int64."""
    n_real, n_req = arrival_us.shape
    cfg = RRCfg(int(n_req), int(N), int(C), int(t_tok_us), int(theta_ppm))
    ws, on = _scratch(ws, lib.maps_rr_pressure_workspace_size(ctypes.byref(cfg), n_real), stream)
    return lib.maps_rr_pressure(ctypes.byref(cfg), n_real, _ptr(arrival_us, torch.int64),
                                _ptr(prompt, torch.int32), _ptr(out_len, torch.int32),
                                _ptr(admit_out, torch.int64), _ptr(done_out, torch.int64),
                                _ptr(stats_out, torch.int64), _ptr(t_sim_out, torch.int64),
                                ws.ptr, ws.nbytes, on)


def maps_block_tables(S: int, held, want, table, free_blocks, n_free, n_free_out, got_out,
                      slot_off_out, slots_out, pos_out=None, order=None,
                      ws: Workspace | None = None, stream=None) -> int:
    """Hands out the KV blocks: table [R][max_blocks] and free_blocks [pool]
    int32 are updated in place; slots_out [cap] int64 holds the new tokens'."""
    R = held.numel()
    rows, max_blocks = table.shape
    cap = slots_out.numel()
    if (want.numel() < R or got_out.numel() < R or slot_off_out.numel() <= R or rows < R or
            order is not None and order.numel() < R or pos_out is not None and pos_out.numel() < cap):
        raise ValueError("want, order, table, got_out, slot_off_out or pos_out has too few elements")
    ws, on = _scratch(ws, _need(None, "maps_block_tables_workspace_size", R), stream)
    return lib.maps_block_tables(R, S, _ptr(held, torch.int32), _ptr(want, torch.int32),
                                 _ptr(order, torch.int32), _ptr(table, torch.int32),
                                 max_blocks, _ptr(free_blocks, torch.int32),
                                 free_blocks.numel(), _ptr(n_free, torch.int32),
                                 _ptr(n_free_out, torch.int32), _ptr(got_out, torch.int32),
                                 _ptr(slot_off_out, torch.int64), _ptr(slots_out, torch.int64),
                                 cap, _ptr(pos_out, torch.int32), ws.ptr, ws.nbytes,
                                 on)


def _rows(t, dtype=None):
    """(pointer, row stride, head stride) of a [rows, heads, channels] tensor
    whose channels are contiguous; any strides otherwise."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("expected a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"expected {dtype}, got {t.dtype}")
    row, head, channel = t.stride()
    if channel != 1 and t.numel() > 0:  # the strides of an empty tensor say nothing
        raise TypeError("expected [rows, heads, channels] with contiguous channels")
    return t.data_ptr(), row, head


_DTYPES = {torch.bfloat16: BF16, torch.float16: F16}


def _dtype(t) -> int:
    try:
        return _DTYPES[t.dtype]
    except KeyError:
        raise TypeError(f"expected torch.bfloat16 or torch.float16, got {t.dtype}") from None


def kv4_cache_shape(n_blocks: int, H: int, S: int, D: int) -> tuple[int, int, int]:
    """Shape of a 4-bit cache (uint8): [blocks][KV heads][record bytes]."""
    nbytes = _need(None, "maps_kv4_record_bytes", S, D)
    if nbytes == 0:
        raise ValueError(f"no 4-bit cache for blocks of {S} tokens and {D} channels")
    return n_blocks, H, nbytes


def _kv4(cache, S: int, D: int, H: int):
    if cache.shape != kv4_cache_shape(cache.shape[0], H, S, D):
        raise ValueError(f"a cache of {H} heads, blocks of {S} and {D} channels does not have shape "
                         f"{tuple(cache.shape)}")
    return _ptr(cache, torch.uint8)


def maps_kv4_append(k, v, slots, cache, S: int, ws: Workspace | None = None, stream=None) -> int:
    """Writes k, v [T, H, D] (bf16 or fp16) to the slots [T] int64 of the cache."""
    T, H, D = k.shape
    if v.shape != k.shape or slots.numel() != T:
        raise ValueError("k, v and slots differ in size")
    ws, on = _scratch(ws, _need(None, "maps_kv4_workspace_size"), stream)
    return lib.maps_kv4_append(_dtype(k), T, H, D, S, *_rows(k), *_rows(v, k.dtype),
                               _ptr(slots, torch.int64), _kv4(cache, S, D, H), cache.shape[0],
                               ws.ptr, ws.nbytes, on)


def maps_kv4_read(slots, cache, S: int, k_out, v_out, ws: Workspace | None = None,
                  stream=None) -> int:
    """Reads the slots [T] of the cache back into k_out, v_out [T, H, D]."""
    T, H, D = k_out.shape
    if v_out.shape != k_out.shape or slots.numel() != T:
        raise ValueError("k_out, v_out and slots differ in size")
    ws, on = _scratch(ws, _need(None, "maps_kv4_workspace_size"), stream)
    return lib.maps_kv4_read(_dtype(k_out), T, H, D, S, _ptr(slots, torch.int64),
                             _kv4(cache, S, D, H), cache.shape[0], *_rows(k_out),
                             *_rows(v_out, k_out.dtype), ws.ptr, ws.nbytes, on)


def maps_kv4_attention(q, qo_off, kv_len, table, cache, S: int, sm_scale: float, out, lse_out=None,
                       causal: bool = True, window: int = 0, ws: Workspace | None = None,
                       stream=None) -> int:
    """Attention of q [T, Hq, D] over the 4-bit cache: qo_off [B + 1] int64,
    kv_len [B] int32, table [B][max_blocks] int32; out like q, lse_out [T][Hq]
    float32 or None."""
    T, Hq, D = q.shape
    B, Hkv = kv_len.numel(), cache.shape[1]
    if out.shape != q.shape or qo_off.numel() != B + 1 or table.shape[0] != B:
        raise ValueError("q, out, qo_off, kv_len and table differ in size")
    if lse_out is not None and tuple(lse_out.shape) != (T, Hq):
        raise ValueError("lse_out is [T, Hq]")
    ws, on = _scratch(ws, _need(torch.cuda.current_device(), "maps_kv4_attention_workspace_size", B, T, Hq, Hkv, D), stream)
    return lib.maps_kv4_attention(_dtype(q), B, T, Hq, Hkv, D, S, *_rows(q),
                                  _ptr(qo_off, torch.int64), _ptr(kv_len, torch.int32),
                                  _ptr(table, torch.int32), table.shape[1],
                                  _kv4(cache, S, D, Hkv), cache.shape[0], float(sm_scale),
                                  int(bool(causal)), int(window), *_rows(out, q.dtype),
                                  _ptr(lse_out, torch.float32), ws.ptr, ws.nbytes,
                                  on)
