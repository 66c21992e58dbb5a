"""ctypes binding of the CUDA library (include/crc.h), names as in the C ABI.

Argument marshalling only: every step of the routing and cache path runs in
the library's kernels.  PyTorch supplies device memory and streams.  There
is no fallback: if libcrc.so is missing or a call fails, an exception is
raised.
"""
from __future__ import annotations

import ctypes
import math
import os
import threading
from dataclasses import dataclass

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_build", "libcrc.so")

(CRC_OK, CRC_EINVAL, CRC_EUNSUPPORTED, CRC_ECUDA, CRC_ETIMEOUT, CRC_ESTATE, CRC_EDEVICE,
 CRC_ENOMEM) = range(8)


class crc_problem(ctypes.Structure):
    _fields_ = [("L", ctypes.c_int32), ("N", ctypes.c_int32), ("K", ctypes.c_int32),
                ("d", ctypes.c_int32), ("C", ctypes.c_int32), ("R", ctypes.c_int32),
                ("B", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("expert_bytes", ctypes.c_uint64)]


class crc_trace(ctypes.Structure):
    _fields_ = [("topk_dev", ctypes.c_void_p), ("misses_dev", ctypes.c_void_p),
                ("proactive_dev", ctypes.c_void_p), ("cache_mid_dev", ctypes.c_void_p),
                ("cache_after_dev", ctypes.c_void_p), ("topk_set_dev", ctypes.c_void_p)]


class crc_transfer(ctypes.Structure):
    _fields_ = [("t", ctypes.c_int32), ("l", ctypes.c_int32), ("expert", ctypes.c_int32),
                ("slot", ctypes.c_int32), ("evicted", ctypes.c_int32),
                ("proactive", ctypes.c_int32)]


TRANSFER_DTYPE = np.dtype([("t", np.int32), ("l", np.int32), ("expert", np.int32),
                           ("slot", np.int32), ("evicted", np.int32), ("proactive", np.int32)])


class crc_stats(ctypes.Structure):
    _fields_ = [("accesses", ctypes.c_uint64), ("hits", ctypes.c_uint64),
                ("misses", ctypes.c_uint64), ("proactive", ctypes.c_uint64),
                ("traffic_bytes", ctypes.c_uint64), ("tokens", ctypes.c_uint64),
                ("error", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]


class crc_report(ctypes.Structure):
    _fields_ = [("hit", ctypes.c_double), ("adj_hit", ctypes.c_double),
                ("traffic_bytes", ctypes.c_double), ("load_per_token_bytes", ctypes.c_double)]


KERNEL_KINDS = {"router": 0, "scan": 1, "state": 2, "synth": 3, "fused": 4, "loss": 5,
                "loss_means": 6, "short": 7, "norm": 8, "quantize": 9, "moe_route": 10, "moe": 11}


class crc_kernel_times(ctypes.Structure):
    _fields_ = [("launches", ctypes.c_uint64 * 12), ("ms", ctypes.c_double * 12)]


class crc_moe(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int32), ("K", ctypes.c_int32), ("d", ctypes.c_int32),
                ("f", ctypes.c_int32), ("slots", ctypes.c_int32),
                ("weight_type", ctypes.c_int32), ("renormalize", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("gate_up_dev", ctypes.c_void_p),
                ("down_dev", ctypes.c_void_p), ("gate_up_stride", ctypes.c_int64),
                ("down_stride", ctypes.c_int64), ("gate_up_scale_dev", ctypes.c_void_p),
                ("down_scale_dev", ctypes.c_void_p), ("gate_up_scale_stride", ctypes.c_int64),
                ("down_scale_stride", ctypes.c_int64), ("router_dev", ctypes.c_void_p),
                ("expert_slot_dev", ctypes.c_void_p)]


class CrcError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: {crc_strerror(code)} (code {code})")


_lib = None
_lock = threading.Lock()

# (name, restype, argtypes) of every exported symbol
P, I32, I64, U32, U64, SZ, D = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32,
                                ctypes.c_uint64, ctypes.c_size_t, ctypes.c_double)
PP = ctypes.POINTER(crc_problem)
EXPORTS = [
    ("crc_state_bytes", SZ, [PP]),
    ("crc_state_init", ctypes.c_int, [PP, P, SZ, P]),
    ("crc_state_read", ctypes.c_int, [PP, P, SZ, ctypes.POINTER(crc_stats), P, P, P, P]),
    ("crc_route_scores", ctypes.c_int, [PP, P, P, I32, I32, P, P]),
    ("crc_cache_scan", ctypes.c_int, [PP, P, I32, P, SZ, ctypes.POINTER(crc_trace), P]),
    ("crc_workspace_bytes", SZ, [PP, I32]),
    ("crc_fused_workspace_bytes", SZ, [PP]),
    ("crc_route_and_cache", ctypes.c_int,
     [PP, P, P, I32, P, SZ, ctypes.POINTER(crc_trace), P, SZ, P]),
    ("crc_route_and_cache_noalloc", ctypes.c_int,
     [PP, P, P, I32, P, SZ, ctypes.POINTER(crc_trace), P]),
    ("crc_host_staging_bytes", SZ, [PP, I32]),
    ("crc_host_alloc", ctypes.c_int, [SZ, ctypes.POINTER(ctypes.c_void_p)]),
    ("crc_host_free", ctypes.c_int, [P]),
    ("crc_wait_probe", ctypes.c_int, [PP, P, SZ, I32, U64, P]),
    ("crc_route_and_cache_host", ctypes.c_int, [PP, P, P, I32, I32, P, SZ, P, SZ, P, SZ, P]),
    ("crc_device_error", ctypes.c_int, []),
    ("crc_cache_scan_policy", ctypes.c_int,
     [PP, P, I32, P, SZ, ctypes.POINTER(crc_trace), I32, I32, P]),
    ("crc_state_read_aux", ctypes.c_int, [PP, P, SZ, P, P]),
    ("crc_loss_workspace_bytes", SZ, [PP, I32]),
    ("crc_transfer_plan", ctypes.c_int, [PP, I32, P, P, P, P, P, ctypes.c_int64, P]),
    ("crc_transfer_replay", ctypes.c_int, [PP, P, ctypes.c_int64, P, ctypes.c_int64, P, P]),
    ("crc_cache_loss", ctypes.c_int, [PP, P, I32, I32, I32, D, D, D, P, P, P, P, SZ, P]),
    ("crc_metrics", ctypes.c_int, [PP, ctypes.POINTER(crc_stats), ctypes.POINTER(crc_report)]),
    ("crc_load_time", ctypes.c_int, [PP, ctypes.POINTER(crc_stats), D, D,
                                      ctypes.POINTER(ctypes.c_double)]),
    ("crc_launch_count", U64, []),
    ("crc_strerror", ctypes.c_char_p, [ctypes.c_int]),
    ("crc_profile_begin", ctypes.c_int, []),
    ("crc_profile_end", ctypes.c_int, [ctypes.POINTER(crc_kernel_times)]),
    ("crc_synth_hidden", ctypes.c_int, [I32, I32, I32, I32, I32, U32, D, D, P, P, P, P]),
    ("crc_synth_weights", ctypes.c_int, [I32, I32, I32, U32, I32, P, P]),
    ("crc_rms_norm", ctypes.c_int, [P, I64, P, P, I32, I64, I32, D, P, P, P, P, P, P]),
    ("crc_rms_norm_grad_workspace_bytes", SZ, [I64, I32]),
    ("crc_rms_norm_grad", ctypes.c_int, [P, P, P, P, P, I32, I64, I32, P, P, P, SZ, P]),
    ("crc_quantize_rows", ctypes.c_int, [P, I64, I64, I32, P, P, P]),
    ("crc_moe_workspace_bytes", SZ, [ctypes.POINTER(crc_moe), I32]),
    ("crc_moe_layer", ctypes.c_int,
     [ctypes.POINTER(crc_moe), P, I64, P, P, P, I64, I32, P, P, P, P, SZ, P]),
]


def load(path: str = LIB_PATH):
    """Load libcrc.so (built by paper_2609_04895_gb300.build); raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(path):
                raise ImportError(
                    f"CUDA library not built: {path} (run paper_2609_04895_gb300.build.build())")
            lib = ctypes.CDLL(path)
            for name, res, args in EXPORTS:
                f = getattr(lib, name)
                f.restype = res
                f.argtypes = args
            _lib = lib
    return _lib


def _ck(rc: int, what: str):
    if rc != CRC_OK:
        raise CrcError(rc, what)


def _stream(stream, dev: int | None = None) -> int:
    """The raw handle; dev: the current device, where the caller has asked for it."""
    if stream is None:
        # the current stream's handle without the Stream object around it, which
        # took 3 of a one-token call's 13 us on the host
        import torch
        if dev is None:
            dev = torch.cuda.current_device()
        return torch._C._cuda_getCurrentRawStream(dev)
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _ptr(t) -> int:
    if t is None:
        return None
    return t.data_ptr()


def _on(stream, device):
    """`stream` as a torch stream, None if it is the current one."""
    import torch
    ptr = _stream(stream)
    if ptr == torch.cuda.current_stream(device).cuda_stream:
        return None
    if isinstance(stream, torch.cuda.Stream):
        return stream
    if ptr == 0:
        return torch.cuda.default_stream(device)
    return torch.cuda.ExternalStream(ptr, device)


def _new(stream, device, shape, dtype, zeros: bool = False):
    """A tensor that a call on `stream` writes.  It comes from that stream's pool: what was
    in its memory before is used up when the call's kernels run, and after the caller's
    last reference the memory waits for them.  The current stream may read it too."""
    import torch
    make = torch.zeros if zeros else torch.empty
    on = None if stream is None else _on(stream, device)
    if on is None:
        return make(shape, dtype=dtype, device=device)
    with torch.cuda.stream(on):
        t = make(shape, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream(device))
    return t


# --------------------------------------------------------------------------- #
# C-ABI names
# --------------------------------------------------------------------------- #
def crc_strerror(code: int) -> str:
    try:
        return load().crc_strerror(code).decode()
    except ImportError:
        return f"error {code}"


def crc_state_bytes(p: crc_problem) -> int:
    return int(load().crc_state_bytes(ctypes.byref(p)))


def crc_state_init(p: crc_problem, state_ptr: int, state_bytes: int, stream=None):
    _ck(load().crc_state_init(ctypes.byref(p), state_ptr, state_bytes, _stream(stream)),
        "crc_state_init")


def crc_state_read(p: crc_problem, state_ptr: int, state_bytes: int, stream=None,
                   want_caches: bool = False, want_retention: bool = False,
                   want_chain_counters: bool = False) -> dict:
    st = crc_stats()
    B, L, N = p.B, p.L, p.N
    bits = np.zeros((B, L, (N + 31) // 32), np.uint32) if want_caches else None
    ret = np.zeros((B, L, N), np.float32) if want_retention else None
    cc = np.zeros((B, L, 3), np.uint64) if want_chain_counters else None
    rc = load().crc_state_read(ctypes.byref(p), state_ptr, state_bytes, ctypes.byref(st),
                               None if bits is None else bits.ctypes.data,
                               None if ret is None else ret.ctypes.data,
                               None if cc is None else cc.ctypes.data, _stream(stream))
    _ck(rc, "crc_state_read")
    out = {f: int(getattr(st, f)) for f, _ in crc_stats._fields_ if f != "reserved"}
    out.update(cache_bits=bits, retention=ret, chain_counters=cc)
    return out


def crc_route_scores(p: crc_problem, hidden_ptr: int, w_ptr: int, T: int, heads: int,
                     scores_ptr: int, stream=None):
    _ck(load().crc_route_scores(ctypes.byref(p), hidden_ptr, w_ptr, T, heads, scores_ptr,
                                _stream(stream)), "crc_route_scores")


def crc_cache_scan(p: crc_problem, scores_ptr: int, T: int, state_ptr: int, state_bytes: int,
                   trace: crc_trace | None = None, stream=None):
    _ck(load().crc_cache_scan(ctypes.byref(p), scores_ptr, T, state_ptr, state_bytes,
                              None if trace is None else ctypes.byref(trace), _stream(stream)),
        "crc_cache_scan")


# comparison policies (crc.h CRC_POLICY_*)
POLICIES = {"lru": 1, "lfu": 2, "lrfu": 3, "spatio_lru": 4}


def crc_cache_scan_policy(p: crc_problem, scores_ptr: int, T: int, state_ptr: int,
                          state_bytes: int, trace: crc_trace | None, policy: int,
                          lambda_halves: int = 1, stream=None):
    _ck(load().crc_cache_scan_policy(ctypes.byref(p), scores_ptr, T, state_ptr, state_bytes,
                                     None if trace is None else ctypes.byref(trace), policy,
                                     lambda_halves, _stream(stream)),
        "crc_cache_scan_policy")


def crc_state_read_aux(p: crc_problem, state_ptr: int, state_bytes: int,
                       stream=None) -> np.ndarray:
    aux = np.zeros((p.B, p.L, p.N), np.uint32)
    _ck(load().crc_state_read_aux(ctypes.byref(p), state_ptr, state_bytes, aux.ctypes.data,
                                  _stream(stream)), "crc_state_read_aux")
    return aux


def crc_loss_workspace_bytes(p: crc_problem, T: int) -> int:
    return int(load().crc_loss_workspace_bytes(ctypes.byref(p), T))


def crc_cache_loss(p: crc_problem, probs_ptr: int, T: int, heads: int, top_b: int, tau: float,
                   w_T: float, w_ST: float, loss_ptr, means_ptr, grad_ptr, ws_ptr, ws_bytes: int,
                   stream=None):
    _ck(load().crc_cache_loss(ctypes.byref(p), probs_ptr, T, heads, top_b, tau, w_T, w_ST,
                              loss_ptr, means_ptr, grad_ptr, ws_ptr, ws_bytes, _stream(stream)),
        "crc_cache_loss")


def crc_transfer_plan(p: crc_problem, T: int, mid_ptr, after_ptr, start_ptr, slot_expert_ptr,
                      out_ptr, max_out: int) -> int:
    n = ctypes.c_int64(0)
    _ck(load().crc_transfer_plan(ctypes.byref(p), T, mid_ptr, after_ptr, start_ptr,
                                 slot_expert_ptr, out_ptr, max_out, ctypes.byref(n)),
        "crc_transfer_plan")
    return int(n.value)


def crc_transfer_replay(p: crc_problem, plan_ptr, n: int, pool_ptr, pool_experts: int,
                        slots_ptr, stream=None):
    _ck(load().crc_transfer_replay(ctypes.byref(p), plan_ptr, n, pool_ptr, pool_experts,
                                   slots_ptr, _stream(stream)), "crc_transfer_replay")


def crc_workspace_bytes(p: crc_problem, chunk_tokens: int) -> int:
    return int(load().crc_workspace_bytes(ctypes.byref(p), chunk_tokens))


def crc_fused_workspace_bytes(p: crc_problem) -> int:
    return int(load().crc_fused_workspace_bytes(ctypes.byref(p)))


def crc_route_and_cache(p: crc_problem, hidden_ptr: int, w_ptr: int, T: int, state_ptr: int,
                        state_bytes: int, trace: crc_trace | None, ws_ptr: int, ws_bytes: int,
                        stream=None):
    _ck(load().crc_route_and_cache(ctypes.byref(p), hidden_ptr, w_ptr, T, state_ptr, state_bytes,
                                   None if trace is None else ctypes.byref(trace), ws_ptr,
                                   ws_bytes, _stream(stream)), "crc_route_and_cache")


def pinned_empty(shape, dtype):
    """A host tensor in pinned huge-page memory from crc_host_alloc, released
    with crc_host_free when the tensor (and every view of it) is gone."""
    import torch
    nbytes = math.prod(shape) * torch.empty((), dtype=dtype).element_size()
    ptr = ctypes.c_void_p()
    _ck(load().crc_host_alloc(max(nbytes, 1), ctypes.byref(ptr)), "crc_host_alloc")
    addr = ptr.value
    lib = load()

    class _Pinned(ctypes.c_uint8 * max(nbytes, 1)):
        def __del__(self):
            lib.crc_host_free(addr)

    buf = _Pinned.from_address(addr)
    return torch.frombuffer(buf, dtype=torch.uint8)[:nbytes].view(dtype).view(shape)


def crc_host_staging_bytes(p: crc_problem, chunk_tokens: int) -> int:
    return int(load().crc_host_staging_bytes(ctypes.byref(p), chunk_tokens))


def crc_route_and_cache_host(p: crc_problem, hidden_host_ptr: int, w_ptr: int, T: int,
                             chunk_tokens: int, state_ptr: int, state_bytes: int,
                             staging_ptr: int, staging_bytes: int, ws_ptr: int, ws_bytes: int,
                             stream=None):
    _ck(load().crc_route_and_cache_host(ctypes.byref(p), hidden_host_ptr, w_ptr, T, chunk_tokens,
                                        state_ptr, state_bytes, staging_ptr, staging_bytes,
                                        ws_ptr, ws_bytes, _stream(stream)),
        "crc_route_and_cache_host")


NOALLOC_SCRATCH_BYTES = 32 << 20


def crc_route_and_cache_noalloc(p: crc_problem, hidden_ptr: int, w_ptr: int, T: int,
                                state_ptr: int, state_bytes: int, trace: crc_trace | None = None,
                                stream=None):
    """crc_route_and_cache using the library's built-in scratch array (no workspace)."""
    _ck(load().crc_route_and_cache_noalloc(ctypes.byref(p), hidden_ptr, w_ptr, T, state_ptr,
                                           state_bytes,
                                           None if trace is None else ctypes.byref(trace),
                                           _stream(stream)), "crc_route_and_cache_noalloc")


def crc_device_error() -> int:
    return int(load().crc_device_error())


def crc_launch_count() -> int:
    return int(load().crc_launch_count())


def crc_profile_begin():
    _ck(load().crc_profile_begin(), "crc_profile_begin")


def crc_profile_end() -> dict:
    kt = crc_kernel_times()
    _ck(load().crc_profile_end(ctypes.byref(kt)), "crc_profile_end")
    return {k: {"launches": int(kt.launches[i]), "ms": float(kt.ms[i])}
            for k, i in KERNEL_KINDS.items()}


def crc_synth_hidden(B, T, L, d, t0, seed, rho_t, rho_l, attempts_ptr, hidden_ptr, carry_ptr,
                     stream=None):
    _ck(load().crc_synth_hidden(B, T, L, d, t0, seed, rho_t, rho_l, attempts_ptr, hidden_ptr,
                                carry_ptr, _stream(stream)), "crc_synth_hidden")


def crc_synth_weights(L, N, d, seed, copy_init, w_ptr, stream=None):
    _ck(load().crc_synth_weights(L, N, d, seed, int(copy_init), w_ptr, _stream(stream)),
        "crc_synth_weights")


# element types (crc.h CRC_BF16 ...)
BF16, F32, E4M3 = 1, 2, 3


def crc_rms_norm(x_ptr, x_stride: int, residual_ptr, weight_ptr, stream_type: int, M: int, d: int,
                 eps: float, residual_out_ptr, out_ptr, out8_ptr, scale8_ptr, rstd_ptr,
                 stream=None):
    _ck(load().crc_rms_norm(x_ptr, x_stride, residual_ptr, weight_ptr, stream_type, M, d, eps,
                            residual_out_ptr, out_ptr, out8_ptr, scale8_ptr, rstd_ptr,
                            _stream(stream)), "crc_rms_norm")


def crc_rms_norm_grad_workspace_bytes(M: int, d: int) -> int:
    return int(load().crc_rms_norm_grad_workspace_bytes(M, d))


def crc_rms_norm_grad(dy_ptr, s_ptr, weight_ptr, rstd_ptr, dres_ptr, stream_type: int, M: int,
                      d: int, dx_ptr, dw_ptr, ws_ptr, ws_bytes: int, stream=None):
    _ck(load().crc_rms_norm_grad(dy_ptr, s_ptr, weight_ptr, rstd_ptr, dres_ptr, stream_type, M, d,
                                 dx_ptr, dw_ptr, ws_ptr, ws_bytes, _stream(stream)),
        "crc_rms_norm_grad")


def crc_quantize_rows(x_ptr, x_stride: int, M: int, d: int, out8_ptr, scale8_ptr, stream=None):
    _ck(load().crc_quantize_rows(x_ptr, x_stride, M, d, out8_ptr, scale8_ptr, _stream(stream)),
        "crc_quantize_rows")


def crc_moe_workspace_bytes(m: crc_moe, M: int) -> int:
    return int(load().crc_moe_workspace_bytes(ctypes.byref(m), M))


def crc_moe_layer(m: crc_moe, x_ptr, x_stride: int, x8_ptr, x8_scale_ptr, scores_ptr,
                  scores_stride: int, M: int, out_ptr, topk_ptr, gates_ptr, ws_ptr, ws_bytes: int,
                  stream=None):
    _ck(load().crc_moe_layer(ctypes.byref(m), x_ptr, x_stride, x8_ptr, x8_scale_ptr, scores_ptr,
                             scores_stride, M, out_ptr, topk_ptr, gates_ptr, ws_ptr, ws_bytes,
                             _stream(stream)), "crc_moe_layer")


# --------------------------------------------------------------------------- #
# torch conveniences (allocation and marshalling only)
#
# `stream`: a torch stream or a raw handle; None is the current one.  Tensors that are
# made for a call (outputs, workspaces) come from its stream's pool and may be read on
# the current stream; tensors that are passed in are the caller's to keep and to order.
# --------------------------------------------------------------------------- #
def problem(L, N, K, d, C, R, B, expert_bytes) -> crc_problem:
    return crc_problem(L=L, N=N, K=K, d=d, C=C, R=R, B=B, reserved=0,
                       expert_bytes=int(expert_bytes))


def problem_of(w) -> crc_problem:
    """crc_problem from an object with fields L, N, K, d, C, R, B, expert_bytes."""
    return problem(w.L, w.N, w.K, w.d, w.C, w.R, w.B, w.expert_bytes)


class State:
    """A cache state in device memory (torch-allocated, 256-byte aligned)."""

    def __init__(self, p: crc_problem, device="cuda", stream=None):
        import torch
        self.p = p
        self.nbytes = crc_state_bytes(p)
        if self.nbytes == 0:
            raise CrcError(CRC_EINVAL, "crc_state_bytes")
        self.buf = _new(stream, torch.device(device), self.nbytes, torch.uint8)
        assert self.buf.data_ptr() % 256 == 0
        self.init(stream)

    @property
    def ptr(self) -> int:
        return self.buf.data_ptr()

    def init(self, stream=None):
        crc_state_init(self.p, self.ptr, self.nbytes, stream)

    def read(self, stream=None, **kw) -> dict:
        return crc_state_read(self.p, self.ptr, self.nbytes, stream, **kw)

    def read_aux(self, stream=None) -> np.ndarray:
        return crc_state_read_aux(self.p, self.ptr, self.nbytes, stream)


@dataclass
class Trace:
    topk: object
    misses: object
    proactive: object
    cache_mid: object = None
    cache_after: object = None
    topk_set: object = None

    @staticmethod
    def alloc(p: crc_problem, T: int, device="cuda", caches: bool = False,
              rank_order: bool = True, topk_set: bool = False) -> "Trace":
        """caches: also the cache sets after the refinement and after the update
        ([B][T][L][NW] uint32 bitmasks); rank_order=False leaves out the Top-K
        in rank order (such a trace keeps crc_route_and_cache on its fused
        kernel); topk_set: the Top-K as a [B][T][L][NW] bitmask."""
        import torch
        nw = (p.N + 31) // 32

        def words(on):
            return torch.zeros((p.B, T, p.L, nw), dtype=torch.int32, device=device) if on else None

        return Trace(torch.zeros((p.B, T, p.L, p.K), dtype=torch.uint8, device=device)
                     if rank_order else None,
                     torch.zeros((p.B, T, p.L), dtype=torch.uint8, device=device),
                     torch.zeros((p.B, T, p.L), dtype=torch.uint8, device=device),
                     words(caches), words(caches), words(topk_set))

    def c(self) -> crc_trace:
        return crc_trace(_ptr(self.topk), _ptr(self.misses), _ptr(self.proactive),
                         _ptr(self.cache_mid), _ptr(self.cache_after), _ptr(self.topk_set))


def transfer_plan(p: crc_problem, cache_mid, cache_after, slot_expert=None, start=None):
    """crc_transfer_plan for one stream: cache_mid / cache_after [T][L][NW]
    (host arrays, uint32 bit patterns).  Returns (plan, slot_expert after the
    last token); plan is a structured array of TRANSFER_DTYPE."""
    mid = np.ascontiguousarray(cache_mid).view(np.uint32)
    aft = np.ascontiguousarray(cache_after).view(np.uint32)
    T = mid.shape[0]
    se = (np.full((p.L, p.C), -1, np.int32) if slot_expert is None
          else np.ascontiguousarray(slot_expert, dtype=np.int32).copy())
    st = None if start is None else np.ascontiguousarray(start).view(np.uint32)
    args = (mid.ctypes.data, aft.ctypes.data, None if st is None else st.ctypes.data)
    scratch = se.copy()                      # the counting pass moves a copy of the map
    n = crc_transfer_plan(p, T, *args, scratch.ctypes.data, None, 0)
    plan = np.zeros(n, TRANSFER_DTYPE)
    crc_transfer_plan(p, T, *args, se.ctypes.data, plan.ctypes.data if n else None, n)
    return plan, se


def transfer_replay(p: crc_problem, plan, pool, slots, pool_experts=None, stream=None):
    """crc_transfer_replay: pool a pinned host tensor of pool_experts expert
    images (default: all of it), slots a device tensor [L][C][expert_bytes]."""
    plan = np.ascontiguousarray(plan, dtype=TRANSFER_DTYPE)
    nbytes = pool.numel() * pool.element_size()
    pe = pool_experts or nbytes // int(p.expert_bytes)
    crc_transfer_replay(p, plan.ctypes.data if len(plan) else None, len(plan), pool.data_ptr(),
                        pe, slots.data_ptr(), stream)


def route_scores(p: crc_problem, hidden, w_cat, heads: int = 3, out=None, stream=None):
    import torch
    B, T, L, d = hidden.shape
    if out is None:
        out = _new(stream, hidden.device, (B, T, L, 3, p.N), torch.float32)
    crc_route_scores(p, hidden.data_ptr(), w_cat.data_ptr(), T, heads, out.data_ptr(), stream)
    return out


def cache_scan(p: crc_problem, scores, state: State, trace: Trace | None = None, stream=None):
    T = scores.shape[1]
    crc_cache_scan(p, scores.data_ptr(), T, state.ptr, state.nbytes,
                   None if trace is None else trace.c(), stream)


def cache_scan_policy(p: crc_problem, scores, state: State, policy, trace: Trace | None = None,
                      lambda_halves: int = 1, stream=None):
    """crc_cache_scan_policy: policy is a CRC_POLICY_* value or one of POLICIES."""
    T = scores.shape[1]
    code = POLICIES[policy] if isinstance(policy, str) else int(policy)
    crc_cache_scan_policy(p, scores.data_ptr(), T, state.ptr, state.nbytes,
                          None if trace is None else trace.c(), code, lambda_halves, stream)


def cache_loss(p: crc_problem, probs, top_b: int, tau: float, w_T: float = 1.0,
               w_ST: float = 1.0, heads: int = 3, grad: bool = True, loss=None, means=None,
               grad_out=None, workspace=None, stream=None):
    """crc_cache_loss over probs [B][T][L][3][N] (fp32, on the device).

    Returns (loss [B][T][L][2] fp32, means [2] fp64 = (L_T, L_ST), grad
    [B][T][L][3][N] fp32 or None); pass preallocated tensors to reuse them."""
    import torch
    B, T, L, H, N = probs.shape
    dev = probs.device
    if loss is None:
        loss = _new(stream, dev, (B, T, L, 2), torch.float32)
    if means is None:
        means = _new(stream, dev, 2, torch.float64)
    if grad and grad_out is None:
        grad_out = _new(stream, dev, (B, T, L, 3, N), torch.float32, zeros=True)
    if workspace is None:
        workspace = _new(stream, dev, max(crc_loss_workspace_bytes(p, T), 256), torch.uint8)
    crc_cache_loss(p, probs.data_ptr(), T, heads, top_b, tau, w_T, w_ST, loss.data_ptr(),
                   means.data_ptr(), grad_out.data_ptr() if grad else None, workspace.data_ptr(),
                   workspace.numel(), stream)
    return loss, means, (grad_out if grad else None)


def route_and_cache(p: crc_problem, hidden, w_cat, state: State, trace: Trace | None = None,
                    workspace=None, stream=None):
    T = hidden.size(1)
    if workspace is None:
        import torch
        workspace = _new(stream, hidden.device, crc_workspace_bytes(p, T), torch.uint8)
    crc_route_and_cache(p, hidden.data_ptr(), w_cat.data_ptr(), T, state.buf.data_ptr(),
                        state.nbytes, None if trace is None else trace.c(),
                        workspace.data_ptr(), workspace.nbytes, stream)
    return workspace


def route_and_cache_host(p: crc_problem, hidden_host, w_cat, state: State, chunk_tokens=128,
                         staging=None, workspace=None, stream=None):
    """The step on hidden states [B][T][L][d] bf16 held in (pinned) host memory:
    chunked copies overlapped with the fused step.  Returns (staging, workspace)
    for reuse; neither may be reused before `stream` has passed this call."""
    import torch
    if hidden_host.device.type != "cpu" or not hidden_host.is_contiguous():
        raise ValueError("hidden_host must be a contiguous host tensor")
    T = hidden_host.shape[1]
    dev = w_cat.device
    chunk = max(1, min(chunk_tokens, T))
    if staging is None:
        staging = _new(stream, dev, crc_host_staging_bytes(p, chunk), torch.uint8)
    if workspace is None:
        workspace = _new(stream, dev, crc_fused_workspace_bytes(p), torch.uint8)
    crc_route_and_cache_host(p, hidden_host.data_ptr(), w_cat.data_ptr(), T, chunk_tokens,
                             state.ptr, state.nbytes, staging.data_ptr(),
                             staging.numel() * staging.element_size(), workspace.data_ptr(),
                             workspace.numel() * workspace.element_size(), stream)
    return staging, workspace


def synth_weights(L, N, d, seed=0, copy_init=False, device="cuda", stream=None):
    import torch
    w = _new(stream, torch.device(device), (L, 3 * N, d), torch.bfloat16)
    crc_synth_weights(L, N, d, seed, copy_init, w.data_ptr(), stream)
    return w


def synth_hidden(B, T, L, d, seed=0, rho_t=0.9, rho_l=0.8, t0=0, carry=None, attempts=None,
                 out=None, device="cuda", stream=None):
    """Tokens [t0, t0+T) of the synthetic hidden-state field; returns (hidden, carry)."""
    import torch
    if out is None:
        out = _new(stream, torch.device(device), (B, T, L, d), torch.bfloat16)
    if carry is None:
        carry = _new(stream, torch.device(device), (B, L, d), torch.float32, zeros=True)
    crc_synth_hidden(B, T, L, d, t0, seed, rho_t, rho_l, _ptr(attempts), out.data_ptr(),
                     carry.data_ptr(), stream)
    return out, carry


def _stream_type(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise ValueError(f"the residual stream is bfloat16 or float32, not {t.dtype}")


def _here(t, name: str) -> int:
    """The current device, where calls are launched; `t` has to lie there."""
    import torch
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{name} must be a CUDA tensor")
    # not torch.cuda.current_device(): t shows that CUDA is up, and a call takes 8 us in all
    if dev != torch._C._cuda_getDevice():
        raise ValueError(f"{name} lies on {t.device}, which is not the current device")
    return dev


def _check(t, name: str, shape, dtype, dev: int, dense: bool = True):
    """The address of a tensor argument of the stated shape and type on device `dev`, or
    None.  (Short on purpose: a one-row norm has six of them, and takes the GPU 2 us.)"""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev:
        raise ValueError(f"{name}: a {dtype} tensor of shape {tuple(shape)} on cuda:{dev} is "
                         f"wanted, got {t.dtype} {tuple(t.shape)} on {t.device}")
    if dense and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _workspace(t, dev: int):
    """Address and bytes of a workspace: any contiguous tensor on device `dev`."""
    if t is None:
        return None, 0
    if t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on cuda:{dev}")
    return t.data_ptr(), t.nbytes


def _rows(t, name: str):
    """(rows, elements a row, elements between rows) of a 2-D tensor."""
    if t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D tensor")
    M, d = t.shape
    if t.stride(1) != 1 and d != 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    return M, d, (t.stride(0) if M > 1 else (d + 7) // 8 * 8)


def rms_norm(x, weight, eps: float = 1e-6, residual=None, residual_out=None, out=None, out8=None,
             scale8=None, rstd=None, stream=None):
    """crc_rms_norm on rows x [M][d] (bf16 or fp32, rows may be strided).

    Writes y = norm(x + residual) * weight to `out` (bf16; made when no output is
    given), to out8 / scale8 (float8_e4m3fn and fp32 [M]) if given, x + residual to
    residual_out and the rows' statistic to rstd (fp32 [M]).  Returns out."""
    import torch
    bf16, f32, dtype = torch.bfloat16, torch.float32, x.dtype
    dev = _here(x, "x")
    M, d, ldx = _rows(x, "x")
    if out is None and out8 is None:
        out = _new(stream, x.device, (M, d), bf16)
    rows = x.shape
    rc = load().crc_rms_norm(
        x.data_ptr(), ldx, _check(residual, "residual", rows, dtype, dev),
        _check(weight, "weight", (d,), bf16, dev), _stream_type(x), M, d, eps,
        _check(residual_out, "residual_out", rows, dtype, dev), _check(out, "out", rows, bf16, dev),
        _check(out8, "out8", rows, torch.float8_e4m3fn, dev),
        _check(scale8, "scale8", (M,), f32, dev), _check(rstd, "rstd", (M,), f32, dev),
        _stream(stream, dev))
    if rc:
        raise CrcError(rc, "crc_rms_norm")
    return out


def rms_norm_grad(dy, s, weight, rstd, dres=None, dx=None, dw=None, want_dw: bool = True,
                  workspace=None, stream=None):
    """crc_rms_norm_grad: (dx, dw) from dy (bf16), s = x + residual and rstd of the
    forward call, and dres, the gradient that arrives at s directly."""
    import torch
    M, d = rows = dy.shape
    dev = _here(dy, "dy")
    bf16, f32 = torch.bfloat16, torch.float32
    if dx is None:
        dx = _new(stream, s.device, s.shape, s.dtype)
    if want_dw and dw is None:
        dw = _new(stream, dy.device, d, f32)
    if dw is not None and workspace is None:
        workspace = _new(stream, dy.device, crc_rms_norm_grad_workspace_bytes(M, d), torch.uint8)
    crc_rms_norm_grad(_check(dy, "dy", rows, bf16, dev), _check(s, "s", rows, s.dtype, dev),
                      _check(weight, "weight", (d,), bf16, dev),
                      _check(rstd, "rstd", (M,), f32, dev),
                      _check(dres, "dres", rows, s.dtype, dev), _stream_type(s), M, d,
                      _check(dx, "dx", rows, s.dtype, dev), _check(dw, "dw", (d,), f32, dev),
                      *_workspace(workspace, dev), _stream(stream, dev))
    return dx, dw


def quantize_rows(x, out8=None, scale=None, stream=None):
    """crc_quantize_rows: bf16 rows [..][d] as (float8_e4m3fn, fp32 scale a row).
    A 2-D x may have strided rows; more dimensions must be contiguous."""
    import torch
    if x.dtype != torch.bfloat16:
        raise ValueError("x must be bfloat16")
    dev = _here(x, "x")
    lead, d = x.shape[:-1], x.shape[-1]
    if x.dim() != 2:
        if not x.is_contiguous():
            raise ValueError("x must be contiguous, or have two dimensions")
        x = x.reshape(-1, d)
    M, d, ldx = _rows(x, "x")
    if out8 is None:
        out8 = _new(stream, x.device, (*lead, d), torch.float8_e4m3fn)
    if scale is None:
        scale = _new(stream, x.device, lead, torch.float32)
    crc_quantize_rows(x.data_ptr(), ldx, M, d,
                      _check(out8, "out8", (*lead, d), torch.float8_e4m3fn, dev),
                      _check(scale, "scale", lead, torch.float32, dev), _stream(stream, dev))
    return out8, scale


def expert_views(slots, f: int, d: int):
    """The matrices in the expert slots [C][3 * f * d] of one layer (bf16 or
    float8_e4m3fn elements, e.g. `slots_dev[l]` of transfer_replay viewed in that
    type): gate_up [C][2][f][d] and down [C][d][f], views of the slots."""
    C, n = slots.shape
    if n < 3 * f * d or (slots.stride(1) != 1):
        raise ValueError("a slot holds 3 * f * d contiguous elements")
    st = slots.stride(0)
    gate_up = slots.as_strided((C, 2, f, d), (st, f * d, d, 1))
    down = slots.as_strided((C, d, f), (st, f, 1), slots.storage_offset() + 2 * f * d)
    return gate_up, down


class MoeLayer:
    """One layer's experts for crc_moe_layer: gate_up [slots][2][f][d] and down
    [slots][d][f], bf16, or float8_e4m3fn with gate_up_scale [slots][2][f] and
    down_scale [slots][d] (the slots may be strided, see expert_views); router
    bf16 [N][d]; expert_slot int32 [N] (None: expert e is in slot e).  Keeps
    references to all of them and no copy: what is written to them later (an
    expert copied to a slot, a new expert_slot map) counts from the next call."""

    def __init__(self, gate_up, down, K: int, router=None, expert_slot=None, gate_up_scale=None,
                 down_scale=None, renormalize: bool = True, N: int | None = None):
        import torch
        if gate_up.dim() != 4 or gate_up.shape[1] != 2:
            raise ValueError("gate_up has the shape [slots][2][f][d]")
        slots, _, f, d = gate_up.shape
        kinds = {torch.bfloat16: BF16, torch.float8_e4m3fn: E4M3}
        if gate_up.dtype not in kinds or not gate_up.is_cuda:
            raise ValueError("gate_up must be a bfloat16 or float8_e4m3fn CUDA tensor")
        dev = gate_up.get_device()
        _check(down, "down", (slots, d, f), gate_up.dtype, dev, dense=False)
        if gate_up.stride()[1:] != (f * d, d, 1) or down.stride()[1:] != (f, 1):
            raise ValueError("an expert's matrices must be contiguous")
        if N is None:
            N = (router.shape[0] if router is not None else
                 expert_slot.shape[0] if expert_slot is not None else slots)
        _check(router, "router", (N, d), torch.bfloat16, dev)
        _check(expert_slot, "expert_slot", (N,), torch.int32, dev)
        if expert_slot is None and N > slots:
            raise ValueError("more experts than slots: an expert_slot map is wanted")
        for t, name, shape in ((gate_up_scale, "gate_up_scale", (slots, 2, f)),
                               (down_scale, "down_scale", (slots, d))):
            if (t is None) != (gate_up.dtype == torch.bfloat16):
                raise ValueError(f"{name} belongs to 8-bit experts")
            _check(t, name, shape, torch.float32, dev, dense=False)
        if gate_up_scale is not None and (gate_up_scale.stride()[1:] != (f, 1)
                                          or down_scale.stride(1) != 1):
            raise ValueError("an expert's scales must be contiguous")
        es = gate_up.element_size()
        self.N, self.K, self.d, self.f, self.device = N, K, d, f, dev
        self.tensors = (gate_up, down, router, expert_slot, gate_up_scale, down_scale)
        self.c = crc_moe(N=N, K=K, d=d, f=f, slots=slots, weight_type=kinds[gate_up.dtype],
                         renormalize=int(renormalize), reserved=0,
                         gate_up_dev=gate_up.data_ptr(), down_dev=down.data_ptr(),
                         gate_up_stride=gate_up.stride(0) * es, down_stride=down.stride(0) * es,
                         gate_up_scale_dev=_ptr(gate_up_scale), down_scale_dev=_ptr(down_scale),
                         gate_up_scale_stride=0 if gate_up_scale is None
                         else gate_up_scale.stride(0) * 4,
                         down_scale_stride=0 if down_scale is None else down_scale.stride(0) * 4,
                         router_dev=_ptr(router), expert_slot_dev=_ptr(expert_slot))
        self._ref = ctypes.byref(self.c)
        if self.workspace_bytes(1) == 0:
            raise CrcError(CRC_EUNSUPPORTED, "crc_moe_workspace_bytes")

    def workspace_bytes(self, M: int) -> int:
        return crc_moe_workspace_bytes(self.c, M)

    def __call__(self, x, out=None, x8=None, x_scale=None, scores=None, topk=None, gates=None,
                 workspace=None, stream=None):
        """out [M][d] of rows x [M][d] (bf16, rows may be strided); x8 / x_scale:
        the rows in 8 bits for the experts; scores: fp32 probabilities [M][N] (rows
        may be strided) in place of the router; topk (uint8) and gates (fp32)
        [M][K] are written if given.  x may be None when x8 and scores are given."""
        import torch
        src = x if x is not None else x8
        if src is None:
            raise ValueError("x or x8 is wanted")
        dev = _here(src, "x")
        if dev != self.device:
            raise ValueError(f"x lies on cuda:{dev}, the experts on cuda:{self.device}")
        M, _, ldx = _rows(src, "x")
        rows, f32 = (M, self.d), torch.float32
        lds = 0 if scores is None else _rows(scores, "scores")[2]
        if out is None:
            out = _new(stream, src.device, rows, torch.bfloat16)
        if workspace is None:
            workspace = _new(stream, src.device, self.workspace_bytes(M), torch.uint8)
        rc = load().crc_moe_layer(
            self._ref, _check(x, "x", rows, torch.bfloat16, dev, False), ldx,
            _check(x8, "x8", rows, torch.float8_e4m3fn, dev),
            _check(x_scale, "x_scale", (M,), f32, dev),
            _check(scores, "scores", (M, self.N), f32, dev, False), lds, M,
            _check(out, "out", rows, torch.bfloat16, dev),
            _check(topk, "topk", (M, self.K), torch.uint8, dev),
            _check(gates, "gates", (M, self.K), f32, dev), *_workspace(workspace, dev),
            _stream(stream, dev))
        if rc:
            raise CrcError(rc, "crc_moe_layer")
        return out


def _stats_struct(stats: dict) -> crc_stats:
    st = crc_stats()
    for f, _ in crc_stats._fields_:
        if f in stats and f != "reserved":
            setattr(st, f, int(stats[f]))
    return st


def load_time(stats: dict, p: crc_problem, c_exp: float, eta: float) -> float:
    """crc_load_time: exposed expert-loading cost per decode token under the
    paper's overlap model, from the totals of crc_state_read (a dict as
    returned by State.read)."""
    if not 0.0 <= eta <= 1.0:
        raise ValueError("eta must lie in [0, 1]")
    out = ctypes.c_double()
    _ck(load().crc_load_time(ctypes.byref(p), ctypes.byref(_stats_struct(stats)), c_exp, eta,
                             ctypes.byref(out)), "crc_load_time")
    return out.value


def metrics(stats: dict, p: crc_problem) -> dict:
    """crc_metrics: Hit, AdjHit, traffic and Load/token (bytes per decode
    token) of Sec. 4.1 from the totals of crc_state_read."""
    r = crc_report()
    _ck(load().crc_metrics(ctypes.byref(p), ctypes.byref(_stats_struct(stats)), ctypes.byref(r)),
        "crc_metrics")
    return {"hit": r.hit, "adj_hit": r.adj_hit, "traffic_bytes": r.traffic_bytes,
            "load_per_token_bytes": r.load_per_token_bytes}
