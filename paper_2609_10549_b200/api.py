"""ctypes binding of libcompass.so: same names as the C ABI, argument
marshalling only.  torch provides device memory and streams; every step of the
path runs inside the library.  There is no fallback: if the library is missing
the first call raises.
"""
from __future__ import annotations

import ctypes as C
import os
import sys
from array import array
from dataclasses import dataclass
from typing import List, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcompass.so")

OK, ERR_INVALID_ARG, ERR_SHAPE, ERR_UNSUPPORTED, ERR_ALIGNMENT, ERR_BUFFER_TOO_SMALL, ERR_CUDA, ERR_TIMEOUT = range(8)
ERR_SCRATCH_LIMIT = 8
NOALLOC_SCRATCH_BYTES = 32 * 1024 * 1024
OP_AG_GEMM, OP_GEMM_RS = 0, 1
DTYPE_BF16, DTYPE_FP32, DTYPE_E4M3, DTYPE_E5M2 = range(4)
INDEX_INT64, INDEX_INT32 = 0, 1
RS_SEGMENTED_K, RS_RING_RMW, RS_RING_RMW_F32 = 0, 1, 2
STRATEGY_INTRAFUSION, STRATEGY_INTERDECOM = 0, 1
ORDER_RANK_MAJOR, ORDER_STEP_MAJOR = 0, 1
COPY_KERNEL, COPY_ENGINES = 0, 1
WS_FUSED, WS_DECOMP, WS_PUSH = 0, 1, 2
ACT_NONE, ACT_GELU_TANH, ACT_SWIGLU = 0, 1, 2
B_NK, B_KN = 0, 1
MAX_P = 16
STATUS_BYTES = 256

# every symbol include/compass.h declares
EXPORTS = (
    "compass_schedule", "compass_ag_gemm", "compass_gemm_rs", "compass_decomp", "compass_select",
    "compass_model_decomp_time", "compass_model_optimal_degree", "compass_model_fusion_time",
    "compass_calib_fit_decomp", "compass_calib_fit_fusion", "compass_workspace_bytes", "compass_workspace_init",
    "compass_read_status", "compass_launch_plan", "compass_fused_host", "compass_status_string",
    "compass_last_cuda_error", "compass_kernel_launch_count", "compass_gemm_rs_sequential_noalloc",
    "compass_set_wait_limit_us", "compass_calib_fit_line", "compass_ag_gemm_push", "compass_read_kernel_clock",
    "compass_mlp_workspace_bytes", "compass_mlp_block", "compass_noalloc_read_status", "compass_select_ex", "compass_test_drop_flag_writes", "compass_tensor_map_cache_stats", "compass_decomp_comm", "compass_tile_plan",
    "compass_embedding", "compass_embedding_workspace_bytes", "compass_embedding_backward",
    "compass_layer_norm", "compass_layer_norm_workspace_bytes", "compass_layer_norm_backward",
    "compass_head_workspace_bytes", "compass_head_loss", "compass_head_loss_backward",
    "compass_rms_norm", "compass_rms_norm_workspace_bytes", "compass_rms_norm_backward", "compass_quantize", "compass_dequantize",
    "compass_8bit_workspace_bytes", "compass_ag_gemm_8bit", "compass_gemm_rs_8bit", "compass_weight_grad_8bit",
)


class CompassError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status}, cuda error {last_cuda_error()})")


class Problem(C.Structure):
    _fields_ = [("op", C.c_int32), ("P", C.c_int32), ("rings", C.c_int32), ("d", C.c_int32),
                ("M", C.c_int64), ("N", C.c_int64), ("K", C.c_int64),
                ("dtype", C.c_int32), ("rs_variant", C.c_int32), ("order", C.c_int32), ("copy_mode", C.c_int32),
                ("b_layout", C.c_int32), ("ring_group", C.c_int32)]


class Mlp(C.Structure):
    _fields_ = [("P", C.c_int32), ("rings", C.c_int32), ("M", C.c_int64), ("hidden", C.c_int64), ("ffn", C.c_int64),
                ("activation", C.c_int32), ("rs_variant", C.c_int32), ("order", C.c_int32), ("b_layout", C.c_int32)]


class Embed(C.Structure):
    _fields_ = [("P", C.c_int32), ("dtype", C.c_int32), ("grad_dtype", C.c_int32), ("index_dtype", C.c_int32),
                ("M", C.c_int64), ("hidden", C.c_int64), ("vocab", C.c_int64), ("scale", C.c_float), ("accumulate", C.c_int32)]


class Norm(C.Structure):
    _fields_ = [("P", C.c_int32), ("dtype", C.c_int32), ("param_dtype", C.c_int32), ("eps", C.c_float),
                ("M", C.c_int64), ("hidden", C.c_int64)]


class Head(C.Structure):
    _fields_ = [("P", C.c_int32), ("dtype", C.c_int32), ("grad_dtype", C.c_int32), ("index_dtype", C.c_int32),
                ("M", C.c_int64), ("hidden", C.c_int64), ("vocab", C.c_int64), ("logit_scale", C.c_float),
                ("label_smoothing", C.c_float)]


class Quant(C.Structure):
    _fields_ = [("P", C.c_int32), ("dtype", C.c_int32), ("format", C.c_int32), ("block_rows", C.c_int32),
                ("M", C.c_int64), ("cols", C.c_int64)]


class SchedEntry(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rank", "step", "ring", "part", "chunk", "peer", "row_begin", "row_count")]


class Calib(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("comp_a", "comp_b", "comm_a", "comm_b",
                                           "alpha_decomp", "beta_decomp", "alpha_fusion", "beta_fusion")]


class Choice(C.Structure):
    _fields_ = [("strategy", C.c_int32), ("d_star", C.c_int32), ("t_fusion", C.c_double), ("t_decomp", C.c_double),
                ("t_comp", C.c_double), ("t_comm", C.c_double), ("lam", C.c_double), ("t_star", C.c_double)]


class TileCounts(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("cta_pairs", "blocks", "rows_per_block", "blocks_per_group", "tiles_512x256",
                                          "tiles_256x256", "tiles_256x128", "tiles_128x256", "total_tiles")]


class PlanBlock(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rank", "step", "ring", "part", "a_tensor", "a_row_begin", "out_tensor",
                                          "out_row_begin", "rows", "first_tile", "tile_count")]


_lib: Optional[C.CDLL] = None


def _torch_device() -> int:
    import torch
    return torch.cuda.current_device()


_raw_stream = None                        # torch's getter of the current stream's handle, once the library is loaded
_current_device = _torch_device           # and of the current device


def lib() -> C.CDLL:
    global _lib, _raw_stream, _current_device
    if _lib is None:
        torch = sys.modules.get("torch")
        if torch is not None:
            _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
            _current_device = getattr(torch._C, "_cuda_getDevice", _torch_device)
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_10549_b200.build` "
                               "(there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        pp = C.POINTER(C.c_void_p)
        L.compass_schedule.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int64, C.POINTER(SchedEntry), C.c_size_t,
                                       C.POINTER(C.c_size_t)]
        for name in ("compass_ag_gemm", "compass_gemm_rs"):
            getattr(L, name).argtypes = [C.POINTER(Problem), pp, pp, pp, C.c_void_p, C.c_size_t, C.c_void_p]
        L.compass_decomp.argtypes = [C.POINTER(Problem), pp, pp, pp, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        L.compass_decomp_comm.argtypes = [C.POINTER(Problem), pp, pp, pp, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        L.compass_ag_gemm_push.argtypes = [C.POINTER(Problem), pp, pp, pp, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        L.compass_mlp_workspace_bytes.argtypes = [C.POINTER(Mlp), C.POINTER(C.c_size_t)]
        L.compass_mlp_block.argtypes = [C.POINTER(Mlp), pp, pp, pp, pp, pp, C.c_void_p, C.c_size_t, C.c_void_p]
        L.compass_select.argtypes = [C.POINTER(Problem), C.POINTER(Calib), C.POINTER(Choice)]
        L.compass_select_ex.argtypes = [C.POINTER(Problem), C.POINTER(Calib), C.c_int, C.POINTER(Choice)]
        L.compass_model_decomp_time.argtypes = [C.c_double] * 4 + [C.c_int, C.POINTER(C.c_double)]
        L.compass_model_optimal_degree.argtypes = [C.c_double] * 4 + [C.c_int, C.c_int, C.POINTER(C.c_int),
                                                                       C.POINTER(C.c_double)]
        L.compass_model_fusion_time.argtypes = [C.c_double, C.c_double, C.c_int, C.c_double, C.c_double, C.c_double,
                                                C.POINTER(C.c_double)]
        dp, ip = C.POINTER(C.c_double), C.POINTER(C.c_int)
        L.compass_calib_fit_decomp.argtypes = [dp, dp, ip, dp, C.c_size_t, dp, dp]
        L.compass_calib_fit_fusion.argtypes = [dp, dp, ip, dp, dp, C.c_size_t, dp, dp]
        L.compass_calib_fit_line.argtypes = [dp, dp, C.c_size_t, dp, dp]
        L.compass_workspace_bytes.argtypes = [C.POINTER(Problem), C.c_int, C.POINTER(C.c_size_t)]
        L.compass_workspace_init.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p]
        L.compass_read_status.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_int)]
        L.compass_read_kernel_clock.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_uint64), C.POINTER(C.c_uint64)]
        L.compass_launch_plan.argtypes = [C.POINTER(Problem), C.POINTER(PlanBlock), C.c_size_t, C.POINTER(C.c_size_t)]
        L.compass_tile_plan.argtypes = [C.POINTER(Problem), C.c_int, C.c_int, C.POINTER(TileCounts)]
        L.compass_fused_host.argtypes = [C.POINTER(Problem), pp, pp, pp, C.c_void_p, C.c_size_t, C.POINTER(C.c_size_t),
                                         C.c_void_p, C.c_size_t, C.c_void_p]
        L.compass_gemm_rs_sequential_noalloc.argtypes = [C.POINTER(Problem), pp, pp, pp, C.c_void_p]
        L.compass_noalloc_read_status.argtypes = [C.c_void_p, C.POINTER(C.c_int)]
        vp = C.c_void_p
        L.compass_embedding.argtypes = [C.POINTER(Embed), vp, pp, pp, vp]
        L.compass_embedding_workspace_bytes.argtypes = [C.POINTER(Embed), C.POINTER(C.c_size_t)]
        L.compass_embedding_backward.argtypes = [C.POINTER(Embed), vp, pp, pp, vp, C.c_size_t, vp]
        L.compass_layer_norm.argtypes = [C.POINTER(Norm), pp, pp, vp, vp, pp, pp, vp, vp, vp]
        L.compass_layer_norm_workspace_bytes.argtypes = [C.POINTER(Norm), C.POINTER(C.c_size_t)]
        L.compass_layer_norm_backward.argtypes = [C.POINTER(Norm), pp, pp, vp, vp, vp, pp, pp, vp, vp, vp, C.c_size_t, vp]
        L.compass_head_workspace_bytes.argtypes = [C.POINTER(Head), C.c_int, C.POINTER(C.c_size_t)]
        L.compass_head_loss.argtypes = [C.POINTER(Head), pp, pp, vp, vp, vp, vp, C.c_size_t, vp]
        L.compass_head_loss_backward.argtypes = [C.POINTER(Head), pp, pp, vp, vp, vp, pp, pp, vp, C.c_size_t, vp]
        # (arrays of pointers by their address: several lie in one)
        L.compass_rms_norm.argtypes = [C.POINTER(Norm), vp, vp, vp, vp, vp, C.c_int, vp, vp, vp, vp]
        L.compass_rms_norm_workspace_bytes.argtypes = [C.POINTER(Norm), C.POINTER(C.c_size_t)]
        L.compass_rms_norm_backward.argtypes = [C.POINTER(Norm), vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.compass_quantize.argtypes = L.compass_dequantize.argtypes = [C.POINTER(Quant), vp, vp, vp, vp]
        L.compass_8bit_workspace_bytes.argtypes = [C.POINTER(Problem), C.POINTER(C.c_size_t)]
        for name in ("compass_ag_gemm_8bit", "compass_gemm_rs_8bit"):
            getattr(L, name).argtypes = [C.POINTER(Problem), vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.compass_weight_grad_8bit.argtypes = [C.POINTER(Problem), C.c_int, C.c_int, vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.compass_set_wait_limit_us.argtypes = [C.c_uint32]
        L.compass_test_drop_flag_writes.argtypes = [C.c_int]
        L.compass_tensor_map_cache_stats.argtypes = [C.POINTER(C.c_uint64), C.POINTER(C.c_uint64)]
        L.compass_status_string.argtypes = [C.c_int]
        L.compass_status_string.restype = C.c_char_p
        L.compass_last_cuda_error.restype = C.c_int
        L.compass_kernel_launch_count.restype = C.c_uint64
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().compass_status_string(int(status)).decode()


def last_cuda_error() -> int:
    return int(lib().compass_last_cuda_error())


def compass_set_wait_limit_us(microseconds: int) -> None:
    _check(lib().compass_set_wait_limit_us(int(microseconds)), "compass_set_wait_limit_us")


def compass_test_drop_flag_writes(count: int) -> None:
    _check(lib().compass_test_drop_flag_writes(int(count)), "compass_test_drop_flag_writes")


def tensor_map_cache_stats():
    """(hits, misses) of the library's table of encoded TMA tensor maps since it was loaded."""
    hits, misses = C.c_uint64(0), C.c_uint64(0)
    _check(lib().compass_tensor_map_cache_stats(C.byref(hits), C.byref(misses)), "compass_tensor_map_cache_stats")
    return int(hits.value), int(misses.value)


def kernel_launch_count() -> int:
    return int(lib().compass_kernel_launch_count())


def _check(status: int, where: str) -> None:
    if status != OK:
        raise CompassError(status, where)


def make_problem(op: int, P: int, M: int, N: int, K: int, rings: int = 2, d: int = 1,
                 rs_variant: int = RS_SEGMENTED_K, dtype: int = DTYPE_BF16, order: int = ORDER_RANK_MAJOR,
                 copy_mode: int = COPY_KERNEL, b_layout: int = B_NK, ring_group: int = 0) -> Problem:
    return Problem(op=op, P=P, rings=rings, d=d, M=M, N=N, K=K, dtype=dtype, rs_variant=rs_variant, order=order,
                   copy_mode=copy_mode, b_layout=b_layout, ring_group=ring_group)


# ---- host-only calls -------------------------------------------------------------

def compass_schedule(op: int, P: int, rings: int, M: int) -> np.ndarray:
    """Returns the schedule as an int32 array [count, 8] (columns as in compass_sched_entry)."""
    n = C.c_size_t(0)
    _check(lib().compass_schedule(op, P, rings, M, None, 0, C.byref(n)), "compass_schedule")
    buf = (SchedEntry * n.value)()
    _check(lib().compass_schedule(op, P, rings, M, buf, n.value, C.byref(n)), "compass_schedule")
    return np.frombuffer(buf, dtype=np.int32).reshape(n.value, 8).copy()


def compass_select(problem: Problem, calib: Calib, eq5_as_printed: bool = False) -> Choice:
    out = Choice()
    if eq5_as_printed:
        _check(lib().compass_select_ex(C.byref(problem), C.byref(calib), 1, C.byref(out)), "compass_select_ex")
    else:
        _check(lib().compass_select(C.byref(problem), C.byref(calib), C.byref(out)), "compass_select")
    return out


def compass_model_decomp_time(t_comp: float, t_comm: float, alpha: float, beta: float, d: int) -> float:
    out = C.c_double()
    _check(lib().compass_model_decomp_time(t_comp, t_comm, alpha, beta, d, C.byref(out)), "compass_model_decomp_time")
    return out.value


def compass_model_optimal_degree(t_comp: float, t_comm: float, alpha: float, beta: float, d_max: int = 16,
                                 as_printed: bool = False):
    d, x = C.c_int(), C.c_double()
    _check(lib().compass_model_optimal_degree(t_comp, t_comm, alpha, beta, d_max, int(as_printed), C.byref(d),
                                              C.byref(x)), "compass_model_optimal_degree")
    return d.value, (x.value if x.value >= 0 else None)


def compass_model_fusion_time(t_comp: float, t_comm: float, n_chunks: int, alpha_f: float, beta_f: float,
                              m_volume: float) -> float:
    out = C.c_double()
    _check(lib().compass_model_fusion_time(t_comp, t_comm, n_chunks, alpha_f, beta_f, m_volume, C.byref(out)),
           "compass_model_fusion_time")
    return out.value


def _darr(xs):
    return (C.c_double * len(xs))(*[float(x) for x in xs])


def _iarr(xs):
    return (C.c_int * len(xs))(*[int(x) for x in xs])


def compass_calib_fit_decomp(t_comp, t_comm, d, t_measured):
    a, b = C.c_double(), C.c_double()
    _check(lib().compass_calib_fit_decomp(_darr(t_comp), _darr(t_comm), _iarr(d), _darr(t_measured), len(d),
                                          C.byref(a), C.byref(b)), "compass_calib_fit_decomp")
    return a.value, b.value


def compass_calib_fit_line(x, y):
    a, b = C.c_double(), C.c_double()
    _check(lib().compass_calib_fit_line(_darr(x), _darr(y), len(x), C.byref(a), C.byref(b)), "compass_calib_fit_line")
    return a.value, b.value


def compass_calib_fit_fusion(t_comp, t_comm, n_chunks, m_volume, t_measured):
    a, b = C.c_double(), C.c_double()
    _check(lib().compass_calib_fit_fusion(_darr(t_comp), _darr(t_comm), _iarr(n_chunks), _darr(m_volume),
                                          _darr(t_measured), len(n_chunks), C.byref(a), C.byref(b)),
           "compass_calib_fit_fusion")
    return a.value, b.value


def compass_workspace_bytes(problem: Problem, which: int = WS_FUSED) -> int:
    n = C.c_size_t(0)
    _check(lib().compass_workspace_bytes(C.byref(problem), which, C.byref(n)), "compass_workspace_bytes")
    return int(n.value)


def compass_tile_plan(problem: Problem, decomposed: bool = False, cta_pairs: int = 74) -> TileCounts:
    out = TileCounts()
    _check(lib().compass_tile_plan(C.byref(problem), int(decomposed), int(cta_pairs), C.byref(out)), "compass_tile_plan")
    return out


def compass_launch_plan(problem: Problem) -> List[PlanBlock]:
    n = C.c_size_t(0)
    _check(lib().compass_launch_plan(C.byref(problem), None, 0, C.byref(n)), "compass_launch_plan")
    buf = (PlanBlock * n.value)()
    _check(lib().compass_launch_plan(C.byref(problem), buf, n.value, C.byref(n)), "compass_launch_plan")
    return list(buf)


# ---- device calls (torch tensors supply the memory) ------------------------------

def _ptr_array(tensors: Sequence) -> C.Array:
    return (C.c_void_p * len(tensors))(*[int(t.data_ptr()) for t in tensors])


def _stream_handle(stream, here: Optional[int] = None) -> C.c_void_p:
    if stream is None:
        if _raw_stream is not None:       # torch.cuda.current_stream() builds an object around it, several microseconds a call
            return C.c_void_p(_raw_stream(_current_device() if here is None else here))
        import torch
        stream = torch.cuda.current_stream()
    return C.c_void_p(int(stream.cuda_stream))


def _ws(workspace):
    return C.c_void_p(int(workspace.data_ptr())), int(workspace.numel() * workspace.element_size())


def compass_workspace_init(workspace, stream=None) -> None:
    p, n = _ws(workspace)
    _check(lib().compass_workspace_init(p, n, _stream_handle(stream)), "compass_workspace_init")


def compass_read_status(workspace, stream=None):
    detail = C.c_int(0)
    p, _ = _ws(workspace)
    st = lib().compass_read_status(p, _stream_handle(stream), C.byref(detail))
    return int(st), int(detail.value)


def compass_read_kernel_clock(workspace, stream=None):
    """(SM cycles, nanoseconds) of CTA 0 of the last GEMM kernel that used this workspace."""
    cycles, ns = C.c_uint64(0), C.c_uint64(0)
    p, _ = _ws(workspace)
    _check(lib().compass_read_kernel_clock(p, _stream_handle(stream), C.byref(cycles), C.byref(ns)),
           "compass_read_kernel_clock")
    return int(cycles.value), int(ns.value)


def compass_ag_gemm(problem: Problem, A: Sequence, B: Sequence, Cout: Sequence, workspace, stream=None) -> None:
    p, n = _ws(workspace)
    _check(lib().compass_ag_gemm(C.byref(problem), _ptr_array(A), _ptr_array(B), _ptr_array(Cout), p, n,
                                 _stream_handle(stream)), "compass_ag_gemm")


def compass_gemm_rs(problem: Problem, A: Sequence, B: Sequence, Out: Sequence, workspace, stream=None) -> None:
    p, n = _ws(workspace)
    _check(lib().compass_gemm_rs(C.byref(problem), _ptr_array(A), _ptr_array(B), _ptr_array(Out), p, n,
                                 _stream_handle(stream)), "compass_gemm_rs")


def compass_ag_gemm_push(problem: Problem, A: Sequence, B: Sequence, Cout: Sequence, workspace, stream_compute,
                         stream_copy) -> None:
    p, n = _ws(workspace)
    _check(lib().compass_ag_gemm_push(C.byref(problem), _ptr_array(A), _ptr_array(B), _ptr_array(Cout), p, n,
                                      _stream_handle(stream_compute), _stream_handle(stream_copy)), "compass_ag_gemm_push")


def make_mlp(P: int, M: int, hidden: int, ffn: int, activation: int = 0, rings: int = 2,
             rs_variant: int = RS_SEGMENTED_K, order: int = ORDER_RANK_MAJOR, b_layout: int = B_NK) -> Mlp:
    return Mlp(P=P, rings=rings, M=M, hidden=hidden, ffn=ffn, activation=activation, rs_variant=rs_variant,
               order=order, b_layout=b_layout)


def compass_mlp_workspace_bytes(mlp: Mlp) -> int:
    n = C.c_size_t(0)
    _check(lib().compass_mlp_workspace_bytes(C.byref(mlp), C.byref(n)), "compass_mlp_workspace_bytes")
    return int(n.value)


def alloc_mlp_workspace(mlp: Mlp, device="cuda"):
    import torch
    ws = torch.empty(compass_mlp_workspace_bytes(mlp), dtype=torch.uint8, device=device)
    compass_workspace_init(ws)
    return ws


def compass_mlp_block(mlp: Mlp, X: Sequence, W0: Sequence, H: Sequence, W1: Sequence, Out: Sequence, workspace,
                      stream=None) -> None:
    p, n = _ws(workspace)
    _check(lib().compass_mlp_block(C.byref(mlp), _ptr_array(X), _ptr_array(W0), _ptr_array(H), _ptr_array(W1),
                                   _ptr_array(Out), p, n, _stream_handle(stream)), "compass_mlp_block")


# ---- around the blocks: embedding, layer norm, output-layer loss -------------------
#
# These take torch tensors and check type, shape, layout and device before the library sees the addresses
# (ValueError); what the library itself refuses raises CompassError.  Everything lies on the current device,
# where the call is launched (`here`, looked up once per call).

_TORCH_DTYPES: dict = {}
_POINTERS = [C.c_void_p * P for P in range(MAX_P + 1)]


def _pointers(addresses: list) -> C.Array:
    n = len(addresses)
    return (_POINTERS[n] if n <= MAX_P else C.c_void_p * n)(*addresses)


def _torch_dtype(kind: int):
    if not _TORCH_DTYPES:
        import torch
        _TORCH_DTYPES.update({DTYPE_BF16: torch.bfloat16, DTYPE_FP32: torch.float32, "index": {INDEX_INT64: torch.int64, INDEX_INT32: torch.int32}})
    if kind not in _TORCH_DTYPES:
        raise ValueError(f"unknown element type {kind}")
    return _TORCH_DTYPES[kind]


def _here() -> Optional[int]:
    """Index of the current device (None without any: then no tensor is on it)."""
    try:
        return _current_device()
    except (RuntimeError, AssertionError):
        return None


def _tensor(name: str, t, dtype, shape, here) -> Optional[int]:
    """Address of a dense tensor of this type and shape on the current device (None stays None)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != here:
        raise ValueError(f"{name}: want a contiguous tensor of {dtype} {tuple(shape)} on the current device (cuda:{here}), got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}, strides {tuple(t.stride())}")
    return t.data_ptr() or None


def _op_workspace(t, here):
    """Address and bytes of a workspace on the current device."""
    if not t.is_contiguous() or t.get_device() != here:
        raise ValueError(f"workspace: want a contiguous tensor on the current device (cuda:{here}), got one on {t.device}, "
                         f"strides {tuple(t.stride())}")
    return _ws(t)


def _row_shards(name: str, tensors: Optional[Sequence], P: int, M: int, hidden: int, kind: int, here):
    if tensors is None:
        return None
    if len(tensors) != P:
        raise ValueError(f"{name}: want {P} shards, got {len(tensors)}")
    dtype, shape = _torch_dtype(kind), (M // P if P else 0, hidden)       # (P = 0 is the library's to refuse)
    return _pointers([_tensor(name, t, dtype, shape, here) for t in tensors])


def vocab_shard_rows(vocab: int, P: int, r: int) -> int:
    """Rows of rank r's shard of a table of `vocab` rows: ceil(vocab / P) each, the last ones fewer."""
    s = -(-vocab // P)
    return max(0, min(s, vocab - s * r))


def _vocab_shards(name: str, tensors: Sequence, P: int, vocab: int, hidden: int, kind: int, here):
    if len(tensors) != P:
        raise ValueError(f"{name}: want {P} shards, got {len(tensors)}")
    dtype = _torch_dtype(kind)
    return _pointers([_tensor(name, t, dtype, (vocab_shard_rows(vocab, P, r), hidden), here) for r, t in enumerate(tensors)])


def _index(name: str, t, kind: int, M: int, here):
    kinds = _torch_dtype("index")
    if kind not in kinds:
        raise ValueError(f"unknown index type {kind}")
    return _tensor(name, t, kinds[kind], (M,), here)


def _vector(name: str, t, n: int, here, kind: int = DTYPE_FP32):
    return _tensor(name, t, _torch_dtype(kind), (n,), here)


def _sized_workspace(nbytes: int, device):
    import torch
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    with torch.cuda.device(ws.device):        # zeroed on the stream that its calls will follow
        compass_workspace_init(ws)
    return ws


def make_embedding(P: int, M: int, hidden: int, vocab: int, scale: float = 1.0, dtype: int = DTYPE_BF16,
                   grad_dtype: Optional[int] = None, index_dtype: int = INDEX_INT64, accumulate: bool = False) -> Embed:
    return Embed(P=P, dtype=dtype, grad_dtype=dtype if grad_dtype is None else grad_dtype, index_dtype=index_dtype, M=M,
                 hidden=hidden, vocab=vocab, scale=scale, accumulate=int(accumulate))


def compass_embedding(embed: Embed, ids, W: Sequence, Out: Sequence, stream=None) -> None:
    """Out[r] = scale * W[ids of rank r's rows]; ids outside the vocabulary give zero rows."""
    e, here = embed, _here()
    _check(lib().compass_embedding(C.byref(e), _index("ids", ids, e.index_dtype, e.M, here), _vocab_shards("W", W, e.P, e.vocab, e.hidden, e.dtype, here),
                                   _row_shards("Out", Out, e.P, e.M, e.hidden, e.dtype, here), _stream_handle(stream, here)), "compass_embedding")


def compass_embedding_workspace_bytes(embed: Embed) -> int:
    n = C.c_size_t(0)
    _check(lib().compass_embedding_workspace_bytes(C.byref(embed), C.byref(n)), "compass_embedding_workspace_bytes")
    return int(n.value)


def alloc_embedding_workspace(embed: Embed, device="cuda"):
    return _sized_workspace(compass_embedding_workspace_bytes(embed), device)


def compass_embedding_backward(embed: Embed, ids, dOut: Sequence, dW: Sequence, workspace, stream=None) -> None:
    """dW (+)= scale * the rows of dOut summed by id, over tokens sorted by id."""
    e, here = embed, _here()
    p, n = _op_workspace(workspace, here)
    _check(lib().compass_embedding_backward(C.byref(e), _index("ids", ids, e.index_dtype, e.M, here),
                                            _row_shards("dOut", dOut, e.P, e.M, e.hidden, e.dtype, here),
                                            _vocab_shards("dW", dW, e.P, e.vocab, e.hidden, e.grad_dtype, here), p, n, _stream_handle(stream, here)),
           "compass_embedding_backward")


def make_layer_norm(P: int, M: int, hidden: int, eps: float = 1e-5, dtype: int = DTYPE_BF16, param_dtype: Optional[int] = None) -> Norm:
    return Norm(P=P, dtype=dtype, param_dtype=dtype if param_dtype is None else param_dtype, eps=eps, M=M, hidden=hidden)


def compass_layer_norm(norm: Norm, X: Sequence, gamma, beta, Y: Sequence, mean=None, rstd=None, residual: Optional[Sequence] = None,
                       summed: Optional[Sequence] = None, stream=None) -> None:
    """Y = layer norm of X, or of summed = X + residual; gamma and beta may be None (1 and 0)."""
    n, here = norm, _here()
    rows = lambda name, t: _row_shards(name, t, n.P, n.M, n.hidden, n.dtype, here)  # noqa: E731
    _check(lib().compass_layer_norm(C.byref(n), rows("X", X), rows("residual", residual), _vector("gamma", gamma, n.hidden, here, n.param_dtype),
                                    _vector("beta", beta, n.hidden, here, n.param_dtype), rows("summed", summed), rows("Y", Y),
                                    _vector("mean", mean, n.M, here), _vector("rstd", rstd, n.M, here), _stream_handle(stream, here)), "compass_layer_norm")


def compass_layer_norm_workspace_bytes(norm: Norm) -> int:
    n = C.c_size_t(0)
    _check(lib().compass_layer_norm_workspace_bytes(C.byref(norm), C.byref(n)), "compass_layer_norm_workspace_bytes")
    return int(n.value)


def alloc_layer_norm_workspace(norm: Norm, device="cuda"):
    return _sized_workspace(compass_layer_norm_workspace_bytes(norm), device)


def compass_layer_norm_backward(norm: Norm, dY: Sequence, X: Sequence, gamma, mean, rstd, dX: Sequence, dgamma, dbeta, workspace,
                                dsum: Optional[Sequence] = None, stream=None) -> None:
    """dX (+ dsum, the gradient that reaches X past the norm), dgamma and dbeta (None: left out) summed over all M rows."""
    n, here = norm, _here()
    p, size = _op_workspace(workspace, here)
    rows = lambda name, t: _row_shards(name, t, n.P, n.M, n.hidden, n.dtype, here)  # noqa: E731
    param = lambda name, t: _vector(name, t, n.hidden, here, n.param_dtype)  # noqa: E731
    _check(lib().compass_layer_norm_backward(C.byref(n), rows("dY", dY), rows("X", X), param("gamma", gamma), _vector("mean", mean, n.M, here),
                                             _vector("rstd", rstd, n.M, here), rows("dsum", dsum), rows("dX", dX), param("dgamma", dgamma),
                                             param("dbeta", dbeta), p, size, _stream_handle(stream, here)), "compass_layer_norm_backward")


def make_head(P: int, M: int, hidden: int, vocab: int, logit_scale: float = 1.0, label_smoothing: float = 0.0, dtype: int = DTYPE_BF16,
              grad_dtype: Optional[int] = None, index_dtype: int = INDEX_INT64) -> Head:
    return Head(P=P, dtype=dtype, grad_dtype=dtype if grad_dtype is None else grad_dtype, index_dtype=index_dtype, M=M, hidden=hidden,
                vocab=vocab, logit_scale=logit_scale, label_smoothing=label_smoothing)


def compass_head_workspace_bytes(head: Head, backward: bool = False) -> int:
    n = C.c_size_t(0)
    _check(lib().compass_head_workspace_bytes(C.byref(head), int(backward), C.byref(n)), "compass_head_workspace_bytes")
    return int(n.value)


def alloc_head_workspace(head: Head, backward: bool = False, device="cuda"):
    return _sized_workspace(compass_head_workspace_bytes(head, backward), device)


def compass_head_loss(head: Head, X: Sequence, W: Sequence, targets, loss, lse, workspace, stream=None) -> None:
    """Cross entropy of every token and its log-sum-exp, without the logits; targets outside the vocabulary take no part."""
    h, here = head, _here()
    p, n = _op_workspace(workspace, here)
    _check(lib().compass_head_loss(C.byref(h), _row_shards("X", X, h.P, h.M, h.hidden, h.dtype, here),
                                   _vocab_shards("W", W, h.P, h.vocab, h.hidden, h.dtype, here), _index("targets", targets, h.index_dtype, h.M, here),
                                   _vector("loss", loss, h.M, here), _vector("lse", lse, h.M, here), p, n, _stream_handle(stream, here)), "compass_head_loss")


def compass_head_loss_backward(head: Head, X: Sequence, W: Sequence, targets, lse, dloss, dX: Sequence, dW: Sequence, workspace,
                               stream=None) -> None:
    """dX and dW from the gradient of every token's loss; the logits are computed again in pieces of the vocabulary.

    The logits' gradient is rounded to BF16 for its products: FP32 in grad_dtype saves dW its own rounding, not that one."""
    h, here = head, _here()
    p, n = _op_workspace(workspace, here)
    _check(lib().compass_head_loss_backward(C.byref(h), _row_shards("X", X, h.P, h.M, h.hidden, h.dtype, here),
                                            _vocab_shards("W", W, h.P, h.vocab, h.hidden, h.dtype, here),
                                            _index("targets", targets, h.index_dtype, h.M, here), _vector("lse", lse, h.M, here),
                                            _vector("dloss", dloss, h.M, here), _row_shards("dX", dX, h.P, h.M, h.hidden, h.dtype, here),
                                            _vocab_shards("dW", dW, h.P, h.vocab, h.hidden, h.grad_dtype, here), p, n, _stream_handle(stream, here)),
           "compass_head_loss_backward")


# ---- a linear block in 8 bits: root-mean-square norm, tensors kept in 8 bits, products, weight gradients ------
#
# 8-bit tensors are torch.float8_e4m3fn or torch.float8_e5m2, their scales torch.float8_e8m0fnu.  Arguments are checked
# as those of the operators around the blocks are.

def scale_shape(rows: int, cols: int, block_rows: int = 1):
    """Shape of the scales of an 8-bit matrix: one for 128 columns of a row, or for each 128 x 128 block."""
    return -(-rows // block_rows), -(-cols // 128)


_TYPES: dict = {}


def _types():
    """torch's types by the library's numbers, and that of the scales."""
    if not _TYPES:
        import torch
        _TYPES.update({DTYPE_BF16: torch.bfloat16, DTYPE_FP32: torch.float32, DTYPE_E4M3: torch.float8_e4m3fn, DTYPE_E5M2: torch.float8_e5m2,
                       "scale": torch.float8_e8m0fnu})
    return _TYPES


_FULL, _EIGHT = (DTYPE_BF16, DTYPE_FP32), (DTYPE_E4M3, DTYPE_E5M2)


def _type(kind: int, which: tuple):
    if kind not in which:
        raise ValueError(f"unknown {'8-bit' if which is _EIGHT else 'element'} type {kind}")
    return _types()[kind]


def _arrays(P: int, here, *groups):
    """Arrays of P pointers to (name, tensors or None, type, shape), one behind the other: what keeps them, and their addresses."""
    flat, at = [], []
    for name, tensors, dtype, shape in groups:
        if tensors is None:
            at.append(None)
            continue
        if len(tensors) != P:
            raise ValueError(f"{name}: want {P} tensors, got {len(tensors)}")
        at.append(len(flat))
        for t in tensors:
            if t is not None and (t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != here):
                _tensor(name, t, dtype, shape, here)       # raises (None is the library's to refuse)
            flat.append(0 if t is None else t.data_ptr())
    kept = array("Q", flat)        # (a quarter of the time of a ctypes array)
    base = kept.buffer_info()[0]
    return kept, [None if i is None else base + 8 * i for i in at]


def alloc_8bit(n: int, rows: int, cols: int, format: int = DTYPE_E4M3, block_rows: int = 1, device="cuda"):
    """n matrices in 8 bits and their scales, not initialised."""
    import torch
    return ([torch.empty(rows, cols, device=device, dtype=_type(format, _EIGHT)) for _ in range(n)],
            [torch.empty(scale_shape(rows, cols, block_rows), device=device, dtype=_types()["scale"]) for _ in range(n)])


def make_rms_norm(P: int, M: int, hidden: int, eps: float = 1e-6, dtype: int = DTYPE_BF16, param_dtype: Optional[int] = None) -> Norm:
    return Norm(P=P, dtype=dtype, param_dtype=dtype if param_dtype is None else param_dtype, eps=eps, M=M, hidden=hidden)


def compass_rms_norm(norm: Norm, X: Sequence, gamma, Y: Optional[Sequence] = None, rstd=None, residual: Optional[Sequence] = None,
                     summed: Optional[Sequence] = None, Y8: Optional[Sequence] = None, scale: Optional[Sequence] = None,
                     format: int = DTYPE_E4M3, stream=None) -> None:
    """Root-mean-square norm of X, or of summed = X + residual, into Y, into Y8 with its scales, or both; gamma may be None (1)."""
    n, here = norm, _here()
    P, M, H, kind = n.P, n.M, n.hidden, _type(n.dtype, _FULL)
    rows = (M // P if P else 0, H)
    kept, at = _arrays(P, here, ("X", X, kind, rows), ("residual", residual, kind, rows), ("summed", summed, kind, rows), ("Y", Y, kind, rows),
                       ("Y8", Y8, None if Y8 is None else _type(format, _EIGHT), rows), ("scale", scale, _types()["scale"], (rows[0], -(-H // 128))))
    _check(lib().compass_rms_norm(C.byref(n), at[0], at[1], _vector("gamma", gamma, H, here, n.param_dtype), at[2], at[3], format, at[4], at[5],
                                  _vector("rstd", rstd, M, here), _stream_handle(stream, here)), "compass_rms_norm")


def compass_rms_norm_workspace_bytes(norm: Norm) -> int:
    n = C.c_size_t(0)
    _check(lib().compass_rms_norm_workspace_bytes(C.byref(norm), C.byref(n)), "compass_rms_norm_workspace_bytes")
    return int(n.value)


def alloc_rms_norm_workspace(norm: Norm, device="cuda"):
    return _sized_workspace(compass_rms_norm_workspace_bytes(norm), device)


def compass_rms_norm_backward(norm: Norm, dY: Sequence, X: Sequence, gamma, rstd, dX: Sequence, dgamma, workspace,
                              dsum: Optional[Sequence] = None, stream=None) -> None:
    """dX (+ dsum, the gradient that reaches X past the norm) and dgamma (None: left out) summed over all M rows."""
    n, here = norm, _here()
    p, size = _op_workspace(workspace, here)
    P, M, H, kind = n.P, n.M, n.hidden, _type(n.dtype, _FULL)
    rows = (M // P if P else 0, H)
    kept, at = _arrays(P, here, ("dY", dY, kind, rows), ("X", X, kind, rows), ("dsum", dsum, kind, rows), ("dX", dX, kind, rows))
    _check(lib().compass_rms_norm_backward(C.byref(n), at[0], at[1], _vector("gamma", gamma, H, here, n.param_dtype), _vector("rstd", rstd, M, here),
                                           at[2], at[3], _vector("dgamma", dgamma, H, here, n.param_dtype), p, size, _stream_handle(stream, here)),
           "compass_rms_norm_backward")


def make_quant(P: int, M: int, cols: int, dtype: int = DTYPE_BF16, format: int = DTYPE_E4M3, block_rows: int = 1) -> Quant:
    return Quant(P=P, dtype=dtype, format=format, block_rows=block_rows, M=M, cols=cols)


def _quant(quant: Quant, X: Sequence, Q: Sequence, scale: Sequence, here):
    q, P = quant, quant.P
    if q.block_rows < 1:
        raise ValueError(f"unknown block of {q.block_rows} rows")
    rows = (q.M // P if P else 0, q.cols)
    return _arrays(P, here, ("X", X, _type(q.dtype, _FULL), rows), ("Q", Q, _type(q.format, _EIGHT), rows),
                   ("scale", scale, _types()["scale"], scale_shape(*rows, q.block_rows)))


def compass_quantize(quant: Quant, X: Sequence, Q: Sequence, scale: Sequence, stream=None) -> None:
    """X in 8 bits: values and a power of two for each run of 128 columns or each 128 x 128 block."""
    here = _here()
    kept, (x, q, s) = _quant(quant, X, Q, scale, here)
    _check(lib().compass_quantize(C.byref(quant), x, q, s, _stream_handle(stream, here)), "compass_quantize")


def compass_dequantize(quant: Quant, Q: Sequence, scale: Sequence, X: Sequence, stream=None) -> None:
    """X = scale * Q."""
    here = _here()
    kept, (x, q, s) = _quant(quant, X, Q, scale, here)
    _check(lib().compass_dequantize(C.byref(quant), q, s, x, _stream_handle(stream, here)), "compass_dequantize")


def compass_8bit_workspace_bytes(problem: Problem) -> int:
    n = C.c_size_t(0)
    _check(lib().compass_8bit_workspace_bytes(C.byref(problem), C.byref(n)), "compass_8bit_workspace_bytes")
    return int(n.value)


def alloc_8bit_workspace(problem: Problem, device="cuda"):
    """For compass_ag_gemm_8bit, compass_gemm_rs_8bit and compass_weight_grad_8bit of this problem."""
    return _sized_workspace(compass_8bit_workspace_bytes(problem), device)


def _product_8bit(name: str, op: int, g: Problem, A: Sequence, A_scale: Sequence, B: Sequence, B_scale: Sequence, out: Sequence, workspace, stream):
    here = _here()
    p, size = _op_workspace(workspace, here)
    P, M, N, K, kinds = g.P, g.M, g.N, g.K, _types()
    each = M // P if P else 0
    a_rows, out_rows = (each, M) if op == OP_AG_GEMM else (M, each)
    b_shape = (K, N) if g.b_layout == B_KN else (N, K)
    kept, at = _arrays(P, here, ("A", A, _type(g.dtype, _EIGHT), (a_rows, K)), ("A_scale", A_scale, kinds["scale"], (a_rows, -(-K // 128))),
                       ("B", B, kinds[DTYPE_E4M3], b_shape), ("B_scale", B_scale, kinds["scale"], (-(-b_shape[0] // 128), -(-b_shape[1] // 128))),
                       ("out", out, kinds[DTYPE_BF16], (out_rows, N)))
    _check(getattr(lib(), name)(C.byref(g), *at, p, size, _stream_handle(stream, here)), name)


def compass_ag_gemm_8bit(problem: Problem, A: Sequence, A_scale: Sequence, B: Sequence, B_scale: Sequence, Cout: Sequence, workspace,
                         stream=None) -> None:
    """C[r] = concat(A) @ B[r].T on 8-bit operands; problem.dtype is the type of A, weights are E4M3 with a scale per 128 x 128."""
    _product_8bit("compass_ag_gemm_8bit", OP_AG_GEMM, problem, A, A_scale, B, B_scale, Cout, workspace, stream)


def compass_gemm_rs_8bit(problem: Problem, A: Sequence, A_scale: Sequence, B: Sequence, B_scale: Sequence, Out: Sequence, workspace,
                         stream=None) -> None:
    """Out[r] = rank r's rows of sum over q of A[q] @ B[q].T on 8-bit operands."""
    _product_8bit("compass_gemm_rs_8bit", OP_GEMM_RS, problem, A, A_scale, B, B_scale, Out, workspace, stream)


def compass_weight_grad_8bit(problem: Problem, G: Sequence, X: Sequence, X_scale: Sequence, dW: Sequence, workspace,
                             grad_dtype: int = DTYPE_BF16, accumulate: bool = False, stream=None) -> None:
    """dW[r] (+)= G[r].T @ X[r] for the product that `problem` describes, X as it was kept in 8 bits.

    AllGather: G[r] is the gradient of C[r], X the row shards.  ReduceScatter: G the gradient of Out in row shards, X[r] rank r's."""
    g, here = problem, _here()
    p, size = _op_workspace(workspace, here)
    P, M, N, K, kinds = g.P, g.M, g.N, g.K, _types()
    each = M // P if P else 0
    g_rows, x_rows = (M, each) if g.op == OP_AG_GEMM else (each, M)
    kept, at = _arrays(P, here, ("G", G, kinds[DTYPE_BF16], (g_rows, N)), ("X", X, _type(g.dtype, _EIGHT), (x_rows, K)),
                       ("X_scale", X_scale, kinds["scale"], (x_rows, -(-K // 128))), ("dW", dW, _type(grad_dtype, _FULL), (N, K)))
    _check(lib().compass_weight_grad_8bit(C.byref(g), grad_dtype, int(accumulate), *at, p, size, _stream_handle(stream, here)),
           "compass_weight_grad_8bit")


def compass_decomp(problem: Problem, A: Sequence, B: Sequence, out: Sequence, workspace, stream_compute=None,
                   stream_copy=None) -> None:
    p, n = _ws(workspace)
    sc = _stream_handle(stream_compute)
    sp = _stream_handle(stream_copy) if stream_copy is not None else sc
    _check(lib().compass_decomp(C.byref(problem), _ptr_array(A), _ptr_array(B), _ptr_array(out), p, n, sc, sp),
           "compass_decomp")


def compass_decomp_comm(problem: Problem, A: Sequence, B: Sequence, out: Sequence, workspace, stream_compute=None,
                        stream_copy=None) -> None:
    """The d sub-collectives of compass_decomp alone (no sub-GEMMs): T_comm, measurable on its own."""
    p, n = _ws(workspace)
    sc = _stream_handle(stream_compute)
    sp = _stream_handle(stream_copy) if stream_copy is not None else sc
    _check(lib().compass_decomp_comm(C.byref(problem), _ptr_array(A), _ptr_array(B), _ptr_array(out), p, n, sc, sp),
           "compass_decomp_comm")


def compass_gemm_rs_sequential_noalloc(problem: Problem, A: Sequence, B: Sequence, Out: Sequence, stream=None) -> None:
    """GEMM+ReduceScatter (sequential form) whose scratch is the library's built-in
    device array: for callers that cannot allocate or pass a workspace (all device
    memory already handed out, or no tolerance for cudaMalloc's device-wide sync).
    Refuses problems needing more than NOALLOC_SCRATCH_BYTES."""
    _check(lib().compass_gemm_rs_sequential_noalloc(C.byref(problem), _ptr_array(A), _ptr_array(B), _ptr_array(Out),
                                                    _stream_handle(stream)), "compass_gemm_rs_sequential_noalloc")


def compass_noalloc_read_status(stream=None):
    """(status, detail) the last compass_gemm_rs_sequential_noalloc on the current device left in the
    built-in array; synchronises the stream, allocates nothing."""
    detail = C.c_int(0)
    st = lib().compass_noalloc_read_status(_stream_handle(stream), C.byref(detail))
    return int(st), int(detail.value)


def compass_fused_host_bytes(problem: Problem) -> int:
    n = C.c_size_t(0)
    _check(lib().compass_fused_host(C.byref(problem), None, None, None, None, 0, C.byref(n), None, 0, None),
           "compass_fused_host")
    return int(n.value)


def compass_fused_host(problem: Problem, A_host: Sequence, B_host: Sequence, out_host: Sequence, staging, workspace,
                       stream=None) -> None:
    """A_host/B_host/out_host: CPU tensors (pinned recommended)."""
    p, n = _ws(workspace)
    sp, sn = _ws(staging)
    need = C.c_size_t(0)
    _check(lib().compass_fused_host(C.byref(problem), _ptr_array(A_host), _ptr_array(B_host), _ptr_array(out_host),
                                    sp, sn, C.byref(need), p, n, _stream_handle(stream)), "compass_fused_host")


# ---- small conveniences (no arithmetic) ------------------------------------------

@dataclass
class DeviceWorkload:
    problem: Problem
    A: list
    B: list
    out: list
    workspace: object


def to_device(bits: np.ndarray, device="cuda"):
    """uint16 BF16 bit patterns -> torch.bfloat16 tensor on the device."""
    import torch
    return torch.from_numpy(bits.view(np.int16)).to(device).view(torch.bfloat16)


def to_bits(t) -> np.ndarray:
    """torch.bfloat16 tensor -> uint16 BF16 bit patterns on the host."""
    import torch
    return t.detach().view(torch.int16).cpu().numpy().view(np.uint16)


def alloc_workspace(problem: Problem, which: int = WS_FUSED, device="cuda"):
    import torch
    n = compass_workspace_bytes(problem, which)
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    compass_workspace_init(ws)
    return ws
