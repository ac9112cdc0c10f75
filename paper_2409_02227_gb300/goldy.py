"""ctypes binding of ``include/goldy.h`` — argument marshalling only.

Every function here has the name of the C entry point it calls and does no
work of its own beyond converting arguments and raising ``GoldyError`` on a
non-zero status.  Device pointers and CUDA streams are plain integers
(``tensor.data_ptr()``, ``torch.cuda.Stream().cuda_stream``).  The library is
``libgoldy.so`` next to this file, built by ``paper_2409_02227_gb300.build``;
importing this module without it raises ImportError — there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgoldy.so")
DEFAULT_LUT = os.path.join(_HERE, "data", "goldy_lut.bin")
DEFAULT_PREDICTOR = os.path.join(_HERE, "data", "goldy_lr.bin")
LR_FEATURES = 18

GOLDY_OK = 0
GOLDY_ERR_INVALID_ARG = 1
GOLDY_ERR_UNSUPPORTED = 2
GOLDY_ERR_LUT = 3
GOLDY_ERR_CUDA = 4
GOLDY_ERR_TIMEOUT = 5
GOLDY_ERR_NOMEM = 6

GOLDY_BF16 = 0
GOLDY_F32 = 1

GOLDY_PLAN_AUTO = 0
GOLDY_PLAN_SEQUENTIAL = 1
GOLDY_PLAN_DEFAULT = 2
GOLDY_PLAN_GO = 3
GOLDY_PLAN_FORCE_CD = 4
GOLDY_PLAN_FUSED = 0x10
GOLDY_MAX_GEMMS = 64
GOLDY_MAX_STREAMS = 16

GOLDY_ACT_NONE = 0
GOLDY_ACT_RELU = 1
GOLDY_ACT_GELU = 2
GOLDY_ACT_GELU_TANH = 3
GOLDY_ACT_SILU = 4
GOLDY_MAX_GROUPS = 4096
GOLDY_ROUTER_ALL = 0
GOLDY_ROUTER_CHOSEN = 1
GOLDY_MAX_SLOTS = 32
GOLDY_NORM_NONE = 0
GOLDY_NORM_LAYER = 1
GOLDY_NORM_RMS = 2
GOLDY_KEEP8_BLOCK = 32


def force_cd(cd: int) -> int:
    """Flags for GOLDY_PLAN_FORCE_CD with concurrency degree ``cd``."""
    return GOLDY_PLAN_FORCE_CD | (int(cd) << 8)


class GoldyError(RuntimeError):
    def __init__(self, status: int, where: str, message: str):
        super().__init__(f"{where}: status {status}: {message}")
        self.status = status


class goldy_ewise_desc(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class goldy_gemm_desc(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64), ("N", ctypes.c_int64), ("K", ctypes.c_int64),
                ("lda", ctypes.c_int64), ("ldb", ctypes.c_int64), ("ldc", ctypes.c_int64),
                ("trans_a", ctypes.c_int32), ("trans_b", ctypes.c_int32),
                ("a_dtype", ctypes.c_int32), ("b_dtype", ctypes.c_int32),
                ("c_dtype", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("batch", ctypes.c_int64), ("stride_a", ctypes.c_int64), ("stride_b", ctypes.c_int64),
                ("stride_c", ctypes.c_int64)]


class goldy_linear_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "in", "out", "ldx", "lddx", "ldw", "ldy", "ldz", "ldr", "stride_w")] + \
               [(n, ctypes.c_int32) for n in ("groups", "act", "act_x", "y_dtype", "dx_dtype", "dw_dtype", "bias_dtype",
                                              "reserved")]


class goldy_layernorm_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "n", "ldx", "ldy")] + \
               [("dtype", ctypes.c_int32), ("param_dtype", ctypes.c_int32), ("eps", ctypes.c_float),
                ("reserved", ctypes.c_int32)]


class goldy_router_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "ld", "ldd")] + \
               [(n, ctypes.c_int32) for n in ("experts", "k", "dtype", "over")] + \
               [("scale", ctypes.c_float), ("reserved", ctypes.c_int32)]


class goldy_route_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "width", "ldx", "lde", "ldr")] + \
               [(n, ctypes.c_int32) for n in ("k", "groups", "dtype", "reserved")]


class goldy_residual_norm_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "n", "ldx", "ldf", "lds", "ldy")] + \
               [(n, ctypes.c_int32) for n in ("dtype", "param_dtype", "norm_f", "norm_y")] + \
               [("eps", ctypes.c_float), ("alpha", ctypes.c_float), ("reserved", ctypes.c_int32)]


class goldy_residual_norm_params(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("gate", "gamma_f", "beta_f", "gamma_y", "beta_y")]


class goldy_keep8_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "n", "ldz", "ldh")] + \
               [(n, ctypes.c_int32) for n in ("dtype", "act", "reserved")]


class goldy_run_opts(ctypes.Structure):
    _fields_ = [("ev_begin", ctypes.POINTER(ctypes.c_void_p)), ("ev_end", ctypes.POINTER(ctypes.c_void_p)),
                ("trace", ctypes.c_void_p), ("trace_ctas", ctypes.c_size_t), ("serial_launch", ctypes.c_int32),
                ("inputs_ready", ctypes.c_int32), ("wait_limit_us", ctypes.c_uint32),
                ("test_stall_first_stage", ctypes.c_int32)]


class goldy_variant_info(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("id", "kind", "mma_m", "mma_n", "swap_ab", "stages", "acc_stages", "tmem_cols",
                 "smem_bytes", "split_k", "rc_div", "ctas_per_sm", "cta_pair")] + [("name", ctypes.c_char * 32)]

    def as_dict(self) -> dict:
        d = {n: getattr(self, n) for n, _ in self._fields_ if n != "name"}
        d["name"] = self.name.decode()
        return d


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with "
                          "`python -c 'import __graft_entry__ as g; g.build()'` (no CPU fallback exists)")
    lib = ctypes.CDLL(LIB_PATH)
    P, I, U32, SZ = ctypes.c_void_p, ctypes.c_int, ctypes.c_uint32, ctypes.c_size_t
    PP = ctypes.POINTER(ctypes.c_void_p)
    IP = ctypes.POINTER(ctypes.c_int)
    DP = ctypes.POINTER(goldy_gemm_desc)
    LP = ctypes.POINTER(goldy_linear_desc)
    NP = ctypes.POINTER(goldy_layernorm_desc)
    RP = ctypes.POINTER(goldy_router_desc)
    TP = ctypes.POINTER(goldy_route_desc)
    SP = ctypes.POINTER(goldy_residual_norm_desc)
    SPP = ctypes.POINTER(goldy_residual_norm_params)
    KP = ctypes.POINTER(goldy_keep8_desc)
    sig = {
        "goldy_abi_version": ([], I),
        "goldy_last_error": ([], ctypes.c_char_p),
        "goldy_variant_count": ([], I),
        "goldy_variant_info_get": ([I, ctypes.POINTER(goldy_variant_info)], I),
        "goldy_lut_load": ([ctypes.c_char_p, PP], I),
        "goldy_lut_from_memory": ([P, SZ, PP], I),
        "goldy_lut_free": ([P], None),
        "goldy_bucket_key": ([DP, ctypes.POINTER(U32)], I),
        "goldy_plan": ([DP, I, P, I, PP], I),
        "goldy_plan_ex": ([DP, I, P, P, I, PP], I),
        "goldy_predictor_load": ([ctypes.c_char_p, PP], I),
        "goldy_predictor_from_memory": ([P, SZ, PP], I),
        "goldy_predictor_free": ([P], None),
        "goldy_lut_lookup": ([P, DP, IP, IP], I),
        "goldy_lr_features": ([DP, P, I, ctypes.POINTER(ctypes.c_double)], I),
        "goldy_predict_cd": ([P, P, DP, IP, ctypes.POINTER(ctypes.c_double)], I),
        "goldy_schedule_build": ([DP, I, IP, IP, IP, I, PP], I),
        "goldy_schedule_query": ([P, IP, IP, IP, ctypes.POINTER(SZ)], I),
        "goldy_schedule_entry": ([P, I, IP, IP, IP, IP], I),
        "goldy_schedule_serialize": ([P, P, SZ, ctypes.POINTER(SZ)], I),
        "goldy_schedule_free": ([P], None),
        "goldy_run": ([P, PP, PP, PP, P, SZ, PP, I], I),
        "goldy_graph_create": ([P, PP, PP, PP, P, SZ, PP, I, PP], I),
        "goldy_run_ex": ([P, PP, PP, PP, P, SZ, PP, I, ctypes.POINTER(goldy_run_opts)], I),
        "goldy_graph_create_ex": ([P, PP, PP, PP, P, SZ, PP, I, ctypes.POINTER(goldy_run_opts), PP], I),
        "goldy_graph_launch": ([P, P], I),
        "goldy_exec_create": ([P, PP, PP, PP, P, SZ, PP, I, ctypes.POINTER(goldy_run_opts), PP], I),
        "goldy_exec_launch": ([P], I),
        "goldy_exec_time": ([PP, I, I, I, ctypes.POINTER(ctypes.c_float)], I),
        "goldy_partition_create": ([I, I, PP], I),
        "goldy_corun_plan": ([DP, ctypes.POINTER(goldy_ewise_desc), P, I, PP], I),
        "goldy_corun_query": ([P, IP, IP, IP, ctypes.POINTER(SZ)], I),
        "goldy_corun_run": ([P, P, P, P, P, SZ, P, P, P, PP, I], I),
        "goldy_corun_exec_create": ([P, P, P, P, P, SZ, P, P, P, PP, I, PP], I),
        "goldy_corun_free": ([P], None),
        "goldy_ewise_add": ([P, P, P, ctypes.c_int64, I, I, P], I),
        "goldy_partition_query": ([P, IP, PP, I], I),
        "goldy_partition_free": ([P], None),
        "goldy_exec_free": ([P], None),
        "goldy_graph_free": ([P], None),
        "goldy_gemm_noalloc": ([DP, I, P, P, P, P], I),
        "goldy_linear_query": ([LP, ctypes.POINTER(SZ)], I),
        "goldy_linear_forward": ([LP, P, P, P, P, P, P, P, P, SZ, P], I),
        "goldy_linear_input_grad": ([LP, P, P, P, P, P, P, P, SZ, P], I),
        "goldy_linear_weight_grad": ([LP, P, P, P, P, I, P, SZ, P], I),
        "goldy_linear_bias_grad": ([LP, P, P, P, P, P, I, P, SZ, P], I),
        "goldy_layernorm_query": ([NP, ctypes.POINTER(SZ)], I),
        "goldy_layernorm_forward": ([NP, P, P, P, P, P, P, P], I),
        "goldy_layernorm_backward": ([NP, P, P, P, P, P, P, P, P, I, P, SZ, P], I),
        "goldy_router_forward": ([RP, P, P, P, P], I),
        "goldy_router_backward": ([RP, P, P, P, P, P], I),
        "goldy_route_query": ([TP, ctypes.POINTER(SZ)], I),
        "goldy_route_sort": ([TP, P, P, P, P, P, SZ, P], I),
        "goldy_route_dispatch": ([TP, P, P, P, P], I),
        "goldy_route_combine": ([TP, P, P, P, P, P, P], I),
        "goldy_route_combine_grad": ([TP, P, P, P, P, P, P, P], I),
        "goldy_residual_norm_query": ([SP, ctypes.POINTER(SZ)], I),
        "goldy_residual_norm_forward": ([SP, SPP, P, P, P, P, P, P], I),
        "goldy_residual_norm_backward": ([SP, SPP, P, P, P, P, P, P, P, SPP, I, P, SZ, P], I),
        "goldy_keep8_query": ([KP, ctypes.POINTER(SZ), ctypes.POINTER(SZ)], I),
        "goldy_keep8_pack": ([KP, P, P, P, P], I),
        "goldy_keep8_unpack": ([KP, P, P, P, P, P], I),
        "goldy_device_error": ([IP, I], I),
        "goldy_device_info": ([I, IP, IP], I),
    }
    for name, (args, res) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    return lib


_lib = _load()


def _check(status: int, where: str) -> None:
    if status != GOLDY_OK:
        raise GoldyError(status, where, _lib.goldy_last_error().decode())


def _ptrs(values: Sequence[int]):
    arr = (ctypes.c_void_p * max(1, len(values)))()
    for i, v in enumerate(values):
        arr[i] = int(v) if v else None
    return arr


def _descs(descs: Sequence[goldy_gemm_desc]):
    arr = (goldy_gemm_desc * max(1, len(descs)))()
    for i, d in enumerate(descs):
        arr[i] = d
    return arr


def desc(M: int, N: int, K: int, c_dtype: int = GOLDY_F32, lda: Optional[int] = None,
         ldb: Optional[int] = None, ldc: Optional[int] = None, batch: int = 1, stride_a: Optional[int] = None,
         stride_b: Optional[int] = None, stride_c: Optional[int] = None) -> goldy_gemm_desc:
    """Descriptor of C (M x N) = A (M x K, row-major) * B (K x N, row-major),
    or of `batch` such products with entries packed back to back (default
    strides M*lda, K*ldb, M*ldc)."""
    lda = K if lda is None else lda
    ldb = N if ldb is None else ldb
    ldc = N if ldc is None else ldc
    return goldy_gemm_desc(M, N, K, lda, ldb, ldc, 0, 0, GOLDY_BF16, GOLDY_BF16, int(c_dtype), 0, int(batch),
                           M * lda if stride_a is None else stride_a, K * ldb if stride_b is None else stride_b,
                           M * ldc if stride_c is None else stride_c)


class _Handle:
    _free = None

    def __init__(self, ptr: ctypes.c_void_p):
        self.ptr = ptr

    def close(self) -> None:
        if self.ptr:
            type(self)._free(self.ptr)
            self.ptr = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Lut(_Handle):
    _free = staticmethod(lambda p: _lib.goldy_lut_free(p))


class Predictor(_Handle):
    _free = staticmethod(lambda p: _lib.goldy_predictor_free(p))


class Schedule(_Handle):
    _free = staticmethod(lambda p: _lib.goldy_schedule_free(p))


class Graph(_Handle):
    _free = staticmethod(lambda p: _lib.goldy_graph_free(p))


class Corun(_Handle):
    _free = staticmethod(lambda p: _lib.goldy_corun_free(p))


class Partition(_Handle):
    _free = staticmethod(lambda p: _lib.goldy_partition_free(p))


class Exec(_Handle):
    _free = staticmethod(lambda p: _lib.goldy_exec_free(p))


def goldy_abi_version() -> int:
    return int(_lib.goldy_abi_version())


def goldy_last_error() -> str:
    return _lib.goldy_last_error().decode()


def goldy_variant_count() -> int:
    return int(_lib.goldy_variant_count())


def goldy_variant_info_get(variant_id: int) -> dict:
    info = goldy_variant_info()
    _check(_lib.goldy_variant_info_get(int(variant_id), ctypes.byref(info)), "goldy_variant_info_get")
    return info.as_dict()


def goldy_lut_load(path: str = DEFAULT_LUT) -> Lut:
    out = ctypes.c_void_p()
    _check(_lib.goldy_lut_load(path.encode(), ctypes.byref(out)), "goldy_lut_load")
    return Lut(out)


def goldy_lut_from_memory(data: bytes) -> Lut:
    out = ctypes.c_void_p()
    buf = ctypes.create_string_buffer(bytes(data), len(data))
    _check(_lib.goldy_lut_from_memory(buf, len(data), ctypes.byref(out)), "goldy_lut_from_memory")
    return Lut(out)


def goldy_bucket_key(d: goldy_gemm_desc) -> int:
    key = ctypes.c_uint32()
    _check(_lib.goldy_bucket_key(ctypes.byref(d), ctypes.byref(key)), "goldy_bucket_key")
    return int(key.value)


def goldy_plan(descs: Sequence[goldy_gemm_desc], lut: Lut, flags: int = GOLDY_PLAN_AUTO) -> Schedule:
    out = ctypes.c_void_p()
    _check(_lib.goldy_plan(_descs(descs), len(descs), lut.ptr if lut else None, int(flags),
                           ctypes.byref(out)), "goldy_plan")
    return Schedule(out)


def goldy_plan_ex(descs: Sequence[goldy_gemm_desc], lut: Lut, predictor: Optional[Predictor],
                  flags: int = GOLDY_PLAN_AUTO) -> Schedule:
    out = ctypes.c_void_p()
    _check(_lib.goldy_plan_ex(_descs(descs), len(descs), lut.ptr if lut else None,
                              predictor.ptr if predictor else None, int(flags), ctypes.byref(out)), "goldy_plan_ex")
    return Schedule(out)


def goldy_predictor_load(path: str = DEFAULT_PREDICTOR) -> Predictor:
    out = ctypes.c_void_p()
    _check(_lib.goldy_predictor_load(path.encode(), ctypes.byref(out)), "goldy_predictor_load")
    return Predictor(out)


def goldy_predictor_from_memory(data: bytes) -> Predictor:
    out = ctypes.c_void_p()
    buf = ctypes.create_string_buffer(bytes(data), len(data))
    _check(_lib.goldy_predictor_from_memory(buf, len(data), ctypes.byref(out)), "goldy_predictor_from_memory")
    return Predictor(out)


def goldy_lut_lookup(lut: Lut, d: goldy_gemm_desc) -> Tuple[int, List[int]]:
    pref = ctypes.c_int()
    vs = (ctypes.c_int * 5)()
    _check(_lib.goldy_lut_lookup(lut.ptr, ctypes.byref(d), ctypes.byref(pref), vs), "goldy_lut_lookup")
    return pref.value, list(vs)


def goldy_lr_features(d: goldy_gemm_desc, lut: Lut, sm_count: int) -> List[float]:
    out = (ctypes.c_double * LR_FEATURES)()
    _check(_lib.goldy_lr_features(ctypes.byref(d), lut.ptr, int(sm_count), out), "goldy_lr_features")
    return list(out)


def goldy_predict_cd(p: Predictor, lut: Lut, d: goldy_gemm_desc) -> Tuple[int, List[float]]:
    cd = ctypes.c_int()
    probs = (ctypes.c_double * 5)()
    _check(_lib.goldy_predict_cd(p.ptr, lut.ptr, ctypes.byref(d), ctypes.byref(cd), probs), "goldy_predict_cd")
    return cd.value, list(probs)


def goldy_schedule_build(descs: Sequence[goldy_gemm_desc], group_of: Sequence[int],
                         variant_of: Sequence[int], slot_of: Sequence[int], flags: int = 0) -> Schedule:
    n = len(descs)
    IA = ctypes.c_int * max(1, n)
    out = ctypes.c_void_p()
    _check(_lib.goldy_schedule_build(_descs(descs), n, IA(*group_of), IA(*variant_of), IA(*slot_of),
                                     int(flags), ctypes.byref(out)), "goldy_schedule_build")
    return Schedule(out)


def goldy_schedule_query(s: Schedule) -> Tuple[int, int, int, int]:
    """(n_gemms, n_groups, max_streams, workspace_bytes)."""
    a, b, c, w = ctypes.c_int(), ctypes.c_int(), ctypes.c_int(), ctypes.c_size_t()
    _check(_lib.goldy_schedule_query(s.ptr, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c),
                                     ctypes.byref(w)), "goldy_schedule_query")
    return a.value, b.value, c.value, int(w.value)


def goldy_schedule_entry(s: Schedule, gemm: int) -> Tuple[int, int, int, int]:
    """(group, variant, slot, cd) of GEMM ``gemm``."""
    g, v, sl, cd = ctypes.c_int(), ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    _check(_lib.goldy_schedule_entry(s.ptr, int(gemm), ctypes.byref(g), ctypes.byref(v),
                                     ctypes.byref(sl), ctypes.byref(cd)), "goldy_schedule_entry")
    return g.value, v.value, sl.value, cd.value


def goldy_schedule_serialize(s: Schedule) -> bytes:
    size = ctypes.c_size_t()
    _lib.goldy_schedule_serialize(s.ptr, None, 0, ctypes.byref(size))
    buf = ctypes.create_string_buffer(size.value)
    _check(_lib.goldy_schedule_serialize(s.ptr, buf, size.value, ctypes.byref(size)),
           "goldy_schedule_serialize")
    return buf.raw[:size.value]


def goldy_run(s: Schedule, A: Sequence[int], B: Sequence[int], C: Sequence[int], workspace: int,
              workspace_bytes: int, streams: Sequence[int]) -> None:
    _check(_lib.goldy_run(s.ptr, _ptrs(A), _ptrs(B), _ptrs(C), int(workspace) or None,
                          int(workspace_bytes), _ptrs(streams), len(streams)), "goldy_run")


def goldy_graph_create(s: Schedule, A: Sequence[int], B: Sequence[int], C: Sequence[int],
                       workspace: int, workspace_bytes: int, streams: Sequence[int]) -> Graph:
    out = ctypes.c_void_p()
    _check(_lib.goldy_graph_create(s.ptr, _ptrs(A), _ptrs(B), _ptrs(C), int(workspace) or None,
                                   int(workspace_bytes), _ptrs(streams), len(streams),
                                   ctypes.byref(out)), "goldy_graph_create")
    return Graph(out)


def _opts(ev_begin: Optional[Sequence[int]], ev_end: Optional[Sequence[int]], trace: int = 0,
          trace_ctas: int = 0, serial_launch: bool = False, inputs_ready: bool = False,
          wait_limit_us: int = 0, test_stall_first_stage: bool = False):
    o = goldy_run_opts()
    o.trace = int(trace) or None
    o.trace_ctas = int(trace_ctas)
    o.serial_launch = 1 if serial_launch else 0
    o.inputs_ready = 1 if inputs_ready else 0
    o.wait_limit_us = int(wait_limit_us)
    o.test_stall_first_stage = 1 if test_stall_first_stage else 0
    keep = []
    if ev_begin is not None:
        arr = _ptrs(ev_begin)
        keep.append(arr)
        o.ev_begin = ctypes.cast(arr, ctypes.POINTER(ctypes.c_void_p))
    if ev_end is not None:
        arr = _ptrs(ev_end)
        keep.append(arr)
        o.ev_end = ctypes.cast(arr, ctypes.POINTER(ctypes.c_void_p))
    return o, keep


def goldy_run_ex(s: Schedule, A: Sequence[int], B: Sequence[int], C: Sequence[int], workspace: int,
                 workspace_bytes: int, streams: Sequence[int], ev_begin: Optional[Sequence[int]] = None,
                 ev_end: Optional[Sequence[int]] = None, trace: int = 0, trace_ctas: int = 0,
                 serial_launch: bool = False, inputs_ready: bool = False, wait_limit_us: int = 0,
                 test_stall_first_stage: bool = False) -> None:
    """goldy_run with per-GEMM timing events (cudaEvent_t handles as ints),
    an optional device phase-trace buffer, the launch mode, early operand
    loads, the bounded-wait limit and the test stall hook (see
    goldy_run_opts)."""
    o, _keep = _opts(ev_begin, ev_end, trace, trace_ctas, serial_launch, inputs_ready, wait_limit_us,
                     test_stall_first_stage)
    _check(_lib.goldy_run_ex(s.ptr, _ptrs(A), _ptrs(B), _ptrs(C), int(workspace) or None,
                             int(workspace_bytes), _ptrs(streams), len(streams), ctypes.byref(o)),
           "goldy_run_ex")


def goldy_graph_create_ex(s: Schedule, A: Sequence[int], B: Sequence[int], C: Sequence[int],
                          workspace: int, workspace_bytes: int, streams: Sequence[int],
                          ev_begin: Optional[Sequence[int]] = None,
                          ev_end: Optional[Sequence[int]] = None, serial_launch: bool = False,
                          inputs_ready: bool = False) -> Graph:
    o, _keep = _opts(ev_begin, ev_end, serial_launch=serial_launch, inputs_ready=inputs_ready)
    out = ctypes.c_void_p()
    _check(_lib.goldy_graph_create_ex(s.ptr, _ptrs(A), _ptrs(B), _ptrs(C), int(workspace) or None,
                                      int(workspace_bytes), _ptrs(streams), len(streams),
                                      ctypes.byref(o), ctypes.byref(out)), "goldy_graph_create_ex")
    return Graph(out)


def goldy_exec_create(s: Schedule, A: Sequence[int], B: Sequence[int], C: Sequence[int], workspace: int,
                      workspace_bytes: int, streams: Sequence[int], ev_begin: Optional[Sequence[int]] = None,
                      ev_end: Optional[Sequence[int]] = None, trace: int = 0, trace_ctas: int = 0,
                      serial_launch: bool = False, inputs_ready: bool = False, wait_limit_us: int = 0) -> Exec:
    o, _keep = _opts(ev_begin, ev_end, trace, trace_ctas, serial_launch, inputs_ready, wait_limit_us)
    out = ctypes.c_void_p()
    _check(_lib.goldy_exec_create(s.ptr, _ptrs(A), _ptrs(B), _ptrs(C), int(workspace) or None,
                                  int(workspace_bytes), _ptrs(streams), len(streams), ctypes.byref(o),
                                  ctypes.byref(out)), "goldy_exec_create")
    return Exec(out)


def goldy_exec_time(execs: Sequence[Exec], warmup: int, reps: int) -> float:
    """Milliseconds per replay (see include/goldy.h)."""
    arr = (ctypes.c_void_p * len(execs))(*[e.ptr for e in execs])
    ms = ctypes.c_float()
    _check(_lib.goldy_exec_time(arr, len(execs), int(warmup), int(reps), ctypes.byref(ms)), "goldy_exec_time")
    return ms.value


def goldy_corun_plan(gemm: goldy_gemm_desc, n: int, dtype: int, lut: Lut, policy: int = GOLDY_PLAN_AUTO) -> Corun:
    """A GEMM co-scheduled with the element-wise add Z = X + Y of n elements."""
    ew = goldy_ewise_desc(int(n), int(dtype), 0)
    out = ctypes.c_void_p()
    _check(_lib.goldy_corun_plan(ctypes.byref(gemm), ctypes.byref(ew), lut.ptr if lut else None, int(policy),
                                 ctypes.byref(out)), "goldy_corun_plan")
    return Corun(out)


def goldy_corun_query(c: Corun) -> Tuple[int, int, int, int]:
    """(concurrent, gemm variant, add grid-cap divisor, workspace bytes)."""
    cc, v, rc, ws = ctypes.c_int(), ctypes.c_int(), ctypes.c_int(), ctypes.c_size_t()
    _check(_lib.goldy_corun_query(c.ptr, ctypes.byref(cc), ctypes.byref(v), ctypes.byref(rc), ctypes.byref(ws)),
           "goldy_corun_query")
    return cc.value, v.value, rc.value, ws.value


def goldy_corun_run(c: Corun, A: int, B: int, C: int, workspace: int, workspace_bytes: int, X: int, Y: int, Z: int,
                    streams: Sequence[int]) -> None:
    _check(_lib.goldy_corun_run(c.ptr, A or None, B or None, C or None, workspace or None, int(workspace_bytes),
                                X or None, Y or None, Z or None, _ptrs(streams), len(streams)), "goldy_corun_run")


def goldy_corun_exec_create(c: Corun, A: int, B: int, C: int, workspace: int, workspace_bytes: int, X: int, Y: int,
                            Z: int, streams: Sequence[int]) -> "Exec":
    out = ctypes.c_void_p()
    _check(_lib.goldy_corun_exec_create(c.ptr, A or None, B or None, C or None, workspace or None,
                                        int(workspace_bytes), X or None, Y or None, Z or None, _ptrs(streams),
                                        len(streams), ctypes.byref(out)), "goldy_corun_exec_create")
    return Exec(out)


def goldy_ewise_add(X: int, Y: int, Z: int, n: int, dtype: int, rc_div: int, stream: int) -> None:
    _check(_lib.goldy_ewise_add(X or None, Y or None, Z or None, int(n), int(dtype), int(rc_div), stream or None),
           "goldy_ewise_add")


def goldy_partition_create(min_sms: int, n_streams: int = 16) -> Partition:
    out = ctypes.c_void_p()
    _check(_lib.goldy_partition_create(int(min_sms), int(n_streams), ctypes.byref(out)), "goldy_partition_create")
    return Partition(out)


def goldy_partition_query(p: Partition, n: int = 0) -> Tuple[int, List[int]]:
    """(SM count, the first n stream handles as integers)."""
    sm = ctypes.c_int()
    arr = (ctypes.c_void_p * max(1, n))()
    _check(_lib.goldy_partition_query(p.ptr, ctypes.byref(sm), arr, int(n)), "goldy_partition_query")
    return sm.value, [int(arr[k] or 0) for k in range(n)]


def goldy_exec_launch(e: Exec) -> None:
    _check(_lib.goldy_exec_launch(e.ptr), "goldy_exec_launch")


def goldy_graph_launch(g: Graph, stream: int) -> None:
    _check(_lib.goldy_graph_launch(g.ptr, int(stream) or None), "goldy_graph_launch")


def goldy_gemm_noalloc(d: goldy_gemm_desc, variant: int, A: int, B: int, C: int, stream: int = 0) -> None:
    """One GEMM with the library's compiled-in split-K scratch (no device
    allocation anywhere); see goldy.h for who needs it and its limits."""
    _check(_lib.goldy_gemm_noalloc(ctypes.byref(d), int(variant), int(A) or None, int(B) or None,
                                   int(C) or None, int(stream) or None), "goldy_gemm_noalloc")


def linear_desc(rows: int, fan_in: int, fan_out: int, groups: int = 0, act: int = GOLDY_ACT_NONE,
                act_x: int = GOLDY_ACT_NONE, y_dtype: int = GOLDY_BF16, dx_dtype: int = GOLDY_BF16,
                dw_dtype: int = GOLDY_F32, bias_dtype: int = GOLDY_BF16, ldx: int = 0, lddx: int = 0, ldw: int = 0,
                ldy: int = 0, ldz: int = 0, ldr: int = 0, stride_w: int = 0) -> goldy_linear_desc:
    """Descriptor of a linear layer Y (rows x fan_out) = act(X (rows x fan_in)
    W (fan_in x fan_out) + b) + R, or of `groups` experts over ragged row
    ranges.  Row strides of 0 stand for dense rows: fp32 rows packed, bf16 rows
    padded to a multiple of 8 elements."""
    return goldy_linear_desc(rows, fan_in, fan_out, ldx, lddx, ldw, ldy, ldz, ldr, stride_w, int(groups), int(act),
                             int(act_x), int(y_dtype), int(dx_dtype), int(dw_dtype), int(bias_dtype), 0)


def goldy_linear_query(d: goldy_linear_desc) -> int:
    """Workspace bytes that cover every call with this descriptor."""
    ws = ctypes.c_size_t()
    _check(_lib.goldy_linear_query(d, ctypes.byref(ws)), "goldy_linear_query")
    return int(ws.value)


def goldy_linear_forward(d: goldy_linear_desc, X: int, W: int, Y: int, bias: int = 0, residual: int = 0, z: int = 0,
                         offsets: int = 0, workspace: int = 0, workspace_bytes: int = 0, stream: int = 0) -> None:
    """Y = act(X W + bias) + residual; z receives X W + bias."""
    _check(_lib.goldy_linear_forward(d, offsets or None, X or None, W or None, bias or None, residual or None,
                                     z or None, Y or None, workspace or None, workspace_bytes, stream or None),
           "goldy_linear_forward")


def goldy_linear_input_grad(d: goldy_linear_desc, dY: int, W: int, dX: int, z: int = 0, residual: int = 0,
                            offsets: int = 0, workspace: int = 0, workspace_bytes: int = 0, stream: int = 0) -> None:
    """dX = (dY W^T) * act_x'(z) + residual."""
    _check(_lib.goldy_linear_input_grad(d, offsets or None, dY or None, W or None, z or None, residual or None,
                                        dX or None, workspace or None, workspace_bytes, stream or None),
           "goldy_linear_input_grad")


def goldy_linear_weight_grad(d: goldy_linear_desc, X: int, dY: int, dW: int, accumulate: bool = False,
                             offsets: int = 0, workspace: int = 0, workspace_bytes: int = 0, stream: int = 0) -> None:
    """dW (+)= X^T dY, per expert."""
    _check(_lib.goldy_linear_weight_grad(d, offsets or None, X or None, dY or None, dW or None, 1 if accumulate else 0,
                                         workspace or None, workspace_bytes, stream or None),
           "goldy_linear_weight_grad")


def goldy_linear_bias_grad(d: goldy_linear_desc, dY: int, db: int, z: int = 0, dz: int = 0, accumulate: bool = False,
                           offsets: int = 0, workspace: int = 0, workspace_bytes: int = 0, stream: int = 0) -> None:
    """db (+)= sum over rows of dz, dz = dY * act'(z) (z = dz = 0: of dY)."""
    _check(_lib.goldy_linear_bias_grad(d, offsets or None, dY or None, z or None, dz or None, db or None,
                                       1 if accumulate else 0, workspace or None, workspace_bytes, stream or None),
           "goldy_linear_bias_grad")


def layernorm_desc(rows: int, n: int, dtype: int = GOLDY_BF16, param_dtype: int = GOLDY_BF16, eps: float = 1e-5,
                   ldx: Optional[int] = None, ldy: Optional[int] = None) -> goldy_layernorm_desc:
    """Descriptor of a layer norm over rows of n elements (default: packed)."""
    return goldy_layernorm_desc(rows, n, n if ldx is None else ldx, n if ldy is None else ldy, int(dtype),
                                int(param_dtype), float(eps), 0)


def goldy_layernorm_query(d: goldy_layernorm_desc) -> int:
    """Workspace bytes of the backward call."""
    ws = ctypes.c_size_t()
    _check(_lib.goldy_layernorm_query(d, ctypes.byref(ws)), "goldy_layernorm_query")
    return int(ws.value)


def goldy_layernorm_forward(d: goldy_layernorm_desc, X: int, gamma: int, beta: int, Y: int, mean: int = 0,
                            rstd: int = 0, stream: int = 0) -> None:
    _check(_lib.goldy_layernorm_forward(d, X or None, gamma or None, beta or None, Y or None, mean or None,
                                        rstd or None, stream or None), "goldy_layernorm_forward")


def goldy_layernorm_backward(d: goldy_layernorm_desc, dY: int, X: int, gamma: int, mean: int, rstd: int, dX: int,
                             dgamma: int = 0, dbeta: int = 0, workspace: int = 0, workspace_bytes: int = 0,
                             stream: int = 0, accumulate: bool = False) -> None:
    _check(_lib.goldy_layernorm_backward(d, dY or None, X or None, gamma or None, mean or None, rstd or None,
                                         dX or None, dgamma or None, dbeta or None, 1 if accumulate else 0,
                                         workspace or None, workspace_bytes, stream or None),
           "goldy_layernorm_backward")


def router_desc(rows: int, experts: int, k: int, dtype: int = GOLDY_F32, over: int = GOLDY_ROUTER_ALL, scale: float = 1.0,
                ld: Optional[int] = None, ldd: Optional[int] = None) -> goldy_router_desc:
    """Descriptor of a router over rows of `experts` logits (default: packed)."""
    return goldy_router_desc(rows, experts if ld is None else ld, experts if ldd is None else ldd, int(experts), int(k),
                             int(dtype), int(over), float(scale), 0)


def goldy_router_forward(d: goldy_router_desc, logits: int, ids: int, weights: int, stream: int = 0) -> None:
    """The k largest logits' ids (int32) and softmax weights (fp32) of each row."""
    _check(_lib.goldy_router_forward(d, logits or None, ids or None, weights or None, stream or None),
           "goldy_router_forward")


def goldy_router_backward(d: goldy_router_desc, logits: int, ids: int, dweights: int, dlogits: int,
                          stream: int = 0) -> None:
    _check(_lib.goldy_router_backward(d, logits or None, ids or None, dweights or None, dlogits or None, stream or None),
           "goldy_router_backward")


def route_desc(rows: int, k: int, groups: int, width: int = 0, dtype: int = GOLDY_BF16, ldx: Optional[int] = None,
               lde: Optional[int] = None, ldr: Optional[int] = None) -> goldy_route_desc:
    """Descriptor of `rows` tokens with k slots each over `groups` experts, and of
    their rows of `width` elements (default: packed)."""
    return goldy_route_desc(rows, width, width if ldx is None else ldx, width if lde is None else lde,
                            width if ldr is None else ldr, int(k), int(groups), int(dtype), 0)


def goldy_route_query(d: goldy_route_desc) -> int:
    """Workspace bytes of the sort."""
    ws = ctypes.c_size_t()
    _check(_lib.goldy_route_query(d, ctypes.byref(ws)), "goldy_route_query")
    return int(ws.value)


def goldy_route_sort(d: goldy_route_desc, ids: int, offsets: int, place: int, source: int = 0, workspace: int = 0,
                     workspace_bytes: int = 0, stream: int = 0) -> None:
    """Slots by expert: offsets per expert, place of each slot, slot at each place."""
    _check(_lib.goldy_route_sort(d, ids or None, offsets or None, place or None, source or None, workspace or None,
                                 workspace_bytes, stream or None), "goldy_route_sort")


def goldy_route_dispatch(d: goldy_route_desc, X: int, place: int, E: int, stream: int = 0) -> None:
    """E[place] = X."""
    _check(_lib.goldy_route_dispatch(d, X or None, place or None, E or None, stream or None), "goldy_route_dispatch")


def goldy_route_combine(d: goldy_route_desc, E: int, place: int, Y: int, weights: int = 0, residual: int = 0,
                        stream: int = 0) -> None:
    """Y = residual + sum over slots of weights * E[place]."""
    _check(_lib.goldy_route_combine(d, E or None, place or None, weights or None, residual or None, Y or None,
                                    stream or None), "goldy_route_combine")


def goldy_route_combine_grad(d: goldy_route_desc, dY: int, E: int, place: int, weights: int, dE: int,
                             dweights: int = 0, stream: int = 0) -> None:
    """dE[place] = weights * dY, dweights = dY . E[place]."""
    _check(_lib.goldy_route_combine_grad(d, dY or None, E or None, place or None, weights or None, dE or None,
                                         dweights or None, stream or None), "goldy_route_combine_grad")


def residual_norm_desc(rows: int, n: int, norm_f: int = GOLDY_NORM_RMS, norm_y: int = GOLDY_NORM_RMS,
                       dtype: int = GOLDY_BF16, param_dtype: int = GOLDY_F32, eps: float = 1e-5, alpha: float = 1.0,
                       ldx: Optional[int] = None, ldf: Optional[int] = None, lds: Optional[int] = None,
                       ldy: Optional[int] = None) -> goldy_residual_norm_desc:
    """Descriptor of S = alpha X + gate * N_f(F), Y = N_y(S) over rows of n
    elements (default: packed)."""
    ld = [n if v is None else v for v in (ldx, ldf, lds, ldy)]
    return goldy_residual_norm_desc(rows, n, *ld, int(dtype), int(param_dtype), int(norm_f), int(norm_y), float(eps),
                                    float(alpha), 0)


def residual_norm_params(gate: int = 0, gamma_f: int = 0, beta_f: int = 0, gamma_y: int = 0,
                         beta_y: int = 0) -> goldy_residual_norm_params:
    """Device pointers of the parameters, or of their fp32 gradients (0: absent)."""
    return goldy_residual_norm_params(gate or None, gamma_f or None, beta_f or None, gamma_y or None, beta_y or None)


def goldy_residual_norm_query(d: goldy_residual_norm_desc) -> int:
    """Workspace bytes of the backward call."""
    ws = ctypes.c_size_t()
    _check(_lib.goldy_residual_norm_query(d, ctypes.byref(ws)), "goldy_residual_norm_query")
    return int(ws.value)


def goldy_residual_norm_forward(d: goldy_residual_norm_desc, params: Optional[goldy_residual_norm_params], X: int, F: int,
                                S: int, Y: int = 0, stats: int = 0, stream: int = 0) -> None:
    _check(_lib.goldy_residual_norm_forward(d, params, X or None, F or None, S or None, Y or None, stats or None,
                                            stream or None), "goldy_residual_norm_forward")


def goldy_residual_norm_backward(d: goldy_residual_norm_desc, params: Optional[goldy_residual_norm_params], dY: int, dS: int,
                                 F: int, S: int, stats: int, dX: int, dF: int,
                                 grads: Optional[goldy_residual_norm_params] = None, workspace: int = 0,
                                 workspace_bytes: int = 0, stream: int = 0, accumulate: bool = False) -> None:
    _check(_lib.goldy_residual_norm_backward(d, params, dY or None, dS or None, F or None, S or None, stats or None,
                                             dX or None, dF or None, grads, 1 if accumulate else 0, workspace or None,
                                             workspace_bytes, stream or None), "goldy_residual_norm_backward")


def keep8_desc(rows: int, n: int, dtype: int = GOLDY_BF16, act: int = GOLDY_ACT_NONE, ldz: Optional[int] = None,
               ldh: Optional[int] = None) -> goldy_keep8_desc:
    """Descriptor of rows of n pre-activations kept in 8 bits (default: packed)."""
    return goldy_keep8_desc(rows, n, n if ldz is None else ldz, n if ldh is None else ldh, int(dtype), int(act), 0)


def goldy_keep8_query(d: goldy_keep8_desc) -> Tuple[int, int]:
    """(bytes of Q, bytes of scales)."""
    q, s = ctypes.c_size_t(), ctypes.c_size_t()
    _check(_lib.goldy_keep8_query(d, ctypes.byref(q), ctypes.byref(s)), "goldy_keep8_query")
    return int(q.value), int(s.value)


def goldy_keep8_pack(d: goldy_keep8_desc, Z: int, Q: int, scales: int, stream: int = 0) -> None:
    _check(_lib.goldy_keep8_pack(d, Z or None, Q or None, scales or None, stream or None), "goldy_keep8_pack")


def goldy_keep8_unpack(d: goldy_keep8_desc, Q: int, scales: int, Z: int = 0, H: int = 0, stream: int = 0) -> None:
    """Z as it was kept, H = act(Z); either may be 0."""
    _check(_lib.goldy_keep8_unpack(d, Q or None, scales or None, Z or None, H or None, stream or None), "goldy_keep8_unpack")


def goldy_device_error(clear: bool = True) -> int:
    code = ctypes.c_int()
    _check(_lib.goldy_device_error(ctypes.byref(code), 1 if clear else 0), "goldy_device_error")
    return code.value


def goldy_device_info(variant_id: int = 0) -> Tuple[int, int]:
    """(SM count, resident CTAs per SM of the variant's kernel)."""
    sm, ctas = ctypes.c_int(), ctypes.c_int()
    _check(_lib.goldy_device_info(int(variant_id), ctypes.byref(sm), ctypes.byref(ctas)),
           "goldy_device_info")
    return sm.value, ctas.value


_SPLITS = (1, 2, 4, 8)
_RC_DIVS = (1, 2, 4)


def variant_id(kind: int, split: int, rc_div: int) -> int:
    """Variant id of (kind, split-K factor, grid-cap divisor): the registry's
    numbering (kind * 4 + split index) * 3 + RC index, checked against it."""
    if split not in _SPLITS or rc_div not in _RC_DIVS:
        raise KeyError((kind, split, rc_div))
    v = (int(kind) * 4 + _SPLITS.index(split)) * 3 + _RC_DIVS.index(rc_div)
    if not 0 <= v < goldy_variant_count():
        raise KeyError((kind, split, rc_div))
    info = goldy_variant_info_get(v)
    if info["kind"] != kind or info["rc_div"] != rc_div or info["split_k"] not in (split, 1):
        raise KeyError((kind, split, rc_div))
    return v


def kind_names() -> List[str]:
    names = {}
    for v in range(goldy_variant_count()):
        info = goldy_variant_info_get(v)
        names.setdefault(info["kind"], info["name"].split("_s")[0])
    return [names[k] for k in sorted(names)]
