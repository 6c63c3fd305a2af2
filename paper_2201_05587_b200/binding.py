"""Python binding of libtt.so: argument marshalling only.

Names mirror ``include/tt.h``.  Torch tensors supply device memory and the current
stream; every step of the hot path runs inside the library's CUDA kernels.  There
is no fallback: if the library is missing or no GPU is present the calls raise.
The calls a program makes per kernel or per pass (``Workload.run``, ``run_chain``) go
through the CPython module ``_ttcall``; the others through ctypes.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import os

from . import build as _build

HERE = os.path.dirname(os.path.abspath(__file__))

# enums
TT_OK, TT_ERR_INVALID_ARG, TT_ERR_INVALID_SCHEDULE, TT_ERR_CLASS_MISMATCH, TT_ERR_RESOURCE, \
    TT_ERR_NOT_APPLIED, TT_ERR_CUDA, TT_ERR_TIMEOUT, TT_ERR_OOM, TT_ERR_NOT_IMPLEMENTED, TT_SKIPPED = range(11)
TT_OP_CONV2D, TT_OP_DWCONV2D, TT_OP_DENSE, TT_OP_BATCH_MATMUL, TT_OP_SOFTMAX = range(5)
TT_ACT_NONE, TT_ACT_RELU, TT_ACT_RELU6, TT_ACT_GELU_ERF = range(4)
TT_FAMILY_GEMM_TC, TT_FAMILY_DW_SIMT, TT_FAMILY_ROW_SIMT = range(3)
TT_MODE_LEGALISE, TT_MODE_STRICT = 0, 1
TT_TYPE_F32, TT_TYPE_F16, TT_TYPE_BF16 = range(3)
TT_RECORD_VERSION = 3
TT_CHG_TILE_M, TT_CHG_TILE_N, TT_CHG_TILE_K, TT_CHG_STAGES, TT_CHG_SPLIT_K, TT_CHG_VEC, TT_CHG_BLOCK, TT_CHG_ITEMS, TT_CHG_SLAB, TT_CHG_ACC, TT_CHG_KORDER, TT_CHG_FORM, \
    TT_CHG_CLUSTER = 1, 2, 4, 8, 16, 32, 64, 128, 256, 512, 1024, 2048, 4096

i32, i64, u32, f32 = C.c_int32, C.c_int64, C.c_uint32, C.c_float


class tt_shapes(C.Structure):
    _fields_ = [(n, i32) for n in ("n", "c", "h", "w", "k", "r", "s", "stride_h", "stride_w", "pad_h", "pad_w",
                                   "batch", "m", "nn", "kk", "trans_b", "has_bias", "has_residual", "act")] + \
               [("scale", f32)]


class tt_schedule_record(C.Structure):
    _fields_ = [("version", u32), ("family", u32), ("origin_op", i32), ("origin", tt_shapes)] + \
               [(n, i32) for n in ("tile_m", "tile_n", "tile_k", "stages", "split_k", "raster", "block_x", "block_y",
                                   "items_per_thread", "vec_width", "unroll", "threads", "mma_m_axis", "slab_tiles", "acc_split", "k_order",
                                   "persistent", "cta_group", "ctas_per_sm", "warp_layout", "precision")]

    FIELDS = ("tile_m", "tile_n", "tile_k", "stages", "split_k", "raster", "block_x", "block_y",
              "items_per_thread", "vec_width", "unroll", "threads", "mma_m_axis", "slab_tiles", "acc_split", "k_order",
              "persistent", "cta_group", "ctas_per_sm", "warp_layout", "precision")

    def as_dict(self):
        d = {"family": int(self.family), "origin_op": int(self.origin_op)}
        d.update({k: int(getattr(self, k)) for k in self.FIELDS})
        return d

    def short(self):
        if self.family == TT_FAMILY_GEMM_TC:
            return (f"tc[{self.tile_m}x{self.tile_n}x{self.tile_k} st{self.stages} sk{self.split_k} "
                    f"r{self.raster} ax{self.mma_m_axis}" + (f" sl{self.slab_tiles}" if self.slab_tiles else "") +
                    (f" acc{self.acc_split}" if self.acc_split > 1 else "") + (" tap" if self.k_order else "") +
                    (" ps" if self.persistent else "") + (f" cg{self.cta_group}" if self.cta_group > 1 else "") +
                    (" 2/sm" if self.ctas_per_sm == 2 else "") + (" x3" if self.precision else "") + "]")
        if self.family == TT_FAMILY_DW_SIMT:
            return (f"dw[c{self.tile_m} {self.block_y}x{self.block_x} it{self.items_per_thread} "
                    f"v{self.vec_width} t{self.threads} u{self.unroll}" + (f" tma st{self.stages}" if self.raster else "") + "]")
        return f"row[{self.block_x}x{self.block_y} v{self.vec_width}]"


class tt_tensors(C.Structure):
    _fields_ = [("x", C.c_void_p), ("w", C.c_void_p), ("bias", C.c_void_p), ("residual", C.c_void_p), ("y", C.c_void_p)]


class tt_chain_step(C.Structure):
    _fields_ = [("workload", C.c_void_p), ("tensors", C.POINTER(tt_tensors)), ("waits", C.POINTER(i32)), ("n_waits", i32), ("lane", i32)]


class tt_gemm_view(C.Structure):
    _fields_ = [("batch", i32), ("gm", i32), ("gn", i32), ("gk", i32), ("flops", C.c_double), ("bytes", C.c_double)]


class tt_apply_info(C.Structure):
    _fields_ = [("legal", tt_schedule_record), ("changed", i32), ("grid_x", i32), ("grid_y", i32), ("grid_z", i32),
                ("threads", i32), ("smem_bytes", i32), ("tmem_cols", i32), ("workspace_bytes", C.c_int64),
                ("launches", i32), ("exchange_kib", i32)]


class tt_timing_opts(C.Structure):
    _fields_ = [("warmup_batches", i32), ("batches", i32), ("min_batch_us", i32), ("max_repeats", i32),
                ("use_graph", i32), ("floor", i32), ("reserved", i32 * 2)]


class tt_timing(C.Structure):
    _fields_ = [("median_us", f32), ("min_us", f32), ("max_us", f32), ("q1_us", f32), ("q3_us", f32),
                ("repeats", i32), ("batches", i32)]


class tt_tune_opts(C.Structure):
    _fields_ = [("timing", tt_timing_opts), ("mode", i32), ("strict_class", i32), ("include_default", i32),
                ("subsample_percent", i32), ("subsample_gain_percent", i32), ("subsample_seed", u32), ("reserved", i32 * 2)]


class tt_tune_result(C.Structure):
    _fields_ = [("chosen", C.POINTER(i32)), ("best_us", C.POINTER(f32)), ("times_us", C.POINTER(f32)),
                ("status", C.POINTER(i32)), ("search_seconds", C.c_double), ("pairs_timed", i32),
                ("pairs_invalid", i32), ("pairs_skipped", i32)]


class tt_quantize_args(C.Structure):
    _fields_ = [("x", C.c_void_p), ("q", C.c_void_p), ("scales", C.c_void_p), ("x_row", i64), ("q_row", i64), ("s_row", i64), ("s_block", i64),
                ("x_type", i32), ("m", i32), ("kk", i32), ("block_rows", i32)]


class tt_dense_quantized_args(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("x", "w", "x_scale", "w_scale", "bias", "y", "status")] + \
               [(n, i64) for n in ("x_row", "w_row", "y_row", "xs_row", "xs_block", "ws_row", "ws_block")] + \
               [(n, i32) for n in ("y_type", "m", "nn", "kk", "act")]


class tt_rotary_args(C.Structure):
    _fields_ = [("x", C.c_void_p * 2), ("y", C.c_void_p * 2), ("x_token", i64 * 2), ("x_head", i64 * 2), ("y_token", i64 * 2), ("y_head", i64 * 2),
                ("positions", C.c_void_p), ("turns", C.c_void_p), ("heads", i32 * 2)] + \
               [(n, i32) for n in ("type", "position_bits", "tokens", "d", "rot", "interleaved", "inverse")] + [("factor", f32)]


class tt_cache(C.Structure):
    _fields_ = [("data", C.c_void_p * 2), ("scale", C.c_void_p * 2), ("page", i64 * 2), ("head", i64 * 2), ("token", i64 * 2), ("s_page", i64 * 2),
                ("s_head", i64 * 2), ("table", C.c_void_p), ("table_row", i64)] + \
               [(n, i32) for n in ("pages", "heads", "block", "d", "batch", "max_pages")]


class tt_cache_append_args(C.Structure):
    _fields_ = [("cache", tt_cache), ("x", C.c_void_p * 2), ("x_token", i64 * 2), ("x_head", i64 * 2), ("starts", C.c_void_p), ("lengths", C.c_void_p),
                ("status", C.c_void_p), ("type", i32), ("tokens", i32)]


class tt_cache_attention_args(C.Structure):
    _fields_ = [("cache", tt_cache), ("q", C.c_void_p), ("y", C.c_void_p), ("q_token", i64), ("q_head", i64), ("y_token", i64), ("y_head", i64),
                ("starts", C.c_void_p), ("lengths", C.c_void_p), ("status", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", i64)] + \
               [(n, i32) for n in ("type", "tokens", "heads_q", "causal", "window", "max_count", "max_length")] + [("scale", f32)]


EXPORTS = {
    "tt_status_string": (C.c_char_p, [i32]),
    "tt_workload_create": (i32, [i32, C.POINTER(tt_shapes), C.POINTER(C.c_void_p)]),
    "tt_workload_destroy": (i32, [C.c_void_p]),
    "tt_workload_key": (i32, [C.c_void_p, C.POINTER(C.c_uint64)]),
    "tt_workload_class": (i32, [C.c_void_p, C.POINTER(C.c_uint64)]),
    "tt_workload_family": (i32, [C.c_void_p, C.POINTER(i32)]),
    "tt_workload_gemm_view": (i32, [C.c_void_p, C.POINTER(tt_gemm_view)]),
    "tt_default_schedule": (i32, [C.c_void_p, C.POINTER(tt_schedule_record)]),
    "tt_schedule_check": (i32, [C.c_void_p, C.POINTER(tt_schedule_record), i32, i32, C.POINTER(tt_apply_info)]),
    "tt_schedule_apply": (i32, [C.c_void_p, C.POINTER(tt_schedule_record), C.POINTER(tt_apply_info)]),
    "tt_schedule_apply_ex": (i32, [C.c_void_p, C.POINTER(tt_schedule_record), i32, i32, C.POINTER(tt_apply_info)]),
    "tt_split_check": (i32, [C.c_int64, C.POINTER(C.c_int64), C.c_size_t, i32, C.POINTER(i32)]),
    "tt_run": (i32, [C.c_void_p, C.POINTER(tt_tensors), C.c_void_p]),
    "tt_run_chain": (i32, [C.POINTER(tt_chain_step), C.c_size_t, C.POINTER(C.c_void_p), C.c_size_t, C.POINTER(C.c_size_t)]),
    "tt_chain_launches": (i32, [C.POINTER(tt_chain_step), C.c_size_t, C.POINTER(C.c_size_t)]),
    "tt_chain_ahead": (i32, [C.POINTER(tt_chain_step), C.c_size_t, C.POINTER(C.c_size_t)]),
    "tt_run_host": (i32, [C.c_void_p, C.POINTER(tt_tensors), C.c_void_p, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]),
    "tt_run_host_async": (i32, [C.c_void_p, C.POINTER(tt_tensors), C.c_void_p, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]),
    "tt_workload_status": (i32, [C.c_void_p, C.c_void_p]),
    "tt_workload_set_constant_weights": (i32, [C.c_void_p, i32]),
    "tt_workload_set_wait_limit": (i32, [C.c_void_p, C.c_uint64]),
    "tt_workload_test_stall": (i32, [C.c_void_p, C.c_uint32]),
    "tt_time": (i32, [C.c_void_p, C.POINTER(tt_tensors), C.c_size_t, C.c_void_p, C.POINTER(tt_timing_opts),
                      C.POINTER(tt_timing)]),
    "tt_select": (i32, [C.POINTER(f32), C.c_size_t, C.c_size_t, C.POINTER(i32)]),
    "tt_model_latency": (i32, [C.POINTER(f32), C.c_size_t, C.c_size_t, C.POINTER(i32), C.POINTER(i32),
                               C.POINTER(C.c_double)]),
    "tt_rank_pools": (i32, [C.POINTER(C.c_double), C.c_size_t, C.POINTER(i32), C.c_size_t, C.POINTER(C.c_double),
                            C.POINTER(i32)]),
    "tt_transfer_tune": (i32, [C.POINTER(C.c_void_p), C.POINTER(tt_tensors), C.c_size_t, C.POINTER(tt_schedule_record),
                               C.c_size_t, C.POINTER(tt_tune_opts), C.c_void_p, C.POINTER(tt_tune_result)]),
    "tt_transfer_tune_sets": (i32, [C.POINTER(C.c_void_p), C.POINTER(tt_tensors), C.POINTER(C.c_size_t), C.c_size_t,
                                    C.POINTER(tt_schedule_record), C.c_size_t, C.POINTER(tt_tune_opts), C.c_void_p,
                                    C.POINTER(tt_tune_result)]),
    "tt_grid_tune": (i32, [C.c_void_p, C.POINTER(tt_tensors), C.c_void_p, C.POINTER(tt_timing_opts), i32, C.c_size_t,
                           C.POINTER(tt_schedule_record), C.POINTER(f32), C.POINTER(C.c_size_t), C.POINTER(i32)]),
    "tt_record_neighbours": (i32, [C.c_void_p, C.POINTER(tt_schedule_record), C.POINTER(tt_schedule_record), C.c_size_t,
                                   C.POINTER(C.c_size_t)]),
    "tt_refine_with": (i32, [C.c_void_p, C.POINTER(tt_schedule_record), C.c_void_p, C.c_void_p, i32, f32,
                             C.POINTER(tt_schedule_record), C.POINTER(f32), C.POINTER(f32), C.POINTER(i32)]),
    "tt_refine": (i32, [C.c_void_p, C.POINTER(tt_tensors), C.c_void_p, C.POINTER(tt_timing_opts),
                        C.POINTER(tt_schedule_record), i32, f32, C.POINTER(tt_schedule_record), C.POINTER(f32),
                        C.POINTER(f32), C.POINTER(i32)]),
    "tt_pool_subsample": (i32, [C.c_size_t, C.c_size_t, C.c_uint64, C.POINTER(i32)]),
    "tt_pool_save": (i32, [C.c_char_p, C.POINTER(tt_schedule_record), C.POINTER(f32), C.c_size_t]),
    "tt_pool_load": (i32, [C.c_char_p, C.POINTER(tt_schedule_record), C.POINTER(f32), C.c_size_t, C.POINTER(C.c_size_t)]),
    "tt_dense_static_scratch": (i32, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, i32, i32, i32, i32,
                                      C.POINTER(tt_schedule_record), C.c_void_p, C.POINTER(C.c_int64)]),
    "tt_quantize": (i32, [C.POINTER(tt_quantize_args), C.c_void_p]),
    "tt_dense_quantized": (i32, [C.POINTER(tt_dense_quantized_args), C.c_void_p]),
    "tt_rotary": (i32, [C.POINTER(tt_rotary_args), C.c_void_p]),
    "tt_rotary_turns": (i32, [C.POINTER(C.c_double), C.c_size_t, C.POINTER(C.c_uint64)]),
    "tt_cache_append": (i32, [C.POINTER(tt_cache_append_args), C.c_void_p]),
    "tt_cache_attention": (i32, [C.POINTER(tt_cache_attention_args), C.c_void_p]),
    "tt_cache_attention_workspace": (i32, [C.POINTER(tt_cache_attention_args), C.POINTER(i64)]),
}

_lib = None
_call = None        # the CPython module of the hot calls, loaded with the library


def lib():
    """Load libtt.so (building it with nvcc first if the sources are newer).  Raises if that fails."""
    global _lib, _call
    if _lib is None:
        path = _build.LIB
        if _build.needs_build():
            path = _build.build()
        handle = C.CDLL(path)
        for name, (res, args) in EXPORTS.items():
            fn = getattr(handle, name)          # AttributeError if a declared symbol is missing
            fn.restype, fn.argtypes = res, args
        spec = importlib.util.spec_from_file_location("_ttcall", _build.CALL_LIB)
        call = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(call)
        call.bind(C.cast(handle.tt_run, C.c_void_p).value, C.cast(handle.tt_run_chain, C.c_void_p).value)
        _call = call
        _lib = handle
    return _lib


class TTError(RuntimeError):
    def __init__(self, status, what=""):
        self.status = int(status)
        msg = lib().tt_status_string(self.status).decode()
        super().__init__(f"{what}: {msg} (tt_status {self.status})" if what else f"{msg} (tt_status {self.status})")


def _check(status, what=""):
    if status != TT_OK:
        raise TTError(status, what)


def status_string(s: int) -> str:
    return lib().tt_status_string(int(s)).decode()


def make_shapes(**kw) -> tt_shapes:
    s = tt_shapes()
    for k, v in kw.items():
        if not hasattr(s, k):
            raise KeyError(k)
        setattr(s, k, v)
    return s


def conv2d_shapes(n, c, h, w, k, r, s, stride=1, pad=0, has_bias=True, act=TT_ACT_RELU, has_residual=False):
    return make_shapes(n=n, c=c, h=h, w=w, k=k, r=r, s=s, stride_h=stride, stride_w=stride, pad_h=pad, pad_w=pad,
                       has_bias=int(has_bias), act=act, has_residual=int(has_residual))


def dense_shapes(m, nn, kk, has_bias=True, act=TT_ACT_NONE):
    return make_shapes(batch=1, m=m, nn=nn, kk=kk, trans_b=1, has_bias=int(has_bias), act=act)


def bmm_shapes(batch, m, nn, kk, trans_b=True):
    return make_shapes(batch=batch, m=m, nn=nn, kk=kk, trans_b=int(trans_b))


def softmax_shapes(batch, m, nn, scale=1.0):
    return make_shapes(batch=batch, m=m, nn=nn, scale=scale)


def make_record(family, **kw) -> tt_schedule_record:
    r = tt_schedule_record()
    r.version = TT_RECORD_VERSION
    r.family = family
    defaults = dict(tile_m=128, tile_n=128, tile_k=32, stages=4, split_k=1, raster=0, block_x=32, block_y=4,
                    items_per_thread=1, vec_width=1, unroll=1, threads=128, mma_m_axis=0, slab_tiles=0, acc_split=1, k_order=0,
                    persistent=0, cta_group=1, ctas_per_sm=0, warp_layout=0, precision=0)
    defaults.update(kw)
    for k, v in defaults.items():
        setattr(r, k, v)
    return r


def split_check(extent, factors, reformulate=False) -> bool:
    arr = (C.c_int64 * len(factors))(*factors)
    v = i32(0)
    _check(lib().tt_split_check(extent, arr, len(factors), int(reformulate), C.byref(v)), "tt_split_check")
    return bool(v.value)


def select(times, n_wl, n_cols):
    arr = (f32 * (n_wl * n_cols))(*[float(t) for t in times])
    out = (i32 * n_wl)()
    _check(lib().tt_select(arr, n_wl, n_cols, out), "tt_select")
    return list(out)


def model_latency(times, n_wl, n_cols, chosen, use_count) -> float:
    arr = (f32 * (n_wl * n_cols))(*[float(t) for t in times])
    ch = (i32 * n_wl)(*chosen)
    uc = (i32 * n_wl)(*use_count)
    out = C.c_double(0)
    _check(lib().tt_model_latency(arr, n_wl, n_cols, ch, uc, C.byref(out)), "tt_model_latency")
    return out.value


def rank_pools(class_share, class_kernels):
    """Equation 1: class_share[c] of the target model, class_kernels[t][c] of each candidate; returns (scores, order)."""
    n_c, n_m = len(class_share), len(class_kernels)
    sh = (C.c_double * n_c)(*[float(v) for v in class_share])
    ck = (i32 * (n_c * max(n_m, 1)))(*[int(v) for row in class_kernels for v in row])
    sc = (C.c_double * max(n_m, 1))()
    od = (i32 * max(n_m, 1))()
    _check(lib().tt_rank_pools(sh, n_c, ck, n_m, sc, od), "tt_rank_pools")
    return list(sc)[:n_m], list(od)[:n_m]


def pool_subsample(n_pool, count, seed):
    """tt_pool_subsample: the first `count` indices of the seeded shuffle of range(n_pool)."""
    out = (i32 * max(count, 1))()
    _check(lib().tt_pool_subsample(n_pool, count, seed, out), "tt_pool_subsample")
    return list(out)[:count]


def pool_save(path, records, us=None):
    """tt_pool_save: write records (and the times they were tuned to) as a text pool file."""
    n = len(records)
    arr = (tt_schedule_record * max(n, 1))(*records)
    uarr = (f32 * max(n, 1))(*[float(v) for v in us]) if us is not None else None
    _check(lib().tt_pool_save(os.fsencode(path), arr, uarr, n), f"tt_pool_save({path})")


def pool_load(path):
    """tt_pool_load: returns (records, times in microseconds)."""
    n = C.c_size_t()
    _check(lib().tt_pool_load(os.fsencode(path), None, None, 0, C.byref(n)), f"tt_pool_load({path})")
    arr = (tt_schedule_record * max(n.value, 1))()
    uarr = (f32 * max(n.value, 1))()
    _check(lib().tt_pool_load(os.fsencode(path), arr, uarr, n.value, C.byref(n)), f"tt_pool_load({path})")
    out = []
    for i in range(n.value):
        r = tt_schedule_record()
        C.memmove(C.byref(r), C.byref(arr[i]), C.sizeof(r))
        out.append(r)
    return out, [float(uarr[i]) for i in range(n.value)]


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def tensors(x, w=None, bias=None, residual=None, y=None) -> tt_tensors:
    """Device pointers of torch CUDA tensors (or host pointers of CPU tensors for tt_run_host)."""
    t = tt_tensors()
    t.x, t.w, t.bias, t.residual, t.y = _ptr(x), _ptr(w), _ptr(bias), _ptr(residual), _ptr(y)
    return t


_torch = None


def _import_torch():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _raw_stream() -> int:
    """The current stream of the current device as an integer (torch's own stream object costs a microsecond to make)."""
    torch = _torch or _import_torch()
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _stream():
    return C.c_void_p(_raw_stream())


def run_chain(wls, steps, tts, plan, streams):
    """tt_run_chain over the nodes of a chain (workloads.run_chain): streams are torch streams, whose device is made current."""
    torch = _torch or _import_torch()
    devices = {s.device_index for s in streams}
    if len(devices) > 1:
        return _run_chain_over_devices(wls, steps, tts, plan, streams)
    if devices == {torch.cuda.current_device()}:
        st, at = _call.run_chain(wls, steps, tts, plan, [s.cuda_stream for s in streams])
    else:
        with torch.cuda.device(streams[0].device):
            st, at = _call.run_chain(wls, steps, tts, plan, [s.cuda_stream for s in streams])
    if st != TT_OK:
        raise TTError(st, f"tt_run({wls[steps[at].kernel].name})" if at >= 0 else "tt_run_chain")


def _query_chain(function, wls, steps, tts, plan):
    st, values = _call.query_chain(wls, steps, tts, plan, C.cast(getattr(lib(), function), C.c_void_p).value)
    _check(st, function)
    return values


def chain_launches(wls, steps, tts, plan):
    """How many kernels run_chain launches for these arguments (tt_chain_launches)."""
    return sum(_query_chain("tt_chain_launches", wls, steps, tts, plan))


def chain_ahead(wls, steps, tts, plan):
    """Per node, how many bytes of weights its launch brings into the L2 for the ones behind it (tt_chain_ahead)."""
    return _query_chain("tt_chain_ahead", wls, steps, tts, plan)


def _run_chain_over_devices(wls, steps, tts, plan, streams):
    """The same pass layer by layer, for lanes on several devices: a native call enqueues on one."""
    needed = {p for pl in plan if pl is not None for p in pl[1]}
    start, events, used = streams[0].record_event(), {}, set()
    for i, (st, tt, pl) in enumerate(zip(steps, tts, plan)):
        if pl is None:
            continue
        lane, waits = pl
        s = streams[lane]
        if lane != 0 and lane not in used:
            s.wait_event(start)
        used.add(lane)
        for p in waits:
            s.wait_event(events[p])
        with _torch.cuda.stream(s):
            wls[st.kernel].run(tt)
        if i in needed:
            events[i] = s.record_event()
    for lane in sorted(used - {0}):
        streams[0].wait_event(streams[lane].record_event())


class Workload:
    """Owns one tt_workload handle."""

    def __init__(self, op, shapes: tt_shapes, name: str = "", use_count: int = 1):
        self.op, self.shapes, self.name, self.use_count = op, shapes, name, use_count
        h = C.c_void_p()
        _check(lib().tt_workload_create(op, C.byref(shapes), C.byref(h)), f"tt_workload_create({name})")
        self.handle, self.address = h, h.value

    def close(self):
        if getattr(self, "handle", None):
            lib().tt_workload_destroy(self.handle)
            self.handle = self.address = None

    __del__ = close

    def key(self) -> int:
        v = C.c_uint64()
        _check(lib().tt_workload_key(self.handle, C.byref(v)))
        return v.value

    def kernel_class(self) -> int:
        v = C.c_uint64()
        _check(lib().tt_workload_class(self.handle, C.byref(v)))
        return v.value

    def family(self) -> int:
        v = i32()
        _check(lib().tt_workload_family(self.handle, C.byref(v)))
        return v.value

    def gemm_view(self) -> tt_gemm_view:
        v = tt_gemm_view()
        _check(lib().tt_workload_gemm_view(self.handle, C.byref(v)))
        return v

    def default_schedule(self) -> tt_schedule_record:
        r = tt_schedule_record()
        _check(lib().tt_default_schedule(self.handle, C.byref(r)))
        return r

    def check(self, rec, mode=TT_MODE_LEGALISE, strict_class=False):
        """Returns (status, tt_apply_info); never raises for an invalid record."""
        info = tt_apply_info()
        st = lib().tt_schedule_check(self.handle, C.byref(rec), mode, int(strict_class), C.byref(info))
        return st, info

    def apply(self, rec, mode=TT_MODE_LEGALISE, strict_class=False) -> tt_apply_info:
        info = tt_apply_info()
        _check(lib().tt_schedule_apply_ex(self.handle, C.byref(rec), mode, int(strict_class), C.byref(info)),
               f"tt_schedule_apply({self.name})")
        return info

    def try_apply(self, rec, mode=TT_MODE_LEGALISE, strict_class=False):
        info = tt_apply_info()
        st = lib().tt_schedule_apply_ex(self.handle, C.byref(rec), mode, int(strict_class), C.byref(info))
        return st, info

    def run(self, t: tt_tensors):
        st = _call.run(self.address or 0, t, _raw_stream())
        if st != TT_OK:
            raise TTError(st, f"tt_run({self.name})")

    def run_host(self, t: tt_tensors):
        up, down = C.c_int64(), C.c_int64()
        _check(lib().tt_run_host(self.handle, C.byref(t), _stream(), C.byref(up), C.byref(down)),
               f"tt_run_host({self.name})")
        return up.value, down.value

    def run_host_async(self, t: tt_tensors, stream=None):
        """tt_run_host_async on `stream` (a torch.cuda.Stream; default: the current one): enqueues only."""
        up, down = C.c_int64(), C.c_int64()
        sp = _stream() if stream is None else C.c_void_p(stream.cuda_stream)
        _check(lib().tt_run_host_async(self.handle, C.byref(t), sp, C.byref(up), C.byref(down)),
               f"tt_run_host_async({self.name})")
        return up.value, down.value

    def status(self, stream=None) -> int:
        sp = _stream() if stream is None else C.c_void_p(stream.cuda_stream)
        return lib().tt_workload_status(self.handle, sp)

    def set_constant_weights(self, on: bool = True):
        _check(lib().tt_workload_set_constant_weights(self.handle, int(bool(on))), "tt_workload_set_constant_weights")

    def set_wait_limit(self, nanoseconds: int):
        _check(lib().tt_workload_set_wait_limit(self.handle, int(nanoseconds)), "tt_workload_set_wait_limit")

    def test_stall(self, extra_bytes: int):
        _check(lib().tt_workload_test_stall(self.handle, int(extra_bytes)), "tt_workload_test_stall")

    def time(self, sets, opts: tt_timing_opts | None = None) -> tt_timing:
        if isinstance(sets, tt_tensors):
            sets = [sets]
        arr = (tt_tensors * len(sets))(*sets)
        out = tt_timing()
        _check(lib().tt_time(self.handle, arr, len(sets), _stream(), C.byref(opts) if opts else None, C.byref(out)),
               f"tt_time({self.name})")
        return out

    def grid_tune(self, t: tt_tensors, opts: tt_timing_opts | None = None, level=0, top_k=1):
        recs = (tt_schedule_record * top_k)()
        us = (f32 * top_k)()
        n = C.c_size_t()
        tried = i32()
        _check(lib().tt_grid_tune(self.handle, C.byref(t), _stream(), C.byref(opts) if opts else None, level, top_k,
                                  recs, us, C.byref(n), C.byref(tried)), f"tt_grid_tune({self.name})")
        out = []
        for i in range(n.value):
            r = tt_schedule_record()
            C.memmove(C.byref(r), C.byref(recs[i]), C.sizeof(r))
            out.append((r, float(us[i])))
        return out, tried.value


    def neighbours(self, rec):
        """tt_record_neighbours: the legalised one-step neighbours of `rec` on this workload."""
        out = (tt_schedule_record * 32)()
        n = C.c_size_t()
        _check(lib().tt_record_neighbours(self.handle, C.byref(rec), out, 32, C.byref(n)), f"tt_record_neighbours({self.name})")
        res = []
        for i in range(n.value):
            r = tt_schedule_record()
            C.memmove(C.byref(r), C.byref(out[i]), C.sizeof(r))
            res.append(r)
        return res

    def refine_with(self, start, time_us, max_rounds=8, min_gain=0.0):
        """tt_refine_with: greedy descent from `start` with a Python timing function rec -> microseconds (negative =
        cannot run).  Returns (best record, best_us, start_us, calls of time_us)."""
        def _cb(_user, rec_ptr):
            return float(time_us(rec_ptr.contents))
        cb = TIME_FN(_cb)
        best, bus, sus, nt = tt_schedule_record(), f32(), f32(), i32()
        _check(lib().tt_refine_with(self.handle, C.byref(start), C.cast(cb, C.c_void_p), None, max_rounds, min_gain,
                                    C.byref(best), C.byref(bus), C.byref(sus), C.byref(nt)), f"tt_refine_with({self.name})")
        return best, bus.value, sus.value, nt.value

    def refine(self, t: tt_tensors, start, opts: tt_timing_opts | None = None, max_rounds=4, min_gain=0.02):
        """tt_refine: the same with device times (median of tt_time); leaves the best record applied."""
        best, bus, sus, nt = tt_schedule_record(), f32(), f32(), i32()
        _check(lib().tt_refine(self.handle, C.byref(t), _stream(), C.byref(opts) if opts else None, C.byref(start),
                               max_rounds, min_gain, C.byref(best), C.byref(bus), C.byref(sus), C.byref(nt)),
               f"tt_refine({self.name})")
        return best, bus.value, sus.value, nt.value


TIME_FN = C.CFUNCTYPE(f32, C.c_void_p, C.POINTER(tt_schedule_record))
TT_STATIC_SCRATCH_BYTES = 8 << 20


def dense_static_scratch(x, w, bias, y, act, rec):
    """tt_dense_static_scratch on torch CUDA tensors x [m,kk], w [nn,kk], bias [nn] or None, y [m,nn]: the dense
    layer under `rec` with its split-K scratch in the library's fixed device array, for callers that cannot
    allocate device memory.  Returns (tt_status, scratch bytes the record needs); never raises."""
    m, kk = x.shape
    nn = w.shape[0]
    used = C.c_int64(0)
    st = lib().tt_dense_static_scratch(_ptr(x), _ptr(w), _ptr(bias), _ptr(y), m, nn, kk, act, C.byref(rec), _stream(),
                                       C.byref(used))
    return st, used.value


# ---- 8-bit operators of a transformer's inference pass ----------------------------------------------------------------------
#
# Each function below checks its tensors and returns a Call: the arguments of the native call, made once, for a program that repeats it
# on the same tensors (Call.run enqueues it on the current stream, which may be capturing).  It keeps references to the tensors.

class Call:
    """One call of an 8-bit operator: ``run`` enqueues it on the current stream of its tensors' device, ``status`` reads what only the
    device has seen.  A call that has a status word or a workspace is made outside of stream captures; its runs share them, so they
    follow each other: the caller orders them when they go to different streams.  It may be dropped while runs are under way on any stream; a
    captured one is kept as long as the graph is replayed, and the tensors that it was made of belong to the caller as ever."""

    def __init__(self, name, args, keep, device, status=None, workspace=None):
        lib()
        self.name, self.args, self._keep, self._status = name, args, keep, status
        self._device, self._index = device, device.index
        self._address = C.cast(getattr(_lib, name), C.c_void_p).value
        # the call's own device words, and the streams that their memory waits for when it is given back
        self._words = [t for t in (status, workspace) if t is not None]
        self._streams = {_torch._C._cuda_getCurrentRawStream(self._index)} if self._words else None

    def run(self):
        torch = _torch
        stream = torch._C._cuda_getCurrentRawStream(self._index)
        if self._words and stream not in self._streams:
            for t in self._words:
                t.record_stream(torch.cuda.current_stream(self._device))
            self._streams.add(stream)
        if torch.cuda.current_device() == self._index:
            st = _call.call(self._address, self.args, stream)
        else:
            with torch.cuda.device(self._index):
                st = _call.call(self._address, self.args, stream)
        if st != TT_OK:
            raise TTError(st, self.name)

    def status(self) -> int:
        """Waits for the runs on the current stream; TT_OK, or what one of them has reported since the last look (and clears it)."""
        if self._status is None:
            _torch.cuda.current_stream(self._device).synchronize()
            return TT_OK
        word = int(self._status.item())
        if word:
            self._status.zero_()
        return word & 0xff


def _need(ok, what):
    if not ok:
        raise TTError(TT_ERR_INVALID_ARG, what)


def _type_of(t):
    torch = _import_torch()
    types = {torch.float32: TT_TYPE_F32, torch.float16: TT_TYPE_F16, torch.bfloat16: TT_TYPE_BF16}
    _need(t.dtype in types, f"elements of {t.dtype}")
    return types[t.dtype]


def _same_device(first, *others):
    _need(first.is_cuda, "tensors live on a GPU")
    _need(all(t is None or t.device == first.device for t in others), "tensors live on one device")
    return first.device


def _is_f8(t):
    torch = _import_torch()
    return t.dtype in (torch.float8_e4m3fn, torch.uint8)


def _inner(t, what):
    _need(t.shape[-1] <= 1 or t.stride(-1) == 1, f"{what}: the last axis is contiguous")


def _row(t):
    """Elements from row to row; a single row's may be anything."""
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _f32(t, shape, what):
    _need(t.dtype == _torch.float32 and tuple(t.shape) == tuple(shape), f"{what}: float32 {tuple(shape)}")


def _device_words(device, n_bytes):
    """Device memory that is zero when this returns, whatever stream is used afterwards."""
    torch = _torch
    _need(not torch.cuda.is_current_stream_capturing(), "a call with device words of its own is made outside of captures")
    t = torch.zeros(max(int(n_bytes), 4), dtype=torch.uint8, device=device)
    torch.cuda.current_stream(device).synchronize()
    return t


def _status_word(device):
    return _device_words(device, 4).view(_torch.int32)


def quantize(x, q, scales, block_rows=1) -> Call:
    """tt_quantize: x [m, k] (float32, float16 or bfloat16) -> q [m, k] (e4m3) and scales [ceil(k / 128), ceil(m / block_rows)] (float32),
    of any strides; the last axis of x and q is contiguous.  For dense_quantized the rows of q start on 16-byte boundaries."""
    _need(x.dim() == 2 and q.shape == x.shape and _is_f8(q), "x [m, k] and q [m, k] in e4m3")
    _need(block_rows in (1, 128), "block_rows is 1 or 128")
    m, k = x.shape
    device = _same_device(x, q, scales)
    _f32(scales, (-(-k // 128), -(-m // block_rows)), "scales")
    _inner(x, "x"), _inner(q, "q")
    a = tt_quantize_args(x=x.data_ptr(), q=q.data_ptr(), scales=scales.data_ptr(), x_row=_row(x), q_row=_row(q), s_row=scales.stride(1),
                            s_block=scales.stride(0), x_type=_type_of(x), m=m, kk=k, block_rows=block_rows)
    return Call("tt_quantize", a, (x, q, scales), device)


def dense_quantized(x, x_scale, w, w_scale, y, bias=None, act=TT_ACT_NONE) -> Call:
    """tt_dense_quantized: y [m, n] = act(x w^T + bias) of x [m, k] and w [n, k] in e4m3 with x_scale [ceil(k / 128), m] and w_scale
    [ceil(n / 128), ceil(k / 128)] (float32, any strides); y float32, float16 or bfloat16, bias float32 [n] or None."""
    _need(x.dim() == 2 and w.dim() == 2 and y.dim() == 2 and _is_f8(x) and _is_f8(w), "x [m, k] and w [n, k] in e4m3")
    (m, k), n = x.shape, w.shape[0]
    _need(w.shape[1] == k and tuple(y.shape) == (m, n), "y [m, n] of x [m, k] and w [n, k]")
    device = _same_device(x, x_scale, w, w_scale, y, bias)
    _f32(x_scale, (-(-k // 128), m), "x_scale")
    _f32(w_scale, (-(-n // 128), -(-k // 128)), "w_scale")
    _inner(x, "x"), _inner(w, "w"), _inner(y, "y")
    if bias is not None:
        _f32(bias, (n,), "bias")
        _inner(bias, "bias")
    pitch = lambda t: _row(t) if t.shape[0] > 1 else -(-t.shape[1] // 16) * 16      # noqa: E731  (a single row has no pitch)
    status = _status_word(device)
    a = tt_dense_quantized_args(x=x.data_ptr(), w=w.data_ptr(), x_scale=x_scale.data_ptr(), w_scale=w_scale.data_ptr(),
                         bias=None if bias is None else bias.data_ptr(), y=y.data_ptr(), status=status.data_ptr(), x_row=pitch(x), w_row=pitch(w),
                         y_row=_row(y), xs_row=x_scale.stride(1), xs_block=x_scale.stride(0), ws_row=w_scale.stride(0), ws_block=w_scale.stride(1),
                         y_type=_type_of(y), m=m, nn=n, kk=k, act=act)
    return Call("tt_dense_quantized", a, (x, x_scale, w, w_scale, y, bias), device, status)


def rotary_frequencies(rot, base=10000.0, scaling=None, factor=1.0, context=4096, slow=1.0, fast=32.0):
    """Angles per position, in radians, of the rot / 2 pairs: base^(-2i / rot), scaled for contexts `factor` times as long as the one that the
    weights were trained on.  scaling: None, "linear" (all positions divided by the factor), "base" (a larger base, so that the slowest
    pair slows down by the factor and the fastest keeps its pace) or "by_parts" (pairs that turn less than `slow` times over the training
    context are divided, those that turn more than `fast` times are kept, the ones between are blended)."""
    _need(rot >= 0 and rot % 2 == 0 and base > 0 and factor > 0 and scaling in (None, "linear", "base", "by_parts") and fast > slow, "rotary_frequencies")
    if scaling == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        return [v / factor for v in f]
    if scaling == "by_parts":
        keep = [min(1.0, max(0.0, (context * v / 6.283185307179586 - slow) / (fast - slow))) for v in f]
        return [v * k + v / factor * (1.0 - k) for v, k in zip(f, keep)]
    return f


def rotary_table(frequencies, device=None):
    """tt_rotary_turns: angles per position (radians; a sequence or a float64 tensor) -> the int64 tensor that rotary takes, on `device` (default:
    the tensor's, or the current GPU)."""
    torch = _import_torch()
    if isinstance(frequencies, torch.Tensor):
        device = device if device is not None else frequencies.device
        frequencies = frequencies.double().tolist()
    n = len(frequencies)
    values, turns = (C.c_double * max(n, 1))(*frequencies), (C.c_uint64 * max(n, 1))()
    _check(lib().tt_rotary_turns(values, n, turns), "tt_rotary_turns")
    signed = [v - (1 << 64) if v >> 63 else v for v in list(turns)[:n]]
    return torch.tensor(signed, dtype=torch.int64, device=device if device is not None else "cuda")


def rotary(x, positions, table, y=None, interleaved=False, factor=1.0, inverse=False) -> Call:
    """tt_rotary: one tensor [tokens, heads, d] or two (queries and keys) turned by positions [tokens] (int32 or int64) times the frequencies of
    `table` [rot / 2] (rotary_table) into y (default: in place).  inverse turns back, which is the gradient of the call."""
    xs = list(x) if isinstance(x, (list, tuple)) else [x]
    ys = xs if y is None else list(y) if isinstance(y, (list, tuple)) else [y]
    torch = _import_torch()
    _need(1 <= len(xs) <= 2 and len(ys) == len(xs) and all(t.dim() == 3 for t in xs), "one or two tensors [tokens, heads, d]")
    tokens, _, d = xs[0].shape
    _need(all(u.shape == t.shape and u.dtype == t.dtype == xs[0].dtype and t.shape[0] == tokens and t.shape[2] == d for t, u in zip(xs, ys)), "tensors of the same tokens, head size and type")
    _need(positions.dtype in (torch.int32, torch.int64) and tuple(positions.shape) == (tokens,) and (tokens <= 1 or positions.stride(0) == 1), "positions [tokens]")
    _need(table.dtype == torch.int64 and table.dim() == 1 and (table.numel() <= 1 or table.stride(0) == 1) and 2 * table.numel() <= d, "table [rot / 2] of rotary_table")
    device = _same_device(xs[0], *xs, *ys, positions, table)
    a = tt_rotary_args(positions=positions.data_ptr(), turns=table.data_ptr(), type=_type_of(xs[0]), position_bits=32 if positions.dtype == torch.int32 else 64,
                       tokens=tokens, d=d, rot=2 * table.numel(), interleaved=int(bool(interleaved)), inverse=int(bool(inverse)), factor=factor)
    for i, (t, u) in enumerate(zip(xs, ys)):
        _inner(t, "x"), _inner(u, "y")
        a.x[i], a.y[i], a.heads[i] = t.data_ptr(), u.data_ptr(), t.shape[1]
        a.x_token[i], a.x_head[i], a.y_token[i], a.y_head[i] = t.stride(0), t.stride(1), u.stride(0), u.stride(1)
    return Call("tt_rotary", a, (xs, ys, positions, table), device)


class Cache:
    """A paged e4m3 cache (tt_cache): k and v [pages, heads, block, d] (any strides that are multiples of 16, the last axis contiguous), k_scale and
    v_scale [pages, heads] float32, table [batch, pages of a sequence] int32."""

    def __init__(self, k, v, k_scale, v_scale, table):
        torch = _import_torch()
        _need(k.dim() == 4 and v.shape == k.shape and _is_f8(k) and _is_f8(v), "k and v [pages, heads, block, d] in e4m3")
        pages, heads, block, d = k.shape
        _need(table.dtype == torch.int32 and table.dim() == 2, "table [batch, pages of a sequence] int32")
        self.device = _same_device(k, v, k_scale, v_scale, table)
        c = tt_cache(table=table.data_ptr(), table_row=_row(table), pages=pages, heads=heads, block=block, d=d, batch=table.shape[0], max_pages=table.shape[1])
        for i, (t, s) in enumerate(((k, k_scale), (v, v_scale))):
            _f32(s, (pages, heads), "scales")
            _inner(t, "k and v")
            c.data[i], c.scale[i] = t.data_ptr(), s.data_ptr()
            c.page[i], c.head[i], c.token[i] = t.stride(0), t.stride(1), t.stride(2)
            c.s_page[i], c.s_head[i] = s.stride(0), s.stride(1)
        _inner(table, "table")
        self.c, self.keep = c, (k, v, k_scale, v_scale, table)

    def _batch(self, starts, lengths):
        torch = _torch
        _need(starts.dtype == lengths.dtype == torch.int32 and starts.is_contiguous() and lengths.is_contiguous(), "starts and lengths are int32")
        _need(tuple(starts.shape) == (self.c.batch + 1,) and tuple(lengths.shape) == (self.c.batch,), "starts [batch + 1], lengths [batch]")


def cache_append(cache, k, v, starts, lengths) -> Call:
    """tt_cache_append: new keys and values [tokens, heads, d] (float32, float16 or bfloat16) of a batch into their pages.  Sequence b has the tokens
    starts[b] .. starts[b + 1] - 1 (int32, on the device), the last of its lengths[b] tokens."""
    _need(k.dim() == 3 and v.shape == k.shape and v.dtype == k.dtype and tuple(k.shape[1:]) == (cache.c.heads, cache.c.d), "k and v [tokens, heads, d] of the cache")
    cache._batch(starts, lengths)
    device = _same_device(k, v, starts, lengths, *cache.keep)
    _inner(k, "k"), _inner(v, "v")
    status = _status_word(device)
    a = tt_cache_append_args(cache=cache.c, starts=starts.data_ptr(), lengths=lengths.data_ptr(), status=status.data_ptr(), type=_type_of(k), tokens=k.shape[0])
    for i, t in enumerate((k, v)):
        a.x[i], a.x_token[i], a.x_head[i] = t.data_ptr(), t.stride(0), t.stride(1)
    return Call("tt_cache_append", a, (cache, k, v, starts, lengths), device, status)


def cache_attention(cache, q, y, starts, lengths, scale, causal=True, window=0, max_count=0, max_length=0) -> Call:
    """tt_cache_attention: y [tokens, heads_q, d] of the queries q [tokens, heads_q, d] (float16 or bfloat16) over the cache, batched as in
    cache_append.  max_count and max_length: bounds on a sequence's queries and on the lengths, where the program knows them; single tokens
    want max_count=1 (without it 64 of them over 4096 tokens take 195 us for 114)."""
    _need(q.dim() == 3 and y.shape == q.shape and y.dtype == q.dtype and q.shape[2] == cache.c.d, "q and y [tokens, heads_q, d] of the cache")
    cache._batch(starts, lengths)
    device = _same_device(q, y, starts, lengths, *cache.keep)
    _inner(q, "q"), _inner(y, "y")
    status = _status_word(device)
    a = tt_cache_attention_args(cache=cache.c, q=q.data_ptr(), y=y.data_ptr(), q_token=q.stride(0), q_head=q.stride(1), y_token=y.stride(0),
                                y_head=y.stride(1), starts=starts.data_ptr(), lengths=lengths.data_ptr(), status=status.data_ptr(), type=_type_of(q),
                                tokens=q.shape[0], heads_q=q.shape[1], causal=int(bool(causal)), window=window, max_count=max_count,
                                max_length=max_length, scale=scale)
    n = i64()
    _check(lib().tt_cache_attention_workspace(C.byref(a), C.byref(n)), "tt_cache_attention")
    workspace = _device_words(device, n.value)
    a.workspace, a.workspace_bytes = workspace.data_ptr(), n.value
    return Call("tt_cache_attention", a, (cache, q, y, starts, lengths), device, status, workspace)


def transfer_tune(workloads, tensor_sets, pool, opts: tt_tune_opts | None = None):
    """Evaluate every workload under the default record and every pool record; returns a dict with
    chosen (column index per workload), best_us, times_us [n_wl][n_pool+1], status, search_seconds, counts."""
    n_wl, n_pool = len(workloads), len(pool)
    n_cols = n_pool + 1
    handles = (C.c_void_p * n_wl)(*[w.handle for w in workloads])
    # an entry of tensor_sets may be one tt_tensors or a list of them (several sets, walked round-robin while timing)
    multi = any(not isinstance(t, tt_tensors) for t in tensor_sets)
    groups = [[t] if isinstance(t, tt_tensors) else list(t) for t in tensor_sets]
    flat_sets = [t for g in groups for t in g]
    tens = (tt_tensors * len(flat_sets))(*flat_sets)
    counts = (C.c_size_t * n_wl)(*[len(g) for g in groups])
    parr = (tt_schedule_record * max(n_pool, 1))(*pool)
    chosen = (i32 * n_wl)()
    best = (f32 * n_wl)()
    times = (f32 * (n_wl * n_cols))()
    status = (i32 * (n_wl * n_cols))()
    res = tt_tune_result()
    res.chosen, res.best_us, res.times_us, res.status = chosen, best, times, status
    if opts is None:
        opts = tt_tune_opts()
        opts.include_default = 1
    if multi:
        _check(lib().tt_transfer_tune_sets(handles, tens, counts, n_wl, parr, n_pool, C.byref(opts), _stream(), C.byref(res)),
               "tt_transfer_tune_sets")
    else:
        _check(lib().tt_transfer_tune(handles, tens, n_wl, parr, n_pool, C.byref(opts), _stream(), C.byref(res)),
               "tt_transfer_tune")
    return {
        "chosen": list(chosen), "best_us": list(best),
        "times_us": [[times[i * n_cols + j] for j in range(n_cols)] for i in range(n_wl)],
        "status": [[status[i * n_cols + j] for j in range(n_cols)] for i in range(n_wl)],
        "search_seconds": res.search_seconds, "pairs_timed": res.pairs_timed, "pairs_invalid": res.pairs_invalid,
        "pairs_skipped": res.pairs_skipped,
    }
