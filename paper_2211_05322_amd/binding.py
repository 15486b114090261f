"""Thin Python binding of libreshard.so (ctypes; argument marshalling only).

The names mirror the C ABI in include/reshard.h.  Buffers are passed as raw
pointers (ints) or torch tensors (their data_ptr()); streams as a
torch.cuda.Stream, a raw hipStream_t int, or None for the current torch
stream.  All data movement happens inside the library's HIP kernel; this
module never copies tensor data.  If the library is missing it raises --
there is no fallback.
"""

from __future__ import annotations

import contextlib
import ctypes
import os
from typing import NamedTuple

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libreshard.so")

RESHARD_OK, RESHARD_EINVAL, RESHARD_EUNSUPPORTED, RESHARD_ENOMEM, RESHARD_EHIP = range(5)
RESHARD_SENDER_NAIVE = 0x1
RESHARD_XCD_REMAP = 0x2
RESHARD_TASK_ORDER = 0x4
RESHARD_NO_REALIGN = 0x8
RESHARD_LDS_STAGING = 0x10
RESHARD_STRATEGY_SENDRECV = 0x20
RESHARD_STRATEGY_ALLGATHER = 0x40
RESHARD_NO_GATHER = 0x100
RESHARD_MAX_BUFFERS = 496

_DTYPES = {"uint8": 0, "int8": 1, "float16": 2, "bfloat16": 3, "float32": 4, "int32": 5,
           "float64": 6, "int64": 7, "uint16": 8, "int16": 9, "uint32": 10, "uint64": 11,
           "float8_e4m3fn": 12, "float8_e8m0fnu": 13}

_STATUS = {RESHARD_EINVAL: "EINVAL", RESHARD_EUNSUPPORTED: "EUNSUPPORTED",
           RESHARD_ENOMEM: "ENOMEM", RESHARD_EHIP: "EHIP"}


class ReshardError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status


class reshard_tuning_t(ctypes.Structure):
    _fields_ = [("chunk_bytes", ctypes.c_int64), ("block_threads", ctypes.c_int32),
                ("max_wgs_per_cu", ctypes.c_int32), ("gather_band", ctypes.c_int32),
                ("reserved", ctypes.c_int32 * 3)]


_lib = _torch = None
_I64P = ctypes.POINTER(ctypes.c_int64)
_VPP = ctypes.POINTER(ctypes.c_void_p)


def load(path=None):
    """Load libreshard.so (built by paper_2211_05322_amd.build); raise if it is missing."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    path = path or LIB_PATH
    if not os.path.exists(path):
        raise ImportError(f"libreshard.so not built at {path}; run `python -m paper_2211_05322_amd.build`")
    # torch first: its HIP runtime (libamdhip64 from its own directory,
    # soname libamdhip64.so.7) then satisfies the library's dependency on
    # libamdhip64.so.7.  Opened the other way round, the process would map
    # the system runtime for the library and torch's for its tensors and
    # streams -- two HIP runtimes, with kernels registered in only one.
    global _torch
    import torch
    _torch = torch
    lib = ctypes.CDLL(path)
    plan_args = [ctypes.c_int, _I64P, ctypes.c_int, ctypes.c_int, _I64P, ctypes.c_char_p,
                 ctypes.c_int, _I64P, ctypes.c_char_p, ctypes.c_uint]
    lib.reshard_plan.argtypes = plan_args + [ctypes.POINTER(ctypes.c_void_p)]
    lib.reshard_plan.restype = ctypes.c_int
    lib.reshard_plan_ex.argtypes = plan_args + [ctypes.POINTER(reshard_tuning_t), ctypes.POINTER(ctypes.c_void_p)]
    _I32P = ctypes.POINTER(ctypes.c_int32)
    lib.reshard_plan_permuted.argtypes = [ctypes.c_int, _I64P, ctypes.c_int, ctypes.c_int, _I64P, ctypes.c_char_p,
                                          _I32P, ctypes.c_int, _I64P, ctypes.c_char_p, _I32P, ctypes.c_uint,
                                          ctypes.POINTER(reshard_tuning_t), ctypes.POINTER(ctypes.c_void_p)]
    lib.reshard_plan_permuted.restype = ctypes.c_int
    lib.reshard_plan_unit_gather_chunks.argtypes = [ctypes.c_void_p]
    lib.reshard_plan_unit_gather_chunks.restype = ctypes.c_int64
    lib.reshard_plan_transpose_chunks.argtypes = [ctypes.c_void_p]
    lib.reshard_plan_transpose_chunks.restype = ctypes.c_int64
    lib.reshard_plan_ex.restype = ctypes.c_int
    lib.reshard_execute.argtypes = [ctypes.c_void_p, _VPP, _VPP, ctypes.c_void_p]
    lib.reshard_execute.restype = ctypes.c_int
    lib.reshard_execute_noalloc.argtypes = [ctypes.c_void_p, _VPP, _VPP, ctypes.c_void_p]
    lib.reshard_execute_noalloc.restype = ctypes.c_int
    lib.reshard_plan_destroy.argtypes = [ctypes.c_void_p]
    lib.reshard_plan_destroy.restype = None
    lib.reshard_plan_local_shape.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, _I64P]
    lib.reshard_plan_local_shape.restype = ctypes.c_int
    lib.reshard_plan_stats.argtypes = [ctypes.c_void_p] + [_I64P] * 5
    lib.reshard_plan_stats.restype = ctypes.c_int
    lib.reshard_plan_alignment.argtypes = [ctypes.c_void_p]
    lib.reshard_plan_alignment.restype = ctypes.c_int64
    lib.reshard_plan_lds_bytes.argtypes = [ctypes.c_void_p]
    lib.reshard_plan_lds_bytes.restype = ctypes.c_int64
    lib.reshard_plan_upload.argtypes = [ctypes.c_void_p]
    lib.reshard_plan_upload.restype = ctypes.c_int
    lib.reshard_plan_gather_chunks.argtypes = [ctypes.c_void_p]
    lib.reshard_plan_gather_chunks.restype = ctypes.c_int64
    lib.reshard_plan_realign_chunks.argtypes = [ctypes.c_void_p]
    lib.reshard_plan_realign_chunks.restype = ctypes.c_int64
    lib.reshard_plan_unaligned_gather_chunks.argtypes = [ctypes.c_void_p]
    lib.reshard_plan_unaligned_gather_chunks.restype = ctypes.c_int64
    lib.reshard_plan_unit_task.argtypes = [ctypes.c_void_p, ctypes.c_int64, _I64P, _I64P, _I64P,
                                           _I64P, ctypes.c_int64, _I64P, _I64P, ctypes.c_int64, _I64P]
    lib.reshard_plan_unit_task.restype = ctypes.c_int
    lib.reshard_debug_execute_host.argtypes = [ctypes.c_void_p, _VPP, _VPP]
    lib.reshard_debug_execute_host.restype = ctypes.c_int
    lib.reshard_schedule.argtypes = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_int,
                                     ctypes.c_int64, ctypes.c_int64, ctypes.c_uint64,
                                     _I64P, _I64P, _I64P, _I64P, _I64P]
    lib.reshard_schedule.restype = ctypes.c_int
    lib.reshard_pipeline_simulate.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_double,
                                              ctypes.c_double, ctypes.c_double, ctypes.c_double, ctypes.c_int32,
                                              ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int32)]
    lib.reshard_pipeline_simulate.restype = ctypes.c_int
    if hasattr(lib, "reshard_matmul"):  # the planner built by itself, without GPU code, lacks the operators
        _declare_operators(lib)
    lib.reshard_last_error.argtypes = []
    lib.reshard_last_error.restype = ctypes.c_char_p
    lib.reshard_version.argtypes = []
    lib.reshard_version.restype = ctypes.c_char_p
    if path == LIB_PATH:
        _lib = lib
    return lib


def _declare_operators(lib):
    i64, vp, ci, fp = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p
    lib.reshard_layer_norm.argtypes = [i64, i64, vp, i64, ci, vp, vp, ci, ctypes.c_double, vp, i64, fp, fp, vp]
    lib.reshard_layer_norm_backward_workspace.argtypes = [i64, i64]
    lib.reshard_layer_norm_backward_workspace.restype = i64
    lib.reshard_layer_norm_backward.argtypes = [i64, i64, vp, i64, vp, i64, ci, vp, ci, fp, fp, vp, i64, fp, fp, ci,
                                                vp, i64, vp]
    lib.reshard_quantize.argtypes = [i64, i64, vp, i64, ci, ci, ci, vp, i64, vp, i64, vp, i64, vp, i64, vp]
    lib.reshard_dequantize.argtypes = [i64, i64, vp, i64, ci, vp, i64, ci, vp, i64, ci, vp]
    lib.reshard_matmul_workspace.argtypes = [i64, i64, i64, ci, ci]
    lib.reshard_matmul_workspace.restype = i64
    lib.reshard_matmul.argtypes = [i64, i64, i64, vp, i64, ci, vp, i64, vp, i64, ci, vp, i64, ci, vp, i64, ci, ci,
                                   vp, i64, vp]
    for f in ("layer_norm", "layer_norm_backward", "quantize", "dequantize", "matmul"):
        getattr(lib, "reshard_" + f).restype = ctypes.c_int


def _check(status):
    if status != RESHARD_OK:
        raise ReshardError(status, load().reshard_last_error().decode())


def _i64(vals):
    vals = [int(v) for v in vals]
    return (ctypes.c_int64 * max(1, len(vals)))(*vals)


_CODES = {}  # what _dtype_code has answered, by the dtype itself


def _dtype_code(dtype):
    code = _CODES.get(dtype)
    if code is None:
        code = _CODES[dtype] = _find_dtype_code(dtype)
    return code


def _find_dtype_code(dtype):
    name = str(dtype).replace("torch.", "")
    if name not in _DTYPES:
        raise ValueError(f"unsupported dtype {dtype}")
    return _DTYPES[name]


def _gapless(shape, strides):
    """Whether elements fill one run of memory, the dimensions in any order (a buffer's need not be the tensor's)."""
    run = 1
    for step, n in sorted((s, n) for n, s in zip(shape, strides) if n != 1):
        if step != run:
            return False
        run *= n
    return True


def _refuse_gaps(shape, strides):
    if 0 not in shape and not _gapless(shape, strides):
        raise ValueError(f"a plan's buffers are dense, got shape {tuple(shape)} with strides {tuple(strides)}")


def _addr(b):
    if b is None or isinstance(b, int):
        return b
    if not b.is_contiguous():
        _refuse_gaps(b.shape, b.stride())
    return b.data_ptr() or None  # NULL for an empty tensor


def pointer_array(bufs):
    """The `void *const *` array reshard_execute takes, built once.

    `bufs` holds tensors (an empty one passes NULL), integer addresses or
    None.  A tensor with gaps between its elements is refused: the plan would
    move what lies in them.  A caller that reshards the same buffers repeatedly can build the
    two arrays once and pass them to every reshard_execute, which then skips
    the per-buffer marshalling.  The array holds addresses only: the tensors
    must stay alive (and unmoved) while it is in use.
    """
    if isinstance(bufs, ctypes.Array):
        return bufs
    return (ctypes.c_void_p * max(1, len(bufs)))(*[_addr(b) for b in bufs])


_ptrs = pointer_array


class Plan:
    """Owns a reshard_plan_t*; destroyed with the object."""

    def __init__(self, handle, shape, src_mesh, dst_mesh, dtype):
        self._h = ctypes.c_void_p(handle)
        self._destroy = load().reshard_plan_destroy  # the library that made the plan frees it
        self.shape = tuple(shape)
        self.ndim = len(self.shape)
        self.src_mesh = tuple(src_mesh)
        self.dst_mesh = tuple(dst_mesh)
        self.dtype = dtype
        n = 1
        for m in self.src_mesh:
            n *= m
        self.n_src = n
        n = 1
        for m in self.dst_mesh:
            n *= m
        self.n_dst = n

    @property
    def handle(self):
        return self._h

    def __del__(self):
        if getattr(self, "_destroy", None) and self._h.value:
            self._destroy(self._h)
            self._h = ctypes.c_void_p(0)


def reshard_plan(shape, dtype, src_mesh, src_spec, dst_mesh, dst_spec, flags=0,
                 chunk_bytes=0, block_threads=0, max_wgs_per_cu=0, gather_band=0, src_perm=None, dst_perm=None):
    """A plan; src_perm / dst_perm (tuples or None) permute each side's local
    buffer layout (buffer dimension k is tensor dimension perm[k])."""
    lib = load()
    h = ctypes.c_void_p()
    args = [len(shape), _i64(shape), _dtype_code(dtype), len(src_mesh), _i64(src_mesh),
            src_spec.encode(), len(dst_mesh), _i64(dst_mesh), dst_spec.encode(), int(flags)]
    if src_perm is not None or dst_perm is not None:
        def perm(p):
            return None if p is None else (ctypes.c_int32 * max(1, len(p)))(*[int(a) for a in p])
        t = reshard_tuning_t(chunk_bytes=int(chunk_bytes), block_threads=int(block_threads),
                             max_wgs_per_cu=int(max_wgs_per_cu), gather_band=int(gather_band))
        _check(lib.reshard_plan_permuted(len(shape), _i64(shape), _dtype_code(dtype), len(src_mesh), _i64(src_mesh),
                                         src_spec.encode(), perm(src_perm), len(dst_mesh), _i64(dst_mesh),
                                         dst_spec.encode(), perm(dst_perm), int(flags), ctypes.byref(t),
                                         ctypes.byref(h)))
    elif chunk_bytes or block_threads or max_wgs_per_cu or gather_band:
        t = reshard_tuning_t(chunk_bytes=int(chunk_bytes), block_threads=int(block_threads),
                             max_wgs_per_cu=int(max_wgs_per_cu), gather_band=int(gather_band))
        _check(lib.reshard_plan_ex(*args, ctypes.byref(t), ctypes.byref(h)))
    else:
        _check(lib.reshard_plan(*args, ctypes.byref(h)))
    return Plan(h.value, shape, src_mesh, dst_mesh, dtype)


def _stream_handle(stream):
    if stream is None:
        import torch
        if torch.cuda.is_initialized():
            # the handle alone: torch.cuda.current_stream() builds a Stream
            # object around it, 2.7 us of a call's 7 (0.2 us this way); a
            # torch without these private functions takes that way
            try:
                return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
            except AttributeError:
                pass
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def reshard_plan_upload(plan):
    """Upload the plan's tables to the current device (then execute is graph-capturable)."""
    _check(load().reshard_plan_upload(plan.handle))


def reshard_execute(plan, src_bufs, dst_bufs, stream=None):
    """Enqueue the reshard kernel on `stream` (default: torch's current stream).

    `src_bufs` / `dst_bufs`: one buffer per device (tensors, addresses or
    None), or arrays from `pointer_array`.
    """
    if len(src_bufs) != plan.n_src or len(dst_bufs) != plan.n_dst:
        raise ValueError(f"need {plan.n_src} source and {plan.n_dst} destination buffers")
    status = (_lib or load()).reshard_execute(plan._h, _ptrs(src_bufs), _ptrs(dst_bufs), _stream_handle(stream))
    if status != RESHARD_OK:
        _check(status)


def reshard_execute_noalloc(plan, src_bufs, dst_bufs, stream=None):
    """reshard_execute that allocates nothing: the plan's tables go to the
    library's fixed per-device scratch array (see the header for its limit
    and for calls that overlap)."""
    if len(src_bufs) != plan.n_src or len(dst_bufs) != plan.n_dst:
        raise ValueError(f"need {plan.n_src} source and {plan.n_dst} destination buffers")
    status = (_lib or load()).reshard_execute_noalloc(plan._h, _ptrs(src_bufs), _ptrs(dst_bufs),
                                                      _stream_handle(stream))
    if status != RESHARD_OK:
        _check(status)


def reshard_debug_execute_host(plan, src_bufs, dst_bufs):
    """Run the descriptor table on host buffers (numpy arrays or CPU tensors)."""
    def ptr(b):
        if b is None:
            return None
        if hasattr(b, "ctypes"):
            _refuse_gaps(b.shape, [s // b.itemsize for s in b.strides])
            return b.ctypes.data if b.size > 0 else None
        return _addr(b)
    if len(src_bufs) != plan.n_src or len(dst_bufs) != plan.n_dst:
        raise ValueError(f"need {plan.n_src} source and {plan.n_dst} destination buffers")
    _check(load().reshard_debug_execute_host(plan.handle, _ptrs([ptr(b) for b in src_bufs]),
                                             _ptrs([ptr(b) for b in dst_bufs])))


def reshard_plan_local_shape(plan, side, device):
    out = (ctypes.c_int64 * plan.ndim)()
    _check(load().reshard_plan_local_shape(plan.handle, int(side), int(device), out))
    return tuple(out)


def reshard_plan_stats(plan):
    vals = [ctypes.c_int64() for _ in range(5)]
    _check(load().reshard_plan_stats(plan.handle, *[ctypes.byref(v) for v in vals]))
    keys = ("bytes_read", "bytes_written", "n_unit_tasks", "n_descriptors", "max_fanout")
    return {k: v.value for k, v in zip(keys, vals)}


def reshard_plan_alignment(plan):
    return int(load().reshard_plan_alignment(plan.handle))


def reshard_plan_lds_bytes(plan):
    return int(load().reshard_plan_lds_bytes(plan.handle))


def reshard_plan_gather_chunks(plan):
    return int(load().reshard_plan_gather_chunks(plan.handle))


def reshard_plan_realign_chunks(plan):
    return int(load().reshard_plan_realign_chunks(plan.handle))


def reshard_plan_unit_gather_chunks(plan):
    return load().reshard_plan_unit_gather_chunks(plan.handle)


def reshard_plan_transpose_chunks(plan):
    return load().reshard_plan_transpose_chunks(plan.handle)


def reshard_plan_unaligned_gather_chunks(plan):
    return int(load().reshard_plan_unaligned_gather_chunks(plan.handle))


def reshard_plan_unit_task(plan, index):
    lo = (ctypes.c_int64 * plan.ndim)()
    hi = (ctypes.c_int64 * plan.ndim)()
    chosen = ctypes.c_int64()
    snd = (ctypes.c_int64 * plan.n_src)()
    rcv = (ctypes.c_int64 * plan.n_dst)()
    ns, nr = ctypes.c_int64(), ctypes.c_int64()
    _check(load().reshard_plan_unit_task(plan.handle, int(index), lo, hi, ctypes.byref(chosen),
                                         snd, plan.n_src, ctypes.byref(ns), rcv, plan.n_dst,
                                         ctypes.byref(nr)))
    return {"box": tuple(zip(tuple(lo), tuple(hi))), "sender": chosen.value,
            "senders": list(snd[:ns.value]), "receivers": list(rcv[:nr.value])}


SCHED_ALGOS = {"naive": 0, "load_balance": 1, "dfs": 2, "randomized": 3, "ensemble": 4}


def reshard_schedule(plan, src_devices_per_host, dst_devices_per_host, algo="ensemble",
                     max_dfs_nodes=200000, random_rounds=16, seed=0):
    """Sender choice and start times under the multi-host model (host-side only)."""
    n = reshard_plan_stats(plan)["n_unit_tasks"]
    snd = (ctypes.c_int64 * max(1, n))()
    st = (ctypes.c_int64 * max(1, n))()
    mk, lb, nodes = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
    _check(load().reshard_schedule(plan.handle, int(src_devices_per_host), int(dst_devices_per_host),
                                   SCHED_ALGOS[algo], int(max_dfs_nodes), int(random_rounds), int(seed),
                                   snd, st, ctypes.byref(mk), ctypes.byref(lb), ctypes.byref(nodes)))
    return {"senders": list(snd[:n]), "starts": list(st[:n]), "makespan": mk.value,
            "lower_bound": lb.value, "dfs_nodes": nodes.value}


def reshard_pipeline_simulate(stages, microbatches, eager, t_fwd, t_bwd, t_comm_fwd, t_comm_bwd=None,
                              serial_links=True):
    """(latency, per-stage peak live micro-batches) of one pipelined iteration."""
    lat = ctypes.c_double()
    peak = (ctypes.c_int32 * max(1, int(stages)))()
    _check(load().reshard_pipeline_simulate(int(stages), int(microbatches), int(bool(eager)), float(t_fwd),
                                            float(t_bwd), float(t_comm_fwd),
                                            float(t_comm_fwd if t_comm_bwd is None else t_comm_bwd),
                                            int(bool(serial_links)), ctypes.byref(lat), peak))
    return lat.value, list(peak[:int(stages)])


# ------------------------------------------- operators at a stage's edge

class Blocked(NamedTuple):
    """A matrix in 8 bits with a scale per block of 128 columns.

    data: float8_e4m3fn [..., cols]; scales: float8_e8m0fnu or float32
    [ceil(rows / block_rows), ceil(cols / 128)]; block_rows: 1 or 128.  Both
    tensors reshard like any other (a plan on each) where they are dense, as
    plans take all buffers: codes made with dense=True, or of a width that 128
    divides."""
    data: object
    scales: object
    block_rows: int = 1


def _matrix(name, t):
    """(rows, cols, pitch) of a tensor whose leading dimensions step evenly and whose last is dense."""
    shape, strides = t.shape, t.stride()
    if len(shape) == 2 and strides[1] == 1:
        return shape[0], shape[1], strides[0]
    if not shape:
        raise ValueError(f"{name} needs at least one dimension")
    cols = shape[-1]
    if cols > 1 and strides[-1] != 1:
        raise ValueError(f"{name}: the last dimension must be dense, its stride is {strides[-1]}")
    if len(shape) == 2:
        return shape[0], cols, strides[0]
    if 0 in shape[:-1]:
        return 0, cols, cols
    rows, pitch = 1, None
    for n, s in zip(reversed(shape[:-1]), reversed(strides[:-1])):
        if n != 1:
            if pitch is None:
                pitch = s
            elif s != rows * pitch:
                raise ValueError(f"{name}: the leading dimensions do not step evenly from row to row")
        rows *= n
    return rows, cols, cols if pitch is None else pitch


def _like(name, t, shape, dtype, device):
    """A caller's output or statistic: the shape, type and device it must have."""
    if t.shape != tuple(shape) or t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be {dtype} {tuple(shape)} on {device}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t


def _dense(name, t, shape, beside, dtype):
    if t.shape != shape or t.dtype != dtype or t.get_device() != beside.get_device() or not t.is_contiguous():
        raise ValueError(f"{name} must be dense, {dtype} {tuple(shape)} on {beside.device}, "
                         f"got {t.dtype} {tuple(t.shape)}, strides {t.stride()}, on {t.device}")
    return t


_HERE = contextlib.nullcontext()


def _on(stream):
    """Memory that a call takes comes from the pool of the stream it runs on.  Its inputs are the caller's to keep until
    that stream has passed the call (record_stream, where they come from another stream's pool)."""
    if stream is None:
        return _HERE
    return _torch.cuda.stream(_torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream)


def _on_gpu(name, t):
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU, got {t.device}")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _result(out, like):
    """(tensor, pitch) of a result of like's shape and type: the caller's, or a dense one."""
    if out is not None:
        return _like("out", out, like.shape, like.dtype, like.device), _matrix("out", out)[2]
    y = _torch.empty_like(like) if like.is_contiguous() else like.new_empty(like.shape)
    return y, like.shape[-1]


def reshard_layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, stream=None):
    """(y, mean, rstd): layer norm over x's last dimension; mean and rstd (float32) are for the backward pass."""
    lib = _lib or load()
    rows, cols, pitch = _matrix("x", x)
    wdt = (weight if weight is not None else bias if bias is not None else x).dtype
    if weight is not None:
        _dense("weight", weight, (cols,), x, wdt)
    if bias is not None:
        _dense("bias", bias, (cols,), x, wdt)
    if out is not None:
        _like("out", out, x.shape, x.dtype, x.device)
    _on_gpu("x", x)
    with _on(stream):
        y, y_pitch = _result(out, x)
        mean, rstd = x.new_empty((2, *x.shape[:-1]), dtype=_torch.float32).unbind()
    status = lib.reshard_layer_norm(rows, cols, x.data_ptr(), pitch, _dtype_code(x.dtype), _ptr(weight), _ptr(bias),
                                    _dtype_code(wdt), eps, y.data_ptr(), y_pitch, mean.data_ptr(), rstd.data_ptr(),
                                    _stream_handle(stream))
    if status != RESHARD_OK:
        _check(status)
    return y, mean, rstd


def reshard_layer_norm_backward(dy, x, weight, mean, rstd, dweight=None, dbias=None, accumulate=False, out=None,
                                stream=None):
    """(dx, dweight, dbias) of reshard_layer_norm.  dweight and dbias are
    float32; given ones are overwritten, or added to with accumulate."""
    lib = _lib or load()
    rows, cols, pitch = _matrix("x", x)
    _like("dy", dy, x.shape, x.dtype, x.device)
    if weight is not None:
        _dense("weight", weight, (cols,), x, weight.dtype)
    _dense("mean", mean, x.shape[:-1], x, _torch.float32)
    _dense("rstd", rstd, x.shape[:-1], x, _torch.float32)
    if accumulate and (dweight is None or dbias is None):
        raise ValueError("accumulate needs the dweight and dbias to add to")
    _on_gpu("x", x)
    need = lib.reshard_layer_norm_backward_workspace(rows, cols)
    with _on(stream):
        dx, dx_pitch = _result(out, x)
        if dweight is None and dbias is None:
            dweight, dbias = x.new_empty((2, cols), dtype=_torch.float32).unbind()
        elif dweight is None:
            dweight = x.new_empty(cols, dtype=_torch.float32)
        elif dbias is None:
            dbias = x.new_empty(cols, dtype=_torch.float32)
        work = x.new_empty(max(0, need), dtype=_torch.uint8)
    _dense("dweight", dweight, (cols,), x, _torch.float32)
    _dense("dbias", dbias, (cols,), x, _torch.float32)
    status = lib.reshard_layer_norm_backward(
        rows, cols, dy.data_ptr(), _matrix("dy", dy)[2], x.data_ptr(), pitch, _dtype_code(x.dtype), _ptr(weight),
        _dtype_code(x.dtype if weight is None else weight.dtype), mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(),
        dx_pitch, dweight.data_ptr(), dbias.data_ptr(), int(accumulate), work.data_ptr(), need, _stream_handle(stream))
    if status != RESHARD_OK:
        _check(status)
    return dx, dweight, dbias


_E4M3, _BLOCK = "float8_e4m3fn", 128


def _empty_blocked(x, rows, cols, block_rows, scale_dtype, dense):
    """(Blocked, codes' pitch, scales' pitch) beside x.  Rows of codes are dense, or padded to whole blocks, so that
    each starts on a 16-byte boundary."""
    across = -(-cols // _BLOCK)
    pitch = cols if dense else across * _BLOCK
    data = x.new_empty((rows, pitch), dtype=_torch.float8_e4m3fn)
    scales = x.new_empty((rows if block_rows == 1 else -(-rows // block_rows), across), dtype=scale_dtype)
    if cols != pitch:
        data = data[:, :cols]
    return Blocked(data, scales, block_rows), pitch, across


def _blocked(name, b):
    """(rows, cols, pitch, scales' pitch) of a Blocked."""
    data, scales, block_rows = b
    rows, cols, pitch = _matrix("data", data)
    if _dtype_code(data.dtype) != _DTYPES[_E4M3]:
        raise ValueError(f"{name}.data must be {_E4M3}, got {data.dtype}")
    if block_rows not in (1, _BLOCK):
        raise ValueError(f"{name}.block_rows must be 1 or {_BLOCK}, got {block_rows}")
    srows, scols, spitch = _matrix("scales", scales)
    if srows != -(-rows // block_rows) or scols != -(-cols // _BLOCK):
        raise ValueError(f"{name}.scales must be {(-(-rows // b.block_rows), -(-cols // _BLOCK))}, "
                         f"got {(srows, scols)}")
    if scales.get_device() != data.get_device():
        raise ValueError(f"{name}.scales are on {b.scales.device}, its data on {b.data.device}")
    return rows, cols, pitch, spitch


def reshard_quantize(x, block_rows=1, transposed=False, scale_dtype=None, stream=None, dense=False):
    """x in 8 bits with a power-of-two scale per block (Blocked; x's leading
    dimensions are kept, and count as rows).  transposed=True: of x as a matrix
    of rows, transposed, with blocks along x's rows; "both": the pair, from one reading of x.  scale_dtype:
    torch.float8_e8m0fnu (default) or torch.float32.  Rows of codes start on
    16-byte boundaries, with room between them where 128 does not divide the
    width: so a product reads them fastest.  dense=True: they follow each
    other, as a plan's buffers do."""
    lib = _lib or load()
    rows, cols, pitch = _matrix("x", x)
    if transposed not in (False, True, "both"):
        raise ValueError(f'transposed must be False, True or "both", got {transposed!r}')
    if transposed != "both":
        transposed = bool(transposed)  # 0 and numpy's False equal False and are not it
    if block_rows not in (1, _BLOCK):
        raise ValueError(f"block_rows must be 1 or {_BLOCK}, got {block_rows}")
    if scale_dtype is None:
        scale_dtype = _torch.float8_e8m0fnu
    _on_gpu("x", x)
    q = t = None
    args = [None, 0, None, 0, None, 0, None, 0]
    with _on(stream):
        if transposed is not True:
            q, pitch_q, pitch_s = _empty_blocked(x, rows, cols, block_rows, scale_dtype, dense)
            args[:4] = q.data.data_ptr(), pitch_q, q.scales.data_ptr(), pitch_s
        if transposed is not False:
            t, pitch_q, pitch_s = _empty_blocked(x, cols, rows, block_rows, scale_dtype, dense)
            args[4:] = t.data.data_ptr(), pitch_q, t.scales.data_ptr(), pitch_s
    status = lib.reshard_quantize(rows, cols, x.data_ptr(), pitch, _dtype_code(x.dtype), block_rows,
                                  _dtype_code(scale_dtype), *args, _stream_handle(stream))
    if status != RESHARD_OK:
        _check(status)
    if q is not None and x.dim() != 2:
        def lead(t):
            return t.unflatten(0, x.shape[:-1]) if x.dim() > 2 else t[0]
        q = Blocked(lead(q.data), lead(q.scales) if block_rows == 1 else q.scales, block_rows)
    return (q, t) if transposed == "both" else q if t is None else t


def reshard_dequantize(b, dtype, out=None, stream=None):
    """The values of a Blocked, rounded once to dtype (torch.float16, bfloat16 or float32)."""
    lib = _lib or load()
    rows, cols, pitch, spitch = _blocked("b", b)
    _on_gpu("b", b.data)
    with _on(stream):
        if out is None:
            y, y_pitch = b.data.new_empty(b.data.shape, dtype=dtype), cols
        else:
            y, y_pitch = _like("out", out, b.data.shape, dtype, b.data.device), _matrix("out", out)[2]
    status = lib.reshard_dequantize(rows, cols, b.data.data_ptr(), pitch, b.block_rows, b.scales.data_ptr(), spitch,
                                    _dtype_code(b.scales.dtype), y.data_ptr(), y_pitch, _dtype_code(dtype),
                                    _stream_handle(stream))
    if status != RESHARD_OK:
        _check(status)
    return y


def reshard_matmul(a, b, out_dtype=None, out=None, accumulate=False, stream=None):
    """a [..., k] times b [n, k] transposed, both Blocked with scales of one
    type; [..., n] of out_dtype (default torch.bfloat16), or into `out`, added
    to what is there with accumulate."""
    lib = _lib or load()
    m, k, a_pitch, a_spitch = _blocked("a", a)
    n, kb, b_pitch, b_spitch = _blocked("b", b)
    if k != kb:
        raise ValueError(f"a has {k} columns and b {kb}")
    if a.scales.dtype != b.scales.dtype:
        raise ValueError(f"a's scales are {a.scales.dtype}, b's {b.scales.dtype}")
    if a.data.get_device() != b.data.get_device():
        raise ValueError(f"a is on {a.data.device}, b on {b.data.device}")
    if accumulate and out is None:
        raise ValueError("accumulate needs the out to add to")
    if out is not None:
        _like("out", out, (*a.data.shape[:-1], n), out_dtype or out.dtype, a.data.device)
    _on_gpu("a", a.data)
    shape = (*a.data.shape[:-1], n)
    out_dtype = out_dtype or (_torch.bfloat16 if out is None else out.dtype)
    sdt, odt = _dtype_code(a.scales.dtype), _dtype_code(out_dtype)
    need = lib.reshard_matmul_workspace(m, n, k, sdt, odt)
    work = None
    with _on(stream):
        if out is None:
            y, y_pitch = a.data.new_empty(shape, dtype=out_dtype), n
        else:
            y, y_pitch = _like("out", out, shape, out_dtype, a.data.device), _matrix("out", out)[2]
        if need > 0:
            work = a.data.new_empty(need, dtype=_torch.uint8)
    status = lib.reshard_matmul(m, n, k, a.data.data_ptr(), a_pitch, a.block_rows, a.scales.data_ptr(), a_spitch,
                                b.data.data_ptr(), b_pitch, b.block_rows, b.scales.data_ptr(), b_spitch, sdt,
                                y.data_ptr(), y_pitch, odt, int(accumulate), _ptr(work), max(0, need),
                                _stream_handle(stream))
    if status != RESHARD_OK:
        _check(status)
    return y


def reshard_last_error():
    return load().reshard_last_error().decode()


def reshard_version():
    return load().reshard_version().decode()


# ------------------------------------------------------------ conveniences

def local_shapes(plan, side):
    n = plan.n_src if side == 0 else plan.n_dst
    return [reshard_plan_local_shape(plan, side, k) for k in range(n)]


def empty_shards(plan, side, device="cuda"):
    """Allocate one dense buffer per device of one side (torch, no data movement)."""
    import torch
    dt = getattr(torch, str(plan.dtype).replace("torch.", ""))
    return [torch.empty(s, dtype=dt, device=device) for s in local_shapes(plan, side)]
