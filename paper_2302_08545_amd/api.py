"""ctypes binding of libthc (include/thc.h).  Argument marshalling only: every step of the path runs
in the HIP kernels.  PyTorch supplies device memory (`tensor.data_ptr()`) and the current stream."""
from __future__ import annotations

import ctypes as C
import os
from array import array
from typing import Optional, Sequence

_LIB = None
LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libthc.so")

THC_MAX_WORKERS = 64
THC_DTYPE_F32, THC_DTYPE_BF16, THC_DTYPE_F16 = 0, 1, 2
THC_NORM_L2, THC_NORM_MAX = 0, 1
THC_ORDER_ASCENDING, THC_ORDER_SPLIT = 0, 1

EXPORTS = ("thc_version", "thc_strerror", "thc_workspace_bytes", "thc_prepare_range", "thc_compress",
           "thc_compress_all", "thc_aggregate", "thc_decompress", "thc_decompress_noalloc",
           "thc_uniform_workspace_bytes",
           "thc_uniform_prepare_range", "thc_uniform_compress", "thc_uniform_decompress", "thc_threshold",
           "thc_solve_table", "thc_solve_table_bruteforce", "thc_describe_plan", "thc_norm_workspace_bytes",
           "thc_grad_norm", "thc_grad_clip", "thc_gather", "thc_scatter")


class thc_params(C.Structure):
    _fields_ = [("d", C.c_uint64), ("block", C.c_uint64), ("n", C.c_uint32), ("b", C.c_uint32),
                ("g", C.c_uint32), ("agg_bits", C.c_uint32), ("in_dtype", C.c_uint32), ("t_p", C.c_float),
                ("seed", C.c_uint64), ("table", C.c_uint8 * 256), ("stage_order", C.c_uint32),
                ("first_block", C.c_uint32), ("group_log2", C.c_uint32), ("single_launch", C.c_uint32)]


class thc_tensors(C.Structure):
    """A list of tensors as the library takes it; made by make_tensors, which keeps the tensors, the memory that they had then
    and their device with it."""
    _fields_ = [("count", C.c_uint64), ("data", C.POINTER(C.c_void_p)), ("numel", C.POINTER(C.c_uint64)),
                ("dtype", C.POINTER(C.c_uint32))]
    tensors: tuple = ()
    storages: tuple = ()     # a tensor that is given other storage lets go of the memory that the list describes
    device: Optional[int] = None


class ThcError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {thc_strerror(status)} ({status})")


def lib():
    """The loaded library.  Raises if it has not been built: there is no fallback path."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2302_08545_amd.build` "
                               "(or __graft_entry__.build()) first")
        L = C.CDLL(LIB_PATH)
        vp, u64, u32 = C.c_void_p, C.c_uint64, C.c_uint32
        pp = C.POINTER(thc_params)
        L.thc_version.restype = C.c_int
        L.thc_strerror.restype = C.c_char_p
        L.thc_strerror.argtypes = [C.c_int]
        L.thc_workspace_bytes.argtypes = [pp, C.c_int, C.POINTER(C.c_size_t)]
        L.thc_uniform_workspace_bytes.argtypes = [pp, C.c_int, C.POINTER(C.c_size_t)]
        L.thc_prepare_range.argtypes = [pp, C.POINTER(vp), C.POINTER(vp), vp, vp, vp]
        L.thc_compress.argtypes = [pp, u32, u64, vp, vp, vp, vp, vp, vp]
        L.thc_compress_all.argtypes = [pp, u64, C.POINTER(vp), C.POINTER(vp), vp, C.POINTER(vp), vp, vp]
        L.thc_aggregate.argtypes = [pp, C.POINTER(vp), vp, vp]
        L.thc_decompress.argtypes = [pp, u64, vp, vp, vp, vp, vp]
        L.thc_decompress_noalloc.argtypes = [pp, u64, vp, vp, vp, vp]
        L.thc_uniform_prepare_range.argtypes = [pp, u64, C.POINTER(vp), C.POINTER(vp), C.c_int, vp, vp, vp, vp]
        L.thc_uniform_compress.argtypes = [pp, u32, u64, vp, vp, C.c_int, vp, vp, vp, vp, vp]
        L.thc_uniform_decompress.argtypes = [pp, u64, vp, C.c_int, vp, vp, vp, vp, vp]
        L.thc_threshold.restype = C.c_double
        L.thc_threshold.argtypes = [C.c_double]
        L.thc_solve_table.argtypes = [u32, u32, C.c_double, C.POINTER(C.c_uint8), C.POINTER(C.c_double)]
        L.thc_solve_table_bruteforce.argtypes = [u32, u32, C.c_double, C.POINTER(C.c_uint8), C.POINTER(C.c_double),
                                                 C.POINTER(C.c_uint64)]
        L.thc_describe_plan.argtypes = [pp, C.POINTER(C.c_uint32), C.c_size_t]
        pt, f32 = C.POINTER(thc_tensors), C.c_float
        L.thc_norm_workspace_bytes.argtypes = [C.POINTER(C.c_size_t)]
        L.thc_grad_norm.argtypes = [pt, C.c_int, f32, vp, vp, vp, vp]
        L.thc_grad_clip.argtypes = [pt, C.c_int, f32, vp, vp, vp, vp]
        L.thc_gather.argtypes = [pp, pt, vp, vp, vp]
        L.thc_scatter.argtypes = [pp, vp, vp, pt, vp]
        _LIB = L
    return _LIB


def make_params(d: int, block: int, n: int, b: int, g: int, t_p: float, seed: int, table: Sequence[int],
                agg_bits: int = 8, in_dtype: int = THC_DTYPE_F32, stage_order: int = THC_ORDER_ASCENDING,
                first_block: int = 0, group_log2: int = 0, single_launch: int = 0) -> thc_params:
    p = thc_params()
    p.stage_order = stage_order
    p.first_block = first_block
    p.group_log2 = group_log2
    p.single_launch = single_launch
    p.d, p.block, p.n, p.b, p.g = d, block, n, b, g
    p.agg_bits, p.in_dtype, p.t_p, p.seed = agg_bits, in_dtype, t_p, seed
    for i, v in enumerate(table):
        p.table[i] = int(v)
    return p


def _ptr(t) -> Optional[int]:
    return None if t is None else (t if isinstance(t, int) else t.data_ptr())


def _ptr_array(ts):
    if ts is None:
        return None
    arr = (C.c_void_p * len(ts))()
    for i, t in enumerate(ts):
        arr[i] = _ptr(t)
    return arr


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        if torch.cuda.is_initialized():   # the handle alone: a Stream object costs a small call more than its launches
            try:
                return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
            except AttributeError:        # names of torch's own that a build may lack: then the public way
                pass
        stream = torch.cuda.current_stream()
    return stream if isinstance(stream, int) else stream.cuda_stream


def _check(rc: int, where: str):
    if rc != 0:
        raise ThcError(rc, where)


def thc_version() -> int:
    return lib().thc_version()


def thc_strerror(status: int) -> str:
    return lib().thc_strerror(status).decode()


def thc_workspace_bytes(p: thc_params, ef_enabled: bool = False) -> int:
    out = C.c_size_t(0)
    _check(lib().thc_workspace_bytes(C.byref(p), int(ef_enabled), C.byref(out)), "thc_workspace_bytes")
    return out.value


def thc_uniform_workspace_bytes(p: thc_params, rotate: bool) -> int:
    out = C.c_size_t(0)
    _check(lib().thc_uniform_workspace_bytes(C.byref(p), int(rotate), C.byref(out)), "thc_uniform_workspace_bytes")
    return out.value


def thc_prepare_range(p: thc_params, grads, ef, range_M, ws, stream=None) -> None:
    _check(lib().thc_prepare_range(C.byref(p), _ptr_array(grads), _ptr_array(ef), _ptr(range_M), _ptr(ws),
                                   _stream(stream)), "thc_prepare_range")


def thc_compress_all(p: thc_params, rnd: int, grads, ef_inout, range_M, packed_out, ws, stream=None) -> None:
    _check(lib().thc_compress_all(C.byref(p), rnd, _ptr_array(grads), _ptr_array(ef_inout), _ptr(range_M),
                                  _ptr_array(packed_out), _ptr(ws), _stream(stream)), "thc_compress_all")


def thc_compress(p: thc_params, worker_id: int, rnd: int, grad, ef_inout, range_M, packed_out, ws,
                 stream=None) -> None:
    _check(lib().thc_compress(C.byref(p), worker_id, rnd, _ptr(grad), _ptr(ef_inout), _ptr(range_M),
                              _ptr(packed_out), _ptr(ws), _stream(stream)), "thc_compress")


def thc_aggregate(p: thc_params, packed, agg_out, stream=None) -> None:
    _check(lib().thc_aggregate(C.byref(p), _ptr_array(packed), _ptr(agg_out), _stream(stream)), "thc_aggregate")


def thc_decompress(p: thc_params, rnd: int, agg, range_M, out, ws, stream=None) -> None:
    _check(lib().thc_decompress(C.byref(p), rnd, _ptr(agg), _ptr(range_M), _ptr(out), _ptr(ws), _stream(stream)),
           "thc_decompress")


def thc_decompress_noalloc(p: thc_params, rnd: int, agg, range_M, out, stream=None) -> None:
    _check(lib().thc_decompress_noalloc(C.byref(p), rnd, _ptr(agg), _ptr(range_M), _ptr(out), _stream(stream)),
           "thc_decompress_noalloc")


def thc_uniform_prepare_range(p: thc_params, rnd: int, grads, ef, rotate: bool, range_m, range_M, ws,
                              stream=None) -> None:
    _check(lib().thc_uniform_prepare_range(C.byref(p), rnd, _ptr_array(grads), _ptr_array(ef), int(rotate),
                                           _ptr(range_m), _ptr(range_M), _ptr(ws), _stream(stream)),
           "thc_uniform_prepare_range")


def thc_uniform_compress(p: thc_params, worker_id: int, rnd: int, grad, ef_inout, rotate: bool, range_m, range_M,
                         packed_out, ws, stream=None) -> None:
    _check(lib().thc_uniform_compress(C.byref(p), worker_id, rnd, _ptr(grad), _ptr(ef_inout), int(rotate),
                                      _ptr(range_m), _ptr(range_M), _ptr(packed_out), _ptr(ws), _stream(stream)),
           "thc_uniform_compress")


def thc_uniform_decompress(p: thc_params, rnd: int, agg, rotate: bool, range_m, range_M, out, ws,
                           stream=None) -> None:
    _check(lib().thc_uniform_decompress(C.byref(p), rnd, _ptr(agg), int(rotate), _ptr(range_m), _ptr(range_M),
                                        _ptr(out), _ptr(ws), _stream(stream)), "thc_uniform_decompress")


# ---- a model's tensors -----------------------------------------------------------------------------
_TORCH = None      # torch, and its types' codes, on first use: importing this module does not import torch
_DTYPES = {}


def _torch():
    global _TORCH
    if _TORCH is None:
        import torch
        _DTYPES.update({torch.float32: THC_DTYPE_F32, torch.bfloat16: THC_DTYPE_BF16, torch.float16: THC_DTYPE_F16})
        _TORCH = torch
    return _TORCH


def _one_run(t) -> bool:
    """Whether a tensor's elements lie in one run of memory, whatever the order of its dimensions."""
    at = 1
    for stride, size in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n != 1):
        if stride != at:
            return False
        at *= size
    return True


def make_tensors(tensors: Sequence) -> thc_tensors:
    """Describes a list of GPU tensors (float32, bfloat16, float16; any mixture) for the calls below.

    Each tensor is taken in the order of its memory, so it has to be one run of memory: contiguous, or with its
    dimensions in another order (channels last, transposed).  The list holds the tensors with the memory that they have
    now, and goes on describing that memory: keep it as long as they stay where they are, and make a new one when a gradient
    is replaced (as torch's zero_grad() does unless set_to_none=False) or given other storage (.data, set_).  Storage must
    not be resized under it."""
    ts, n = tuple(tensors), 0
    _torch()
    try:                   # a training step may make a list of hundreds: each property of all of them in one go
        n = len(ts)
        types = array("I", [_DTYPES[t.dtype] for t in ts])
        devices = {t.get_device() for t in ts}
        data = array("Q", [t.data_ptr() for t in ts])
        numel = array("Q", [t.numel() for t in ts])
        storages = tuple([t.untyped_storage() for t in ts])
    except (AttributeError, KeyError, RuntimeError, TypeError):
        devices = {-1}
    if -1 in devices:
        raise ValueError("make_tensors: takes dense float32, bfloat16 and float16 tensors on the GPU")
    if len(devices) > 1:
        raise ValueError("make_tensors: all tensors have to be on one device")
    for t in ts:
        if t.is_neg():
            raise ValueError("make_tensors: a tensor's memory holds its negative (part of a conjugate): resolve_neg() first")
        if not t.is_contiguous() and not _one_run(t):
            raise ValueError(f"make_tensors: a tensor of shape {tuple(t.shape)} with strides {tuple(t.stride())} is not one "
                             "run of memory")
    out = thc_tensors(n, (C.c_void_p * n).from_buffer(data), (C.c_uint64 * n).from_buffer(numel),
                      (C.c_uint32 * n).from_buffer(types)) if n else thc_tensors()
    out.tensors, out.storages, out.device = ts, storages, devices.pop() if n else None
    return out


def _current_device() -> int:
    try:
        return (_TORCH or _torch())._C._cuda_getDevice()
    except AttributeError:                       # a name of torch's own that a build may lack
        return _TORCH.cuda.current_device()


def _list_and_stream(tensors, stream, where: str):
    """The list as the library takes it, the stream's handle, and the device (None: not known).  The tensors have to be on
    the stream's device.  That is the current device for the current stream, and for the null stream (handles up to 2, as
    legacy and per thread), which is the same number on every device; other streams say it themselves.  A bare handle of
    such a stream does not: there the caller answers for it."""
    t = tensors if type(tensors) is thc_tensors else make_tensors(tensors)
    own, whose = t.device, "current device"
    if stream is None:
        at = _current_device()
    else:
        handle = _stream(stream)
        if handle > 2:
            device, whose = getattr(stream, "device", None), "stream's device"
            at = own if device is None else device.index
        else:
            at = _current_device() if own is not None or _torch().cuda.is_available() else None
    if own is not None and at != own:
        raise ValueError(f"{where}: the tensors are on cuda:{own}, the {whose} is cuda:{at}")
    if stream is None:
        try:
            handle = _TORCH._C._cuda_getCurrentRawStream(at)
        except AttributeError:
            handle = _stream(None)
    return t, handle, at


def _buffer(b, name: str, where: str, count: int, dtype: Optional[int], device: Optional[int]) -> Optional[int]:
    """The address of a tensor on the call's GPU that has to hold `count` elements of a type (None: bytes) in one run;
    addresses as they are."""
    if b is None or type(b) is int:
        return b
    if dtype is None:
        ok = b.nbytes >= count
    else:
        if _TORCH is None:
            _torch()
        ok = b.numel() >= count and _DTYPES.get(b.dtype) == dtype and not b.is_neg()   # its memory then holds the negative
    if not (ok and b.is_contiguous() and (b.is_cuda if device is None else b.get_device() == device)):
        raise ValueError(f"{where}: {name} has to be a contiguous tensor on {'the GPU' if device is None else f'cuda:{device}'} "
                         f"with room for {count} {'bytes' if dtype is None else 'values of its type'}")
    return b.data_ptr()


_NORM_WS = 0


def thc_norm_workspace_bytes() -> int:
    out = C.c_size_t(0)
    _check(lib().thc_norm_workspace_bytes(C.byref(out)), "thc_norm_workspace_bytes")
    return out.value


def _norm_call(call, where: str, tensors, kind, max_norm, norm_out, scale_out, ws, stream) -> None:
    global _NORM_WS
    if not _NORM_WS:
        _NORM_WS = thc_norm_workspace_bytes()
    t, stream, at = _list_and_stream(tensors, stream, where)
    rc = call(t, kind, max_norm, _buffer(norm_out, "norm_out", where, 1, THC_DTYPE_F32, at),
              _buffer(scale_out, "scale_out", where, 1, THC_DTYPE_F32, at), _buffer(ws, "ws", where, _NORM_WS, None, at), stream)
    if rc != 0:
        raise ThcError(rc, where)


def thc_grad_norm(tensors, kind: int, max_norm: float, norm_out, scale_out, ws, stream=None) -> None:
    """Global norm of a list of tensors (thc_tensors, or a sequence of tensors) and, unless scale_out is None, the factor
    that clips it to max_norm; both are one float32 on the GPU.  max_norm is taken as float32: the factor is that of the
    rounded limit, up to half a step (2^-24) off that of a Python float."""
    _norm_call((_LIB or lib()).thc_grad_norm, "thc_grad_norm", tensors, kind, max_norm, norm_out, scale_out, ws, stream)


def thc_grad_clip(tensors, kind: int, max_norm: float, norm_out, scale_out, ws, stream=None) -> None:
    """thc_grad_norm, and the tensors scaled in place where the norm exceeds max_norm."""
    _norm_call((_LIB or lib()).thc_grad_clip, "thc_grad_clip", tensors, kind, max_norm, norm_out, scale_out, ws, stream)


def thc_gather(p: thc_params, tensors, scale, grad_out, stream=None) -> None:
    """The tensors one after another into the padded vector grad_out (p.d values of p.in_dtype), times *scale (None: 1)."""
    t, stream, at = _list_and_stream(tensors, stream, "thc_gather")
    _check((_LIB or lib()).thc_gather(p, t, _buffer(scale, "scale", "thc_gather", 1, THC_DTYPE_F32, at),
                                      _buffer(grad_out, "grad_out", "thc_gather", p.d, p.in_dtype, at), stream), "thc_gather")


def thc_scatter(p: thc_params, flat, scale, tensors, stream=None) -> None:
    """The estimate `flat` (p.d float32 values) over the tensors, times *scale (None: 1)."""
    t, stream, at = _list_and_stream(tensors, stream, "thc_scatter")
    _check((_LIB or lib()).thc_scatter(p, _buffer(flat, "flat", "thc_scatter", p.d, THC_DTYPE_F32, at),
                                       _buffer(scale, "scale", "thc_scatter", 1, THC_DTYPE_F32, at), t, stream), "thc_scatter")


def thc_threshold(p: float) -> float:
    return lib().thc_threshold(p)


def thc_solve_table(b: int, g: int, p: float):
    """Returns (table as a list of 2^b ints, cost in sigma^2 units)."""
    out = (C.c_uint8 * 256)()
    cost = C.c_double(0.0)
    _check(lib().thc_solve_table(b, g, p, out, C.byref(cost)), "thc_solve_table")
    return [int(out[i]) for i in range(2 ** b)], cost.value


def thc_solve_table_bruteforce(b: int, g: int, p: float):
    """Exhaustive search over Alg. 4's enumeration.  Returns (table, cost, number of candidates visited)."""
    out = (C.c_uint8 * 256)()
    cost = C.c_double(0.0)
    count = C.c_uint64(0)
    _check(lib().thc_solve_table_bruteforce(b, g, p, out, C.byref(cost), C.byref(count)), "thc_solve_table_bruteforce")
    return [int(out[i]) for i in range(2 ** b)], cost.value, count.value


THC_PLAN_RECORD_WORDS = 40


def thc_describe_plan(p: thc_params):
    """The passes of the transform for these parameters: a list of dicts (kind, bits, tiling fields)."""
    n = lib().thc_describe_plan(C.byref(p), None, 0)
    _check(min(n, 0), "thc_describe_plan")
    buf = (C.c_uint32 * (n * THC_PLAN_RECORD_WORDS))()
    _check(min(lib().thc_describe_plan(C.byref(p), buf, n), 0), "thc_describe_plan")
    names = ("L", "logw", "nrows", "nfixed", "n0", "sh0", "sh1")
    out = []
    for k in range(n):
        r = buf[k * THC_PLAN_RECORD_WORDS:(k + 1) * THC_PLAN_RECORD_WORDS]
        rec = {"kind": r[0], "bits": list(r[2:2 + r[1]])}
        rec.update(zip(names, r[18:25]))
        rec["fcum"], rec["fmask"], rec["fpos"] = list(r[25:29]), list(r[29:33]), list(r[33:37])
        out.append(rec)
    return out
