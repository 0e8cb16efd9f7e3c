"""Python binding of libspccl.so, the gfx950 Pici hot path (SpCCL, arXiv 2607.04676).

Argument marshalling only: every step runs in the HIP library.  Functions keep
the C names of include/spccl.h and take torch tensors for device buffers (their
data pointers and byte sizes are passed through) and an optional torch stream
(default: the current stream).  A nonzero status raises SpcclError.  There is
no fallback: if the library is missing, importing this package fails.
"""
from __future__ import annotations

import ctypes
import os
from bisect import bisect_left

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspccl.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                      "(or python paper_2607_04676_amd/build.py)")

_lib = ctypes.CDLL(LIB_PATH)

SPCCL_OK = 0
STATUS_NAMES = {0: "OK", 1: "ERR_INVALID_ARG", 2: "ERR_CAPACITY", 3: "ERR_UNSUPPORTED",
                4: "ERR_CORRUPT_STREAM", 5: "ERR_WORKSPACE", 6: "ERR_HIP", 7: "ERR_TIMEOUT"}
SPCCL_F32, SPCCL_BF16 = 0, 1
SPCCL_FMT_DENSE, SPCCL_FMT_PICI, SPCCL_FMT_COO = 0, 1, 2
SPCCL_ARRAY, SPCCL_STREAM = 0, 1
SPCCL_STATE_F32, SPCCL_STATE_F8 = 0, 1
SPCCL_STATE_BLOCK = 32
HEADER_BYTES = 48
CONTROL_BYTES = 256
NNZ_UNKNOWN = (1 << 64) - 1

# every symbol the C header declares
EXPORTS = ("spccl_num_tiles", "spccl_pici_bytes", "spccl_stream_bound", "spccl_workspace_bytes",
           "spccl_workspace_min_bytes",
           "spccl_workspace_init", "spccl_compress", "spccl_decompress", "spccl_encode_dense",
           "spccl_reduce", "spccl_gather_expand", "spccl_copy_message", "spccl_read_header",
           "spccl_read_status", "spccl_status_string", "spccl_vr_scratch_bytes",
           "spccl_vr_reduce_scatter", "spccl_vr_all_gather", "spccl_vr_all_reduce",
           "spccl_slice_count", "spccl_slice_bytes", "spccl_compress_sliced", "spccl_decompress_sliced",
           "spccl_reduce_sliced", "spccl_copy_sliced", "spccl_coo_bytes", "spccl_message_bound",
           "spccl_compress_coo", "spccl_slice_tracker_bytes", "spccl_compress_sliced_tracked",
           "spccl_reduce_sliced_tracked", "spccl_vr_sliced_scratch_bytes", "spccl_vr_reduce_scatter_sliced",
           "spccl_vr_all_gather_sliced", "spccl_vr_all_reduce_sliced", "spccl_compress_static",
           "spccl_set_single_pass_limit", "spccl_layer_norm", "spccl_layer_norm_scratch_bytes",
           "spccl_layer_norm_backward", "spccl_prune", "spccl_adamw_plan_bytes", "spccl_adamw_plan",
           "spccl_adamw_step")


class spccl_operand_t(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("fmt", ctypes.c_int32), ("ptr", ctypes.c_void_p),
                ("bytes", ctypes.c_uint64)]


class spccl_header_t(ctypes.Structure):
    _fields_ = [("magic", ctypes.c_uint32), ("format", ctypes.c_uint16), ("dtype", ctypes.c_uint16),
                ("n", ctypes.c_uint64), ("nnz", ctypes.c_uint64), ("off_I", ctypes.c_uint64),
                ("off_A", ctypes.c_uint64), ("total_bytes", ctypes.c_uint64)]


class spccl_policy_t(ctypes.Structure):
    _fields_ = [("intra_thresh", ctypes.c_double), ("inter_thresh", ctypes.c_double),
                ("ag_thresh", ctypes.c_double), ("ranks_per_node", ctypes.c_int32),
                ("adaptive", ctypes.c_int32), ("sparse_fmt", ctypes.c_int32)]


class spccl_trace_t(ctypes.Structure):
    _fields_ = [("step", ctypes.c_int32), ("rank", ctypes.c_int32), ("fmt", ctypes.c_int32),
                ("measured", ctypes.c_int32), ("bytes", ctypes.c_uint64), ("nnz", ctypes.c_uint64),
                ("sigma", ctypes.c_double)]


class spccl_adamw_tensor_t(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("model", ctypes.c_void_p), ("grad", spccl_operand_t),
                ("grad_offset", ctypes.c_uint64), ("grad_n", ctypes.c_uint64), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("n", ctypes.c_uint64), ("weight_decay", ctypes.c_double)]


class spccl_adamw_plan_t(ctypes.Structure):
    _fields_ = [("magic", ctypes.c_uint32), ("param_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32),
                ("state", ctypes.c_int32), ("count", ctypes.c_int32), ("pad", ctypes.c_int32),
                ("array_chunks", ctypes.c_uint64), ("stream_chunks", ctypes.c_uint64), ("table", ctypes.c_void_p)]
    _written = ((), ())       # the starts and the ends of what a step writes


class spccl_adamw_t(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", ctypes.c_uint64), ("seed", ctypes.c_uint64)]


_u64, _i32, _vp = ctypes.c_uint64, ctypes.c_int32, ctypes.c_void_p
_sigs = {
    "spccl_num_tiles": (_u64, [_u64]),
    "spccl_pici_bytes": (_u64, [_u64, _i32, _u64]),
    "spccl_stream_bound": (_u64, [_u64, _i32]),
    "spccl_workspace_bytes": (_u64, [_u64, _i32]),
    "spccl_workspace_min_bytes": (_u64, [_u64, _i32]),
    "spccl_workspace_init": (_i32, [_vp, _u64, _vp]),
    "spccl_set_single_pass_limit": (ctypes.c_uint32, [ctypes.c_uint32]),
    "spccl_compress": (_i32, [_vp, _u64, _i32, _vp, _u64, _vp, _u64, _vp]),
    "spccl_compress_coo": (_i32, [_vp, _u64, _i32, _vp, _u64, _vp, _u64, _vp]),
    "spccl_compress_static": (_i32, [_vp, _u64, _i32, _vp, _u64, _vp]),
    "spccl_coo_bytes": (_u64, [_i32, _u64]),
    "spccl_message_bound": (_u64, [_u64, _i32, _i32]),
    "spccl_decompress": (_i32, [_vp, _u64, _vp, _u64, _i32, _vp, _u64, _vp]),
    "spccl_encode_dense": (_i32, [_vp, _u64, _i32, _vp, _u64, _vp]),
    "spccl_reduce": (_i32, [spccl_operand_t, spccl_operand_t, spccl_operand_t, _u64, _i32, _vp, _u64, _vp]),
    "spccl_gather_expand": (_i32, [ctypes.POINTER(spccl_operand_t), _i32, _u64, _i32, _vp, _u64, _vp, _u64,
                                   _vp]),
    "spccl_copy_message": (_i32, [_vp, _u64, _vp, _u64, _vp, _u64, _vp]),
    "spccl_read_header": (_i32, [_vp, ctypes.POINTER(spccl_header_t), _vp]),
    "spccl_read_status": (_i32, [_vp, _i32, _vp]),
    "spccl_status_string": (ctypes.c_char_p, [_i32]),
    "spccl_vr_scratch_bytes": (_u64, [_i32, _u64, _i32]),
    "spccl_vr_reduce_scatter": (_i32, [ctypes.POINTER(_vp), ctypes.POINTER(_vp), _i32, _u64, _i32,
                                       ctypes.POINTER(spccl_policy_t), _vp, _u64, ctypes.POINTER(spccl_trace_t),
                                       _vp]),
    "spccl_vr_all_gather": (_i32, [ctypes.POINTER(_vp), ctypes.POINTER(_vp), _i32, _u64, _i32,
                                   ctypes.POINTER(spccl_policy_t), _vp, _u64, ctypes.POINTER(spccl_trace_t), _vp]),
    "spccl_vr_all_reduce": (_i32, [ctypes.POINTER(_vp), ctypes.POINTER(_vp), _i32, _u64, _i32,
                                   ctypes.POINTER(spccl_policy_t), _vp, _u64, ctypes.POINTER(spccl_trace_t),
                                   _vp]),
    "spccl_slice_count": (_u64, [_u64]),
    "spccl_slice_bytes": (_u64, [_i32]),
    "spccl_compress_sliced": (_i32, [_vp, _u64, _i32, ctypes.c_double, _vp, _u64, _vp, _u64, _vp]),
    "spccl_decompress_sliced": (_i32, [_vp, _u64, _vp, _u64, _i32, _vp, _u64, _vp]),
    "spccl_reduce_sliced": (_i32, [_vp, _vp, _u64, _vp, _u64, _i32, ctypes.c_double, _u64, _i32, _vp, _u64, _vp]),
    "spccl_copy_sliced": (_i32, [_vp, _u64, _vp, _u64, _u64, _i32, _vp, _u64, _vp]),
    "spccl_slice_tracker_bytes": (_u64, [_u64]),
    "spccl_compress_sliced_tracked": (_i32, [_vp, _u64, _i32, ctypes.c_double, _vp, _u64, _vp, _u64, _vp, _vp,
                                             _u64, _vp]),
    "spccl_reduce_sliced_tracked": (_i32, [_vp, _vp, _u64, _vp, _u64, ctypes.c_double, _vp, _u64, _vp, _u64, _i32,
                                           _vp, _u64, _vp]),
    "spccl_vr_sliced_scratch_bytes": (_u64, [_i32, _u64, _i32]),
    "spccl_vr_reduce_scatter_sliced": (_i32, [ctypes.POINTER(_vp), ctypes.POINTER(_vp), _i32, _u64, _i32,
                                              ctypes.POINTER(spccl_policy_t), _vp, _u64, _vp, _vp]),
    "spccl_vr_all_gather_sliced": (_i32, [ctypes.POINTER(_vp), ctypes.POINTER(_vp), _i32, _u64, _i32, _vp, _u64,
                                          _vp, _vp]),
    "spccl_vr_all_reduce_sliced": (_i32, [ctypes.POINTER(_vp), ctypes.POINTER(_vp), _i32, _u64, _i32,
                                          ctypes.POINTER(spccl_policy_t), _vp, _u64, _vp, _vp, _vp]),
    "spccl_layer_norm": (_i32, [_vp, _u64, _vp, _vp, _vp, _u64, _vp, _vp, _u64, _u64, _i32, _i32, ctypes.c_double, _vp]),
    "spccl_layer_norm_scratch_bytes": (_u64, [_u64, _u64]),
    "spccl_layer_norm_backward": (_i32, [_vp, _u64, _vp, _u64, _vp, _vp, _vp, _vp, _u64, _vp, _vp, _u64, _u64, _i32, _i32,
                                         _i32, _i32, _vp, _u64, _vp]),
    "spccl_prune": (_i32, [_vp, _vp, _vp, ctypes.c_double, _vp, _u64, _i32, _vp]),
    "spccl_adamw_plan_bytes": (_u64, [ctypes.POINTER(spccl_adamw_tensor_t), _i32]),
    "spccl_adamw_plan": (_i32, [ctypes.POINTER(spccl_adamw_tensor_t), _i32, _i32, _i32, _i32, _vp, _u64,
                                ctypes.POINTER(spccl_adamw_plan_t), _vp]),
    "spccl_adamw_step": (_i32, [ctypes.POINTER(spccl_adamw_plan_t), ctypes.POINTER(spccl_adamw_t), _vp, _vp, _u64, _vp]),
}
for _name, (_res, _args) in _sigs.items():
    _f = getattr(_lib, _name)
    _f.restype = _res
    _f.argtypes = _args


class SpcclError(RuntimeError):
    def __init__(self, status: int, what: str):
        msg = _lib.spccl_status_string(status).decode()
        super().__init__(f"{what}: {STATUS_NAMES.get(status, status)} ({msg})")
        self.status = status


def _check(st: int, what: str) -> None:
    if st != SPCCL_OK:
        raise SpcclError(st, what)


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return SPCCL_F32
    if t.dtype in (torch.bfloat16, torch.int16, torch.uint16):
        return SPCCL_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


# the current stream's handle without a Stream object (0.1 us against 2.8)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _nbytes(t: torch.Tensor) -> int:
    return t.numel() * t.element_size()


def operand(t: torch.Tensor, kind: int = SPCCL_ARRAY, fmt: int = SPCCL_FMT_DENSE) -> spccl_operand_t:
    """The C operand of a device tensor.  It holds a reference to the tensor,
    so an operand made from a temporary keeps that memory alive as long as
    the operand itself."""
    o = spccl_operand_t(kind, fmt, t.data_ptr(), _nbytes(t))
    o._tensor = t
    return o


# ---- sizes --------------------------------------------------------------------------

def spccl_num_tiles(n: int) -> int:
    return _lib.spccl_num_tiles(n)


def spccl_pici_bytes(n: int, dtype: int, nnz: int) -> int:
    return _lib.spccl_pici_bytes(n, dtype, nnz)


def spccl_stream_bound(n: int, dtype: int) -> int:
    return _lib.spccl_stream_bound(n, dtype)


def spccl_workspace_bytes(n: int, dtype: int) -> int:
    return _lib.spccl_workspace_bytes(n, dtype)


def spccl_workspace_min_bytes(n: int, dtype: int) -> int:
    return _lib.spccl_workspace_min_bytes(n, dtype)


def spccl_set_single_pass_limit(max_partitions: int) -> int:
    """Upper bound (in 16384-element partitions) on the Pici outputs written in
    one launch with a full workspace (0: always two passes; default 2**32 - 1,
    the library's own limits); returns the previous bound."""
    return _lib.spccl_set_single_pass_limit(max_partitions)


def spccl_coo_bytes(dtype: int, nnz: int) -> int:
    return _lib.spccl_coo_bytes(dtype, nnz)


def spccl_message_bound(n: int, dtype: int, fmt: int) -> int:
    return _lib.spccl_message_bound(n, dtype, fmt)


def spccl_vr_scratch_bytes(P: int, msg_elems: int, dtype: int) -> int:
    return _lib.spccl_vr_scratch_bytes(P, msg_elems, dtype)


# ---- entry points ------------------------------------------------------------------

def spccl_workspace_init(ws: torch.Tensor, stream=None) -> None:
    _check(_lib.spccl_workspace_init(ws.data_ptr(), _nbytes(ws), _stream(stream)), "spccl_workspace_init")


def spccl_compress(dense: torch.Tensor, out: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    _check(_lib.spccl_compress(dense.data_ptr(), dense.numel(), _dt(dense), out.data_ptr(), _nbytes(out),
                               ws.data_ptr(), _nbytes(ws), _stream(stream)), "spccl_compress")


def spccl_compress_static(dense: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    """spccl_compress without a workspace (its scratch is the library's own
    static device array; n <= SPCCL_STATIC_MAX_ELEMS)."""
    _check(_lib.spccl_compress_static(dense.data_ptr(), dense.numel(), _dt(dense), out.data_ptr(), _nbytes(out),
                                      _stream(stream)), "spccl_compress_static")


SPCCL_STATIC_MAX_ELEMS = 1 << 28


def spccl_compress_coo(dense: torch.Tensor, out: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    _check(_lib.spccl_compress_coo(dense.data_ptr(), dense.numel(), _dt(dense), out.data_ptr(), _nbytes(out),
                                   ws.data_ptr(), _nbytes(ws), _stream(stream)), "spccl_compress_coo")


def spccl_decompress(msg: torch.Tensor, dense: torch.Tensor, ws: torch.Tensor, stream=None,
                     msg_bytes: int | None = None) -> None:
    _check(_lib.spccl_decompress(msg.data_ptr(), _nbytes(msg) if msg_bytes is None else msg_bytes,
                                 dense.data_ptr(), dense.numel(), _dt(dense), ws.data_ptr(), _nbytes(ws),
                                 _stream(stream)), "spccl_decompress")


def spccl_encode_dense(dense: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    _check(_lib.spccl_encode_dense(dense.data_ptr(), dense.numel(), _dt(dense), out.data_ptr(), _nbytes(out),
                                   _stream(stream)), "spccl_encode_dense")


def spccl_reduce(a: spccl_operand_t, b: spccl_operand_t, out: spccl_operand_t, n: int, dtype: int,
                 ws: torch.Tensor, stream=None) -> None:
    _check(_lib.spccl_reduce(a, b, out, n, dtype, ws.data_ptr(), _nbytes(ws), _stream(stream)), "spccl_reduce")


def spccl_gather_expand(parts: list, n_per_part: int, dtype: int, dense_out: torch.Tensor, ws: torch.Tensor,
                        stream=None) -> None:
    arr = (spccl_operand_t * len(parts))(*parts)
    _check(_lib.spccl_gather_expand(arr, len(parts), n_per_part, dtype, dense_out.data_ptr(), _nbytes(dense_out),
                                    ws.data_ptr(), _nbytes(ws), _stream(stream)), "spccl_gather_expand")


def spccl_copy_message(src: torch.Tensor, dst: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    _check(_lib.spccl_copy_message(src.data_ptr(), _nbytes(src), dst.data_ptr(), _nbytes(dst), ws.data_ptr(),
                                   _nbytes(ws), _stream(stream)), "spccl_copy_message")


def spccl_read_header(msg: torch.Tensor, stream=None) -> dict:
    h = spccl_header_t()
    _check(_lib.spccl_read_header(msg.data_ptr(), ctypes.byref(h), _stream(stream)), "spccl_read_header")
    return {f: getattr(h, f) for f, _ in spccl_header_t._fields_}


def spccl_read_status(ws: torch.Tensor, clear: bool = True, stream=None) -> int:
    return _lib.spccl_read_status(ws.data_ptr(), 1 if clear else 0, _stream(stream))


def spccl_status_string(status: int) -> str:
    return _lib.spccl_status_string(status).decode()


def _policy(policy) -> spccl_policy_t:
    if policy is None:
        return spccl_policy_t(0.6, 0.5, 0.1, 0, 1, SPCCL_FMT_PICI)
    if isinstance(policy, spccl_policy_t):
        return policy
    return spccl_policy_t(policy.intra_thresh, policy.inter_thresh, policy.ag_thresh, policy.ranks_per_node,
                          policy.adaptive, getattr(policy, "sparse_fmt", SPCCL_FMT_PICI))


def _ptrs(ts) -> ctypes.Array:
    return (ctypes.c_void_p * len(ts))(*[t.data_ptr() for t in ts])


def _trace(tr, count) -> list:
    return [(tr[i].step, tr[i].rank, tr[i].fmt, tr[i].measured, tr[i].bytes, tr[i].nnz, tr[i].sigma)
            for i in range(count)]


def spccl_vr_reduce_scatter(send: list, recv: list, scratch: torch.Tensor, policy=None, stream=None) -> list:
    P, n = len(send), send[0].numel()
    tr = (spccl_trace_t * max(1, P * (P - 1)))()
    pol = _policy(policy)
    _check(_lib.spccl_vr_reduce_scatter(_ptrs(send), _ptrs(recv), P, n, _dt(send[0]), ctypes.byref(pol),
                                        scratch.data_ptr(), _nbytes(scratch), tr, _stream(stream)),
           "spccl_vr_reduce_scatter")
    return _trace(tr, P * (P - 1))


def spccl_vr_all_gather(send: list, recv: list, scratch: torch.Tensor, policy=None, stream=None) -> list:
    P, n = len(send), send[0].numel()
    tr = (spccl_trace_t * P)()
    pol = _policy(policy)
    _check(_lib.spccl_vr_all_gather(_ptrs(send), _ptrs(recv), P, n, _dt(send[0]), ctypes.byref(pol),
                                    scratch.data_ptr(), _nbytes(scratch), tr, _stream(stream)), "spccl_vr_all_gather")
    return _trace(tr, P)


def spccl_vr_all_reduce(send: list, recv: list, scratch: torch.Tensor, policy=None, stream=None) -> list:
    P, n = len(send), send[0].numel()
    tr = (spccl_trace_t * (P * (P - 1) + P))()
    pol = _policy(policy)
    _check(_lib.spccl_vr_all_reduce(_ptrs(send), _ptrs(recv), P, n, _dt(send[0]), ctypes.byref(pol),
                                    scratch.data_ptr(), _nbytes(scratch), tr, _stream(stream)),
           "spccl_vr_all_reduce")
    return _trace(tr, P * (P - 1) + P)


# ---- sliced streams -----------------------------------------------------------------

SPCCL_SLICE_ELEMS = 16384


def spccl_slice_count(n: int) -> int:
    return _lib.spccl_slice_count(n)


def spccl_slice_bytes(dtype: int) -> int:
    return _lib.spccl_slice_bytes(dtype)


def spccl_compress_sliced(dense: torch.Tensor, out: torch.Tensor, ws: torch.Tensor, dense_thresh: float = -1.0,
                          stream=None) -> None:
    _check(_lib.spccl_compress_sliced(dense.data_ptr(), dense.numel(), _dt(dense), float(dense_thresh),
                                      out.data_ptr(), _nbytes(out), ws.data_ptr(), _nbytes(ws), _stream(stream)),
           "spccl_compress_sliced")


def spccl_decompress_sliced(inp: torch.Tensor, dense: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    _check(_lib.spccl_decompress_sliced(inp.data_ptr(), _nbytes(inp), dense.data_ptr(), dense.numel(), _dt(dense),
                                        ws.data_ptr(), _nbytes(ws), _stream(stream)), "spccl_decompress_sliced")


def spccl_reduce_sliced(a: torch.Tensor, b: torch.Tensor, out: torch.Tensor, ws: torch.Tensor, out_sliced: bool,
                        dense_thresh: float = -1.0, stream=None) -> None:
    """out = a (dense) (+) b (sliced stream); out is a sliced stream or a dense array."""
    _check(_lib.spccl_reduce_sliced(a.data_ptr(), b.data_ptr(), _nbytes(b), out.data_ptr(), _nbytes(out),
                                    1 if out_sliced else 0, float(dense_thresh), a.numel(), _dt(a), ws.data_ptr(),
                                    _nbytes(ws), _stream(stream)), "spccl_reduce_sliced")


def spccl_copy_sliced(src: torch.Tensor, dst: torch.Tensor, n: int, dtype: int, ws: torch.Tensor,
                      stream=None) -> None:
    _check(_lib.spccl_copy_sliced(src.data_ptr(), _nbytes(src), dst.data_ptr(), _nbytes(dst), n, dtype,
                                  ws.data_ptr(), _nbytes(ws), _stream(stream)), "spccl_copy_sliced")


def spccl_slice_tracker_bytes(n: int) -> int:
    return _lib.spccl_slice_tracker_bytes(n)


def _ptr_or_null(t) -> int | None:
    return None if t is None else t.data_ptr()


def spccl_compress_sliced_tracked(dense: torch.Tensor, out: torch.Tensor, tracker: torch.Tensor, ws: torch.Tensor,
                                  tau: float, fmt_out: torch.Tensor | None = None, stream=None) -> None:
    _check(_lib.spccl_compress_sliced_tracked(dense.data_ptr(), dense.numel(), _dt(dense), float(tau),
                                              out.data_ptr(), _nbytes(out), tracker.data_ptr(), _nbytes(tracker),
                                              _ptr_or_null(fmt_out), ws.data_ptr(), _nbytes(ws), _stream(stream)),
           "spccl_compress_sliced_tracked")


def spccl_reduce_sliced_tracked(a: torch.Tensor, b: torch.Tensor, out: torch.Tensor, tracker: torch.Tensor,
                                ws: torch.Tensor, tau: float, fmt_out: torch.Tensor | None = None,
                                stream=None) -> None:
    _check(_lib.spccl_reduce_sliced_tracked(a.data_ptr(), b.data_ptr(), _nbytes(b), out.data_ptr(), _nbytes(out),
                                            float(tau), tracker.data_ptr(), _nbytes(tracker), _ptr_or_null(fmt_out),
                                            a.numel(), _dt(a), ws.data_ptr(), _nbytes(ws), _stream(stream)),
           "spccl_reduce_sliced_tracked")


def spccl_vr_sliced_scratch_bytes(P: int, msg_elems: int, dtype: int) -> int:
    return _lib.spccl_vr_sliced_scratch_bytes(P, msg_elems, dtype)


def spccl_vr_reduce_scatter_sliced(send: list, recv: list, scratch: torch.Tensor, policy=None, stream=None):
    """Returns the per-slice formats sent, shape (P-1, P, S)."""
    import numpy as np
    P, n = len(send), send[0].numel()
    S = spccl_slice_count(n // P)
    fm = np.zeros(max(1, (P - 1) * P * S), dtype=np.uint8)
    pol = _policy(policy)
    _check(_lib.spccl_vr_reduce_scatter_sliced(_ptrs(send), _ptrs(recv), P, n, _dt(send[0]), ctypes.byref(pol),
                                               scratch.data_ptr(), _nbytes(scratch), fm.ctypes.data,
                                               _stream(stream)), "spccl_vr_reduce_scatter_sliced")
    return fm[:(P - 1) * P * S].reshape(max(P - 1, 0), P, S)


def spccl_vr_all_gather_sliced(send: list, recv: list, scratch: torch.Tensor, stream=None):
    """Returns the per-slice formats sent, shape (P, S)."""
    import numpy as np
    P, n = len(send), send[0].numel()
    S = spccl_slice_count(n)
    fm = np.zeros(max(1, P * S), dtype=np.uint8)
    _check(_lib.spccl_vr_all_gather_sliced(_ptrs(send), _ptrs(recv), P, n, _dt(send[0]), scratch.data_ptr(),
                                           _nbytes(scratch), fm.ctypes.data, _stream(stream)),
           "spccl_vr_all_gather_sliced")
    return fm[:P * S].reshape(P, S)


def spccl_vr_all_reduce_sliced(send: list, recv: list, scratch: torch.Tensor, policy=None, stream=None):
    """Returns the per-slice formats (reduce-scatter (P-1, P, S), all-gather (P, S))."""
    import numpy as np
    P, n = len(send), send[0].numel()
    S = spccl_slice_count(n // P)
    frs = np.zeros(max(1, (P - 1) * P * S), dtype=np.uint8)
    fag = np.zeros(max(1, P * S), dtype=np.uint8)
    pol = _policy(policy)
    _check(_lib.spccl_vr_all_reduce_sliced(_ptrs(send), _ptrs(recv), P, n, _dt(send[0]), ctypes.byref(pol),
                                           scratch.data_ptr(), _nbytes(scratch), frs.ctypes.data, fag.ctypes.data,
                                           _stream(stream)), "spccl_vr_all_reduce_sliced")
    return frs[:(P - 1) * P * S].reshape(max(P - 1, 0), P, S), fag[:P * S].reshape(P, S)


def alloc_sliced(n: int, dtype: int, device="cuda") -> torch.Tensor:
    """A uint8 buffer with every slot of an n-element sliced stream."""
    return torch.empty(max(spccl_slice_count(n) * spccl_slice_bytes(dtype), 16), dtype=torch.uint8, device=device)


# ---- layer norm ---------------------------------------------------------------------

def _matrix(t: torch.Tensor, like: torch.Tensor, what: str) -> int:
    """The row pitch of a matrix whose rows are contiguous, of the same shape
    and dtype as `like`."""
    if t is not like and (t.shape != like.shape or t.dtype != like.dtype):
        raise ValueError(f"{what}: {tuple(t.shape)} {t.dtype} does not match {tuple(like.shape)} {like.dtype}")
    strides = t.stride()
    if len(strides) != 2 or (strides[1] != 1 and t.shape[1] > 1):
        raise ValueError(f"{what}: a matrix with contiguous rows is needed, got shape {tuple(t.shape)} strides {strides}")
    return strides[0] if t.shape[0] > 1 else max(t.shape[1], 1)


def _vector(t: torch.Tensor, n: int, what: str, dtype) -> int:
    """The address of n contiguous elements of a dtype."""
    if t.shape != (n,) or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{what}: {n} contiguous elements of {dtype} are needed, got shape {tuple(t.shape)} {t.dtype}")
    return t.data_ptr()


def _vectors(a: torch.Tensor | None, b: torch.Tensor | None, n: int, what: str, otherwise: int) -> tuple:
    """Addresses of two vectors of one dtype (either may be None), and the dtype."""
    if a is None and b is None:
        return None, None, otherwise
    dtype = (b if a is None else a).dtype
    return (None if a is None else _vector(a, n, what, dtype), None if b is None else _vector(b, n, what, dtype),
            _dt(b if a is None else a))


def spccl_layer_norm(x: torch.Tensor, weight: torch.Tensor | None, bias: torch.Tensor | None, y: torch.Tensor,
                     mean: torch.Tensor | None = None, rstd: torch.Tensor | None = None, eps: float = 1e-5,
                     stream=None) -> None:
    """y = layer norm of x's rows; mean and rstd (fp32, one per row) are written
    for the backward pass."""
    ldx, ldy = _matrix(x, x, "x"), _matrix(y, x, "y")
    rows, cols = x.shape
    w, b, wdt = _vectors(weight, bias, cols, "weight and bias", SPCCL_F32)
    m = None if mean is None else _vector(mean, rows, "mean", torch.float32)
    r = None if rstd is None else _vector(rstd, rows, "rstd", torch.float32)
    _check(_lib.spccl_layer_norm(x.data_ptr(), ldx, w, b, y.data_ptr(), ldy, m, r, rows, cols, _dt(x), wdt, eps,
                                 _stream(stream)), "spccl_layer_norm")


def spccl_layer_norm_scratch_bytes(rows: int, cols: int) -> int:
    return _lib.spccl_layer_norm_scratch_bytes(rows, cols)


def spccl_layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor | None, mean: torch.Tensor,
                              rstd: torch.Tensor, dx: torch.Tensor | None, dweight: torch.Tensor | None,
                              dbias: torch.Tensor | None, scratch: torch.Tensor | None = None,
                              accumulate: bool = False, stream=None) -> None:
    """The gradients of sum(dy * y): dx, and the weight's and the bias's (any
    None: not wanted), added to what they hold if `accumulate`."""
    ldx, lddy = _matrix(x, x, "x"), _matrix(dy, x, "dy")
    lddx = 0 if dx is None else _matrix(dx, x, "dx")
    rows, cols = x.shape
    w, _, wdt = _vectors(weight, None, cols, "weight", SPCCL_F32)
    dw, db, gdt = _vectors(dweight, dbias, cols, "dweight and dbias", SPCCL_F32)
    _check(_lib.spccl_layer_norm_backward(
        dy.data_ptr(), lddy, x.data_ptr(), ldx, w, _vector(mean, rows, "mean", torch.float32),
        _vector(rstd, rows, "rstd", torch.float32), _ptr_or_null(dx), lddx, dw, db, rows, cols, _dt(x), wdt, gdt,
        1 if accumulate else 0, _ptr_or_null(scratch), 0 if scratch is None else _nbytes(scratch), _stream(stream)),
        "spccl_layer_norm_backward")


# ---- pruning and AdamW ---------------------------------------------------------------

def _device_value(t: torch.Tensor, what: str) -> None:
    """A single value that kernels read: one in pageable host memory, as
    torch.tensor makes it without a device, would fault there."""
    if t.numel() != 1 or t.dtype != torch.float32 or not (t.is_cuda or t.is_pinned()):
        raise ValueError(f"{what} is one fp32 in device memory, got {tuple(t.shape)} {t.dtype} on {t.device}")


def spccl_prune(grad: torch.Tensor, residual: torch.Tensor, threshold: torch.Tensor, leak: float, out: torch.Tensor,
                stream=None) -> None:
    """Split grad + leak * residual: what reaches the threshold (a device value)
    goes to out (which may be grad), the rest stays in residual (fp32)."""
    n = grad.numel()
    if not (grad.is_contiguous() and residual.is_contiguous() and out.is_contiguous()):
        raise ValueError("spccl_prune: contiguous tensors are needed")
    if residual.numel() != n or out.numel() != n or out.dtype != grad.dtype or residual.dtype != torch.float32:
        raise ValueError("spccl_prune: residual (fp32) and out (grad's dtype) hold grad's elements")
    _device_value(threshold, "spccl_prune: threshold")
    _check(_lib.spccl_prune(grad.data_ptr(), residual.data_ptr(), threshold.data_ptr(), float(leak), out.data_ptr(), n,
                            _dt(grad), _stream(stream)), "spccl_prune")


def adamw_tensor(param: torch.Tensor, grad, m: torch.Tensor, v: torch.Tensor, m_scale: torch.Tensor | None = None,
                 v_scale: torch.Tensor | None = None, model: torch.Tensor | None = None, weight_decay: float = 0.0,
                 grad_dtype: int | None = None, grad_offset: int = 0, grad_n: int = 0) -> spccl_adamw_tensor_t:
    """One tensor of an AdamW plan.  grad is a tensor of param's elements, or an
    operand: then grad_dtype (SPCCL_F32 or SPCCL_BF16) and, for a message, the
    tensor's place grad_offset among its grad_n elements are given too.  m and v
    are fp32, or one byte per element (float8_e4m3fn or uint8) with m_scale and
    v_scale (float8_e8m0fnu or uint8), one per SPCCL_STATE_BLOCK elements.  It
    holds references to its tensors."""
    n = param.numel()
    eight = m.dtype != torch.float32
    tensors = [("param", param, n, None), ("m", m, n, None), ("v", v, n, m.dtype)]
    if model is not None:
        tensors.append(("model", model, n, torch.bfloat16))
    if isinstance(grad, torch.Tensor):
        tensors.append(("grad", grad, n, None))
    if eight:
        if m.element_size() != 1 or m_scale is None or v_scale is None:
            raise ValueError("adamw_tensor: 8-bit moments take one byte per element and their scales")
        blocks = -(-n // SPCCL_STATE_BLOCK)
        tensors += [("m_scale", m_scale, blocks, None), ("v_scale", v_scale, blocks, m_scale.dtype)]
        if m_scale.element_size() != 1:
            raise ValueError("adamw_tensor: a scale is one byte")
    elif m_scale is not None or v_scale is not None:
        raise ValueError("adamw_tensor: fp32 moments have no scales")
    for what, t, size, dt in tensors:
        if t.numel() != size or not t.is_contiguous() or (dt is not None and t.dtype != dt):
            raise ValueError(f"adamw_tensor: {what} needs {size} contiguous elements{f' of {dt}' if dt else ''}, got "
                             f"{tuple(t.shape)} {t.dtype}")
    if isinstance(grad, torch.Tensor):
        op, gdt = operand(grad), _dt(grad)
    elif grad_dtype is None:
        raise ValueError("adamw_tensor: an operand's grad_dtype is needed")
    else:
        op, gdt = grad, grad_dtype
    t = spccl_adamw_tensor_t(param.data_ptr(), _ptr_or_null(model), op, grad_offset, grad_n, m.data_ptr(), v.data_ptr(),
                             _ptr_or_null(m_scale), _ptr_or_null(v_scale), n, weight_decay)
    t._types = (_dt(param), gdt, SPCCL_STATE_F8 if eight else SPCCL_STATE_F32)
    t._tensors = (param, grad, m, v, m_scale, v_scale, model)
    return t


def alloc_adamw_state(n: int, state: int = SPCCL_STATE_F32, device="cuda") -> dict:
    """Zeroed moments of n elements, as adamw_tensor's keywords m, v (and m_scale, v_scale)."""
    if state == SPCCL_STATE_F32:
        return {k: torch.zeros(n, dtype=torch.float32, device=device) for k in ("m", "v")}
    blocks = -(-n // SPCCL_STATE_BLOCK)
    out = {k: torch.zeros(n, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn) for k in ("m", "v")}
    for k in ("m_scale", "v_scale"):
        out[k] = torch.zeros(blocks, dtype=torch.uint8, device=device).view(torch.float8_e8m0fnu)
    return out


def spccl_adamw_plan_bytes(tensors: list) -> int:
    return _lib.spccl_adamw_plan_bytes((spccl_adamw_tensor_t * len(tensors))(*tensors), len(tensors))


def spccl_adamw_plan(tensors: list, table: torch.Tensor, stream=None) -> spccl_adamw_plan_t:
    """A plan over tensors made by adamw_tensor, laid out in table (bytes on the
    device).  It holds references to both."""
    kinds = {t._types for t in tensors}
    if len(kinds) > 1:
        raise ValueError(f"spccl_adamw_plan: (param, gradient, state) types differ: {sorted(kinds)}")
    pdt, gdt, state = kinds.pop() if kinds else (SPCCL_F32, SPCCL_F32, SPCCL_STATE_F32)
    plan = spccl_adamw_plan_t()
    _check(_lib.spccl_adamw_plan((spccl_adamw_tensor_t * len(tensors))(*tensors), len(tensors), pdt, gdt, state,
                                 table.data_ptr(), _nbytes(table), ctypes.byref(plan), _stream(stream)),
           "spccl_adamw_plan")
    plan._tensors = (list(tensors), table)
    plan._written = _written(tensors, pdt, state)
    return plan


def _written(tensors: list, pdt: int, state: int) -> tuple:
    """The starts and the ends of what a step writes, in order (the plan has
    refused overlaps among them)."""
    p, s = (4 if pdt == SPCCL_F32 else 2), (4 if state == SPCCL_STATE_F32 else 1)
    spans = []
    for t in tensors:
        n, model = t.n, t.model
        if not n:
            continue
        for a, size in ((t.param, p * n), (t.m, s * n), (t.v, s * n)):
            spans.append((a, a + size))
        if model:
            spans.append((model, model + 2 * n))
        if state == SPCCL_STATE_F8:
            for a in (t.m_scale, t.v_scale):
                spans.append((a, a + -(-n // SPCCL_STATE_BLOCK)))
    spans.sort()
    return [a for a, _ in spans], [b for _, b in spans]


def _meets(written: tuple, at: int, nbytes: int) -> bool:
    """Whether nbytes from an address on share a byte with the written spans."""
    k = bisect_left(written[0], at + nbytes)
    return k > 0 and written[1][k - 1] > at


def spccl_adamw_step(plan: spccl_adamw_plan_t, ws: torch.Tensor, lr: float, beta1: float = 0.9, beta2: float = 0.999,
                     eps: float = 1e-8, step: int = 1, seed: int | None = None, grad_scale: torch.Tensor | None = None,
                     stream=None) -> None:
    """One AdamW step over the plan's tensors; gradients are multiplied by
    grad_scale (one fp32 on the device) first.  seed: of the stochastic rounding
    of 8-bit moments and bf16 parameters, another for each step, or rounding the
    same way each time holds small changes back; the step's number if none is
    given."""
    written, at, scale = plan._written, ws.data_ptr(), None
    if grad_scale is not None:
        _device_value(grad_scale, "spccl_adamw_step: grad_scale")
        scale = grad_scale.data_ptr()
        if _meets(written, scale, 4):
            raise ValueError("spccl_adamw_step: grad_scale overlaps what the step writes")
    if _meets(written, at, CONTROL_BYTES):
        raise ValueError("spccl_adamw_step: the workspace's control block overlaps what the step writes")
    h = spccl_adamw_t(lr, beta1, beta2, eps, step, step if seed is None else seed)
    _check(_lib.spccl_adamw_step(ctypes.byref(plan), ctypes.byref(h), scale, at, ws.nbytes, _stream(stream)),
           "spccl_adamw_step")


# ---- tensor helpers (allocation stays with the caller; these only size buffers) -----

def alloc_stream(n: int, dtype: int, device="cuda", fmt: int = SPCCL_FMT_PICI) -> torch.Tensor:
    """A uint8 buffer able to hold any n-element message of format fmt (or dense)."""
    return torch.empty(spccl_message_bound(n, dtype, fmt), dtype=torch.uint8, device=device)


def alloc_workspace(n: int, dtype: int, device="cuda", stream=None, minimal: bool = False) -> torch.Tensor:
    """A zeroed workspace for messages of up to n elements.  minimal=True
    sizes it for the one-launch kernels only (no per-partition slots)."""
    need = spccl_workspace_min_bytes(n, dtype) if minimal else spccl_workspace_bytes(n, dtype)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    spccl_workspace_init(ws, stream)
    return ws
