"""Thin ctypes binding of libftc.so: same names as the C ABI (include/ftc.h), argument marshalling only.

Device buffers are torch CUDA tensors (torch supplies memory and streams, nothing else); host buffers for
the *_host variants are numpy arrays or CPU tensors. There is no CPU or PyTorch fallback: if the library
is missing or fails to load, importing a function from here raises.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libftc.so")

FTC_I32, FTC_I64, FTC_U64, FTC_F32 = 0, 1, 2, 3
FTC_BF16, FTC_F16 = 4, 5                 # training operators only
FTC_SUM, FTC_MAX, FTC_XOR = 0, 1, 2
FTC_OK, FTC_EINVAL, FTC_EUNSUPPORTED, FTC_EWORKSPACE, FTC_ECUDA, FTC_ETOOLARGE = 0, -1, -2, -3, -4, -5
FTC_NOALLOC_SCRATCH_BYTES = 8 << 20
FTC_ST_OK, FTC_ST_ROOT_FAILED, FTC_ST_NO_CLEAN_SUBTREE, FTC_ST_NO_LIVE_ROOT_CANDIDATE = 0, 1, 2, 3
FTC_ST_PRECONDITION_INOP_ROOT, FTC_ST_BAD_ROOT, FTC_ST_INTERNAL_TIMEOUT = 4, 5, 6
FTC_STATUS_WORDS = 4
FTC_MSG_WORDS = 8
FTC_INOP_UNUSED = 0xFFFFFFFF
FTC_OUT_EXPANDED = 0x1
FTC_KERNEL_GENERIC = 0x100
FTC_MAX_ARITY = 32
FTC_TREE_BINOMIAL = 0x1000000
FTC_PARTNERS_DESCENDING = 0x2000000


def FTC_TREE_ARITY(a: int) -> int:
    """Flag bits asking for a-ary heaps below the root's children."""
    return (a & 0xFF) << 16

FTC_KERNEL_DIRECT = 0x200
FTC_KERNEL_LEVELS = 0x400
FTC_DEBUG_ONE_POLL = 0x4000000
OPS = {"sum": FTC_SUM, "max": FTC_MAX, "xor": FTC_XOR}

EXPORTS = ["ftc_reduce_batch", "ftc_allreduce_batch", "ftc_reduce_batch_noalloc", "ftc_candidates_batch",
           "ftc_candidates_workspace_bytes", "ftc_candidates_kernel_name", "ftc_message_counts_batch", "ftc_failed_list_batch", "ftc_workspace_bytes", "ftc_reduce_batch_host",
           "ftc_allreduce_batch_host", "ftc_host_staging_bytes", "ftc_schedule_info", "ftc_fill_inputs",
           "ftc_kernel_name", "ftc_kernel_variant", "ftc_launch_blocks", "ftc_read_bandwidth_probe", "ftc_strerror", "ftc_version",
           "ftc_layernorm_forward", "ftc_layernorm_backward", "ftc_layernorm_workspace_bytes", "ftc_param_table_bytes",
           "ftc_param_table_build", "ftc_param_table_blocks", "ftc_grad_norm", "ftc_grad_norm_workspace_bytes", "ftc_adamw_step",
           "ftc_adamw_states", "ftc_embedding_forward", "ftc_embedding_backward", "ftc_embedding_workspace_bytes", "ftc_token_logprobs",
           "ftc_token_logprobs_backward", "ftc_muon_plan_bytes", "ftc_muon_plan_build", "ftc_muon_plan_blocks", "ftc_muon_workspace_bytes",
           "ftc_muon_step"]
FTC_STATE_BLOCK = 256


class ftc_desc_t(C.Structure):
    _fields_ = [("P", C.c_uint32), ("f", C.c_uint32), ("k", C.c_uint32), ("dtype", C.c_uint32), ("op", C.c_uint32),
                ("root", C.c_int32), ("max_inop", C.c_uint32), ("flags", C.c_uint32)]


class ftc_sched_t(C.Structure):
    _fields_ = [("q", C.c_uint32), ("r", C.c_uint32), ("H", C.c_uint32), ("rounds_reduce", C.c_uint32),
                ("rounds_attempt", C.c_uint32), ("msgs_upcorrection", C.c_uint64), ("msgs_tree", C.c_uint64)]


class ftc_norm_t(C.Structure):
    _fields_ = [("H", C.c_uint32), ("P", C.c_uint32), ("k", C.c_uint32), ("dtype", C.c_uint32), ("wdtype", C.c_uint32),
                ("eps", C.c_float)]


class ftc_param_t(C.Structure):
    _fields_ = [("param", C.c_void_p), ("master", C.c_void_p), ("grad", C.c_void_p), ("status", C.c_void_p), ("n", C.c_uint64),
                ("k", C.c_uint32), ("param_dtype", C.c_uint32), ("grad_dtype", C.c_uint32), ("lr_scale", C.c_float),
                ("weight_decay", C.c_float), ("reserved", C.c_uint32)]


class ftc_adamw_t(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("step", C.c_uint64),
                ("state_bits", C.c_uint32), ("reserved", C.c_uint32)]


class ftc_embed_t(C.Structure):
    _fields_ = [("V", C.c_uint32), ("H", C.c_uint32), ("P", C.c_uint32), ("k", C.c_uint32), ("dtype", C.c_uint32), ("wdtype", C.c_uint32),
                ("token_bits", C.c_uint32), ("scale", C.c_float)]


class ftc_logprob_t(C.Structure):
    _fields_ = [("V", C.c_uint32), ("dtype", C.c_uint32), ("token_bits", C.c_uint32), ("top", C.c_uint32), ("scale", C.c_float)]


class ftc_matrix_t(C.Structure):
    _fields_ = [("tensor", ftc_param_t), ("rows", C.c_uint32), ("cols", C.c_uint32)]


class ftc_muon_t(C.Structure):
    _fields_ = [("lr", C.c_double), ("momentum", C.c_double), ("eps", C.c_double), ("steps", C.c_uint32), ("nesterov", C.c_uint32),
                ("products", C.c_uint32), ("reserved", C.c_uint32)]


class FtcError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {ftc_strerror(code)} ({code})")


_lib = None


def load():
    """Load libftc.so (built in-tree by paper_2602_22445_b200.build). Raises if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2602_22445_b200.build` "
                          "(there is no fallback implementation)")
    lib = C.CDLL(LIB_PATH)
    vp, u64, u32, sz = C.c_void_p, C.c_uint64, C.c_uint32, C.c_size_t
    dp = C.POINTER(ftc_desc_t)
    batch_args = [dp, u64, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    for name in ("ftc_reduce_batch", "ftc_allreduce_batch", "ftc_reduce_batch_host", "ftc_allreduce_batch_host"):
        getattr(lib, name).restype = C.c_int
        getattr(lib, name).argtypes = batch_args
    lib.ftc_reduce_batch_noalloc.restype = C.c_int
    lib.ftc_reduce_batch_noalloc.argtypes = [dp, u64, vp, vp, vp, vp, vp, vp, vp]
    lib.ftc_candidates_batch.restype = C.c_int
    lib.ftc_candidates_batch.argtypes = [dp, u64, C.c_int, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.ftc_candidates_workspace_bytes.restype = sz
    lib.ftc_candidates_workspace_bytes.argtypes = [dp, u64]
    lib.ftc_candidates_kernel_name.restype = C.c_char_p
    lib.ftc_candidates_kernel_name.argtypes = [dp]
    lib.ftc_message_counts_batch.restype = C.c_int
    lib.ftc_message_counts_batch.argtypes = [dp, u64, C.c_int, vp, vp, vp, vp, vp]
    lib.ftc_failed_list_batch.restype = C.c_int
    lib.ftc_failed_list_batch.argtypes = [dp, u64, C.c_int, vp, vp, vp, vp, vp, vp]
    lib.ftc_workspace_bytes.restype = sz
    lib.ftc_workspace_bytes.argtypes = [dp, u64, C.c_int]
    lib.ftc_host_staging_bytes.restype = sz
    lib.ftc_host_staging_bytes.argtypes = [dp, u64]
    lib.ftc_schedule_info.restype = C.c_int
    lib.ftc_schedule_info.argtypes = [dp, C.POINTER(ftc_sched_t)]
    lib.ftc_fill_inputs.restype = C.c_int
    lib.ftc_fill_inputs.argtypes = [u32, u64, u64, u64, u32, u32, vp, vp]
    lib.ftc_kernel_name.restype = C.c_char_p
    lib.ftc_kernel_name.argtypes = [dp, C.c_int]
    lib.ftc_kernel_variant.restype = C.c_char_p
    lib.ftc_kernel_variant.argtypes = [dp, C.c_int]
    lib.ftc_launch_blocks.restype = C.c_int
    lib.ftc_launch_blocks.argtypes = [dp, u64, C.c_int, C.POINTER(u32)]
    lib.ftc_read_bandwidth_probe.restype = C.c_int
    lib.ftc_read_bandwidth_probe.argtypes = [u32, vp, u64, vp, vp]
    np_, ap = C.POINTER(ftc_norm_t), C.POINTER(ftc_adamw_t)
    lib.ftc_layernorm_forward.restype = C.c_int
    lib.ftc_layernorm_forward.argtypes = [np_, u64, vp, u64, vp, vp, vp, u64, vp, vp, vp]
    lib.ftc_layernorm_backward.restype = C.c_int
    lib.ftc_layernorm_backward.argtypes = [np_, u64, vp, u64, vp, u64, vp, vp, vp, vp, vp, u64, vp, vp, vp, sz, vp]
    lib.ftc_layernorm_workspace_bytes.restype = sz
    lib.ftc_layernorm_workspace_bytes.argtypes = [np_, u64]
    lib.ftc_param_table_bytes.restype = sz
    lib.ftc_param_table_bytes.argtypes = [vp, u32]
    lib.ftc_param_table_build.restype = C.c_int
    lib.ftc_param_table_build.argtypes = [vp, u32, vp, sz]
    lib.ftc_param_table_blocks.restype = u64
    lib.ftc_param_table_blocks.argtypes = [vp]
    lib.ftc_grad_norm.restype = C.c_int
    lib.ftc_grad_norm.argtypes = [vp, vp, C.c_float, vp, vp, vp, sz, vp]
    lib.ftc_grad_norm_workspace_bytes.restype = sz
    lib.ftc_grad_norm_workspace_bytes.argtypes = [vp]
    lib.ftc_adamw_step.restype = C.c_int
    lib.ftc_adamw_step.argtypes = [ap, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.ftc_adamw_states.restype = C.c_int
    lib.ftc_adamw_states.argtypes = [u64, vp, vp, vp, vp, vp, vp, vp]
    ep, lp, mp = C.POINTER(ftc_embed_t), C.POINTER(ftc_logprob_t), C.POINTER(ftc_muon_t)
    lib.ftc_embedding_forward.restype = C.c_int
    lib.ftc_embedding_forward.argtypes = [ep, u64, vp, vp, u64, vp, u64, vp]
    lib.ftc_embedding_backward.restype = C.c_int
    lib.ftc_embedding_backward.argtypes = [ep, u64, vp, vp, u64, vp, vp, vp, sz, vp]
    lib.ftc_embedding_workspace_bytes.restype = sz
    lib.ftc_embedding_workspace_bytes.argtypes = [ep, u64]
    lib.ftc_token_logprobs.restype = C.c_int
    lib.ftc_token_logprobs.argtypes = [lp, u64, vp, u64, vp, vp, vp, vp, vp, vp, vp]
    lib.ftc_token_logprobs_backward.restype = C.c_int
    lib.ftc_token_logprobs_backward.argtypes = [lp, u64, vp, u64, vp, vp, vp, vp, vp, vp, u64, vp]
    lib.ftc_muon_plan_bytes.restype = sz
    lib.ftc_muon_plan_bytes.argtypes = [vp, u32]
    lib.ftc_muon_plan_build.restype = C.c_int
    lib.ftc_muon_plan_build.argtypes = [vp, u32, vp, sz]
    lib.ftc_muon_plan_blocks.restype = u64
    lib.ftc_muon_plan_blocks.argtypes = [vp]
    lib.ftc_muon_workspace_bytes.restype = sz
    lib.ftc_muon_workspace_bytes.argtypes = [vp, u32]
    lib.ftc_muon_step.restype = C.c_int
    lib.ftc_muon_step.argtypes = [mp, vp, vp, vp, vp, vp, sz, vp]
    lib.ftc_strerror.restype = C.c_char_p
    lib.ftc_strerror.argtypes = [C.c_int]
    lib.ftc_version.restype = u32
    lib.ftc_version.argtypes = []
    _lib = lib
    return lib


def _torch():
    import torch
    return torch


def dtype_code(dt) -> int:
    """FTC_* code of a torch or numpy dtype."""
    name = str(dt).replace("torch.", "")
    return {"int32": FTC_I32, "int64": FTC_I64, "uint64": FTC_U64, "float32": FTC_F32}[name]


def make_desc(P, f, k, dtype, op, root=0, max_inop=0, flags=0) -> ftc_desc_t:
    return ftc_desc_t(P, f, k, dtype if isinstance(dtype, int) else dtype_code(dtype),
                      OPS[op] if isinstance(op, str) else op, root, max_inop, flags)


def _dev_ptr(t):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("device arguments must be contiguous CUDA tensors")
    return t.data_ptr()


def _host_ptr(a):
    if a is None:
        return None
    if isinstance(a, np.ndarray):
        if not a.flags["C_CONTIGUOUS"]:
            raise ValueError("host arrays must be C-contiguous")
        return a.ctypes.data
    if a.is_cuda or not a.is_contiguous():
        raise ValueError("host arguments must be contiguous CPU tensors or numpy arrays")
    return a.data_ptr()


_raw_stream = None


def _find_raw_stream():
    """How to ask torch for the current stream's handle: its own short way (a tenth of the public call's microseconds) where this
    version has it."""
    torch = _torch()
    try:
        device, stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
    except AttributeError:
        return lambda: torch.cuda.current_stream().cuda_stream
    torch.cuda.current_stream()                       # torch's CUDA state exists from here on
    return lambda: stream(device())


def _stream(stream):
    global _raw_stream
    if stream is None:
        if _raw_stream is None:
            _raw_stream = _find_raw_stream()
        return _raw_stream()
    return stream if isinstance(stream, int) else stream.cuda_stream


def ftc_strerror(code: int) -> str:
    return load().ftc_strerror(code).decode()


def ftc_version() -> int:
    return load().ftc_version()


def ftc_kernel_name(desc, is_allreduce=False) -> str:
    return load().ftc_kernel_name(C.byref(desc), int(is_allreduce)).decode()


def ftc_kernel_variant(desc, is_allreduce=False) -> str:
    return load().ftc_kernel_variant(C.byref(desc), int(is_allreduce)).decode()


def ftc_launch_blocks(desc, S, is_allreduce=False) -> int:
    out = C.c_uint32(0)
    rc = load().ftc_launch_blocks(C.byref(desc), S, int(is_allreduce), C.byref(out))
    if rc != FTC_OK:
        raise FtcError(rc, "ftc_launch_blocks")
    return out.value


def ftc_workspace_bytes(desc, S, is_allreduce=False) -> int:
    return load().ftc_workspace_bytes(C.byref(desc), S, int(is_allreduce))


def ftc_host_staging_bytes(desc, chunk_scenarios) -> int:
    return load().ftc_host_staging_bytes(C.byref(desc), chunk_scenarios)


def ftc_schedule_info(desc) -> dict:
    out = ftc_sched_t()
    rc = load().ftc_schedule_info(C.byref(desc), C.byref(out))
    if rc != FTC_OK:
        raise FtcError(rc, "ftc_schedule_info")
    return {n: getattr(out, n) for n, _ in ftc_sched_t._fields_}


def _batch(fn_name, desc, S, d_in, d_prefail, d_inop, d_roots, d_out, d_status, d_workspace, stream, check):
    ws_bytes = 0 if d_workspace is None else d_workspace.numel() * d_workspace.element_size()
    rc = getattr(load(), fn_name)(C.byref(desc), S, _dev_ptr(d_in), _dev_ptr(d_prefail), _dev_ptr(d_inop),
                                  _dev_ptr(d_roots), _dev_ptr(d_out), _dev_ptr(d_status), _dev_ptr(d_workspace),
                                  ws_bytes, _stream(stream))
    if check and rc != FTC_OK:
        raise FtcError(rc, fn_name)
    return rc


def ftc_reduce_batch(desc, S, d_in, d_prefail, d_inop, d_roots, d_out, d_status, d_workspace=None, stream=None,
                     check=True) -> int:
    return _batch("ftc_reduce_batch", desc, S, d_in, d_prefail, d_inop, d_roots, d_out, d_status, d_workspace,
                  stream, check)


def ftc_allreduce_batch(desc, S, d_in, d_prefail, d_inop, d_roots, d_out, d_status, d_workspace=None, stream=None,
                        check=True) -> int:
    return _batch("ftc_allreduce_batch", desc, S, d_in, d_prefail, d_inop, d_roots, d_out, d_status, d_workspace,
                  stream, check)


def ftc_reduce_batch_noalloc(desc, S, d_in, d_prefail, d_inop, d_roots, d_out, d_status, stream=None,
                             check=True) -> int:
    """Reduce on the library's built-in scratch array: for callers that can neither pass a workspace nor
    allocate one. Marshals the pointers only; no tensor is created here."""
    rc = load().ftc_reduce_batch_noalloc(C.byref(desc), S, _dev_ptr(d_in), _dev_ptr(d_prefail), _dev_ptr(d_inop),
                                         _dev_ptr(d_roots), _dev_ptr(d_out), _dev_ptr(d_status), _stream(stream))
    if check and rc != FTC_OK:
        raise FtcError(rc, "ftc_reduce_batch_noalloc")
    return rc


def ftc_candidates_kernel_name(desc) -> str:
    return load().ftc_candidates_kernel_name(C.byref(desc)).decode()


def ftc_candidates_workspace_bytes(desc, S) -> int:
    return load().ftc_candidates_workspace_bytes(C.byref(desc), S)


def ftc_candidates_batch(desc, S, is_allreduce, d_in, d_prefail, d_inop, d_roots, d_cand, d_cand_info, d_workspace,
                         stream=None, check=True) -> int:
    ws_bytes = 0 if d_workspace is None else d_workspace.numel() * d_workspace.element_size()
    rc = load().ftc_candidates_batch(C.byref(desc), S, int(is_allreduce), _dev_ptr(d_in), _dev_ptr(d_prefail),
                                     _dev_ptr(d_inop), _dev_ptr(d_roots), _dev_ptr(d_cand), _dev_ptr(d_cand_info),
                                     _dev_ptr(d_workspace), ws_bytes, _stream(stream))
    if check and rc != FTC_OK:
        raise FtcError(rc, "ftc_candidates_batch")
    return rc


def ftc_message_counts_batch(desc, S, is_allreduce, d_prefail, d_inop, d_roots, d_msgs, stream=None, check=True) -> int:
    rc = load().ftc_message_counts_batch(C.byref(desc), S, int(is_allreduce), _dev_ptr(d_prefail), _dev_ptr(d_inop),
                                         _dev_ptr(d_roots), _dev_ptr(d_msgs), _stream(stream))
    if check and rc != FTC_OK:
        raise FtcError(rc, "ftc_message_counts_batch")
    return rc


def ftc_failed_list_batch(desc, S, is_allreduce, d_prefail, d_inop, d_roots, d_failed, d_nfail, stream=None, check=True) -> int:
    rc = load().ftc_failed_list_batch(C.byref(desc), S, int(is_allreduce), _dev_ptr(d_prefail), _dev_ptr(d_inop),
                                      _dev_ptr(d_roots), _dev_ptr(d_failed), _dev_ptr(d_nfail), _stream(stream))
    if check and rc != FTC_OK:
        raise FtcError(rc, "ftc_failed_list_batch")
    return rc


def _batch_host(fn_name, desc, S, h_in, h_prefail, h_inop, h_roots, h_out, h_status, d_staging, stream, check):
    st_bytes = d_staging.numel() * d_staging.element_size()
    rc = getattr(load(), fn_name)(C.byref(desc), S, _host_ptr(h_in), _host_ptr(h_prefail), _host_ptr(h_inop),
                                  _host_ptr(h_roots), _host_ptr(h_out), _host_ptr(h_status), _dev_ptr(d_staging),
                                  st_bytes, _stream(stream))
    if check and rc != FTC_OK:
        raise FtcError(rc, fn_name)
    return rc


def ftc_reduce_batch_host(desc, S, h_in, h_prefail, h_inop, h_roots, h_out, h_status, d_staging, stream=None,
                          check=True) -> int:
    return _batch_host("ftc_reduce_batch_host", desc, S, h_in, h_prefail, h_inop, h_roots, h_out, h_status,
                       d_staging, stream, check)


def ftc_allreduce_batch_host(desc, S, h_in, h_prefail, h_inop, h_roots, h_out, h_status, d_staging, stream=None,
                             check=True) -> int:
    return _batch_host("ftc_allreduce_batch_host", desc, S, h_in, h_prefail, h_inop, h_roots, h_out, h_status,
                       d_staging, stream, check)


def ftc_read_bandwidth_probe(mode, d_buf, nbytes, d_sink, stream=None) -> int:
    rc = load().ftc_read_bandwidth_probe(mode, _dev_ptr(d_buf), nbytes, _dev_ptr(d_sink), _stream(stream))
    if rc != FTC_OK:
        raise FtcError(rc, "ftc_read_bandwidth_probe")
    return rc


def ftc_fill_inputs(kind, seed, first_scenario, S, P, k, d_out, stream=None) -> int:
    rc = load().ftc_fill_inputs(kind, seed & 0xFFFFFFFFFFFFFFFF, first_scenario, S, P, k, _dev_ptr(d_out),
                                _stream(stream))
    if rc != FTC_OK:
        raise FtcError(rc, "ftc_fill_inputs")
    return rc


# ---- training operators: layer norm, many-tensor gradient norm and AdamW ----

_FLOAT_CODES = {"float32": FTC_F32, "bfloat16": FTC_BF16, "float16": FTC_F16}


def _float_code(dt) -> int:
    """FTC_* code of the floating types the training operators take (torch's types are added to the names as they are met)."""
    code = _FLOAT_CODES.get(dt)
    if code is None:
        code = _FLOAT_CODES.get(str(dt).replace("torch.", ""))
        if code is None:
            raise ValueError(f"float32, bfloat16 or float16 wanted, got {dt}")
        _FLOAT_CODES[dt] = code
    return code


def make_norm_desc(H, dtype, wdtype=None, P=1, k=None, eps=1e-5) -> ftc_norm_t:
    """Rows of H elements of `dtype`, weights of `wdtype` (default: `dtype`); P and k: processes and message length of the weight
    gradients (default: one process, one message of H elements)."""
    dtype = dtype if isinstance(dtype, int) else _float_code(dtype)
    wdtype = dtype if wdtype is None else wdtype if isinstance(wdtype, int) else _float_code(wdtype)
    return ftc_norm_t(H, P, H if k is None else k, dtype, wdtype, eps)


def _rows_ptr(desc, t, what, rows):
    """Address and row stride of a [rows][H] tensor of the descriptor's type whose rows are contiguous."""
    if t is None:
        return None, 0
    H = desc.H
    if t.shape != (rows, H) or not t.is_cuda:
        raise ValueError(f"{what}: a CUDA tensor [{rows}][{H}] is wanted")
    if _FLOAT_CODES.get(t.dtype) != desc.dtype and _float_code(t.dtype) != desc.dtype:
        raise ValueError(f"{what}: its type is not the descriptor's")
    stride, inner = t.stride()
    if inner != 1 and H > 1:
        raise ValueError(f"{what}: contiguous rows are wanted")
    return t.data_ptr(), stride if rows > 1 or stride >= H else H


def _vector_ptr(t, what, n, code=FTC_F32):
    """Address of n contiguous elements of a floating type."""
    if t is None:
        return None
    if t.numel() != n or not t.is_cuda or not t.is_contiguous() or (_FLOAT_CODES.get(t.dtype) != code and _float_code(t.dtype) != code):
        raise ValueError(f"{what}: {n} contiguous CUDA elements of the right type are wanted")
    return t.data_ptr()


def ftc_layernorm_forward(desc, d_x, d_gamma, d_beta, d_y, d_mean, d_rstd, stream=None, check=True) -> int:
    rows = d_x.shape[0]
    x, xs = _rows_ptr(desc, d_x, "d_x", rows)
    y, ys = _rows_ptr(desc, d_y, "d_y", rows)
    H, code = desc.H, desc.wdtype
    rc = (_lib or load()).ftc_layernorm_forward(desc, rows, x, xs, _vector_ptr(d_gamma, "d_gamma", H, code),
                                                _vector_ptr(d_beta, "d_beta", H, code), y, ys, _vector_ptr(d_mean, "d_mean", rows),
                                                _vector_ptr(d_rstd, "d_rstd", rows), _stream(stream))
    if rc and check:
        raise FtcError(rc, "ftc_layernorm_forward")
    return rc


def ftc_layernorm_workspace_bytes(desc, rows) -> int:
    return load().ftc_layernorm_workspace_bytes(C.byref(desc), rows)


def ftc_layernorm_backward(desc, d_dy, d_x, d_gamma, d_mean, d_rstd, d_row_splits, d_dx, d_dgamma, d_dbeta, d_workspace,
                           stream=None, check=True) -> int:
    rows = d_x.shape[0]
    dy, dys = _rows_ptr(desc, d_dy, "d_dy", rows)
    x, xs = _rows_ptr(desc, d_x, "d_x", rows)
    dx, dxs = _rows_ptr(desc, d_dx, "d_dx", rows)
    n = -(-desc.H // desc.k) * desc.P * desc.k
    if d_row_splits is not None and (d_row_splits.numel() != desc.P + 1 or _whole_bytes(d_row_splits) != 8):
        raise ValueError("d_row_splits: P + 1 whole numbers of 64 bits are wanted")
    ws_bytes = 0 if d_workspace is None else d_workspace.numel() * d_workspace.element_size()
    rc = (_lib or load()).ftc_layernorm_backward(desc, rows, dy, dys, x, xs, _vector_ptr(d_gamma, "d_gamma", desc.H, desc.wdtype),
                                       _vector_ptr(d_mean, "d_mean", rows), _vector_ptr(d_rstd, "d_rstd", rows),
                                       _dev_ptr(d_row_splits), dx, dxs, _vector_ptr(d_dgamma, "d_dgamma", n),
                                       _vector_ptr(d_dbeta, "d_dbeta", n), _dev_ptr(d_workspace), ws_bytes, _stream(stream))
    if check and rc != FTC_OK:
        raise FtcError(rc, "ftc_layernorm_backward")
    return rc


def make_param(param, grad, master=None, status=None, k=0, lr_scale=1.0, weight_decay=0.0):
    """One tensor of a table: the arguments of ftc_param_t, as tensors. A table keeps them alive."""
    n = grad.numel()
    for t, what in ((param, "param"), (master, "master")):
        if t is not None and t.numel() != n:
            raise ValueError(f"{what}: {n} elements are wanted, as in grad")
    if master is not None and _float_code(master.dtype) != FTC_F32:
        raise ValueError("master: float32 is wanted")
    if status is not None and (k < 1 or status.numel() != -(-n // k) * FTC_STATUS_WORDS or status.element_size() != 4):
        raise ValueError("status: one record of 4 words of 32 bits for each message of k elements is wanted")
    entry = ftc_param_t(_dev_ptr(param), _dev_ptr(master), _dev_ptr(grad), _dev_ptr(status), n, k if status is not None else 0,
                        FTC_F32 if param is None else _float_code(param.dtype), _float_code(grad.dtype), lr_scale, weight_decay, 0)
    return entry, (param, grad, master, status)


class ParamTable:
    """A table of tensors (ftc_param_table_build) on the host and on the device, with the tensors that it points to."""

    def __init__(self, params, device="cuda"):
        torch = _torch()
        entries = (ftc_param_t * max(1, len(params)))(*[p[0] for p in params])
        size = load().ftc_param_table_bytes(entries, len(params))
        self.host = np.zeros(max(size, 8) // 8, dtype=np.uint64)
        rc = load().ftc_param_table_build(entries, len(params), self.host.ctypes.data, size)
        if rc != FTC_OK:
            raise FtcError(rc, "ftc_param_table_build")
        self.keeps = [p[1] for p in params]
        self.n_params = len(params)
        self.h_ptr = self.host.ctypes.data
        self.blocks = load().ftc_param_table_blocks(self.h_ptr)
        self.device = torch.from_numpy(self.host.view(np.int64)).to(device)
        self.d_ptr = self.device.data_ptr()


def make_param_table(params, device="cuda") -> ParamTable:
    """The table of a list of make_param()s. Tensors that move need a new one."""
    return ParamTable(params, device)


def ftc_grad_norm_workspace_bytes(table) -> int:
    return load().ftc_grad_norm_workspace_bytes(table.h_ptr)


def ftc_grad_norm(table, max_norm, d_norm, d_norms, d_workspace, stream=None, check=True) -> int:
    ws_bytes = 0 if d_workspace is None else d_workspace.numel() * d_workspace.element_size()
    rc = (_lib or load()).ftc_grad_norm(table.h_ptr, table.d_ptr, max_norm, _vector_ptr(d_norm, "d_norm", 2),
                              _vector_ptr(d_norms, "d_norms", table.n_params), _dev_ptr(d_workspace), ws_bytes, _stream(stream))
    if check and rc != FTC_OK:
        raise FtcError(rc, "ftc_grad_norm")
    return rc


def make_adamw(lr, beta1=0.9, beta2=0.999, eps=1e-8, step=1) -> ftc_adamw_t:
    return ftc_adamw_t(lr, beta1, beta2, eps, step, 32, 0)


def _states(table, d_m, d_v, d_m_scale, d_v_scale):
    """The states' bits and addresses, sizes checked."""
    n = table.blocks * FTC_STATE_BLOCK
    bits = 8 * d_m.element_size()
    if bits != 8 * d_v.element_size() or d_m.numel() != n or d_v.numel() != n or (bits != 8 and d_m.dtype != d_v.dtype):
        raise ValueError(f"states: {n} elements each, float32 or 8-bit, are wanted")
    if bits == 8 and (d_m_scale is None or d_v_scale is None):
        raise ValueError("states in 8 bits: scales are wanted")
    if bits != 8 and _float_code(d_m.dtype) != FTC_F32:
        raise ValueError("states: float32 or 8-bit elements are wanted")
    scales = [_vector_ptr(t, "scales", table.blocks) if bits == 8 else None for t in (d_m_scale, d_v_scale)]
    return bits, [_dev_ptr(d_m), _dev_ptr(d_v), *scales]


def ftc_adamw_step(hyper, table, d_m, d_v, d_m_scale=None, d_v_scale=None, d_grad_scale=None, stream=None, check=True) -> int:
    bits, states = _states(table, d_m, d_v, d_m_scale, d_v_scale)
    if hyper.state_bits != bits:                      # never the caller's own: another thread may use it over states of other bits
        hyper = ftc_adamw_t.from_buffer_copy(hyper)
        hyper.state_bits = bits
    rc = (_lib or load()).ftc_adamw_step(hyper, table.h_ptr, table.d_ptr, *states, _vector_ptr(d_grad_scale, "d_grad_scale", 1),
                               _stream(stream))
    if check and rc != FTC_OK:
        raise FtcError(rc, "ftc_adamw_step")
    return rc


def ftc_adamw_states(table, d_m, d_v, d_m_scale, d_v_scale, d_m_out, d_v_out, stream=None, check=True) -> int:
    bits, states = _states(table, d_m, d_v, d_m_scale, d_v_scale)
    if bits != 8:
        raise ValueError("states in 8 bits are wanted")
    n = table.blocks * FTC_STATE_BLOCK
    rc = load().ftc_adamw_states(table.blocks, *states, _vector_ptr(d_m_out, "d_m_out", n), _vector_ptr(d_v_out, "d_v_out", n),
                                 _stream(stream))
    if check and rc != FTC_OK:
        raise FtcError(rc, "ftc_adamw_states")
    return rc


# ---- the two ends of a language model: embedding, token log probabilities; the orthogonalised update of its matrices ----

def make_embed_desc(V, H, dtype, wdtype=None, P=1, k=None, scale=1.0) -> ftc_embed_t:
    """A table of V rows of H elements of `wdtype` (default: `dtype`), y and dy of `dtype`; P and k: processes and message length of the
    gradient (default: one process, [V][H]). The tokens' width is taken from the tensor that a call gets."""
    dtype = dtype if isinstance(dtype, int) else _float_code(dtype)
    wdtype = dtype if wdtype is None else wdtype if isinstance(wdtype, int) else _float_code(wdtype)
    return ftc_embed_t(V, H, P, H if k is None else k, dtype, wdtype, 64, scale)


def make_logprob_desc(V, dtype, top=0, scale=1.0) -> ftc_logprob_t:
    """Rows of V logits of `dtype`, multiplied by `scale`; `top`: how many alternatives are listed (0 .. 32)."""
    return ftc_logprob_t(V, dtype if isinstance(dtype, int) else _float_code(dtype), 64, top, scale)


def _matrix_ptr(t, what, rows, cols, code):
    """Address and row stride of a [rows][cols] tensor of a floating type whose rows are contiguous."""
    if t.shape != (rows, cols) or not t.is_cuda or (_FLOAT_CODES.get(t.dtype) != code and _float_code(t.dtype) != code):
        raise ValueError(f"{what}: a CUDA tensor [{rows}][{cols}] of the descriptor's type is wanted")
    stride, inner = t.stride()
    if inner != 1 and cols > 1:
        raise ValueError(f"{what}: contiguous rows are wanted")
    return t.data_ptr(), stride if rows > 1 or stride >= cols else cols


_WHOLE = {}


def _whole_bytes(t) -> int:
    """The size of its elements if they are whole numbers of 32 or 64 bits, else 0 (complex and quantised ones are no floating point numbers
    either). Types are looked up as they were met."""
    size = _WHOLE.get(t.dtype)
    if size is None:
        size = _WHOLE[t.dtype] = {"int32": 4, "uint32": 4, "int64": 8, "uint64": 8}.get(str(t.dtype).rsplit(".", 1)[-1], 0)
    return size


def _tokens_ptr(desc, t, what="d_tokens"):
    """The descriptor for these tokens' width (the caller's own is left as it is: another thread may use it over others), their number and
    address."""
    size = _whole_bytes(t)
    if not size or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous CUDA whole numbers of 32 or 64 bits are wanted")
    if desc.token_bits != 8 * size:
        desc = type(desc).from_buffer_copy(desc)
        desc.token_bits = 8 * size
    return desc, t.numel(), t.data_ptr()


def ftc_embedding_forward(desc, d_tokens, d_table, d_y, stream=None, check=True) -> int:
    desc, n, tokens = _tokens_ptr(desc, d_tokens)
    table, ts = _matrix_ptr(d_table, "d_table", desc.V, desc.H, desc.wdtype)
    y, ys = _matrix_ptr(d_y, "d_y", n, desc.H, desc.dtype)
    rc = (_lib or load()).ftc_embedding_forward(desc, n, tokens, table, ts, y, ys, _stream(stream))
    if rc and check:
        raise FtcError(rc, "ftc_embedding_forward")
    return rc


def ftc_embedding_workspace_bytes(desc, n) -> int:
    return load().ftc_embedding_workspace_bytes(C.byref(desc), n)


def ftc_embedding_backward(desc, d_tokens, d_dy, d_row_splits, d_dtable, d_workspace, stream=None, check=True) -> int:
    desc, n, tokens = _tokens_ptr(desc, d_tokens)
    dy, dys = _matrix_ptr(d_dy, "d_dy", n, desc.H, desc.dtype)
    if d_row_splits is not None and (d_row_splits.numel() != desc.P + 1 or _whole_bytes(d_row_splits) != 8):
        raise ValueError("d_row_splits: P + 1 whole numbers of 64 bits are wanted")
    out = -(-desc.V * desc.H // desc.k) * desc.P * desc.k
    ws_bytes = 0 if d_workspace is None else d_workspace.numel() * d_workspace.element_size()
    rc = (_lib or load()).ftc_embedding_backward(desc, n, tokens, dy, dys, _dev_ptr(d_row_splits), _vector_ptr(d_dtable, "d_dtable", out),
                                                 _dev_ptr(d_workspace), ws_bytes, _stream(stream))
    if rc and check:
        raise FtcError(rc, "ftc_embedding_backward")
    return rc


def _given_tokens(desc, d_tokens, rows):
    if d_tokens is None:
        return desc, None
    desc, n, tokens = _tokens_ptr(desc, d_tokens)
    if n != rows:
        raise ValueError(f"d_tokens: {rows} tokens are wanted, one for each row")
    return desc, tokens


def ftc_token_logprobs(desc, d_logits, d_tokens, d_logprob, d_entropy=None, d_lse=None, d_top_logprob=None, d_top_token=None, stream=None,
                       check=True) -> int:
    rows = d_logits.shape[0]
    desc, tokens = _given_tokens(desc, d_tokens, rows)
    x, xs = _matrix_ptr(d_logits, "d_logits", rows, desc.V, desc.dtype)
    if d_top_token is not None and (d_top_token.numel() != rows * desc.top or _whole_bytes(d_top_token) != 4):
        raise ValueError("d_top_token: `top` whole numbers of 32 bits for each row are wanted")
    rc = (_lib or load()).ftc_token_logprobs(desc, rows, x, xs, tokens, _vector_ptr(d_logprob, "d_logprob", rows), _vector_ptr(d_entropy, "d_entropy", rows),
                                             _vector_ptr(d_lse, "d_lse", rows), _vector_ptr(d_top_logprob, "d_top_logprob", rows * desc.top),
                                             _dev_ptr(d_top_token), _stream(stream))
    if rc and check:
        raise FtcError(rc, "ftc_token_logprobs")
    return rc


def ftc_token_logprobs_backward(desc, d_logits, d_tokens, d_lse, d_entropy, d_dlogprob, d_dentropy, d_dlogits, stream=None, check=True) -> int:
    rows = d_logits.shape[0]
    desc, tokens = _given_tokens(desc, d_tokens, rows)
    x, xs = _matrix_ptr(d_logits, "d_logits", rows, desc.V, desc.dtype)
    d, ds = _matrix_ptr(d_dlogits, "d_dlogits", rows, desc.V, desc.dtype)
    rc = (_lib or load()).ftc_token_logprobs_backward(desc, rows, x, xs, tokens, _vector_ptr(d_lse, "d_lse", rows), _vector_ptr(d_entropy, "d_entropy", rows),
                                                      _vector_ptr(d_dlogprob, "d_dlogprob", rows), _vector_ptr(d_dentropy, "d_dentropy", rows), d, ds,
                                                      _stream(stream))
    if rc and check:
        raise FtcError(rc, "ftc_token_logprobs_backward")
    return rc


def make_matrix(param, grad, master=None, status=None, k=0, lr_scale=1.0, weight_decay=0.0):
    """One matrix of a plan: the arguments of make_param(), `param` with two dimensions. A plan keeps them alive."""
    if param.dim() != 2:
        raise ValueError("param: a matrix is wanted")
    entry, keeps = make_param(param, grad, master, status, k, lr_scale, weight_decay)
    return ftc_matrix_t(entry, param.shape[0], param.shape[1]), keeps


class MuonPlan:
    """A plan of matrices (ftc_muon_plan_build) on the host and on the device, with the tensors that it points to."""

    def __init__(self, matrices, device="cuda"):
        torch = _torch()
        entries = (ftc_matrix_t * max(1, len(matrices)))(*[m[0] for m in matrices])
        size = load().ftc_muon_plan_bytes(entries, len(matrices))
        self.host = np.zeros(max(size, 8) // 8, dtype=np.uint64)
        rc = load().ftc_muon_plan_build(entries, len(matrices), self.host.ctypes.data, size)
        if rc != FTC_OK:
            raise FtcError(rc, "ftc_muon_plan_build")
        self.keeps = [m[1] for m in matrices]
        self.h_ptr = self.host.ctypes.data
        self.blocks = load().ftc_muon_plan_blocks(self.h_ptr)
        self.device = torch.from_numpy(self.host.view(np.int64)).to(device)
        self.d_ptr = self.device.data_ptr()


def make_muon_plan(matrices, device="cuda") -> MuonPlan:
    """The plan of a list of make_matrix()s. Tensors that move need a new one."""
    return MuonPlan(matrices, device)


def make_muon(lr, momentum=0.95, eps=1e-7, steps=5, nesterov=True, products=32) -> ftc_muon_t:
    """`products`: 32, or 16 for updates that may be off by a thousandth (weights in 16 bits), at half the time."""
    return ftc_muon_t(lr, momentum, eps, steps, int(nesterov), products, 0)


def ftc_muon_workspace_bytes(plan, products=32) -> int:
    return load().ftc_muon_workspace_bytes(plan.h_ptr, products)


def ftc_muon_step(hyper, plan, d_momentum, d_grad_scale, d_workspace, stream=None, check=True) -> int:
    ws_bytes = 0 if d_workspace is None else d_workspace.numel() * d_workspace.element_size()
    rc = (_lib or load()).ftc_muon_step(hyper, plan.h_ptr, plan.d_ptr, _vector_ptr(d_momentum, "d_momentum", plan.blocks * FTC_STATE_BLOCK),
                                        _vector_ptr(d_grad_scale, "d_grad_scale", 1), _dev_ptr(d_workspace), ws_bytes, _stream(stream))
    if rc and check:
        raise FtcError(rc, "ftc_muon_step")
    return rc


def check_muon(d_workspace) -> None:
    """Waits for the current stream and raises FtcError where a wait inside the last ftc_muon_step() with this workspace gave up: its weights have not
    moved then, its momentum has. A step itself does not wait for the device and cannot say so."""
    word = d_workspace.view(-1)[:max(1, 4 // d_workspace.element_size())].view(_torch().int32)
    if int(word[0]):
        raise FtcError(FTC_ECUDA, "ftc_muon_step gave up on a wait")
