"""Python binding of the paged decode-attention C ABI (the headers under include/).

Argument marshalling only: every step of the computation runs in the HIP
kernels of libpda.so.  The library must have been built in-tree
(``paper_2405_11143_amd/build.py``); if it is missing, loading fails with an
error -- there is no fallback implementation.  PyTorch supplies device
memory and streams.
"""
from __future__ import annotations

import ctypes
import os
from typing import Tuple

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libpda.so")

PDA_OK, PDA_ERR_NULL, PDA_ERR_SHAPE, PDA_ERR_UNSUPPORTED = 0, 1, 2, 3
PDA_ERR_WORKSPACE, PDA_ERR_ALIGNMENT, PDA_ERR_VALUE, PDA_ERR_HIP, PDA_ERR_SCRATCH = 4, 5, 6, 7, 8
PDA_NOALLOC_SCRATCH_BYTES = 64 << 20  # the static scratch of pda_decode_noalloc

# Every function the headers under include/ declare.
EXPORTED = ("pda_plan", "pda_workspace_bytes", "pda_decode", "pda_partition_attention",
            "pda_merge_partitions", "pda_plan_shared_prefix", "pda_decode_shared_prefix", "pda_append_kv",
            "pda_step_graph_create", "pda_step_graph_launch", "pda_step_graph_destroy", "pda_token_logprobs",
            "pda_logprob_workspace_bytes",
            "pda_validate_host", "pda_work_order", "pda_decode_reusing_order",
            "pda_partition_attention_reusing_order", "pda_decode_noalloc",
            "pda_gather_ceiling", "pda_stream_ceiling", "pda_model_step_graph_create", "pda_decode_append",
            "pda_rotary_inv_freq", "pda_rotary_apply", "pda_append_kv_fp8", "pda_plan_fp8", "pda_decode_fp8",
            "pda_read_kv_fp8",
            "pda_norm_rotary", "pda_norm_rotary_workspace_bytes", "pda_norm_rotary_backward", "pda_norm_rotary_append",
            "pda_plan_window", "pda_decode_window", "pda_blocks_workspace_bytes", "pda_blocks_resize", "pda_slot_map",
            "pda_status_string")
PDA_DTYPE_BF16, PDA_DTYPE_F32 = 0, 1
PDA_ROTARY_PLAIN, PDA_ROTARY_LINEAR, PDA_ROTARY_BASE, PDA_ROTARY_BANDS, PDA_ROTARY_RAMP = 0, 1, 2, 3, 4


class pda_problem(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in (
        "num_seqs", "num_q_heads", "num_kv_heads", "head_dim", "block_size", "num_blocks",
        "max_blocks_per_seq", "max_context_len", "partition_tokens", "num_query_tokens")]


class pda_plan_info(ctypes.Structure):
    _fields_ = [("partition_tokens", ctypes.c_int32), ("num_partitions", ctypes.c_int32),
                ("workspace_bytes", ctypes.c_size_t)]

    def as_dict(self):
        return {name: getattr(self, name) for name, _ in self._fields_}


class pda_prefix_groups(ctypes.Structure):
    _fields_ = [("num_groups", ctypes.c_int32), ("max_group_size", ctypes.c_int32),
                ("max_prefix_len", ctypes.c_int32), ("group_start", ctypes.c_void_p),
                ("group_prefix_len", ctypes.c_void_p)]


class pda_layer_buffers(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k_new", ctypes.c_void_p), ("v_new", ctypes.c_void_p),
                ("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p), ("out", ctypes.c_void_p)]


class pda_rotary(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("backward", ctypes.c_int32),
                ("magnitude", ctypes.c_float), ("inv_freq", ctypes.c_void_p)]


class pda_rotary_scaling(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("factor", ctypes.c_double), ("original_len", ctypes.c_double),
                ("low", ctypes.c_double), ("high", ctypes.c_double)]


class pda_head_norm(ctypes.Structure):
    _fields_ = [("eps", ctypes.c_float), ("weight_offset", ctypes.c_float), ("weight_dtype", ctypes.c_int32),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p)]


class pda_rotary_axes(ctypes.Structure):
    _fields_ = [("num_axes", ctypes.c_int32), ("axis_of_pair", ctypes.c_void_p), ("position_stride", ctypes.c_int64)]


class pda_window(ctypes.Structure):
    _fields_ = [("window", ctypes.c_int32), ("num_sinks", ctypes.c_int32)]


class pda_block_pool(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32), ("num_blocks", ctypes.c_int32), ("max_blocks_per_seq", ctypes.c_int32),
                ("block_table", ctypes.c_void_p), ("held", ctypes.c_void_p), ("free_blocks", ctypes.c_void_p),
                ("counts", ctypes.c_void_p)]


class pda_token_rows(ctypes.Structure):
    _fields_ = [("num_rows", ctypes.c_int32), ("row_start", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("slots", ctypes.c_void_p)]


class PdaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {pda_status_string(status)} (status {status})")


_lib = None


def load_library(path: str = LIB_PATH):
    """Load libpda.so (raises if it has not been built)."""
    global _lib
    if _lib is not None and path == LIB_PATH:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with paper_2405_11143_amd/build.py "
                           "(there is no fallback implementation)")
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER(pda_problem)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    lib.pda_plan.argtypes = [P, ctypes.POINTER(pda_plan_info)]
    lib.pda_workspace_bytes.argtypes = [P, ctypes.POINTER(sz)]
    step = [P, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, sz, vp]
    lib.pda_decode.argtypes = step
    lib.pda_partition_attention.argtypes = step
    lib.pda_decode_reusing_order.argtypes = step
    lib.pda_partition_attention_reusing_order.argtypes = step
    lib.pda_decode_noalloc.argtypes = [P, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp]
    lib.pda_gather_ceiling.argtypes = [i32, i32, i32, vp, vp, vp, i32, i32, vp, vp]
    lib.pda_stream_ceiling.argtypes = [vp, sz, i32, vp, vp]
    lib.pda_work_order.argtypes = [P, vp, vp, sz, vp]
    lib.pda_merge_partitions.argtypes = [P, vp, vp, vp, sz, vp]
    G = ctypes.POINTER(pda_prefix_groups)
    lib.pda_plan_shared_prefix.argtypes = [P, G, ctypes.POINTER(pda_plan_info)]
    lib.pda_decode_shared_prefix.argtypes = [P, G, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, sz, vp]
    lib.pda_append_kv.argtypes = [P, vp, vp, vp, vp, vp, vp, vp]
    lib.pda_decode_append.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, sz, vp]
    lib.pda_step_graph_create.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, sz,
                                          ctypes.POINTER(vp)]
    lib.pda_step_graph_launch.argtypes = [vp, vp]
    lib.pda_model_step_graph_create.argtypes = [P, ctypes.c_int32, ctypes.POINTER(pda_layer_buffers), vp, vp,
                                                ctypes.c_float, vp, sz, ctypes.POINTER(vp)]
    lib.pda_step_graph_destroy.argtypes = [vp]
    lib.pda_token_logprobs.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int64, ctypes.c_int32, vp, vp,
                                       ctypes.c_float, vp, vp, vp, sz, vp]
    lib.pda_logprob_workspace_bytes.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(sz)]
    lib.pda_validate_host.argtypes = [P, vp, vp, ctypes.POINTER(ctypes.c_int64)]
    c32, c64, dbl = ctypes.c_int32, ctypes.c_int64, ctypes.c_double
    R = ctypes.POINTER(pda_rotary)
    lib.pda_rotary_inv_freq.argtypes = [c32, dbl, ctypes.POINTER(pda_rotary_scaling), vp, ctypes.POINTER(ctypes.c_float)]
    lib.pda_rotary_apply.argtypes = [R, c32, c32, c32, c32, c32, vp] + [vp, c64] * 4 + [vp]
    lib.pda_append_kv_fp8.argtypes = [P, R] + [vp] * 9 + [vp]
    lib.pda_plan_fp8.argtypes = [P, ctypes.POINTER(pda_plan_info)]
    lib.pda_decode_fp8.argtypes = [P, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, sz, vp]
    lib.pda_read_kv_fp8.argtypes = [P] + [vp] * 7 + [c32, vp, vp, vp]
    N, A = ctypes.POINTER(pda_head_norm), ctypes.POINTER(pda_rotary_axes)
    lib.pda_norm_rotary.argtypes = [N, R, A, c32, c32, c32, c32, c32, vp] + [vp, c64] * 4 + [vp]
    lib.pda_norm_rotary_workspace_bytes.argtypes = [c32, c32, c32, c32, ctypes.POINTER(sz)]
    lib.pda_norm_rotary_backward.argtypes = [N, R, A, c32, c32, c32, c32, c32, vp] + [vp, c64] * 6 + [vp, vp, vp, sz, vp]
    lib.pda_norm_rotary_append.argtypes = [N, R, A, c32, c32, c32, c32, c32, vp, vp] + [vp, c64] * 4 + [vp, vp, vp]
    W = ctypes.POINTER(pda_window)
    lib.pda_plan_window.argtypes = [P, W, ctypes.POINTER(pda_plan_info)]
    lib.pda_decode_window.argtypes = [P, W, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, sz, vp]
    BP, TR = ctypes.POINTER(pda_block_pool), ctypes.POINTER(pda_token_rows)
    lib.pda_blocks_workspace_bytes.argtypes = [BP, ctypes.POINTER(sz)]
    lib.pda_blocks_resize.argtypes = [BP, vp, TR, vp, sz, vp]
    lib.pda_slot_map.argtypes = [c32, c32, c32, vp, vp, TR, vp]
    lib.pda_status_string.argtypes = [i32]
    lib.pda_status_string.restype = ctypes.c_char_p
    for name in EXPORTED[:-1]:
        getattr(lib, name).restype = i32
    if path == LIB_PATH:
        _lib = lib
    return lib


def pda_status_string(status: int) -> str:
    return load_library().pda_status_string(int(status)).decode()


def make_problem(num_seqs, num_q_heads, num_kv_heads, head_dim, num_blocks, max_blocks_per_seq,
                 max_context_len, partition_tokens=0, block_size=16, num_query_tokens=1) -> pda_problem:
    return pda_problem(int(num_seqs), int(num_q_heads), int(num_kv_heads), int(head_dim), int(block_size),
                       int(num_blocks), int(max_blocks_per_seq), int(max_context_len), int(partition_tokens),
                       int(num_query_tokens))


def pda_plan(prob: pda_problem) -> dict:
    """The plan of a problem: partition_tokens, num_partitions, workspace_bytes."""
    info = pda_plan_info()
    rc = load_library().pda_plan(ctypes.byref(prob), ctypes.byref(info))
    if rc != PDA_OK:
        raise PdaError(rc, "pda_plan")
    return info.as_dict()


def make_prefix_groups(num_groups, max_group_size, max_prefix_len, group_start=None,
                       group_prefix_len=None) -> pda_prefix_groups:
    """Host bounds plus the two device arrays (torch int32 tensors or raw pointers)."""
    ptr = lambda t: (t.data_ptr() if hasattr(t, "data_ptr") else t)
    return pda_prefix_groups(int(num_groups), int(max_group_size), int(max_prefix_len), ptr(group_start),
                             ptr(group_prefix_len))


def pda_plan_shared_prefix(prob: pda_problem, groups: pda_prefix_groups) -> dict:
    info = pda_plan_info()
    rc = load_library().pda_plan_shared_prefix(ctypes.byref(prob), ctypes.byref(groups), ctypes.byref(info))
    if rc != PDA_OK:
        raise PdaError(rc, "pda_plan_shared_prefix")
    return info.as_dict()


def pda_workspace_bytes(prob: pda_problem) -> int:
    ws = ctypes.c_size_t()
    rc = load_library().pda_workspace_bytes(ctypes.byref(prob), ctypes.byref(ws))
    if rc != PDA_OK:
        raise PdaError(rc, "pda_workspace_bytes")
    return ws.value


def pda_validate_host(prob: pda_problem, block_table, context_lens) -> Tuple[int, int]:
    """Check host copies of the device contents; returns (status, first_bad_index)."""
    bt = np.ascontiguousarray(block_table, dtype=np.int32)
    lens = np.ascontiguousarray(context_lens, dtype=np.int32)
    bad = ctypes.c_int64(-1)
    rc = load_library().pda_validate_host(ctypes.byref(prob), bt.ctypes.data, lens.ctypes.data,
                                          ctypes.byref(bad))
    return rc, bad.value


def _query_shape(q):
    """(B, n, Hq, D) of q [B][Hq][D] (n = 1) or [B][n][Hq][D]."""
    if q.dim() == 3:
        return q.shape[0], 1, q.shape[1], q.shape[2]
    if q.dim() == 4:
        return tuple(q.shape)
    raise ValueError("q must be [B][Hq][D] or [B][n][Hq][D]")


def _problem_from(q, k_cache, block_table, max_context_len, partition_tokens) -> pda_problem:
    if k_cache.dim() != 5 or block_table.dim() != 2:
        raise ValueError("k_cache [num_blocks][Hkv][D/8][16][8], block_table [B][max_blocks]")
    B, n, Hq, D = _query_shape(q)
    NB, Hkv, C, BS, E = k_cache.shape
    if C * E != D or E != 8 or block_table.shape[0] != B:
        raise ValueError("q, k_cache and block_table shapes disagree")
    if max_context_len is None:
        raise ValueError("max_context_len must be given (the host bound on context_lens)")
    return make_problem(B, Hq, Hkv, D, NB, block_table.shape[1], max_context_len, partition_tokens, BS, n)


def _require(name, t, dtype):
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _check_tensors(q, k_cache, v_cache, block_table, context_lens, out):
    import torch

    for name, t, dt in (("q", q, torch.bfloat16), ("k_cache", k_cache, torch.bfloat16),
                        ("v_cache", v_cache, torch.bfloat16), ("block_table", block_table, torch.int32),
                        ("context_lens", context_lens, torch.int32), ("out", out, torch.float32)):
        _require(name, t, dt)
    NB, Hkv, C, BS, E = k_cache.shape
    if tuple(v_cache.shape) != (NB, Hkv, BS, C * E):
        raise ValueError("v_cache must be [num_blocks][Hkv][16][D] (k_cache is [num_blocks][Hkv][D/8][16][8])")
    if out.shape != q.shape:
        raise ValueError("out must have the shape of q")
    if context_lens.shape != (q.shape[0],):
        raise ValueError("context_lens must be [B]")


def _check_new_kv(k_new, v_new, q_shape, k_cache):
    import torch

    _require("k_new", k_new, torch.bfloat16)
    _require("v_new", v_new, torch.bfloat16)
    B, n, _, D = q_shape
    Hkv = k_cache.shape[1]
    if tuple(k_new.shape) != (B, n, Hkv, D) or tuple(v_new.shape) != (B, n, Hkv, D):
        raise ValueError(f"k_new and v_new must be [B][n][Hkv][D] = {(B, n, Hkv, D)}")


def _stream_handle(stream, device):
    import torch

    if stream is None:
        stream = torch.cuda.current_stream(device)
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _as_stream(stream, device):
    import torch

    if hasattr(stream, "cuda_stream"):
        return stream
    if int(stream) == 0:  # (an ExternalStream of handle 0 is a new stream)
        return torch.cuda.default_stream(device)
    return torch.cuda.ExternalStream(int(stream), device=device)


def _empty(shape, dtype, device, stream, result=True):
    """Memory for a call on `stream` (None: the current one), taken from that
    stream's own: what the current stream has freed may still be in use by work it
    has queued, which nothing orders before the call.  A `result` is handed back to
    the current stream: it is not reused before that one is done with it, either."""
    import torch

    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    stream = _as_stream(stream, device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    if result:
        t.record_stream(torch.cuda.current_stream(device))
    return t


def _hold(stream, *tensors):
    """Tensors that a call on a stream other than the current one uses and hands
    back: their memory is not reused before the stream is done with them."""
    if stream is not None:
        for t in tensors:
            if t is not None:
                t.record_stream(_as_stream(stream, t.device))


def _workspace(prob, workspace, device, stream=None):
    import torch

    need = pda_workspace_bytes(prob)
    if workspace is None and need > 0:
        workspace = _empty((need,), torch.uint8, device, stream, result=False)
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    return workspace, ws_ptr, ws_bytes


def _step(fn_name, q, k_cache, v_cache, block_table, context_lens, scale, out, max_context_len,
          partition_tokens, workspace, stream):
    return bind_decode(q, k_cache, v_cache, block_table, context_lens, scale, out, max_context_len=max_context_len,
                       partition_tokens=partition_tokens, workspace=workspace, stream=stream,
                       pass1_only=fn_name == "pda_partition_attention")()


def pda_decode(q, k_cache, v_cache, block_table, context_lens, scale: float, out=None, *,
               max_context_len: int, partition_tokens: int = 0, workspace=None, stream=None):
    """One attention step (both passes).  Tensors on the GPU: q bf16
    [B][Hq][D] (a decode step) or [B][n][Hq][D] (n new tokens per sequence,
    the last n of its context, attending causally), k_cache bf16
    [num_blocks][Hkv][D/8][16][8] (each block's keys as D/8 chunks of 16 slots
    x 8 elements), v_cache bf16 [num_blocks][Hkv][16][D], block_table int32
    [B][max_blocks], context_lens int32 [B], out fp32 shaped like q.
    `workspace` (uint8, >= pda_workspace_bytes) is allocated when not given;
    partition_tokens > 0 fixes the split-K partition size."""
    return _step("pda_decode", q, k_cache, v_cache, block_table, context_lens, scale, out, max_context_len,
                 partition_tokens, workspace, stream)


def pda_partition_attention(q, k_cache, v_cache, block_table, context_lens, scale: float, out=None, *,
                            max_context_len: int, partition_tokens: int = 0, workspace=None, stream=None):
    """Pass 1 only (see pda_decode)."""
    return _step("pda_partition_attention", q, k_cache, v_cache, block_table, context_lens, scale, out,
                 max_context_len, partition_tokens, workspace, stream)


def pda_merge_partitions(prob: pda_problem, context_lens, out, workspace, stream=None):
    """Pass 2 only: merge the partial states pass 1 left in `workspace`."""
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    rc = load_library().pda_merge_partitions(ctypes.byref(prob), context_lens.data_ptr(), out.data_ptr(),
                                             ws_ptr, ws_bytes, _stream_handle(stream, out.device))
    if rc != PDA_OK:
        raise PdaError(rc, "pda_merge_partitions")
    return out


def pda_append_kv(k_new, v_new, block_table, context_lens, k_cache, v_cache, *, max_context_len: int,
                  num_q_heads: int = None, stream=None):
    """Store the K/V rows of each sequence's n new tokens (bf16 [B][n][Hkv][D])
    at positions L - n .. L - 1 of its paged cache, in place."""
    bind_append_kv(k_new, v_new, block_table, context_lens, k_cache, v_cache, max_context_len=max_context_len,
                   num_q_heads=num_q_heads, stream=stream)()


class BoundCall:
    """One entry point with its arguments bound once, for a serving loop that
    runs the same step on the same buffers again and again: the Python checks,
    the problem descriptor, the workspace and the stream are prepared when the
    call is built, and each call is then a single foreign-function call (the
    library still validates the descriptor, plans the step and launches its
    kernels every time).  The bound tensors are kept alive and must keep their
    storage; their contents may change between calls."""

    def __init__(self, fn_name, args, keep, result=None):
        self._fn = getattr(load_library(), fn_name)
        self._name = fn_name
        self._args = args
        self._keep = keep
        self.result = result

    def __call__(self):
        rc = self._fn(*self._args)
        if rc != PDA_OK:
            raise PdaError(rc, self._name)
        return self.result


def bind_decode(q, k_cache, v_cache, block_table, context_lens, scale: float, out=None, *, max_context_len: int,
                partition_tokens: int = 0, workspace=None, stream=None, pass1_only: bool = False,
                reuse_order: bool = False) -> BoundCall:
    """pda_decode (or, with pass1_only, pda_partition_attention; with
    reuse_order, pda_decode_reusing_order; with both,
    pda_partition_attention_reusing_order) bound to these tensors and the
    given (else the current) stream; call it to run a step.  The arguments
    are those of pda_decode."""
    import torch

    if out is None:
        out = _empty(q.shape, torch.float32, q.device, stream)
    _check_tensors(q, k_cache, v_cache, block_table, context_lens, out)
    prob = _problem_from(q, k_cache, block_table, max_context_len, partition_tokens)
    workspace, ws_ptr, ws_bytes = _workspace(prob, workspace, q.device, stream)
    args = (ctypes.byref(prob), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), block_table.data_ptr(),
            context_lens.data_ptr(), ctypes.c_float(scale), out.data_ptr(), ws_ptr, ws_bytes,
            _stream_handle(stream, q.device))
    keep = (prob, q, k_cache, v_cache, block_table, context_lens, out, workspace)
    name = {(False, False): "pda_decode", (True, False): "pda_partition_attention",
            (False, True): "pda_decode_reusing_order",
            (True, True): "pda_partition_attention_reusing_order"}[(bool(pass1_only), bool(reuse_order))]
    return BoundCall(name, args, keep, out)


def bind_decode_append(q, k_new, v_new, k_cache, v_cache, block_table, context_lens, scale: float, out=None, *,
                       max_context_len: int, partition_tokens: int = 0, workspace=None, stream=None) -> BoundCall:
    """pda_decode_append bound to these tensors: the append of each sequence's
    new token (k_new/v_new bf16 [B][1][Hkv][D]) folded into the decode step."""
    import torch

    if out is None:
        out = _empty(q.shape, torch.float32, q.device, stream)
    _check_tensors(q, k_cache, v_cache, block_table, context_lens, out)
    _check_new_kv(k_new, v_new, _query_shape(q), k_cache)
    prob = _problem_from(q, k_cache, block_table, max_context_len, partition_tokens)
    workspace, ws_ptr, ws_bytes = _workspace(prob, workspace, q.device, stream)
    args = (ctypes.byref(prob), q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), k_cache.data_ptr(),
            v_cache.data_ptr(), block_table.data_ptr(), context_lens.data_ptr(), ctypes.c_float(scale),
            out.data_ptr(), ws_ptr, ws_bytes, _stream_handle(stream, q.device))
    keep = (prob, q, k_new, v_new, k_cache, v_cache, block_table, context_lens, out, workspace)
    return BoundCall("pda_decode_append", args, keep, out)


def pda_decode_append(q, k_new, v_new, k_cache, v_cache, block_table, context_lens, scale: float, out=None, *,
                      max_context_len: int, partition_tokens: int = 0, workspace=None, stream=None):
    """pda_append_kv + pda_decode in the launches of pda_decode alone (one new
    token per sequence)."""
    return bind_decode_append(q, k_new, v_new, k_cache, v_cache, block_table, context_lens, scale, out,
                              max_context_len=max_context_len, partition_tokens=partition_tokens,
                              workspace=workspace, stream=stream)()


def pda_work_order(prob: pda_problem, context_lens, workspace, stream=None):
    """The step's work order into `workspace` (see include/pda.h): computed
    once per decode step, reused by every layer's pda_decode_reusing_order."""
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    rc = load_library().pda_work_order(ctypes.byref(prob), context_lens.data_ptr(),
                                       workspace.data_ptr() if workspace is not None else None, ws_bytes,
                                       _stream_handle(stream, context_lens.device))
    if rc != PDA_OK:
        raise PdaError(rc, "pda_work_order")


def pda_decode_reusing_order(q, k_cache, v_cache, block_table, context_lens, scale: float, out=None, *,
                             max_context_len: int, partition_tokens: int = 0, workspace, stream=None):
    """pda_decode with the work order already in `workspace` (pda_work_order
    or an earlier pda_decode on it, same descriptor)."""
    return bind_decode(q, k_cache, v_cache, block_table, context_lens, scale, out, max_context_len=max_context_len,
                       partition_tokens=partition_tokens, workspace=workspace, stream=stream, reuse_order=True)()


def bind_decode_noalloc(q, k_cache, v_cache, block_table, context_lens, scale: float, out=None, *,
                        max_context_len: int, partition_tokens: int = 0, stream=None) -> BoundCall:
    """pda_decode_noalloc bound to these tensors and the given (else the
    current) stream: the step of pda_decode with its workspace in the
    library's static scratch, so no call allocates (`out` is allocated here,
    once, when not given)."""
    import torch

    if out is None:
        out = _empty(q.shape, torch.float32, q.device, stream)
    _check_tensors(q, k_cache, v_cache, block_table, context_lens, out)
    prob = _problem_from(q, k_cache, block_table, max_context_len, partition_tokens)
    args = (ctypes.byref(prob), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), block_table.data_ptr(),
            context_lens.data_ptr(), ctypes.c_float(scale), out.data_ptr(), _stream_handle(stream, q.device))
    return BoundCall("pda_decode_noalloc", args, (prob, q, k_cache, v_cache, block_table, context_lens, out), out)


def pda_decode_noalloc(q, k_cache, v_cache, block_table, context_lens, scale: float, out=None, *,
                       max_context_len: int, partition_tokens: int = 0, stream=None):
    """pda_decode without a workspace argument (see include/pda.h): raises
    PdaError with PDA_ERR_SCRATCH when the step needs more than
    PDA_NOALLOC_SCRATCH_BYTES of workspace."""
    return bind_decode_noalloc(q, k_cache, v_cache, block_table, context_lens, scale, out,
                               max_context_len=max_context_len, partition_tokens=partition_tokens, stream=stream)()


def bind_append_kv(k_new, v_new, block_table, context_lens, k_cache, v_cache, *, max_context_len: int,
                   num_q_heads: int = None, stream=None) -> BoundCall:
    """pda_append_kv bound to these tensors and the given (else the current)
    stream; the arguments are those of pda_append_kv."""
    import torch

    if k_new.dim() != 4:
        raise ValueError("k_new must be [B][n][Hkv][D]")
    B, n, Hkv, D = k_new.shape
    for name, t, dt in (("k_cache", k_cache, torch.bfloat16), ("v_cache", v_cache, torch.bfloat16),
                        ("block_table", block_table, torch.int32), ("context_lens", context_lens, torch.int32)):
        _require(name, t, dt)
    q_shape = (B, n, Hkv if num_q_heads is None else num_q_heads, D)
    _check_new_kv(k_new, v_new, q_shape, k_cache)
    NB, Hkv_c, C, BS, E = k_cache.shape
    if Hkv_c != Hkv or C * E != D or tuple(v_cache.shape) != (NB, Hkv, BS, D):
        raise ValueError("k_new/v_new and the caches disagree")
    if block_table.dim() != 2 or block_table.shape[0] != B or context_lens.shape != (B,):
        raise ValueError("block_table [B][max_blocks], context_lens [B]")
    prob = make_problem(B, q_shape[2], Hkv, D, NB, block_table.shape[1], max_context_len, 0, BS, n)
    args = (ctypes.byref(prob), k_new.data_ptr(), v_new.data_ptr(), block_table.data_ptr(), context_lens.data_ptr(),
            k_cache.data_ptr(), v_cache.data_ptr(), _stream_handle(stream, k_cache.device))
    keep = (prob, k_new, v_new, block_table, context_lens, k_cache, v_cache)
    return BoundCall("pda_append_kv", args, keep)


class _MadeForGraph:
    """Tensors allocated here for a captured graph, which is launched on any stream:
    when it is made, nothing uses their memory any more, and that memory is not
    reused before every stream it was launched on is done with it."""

    def __init__(self, device, *tensors):
        import torch

        self._device, self._tensors, self._streams = device, [t for t in tensors if t is not None], set()
        if self._tensors:
            torch.cuda.current_stream(device).synchronize()

    def stream_handle(self, stream):
        """The handle of the stream (None: the current one) of a launch."""
        handle = _stream_handle(stream, self._device)
        if handle.value not in self._streams:
            self._streams.add(handle.value)
            _hold(handle.value or 0, *self._tensors)
        return handle


class ModelStepGraph:
    """pda_model_step_graph_create: a model's decode step over `layers` (a list
    of dicts with q, k_new, v_new, k_cache, v_cache and out tensors, one per
    layer) captured as one HIP graph -- per layer the KV append and the
    attention step, the work order computed once.  launch() replays it on a
    stream and reads the buffers' current contents."""

    def __init__(self, layers, block_table, context_lens, scale: float, *, max_context_len: int,
                 partition_tokens: int = 0, workspace=None):
        import torch

        if not layers:
            raise ValueError("at least one layer")
        arr = (pda_layer_buffers * len(layers))()
        for i, L in enumerate(layers):
            _check_tensors(L["q"], L["k_cache"], L["v_cache"], block_table, context_lens, L["out"])
            _check_new_kv(L["k_new"], L["v_new"], _query_shape(L["q"]), L["k_cache"])
            arr[i] = pda_layer_buffers(L["q"].data_ptr(), L["k_new"].data_ptr(), L["v_new"].data_ptr(),
                                       L["k_cache"].data_ptr(), L["v_cache"].data_ptr(), L["out"].data_ptr())
        L0 = layers[0]
        self.prob = _problem_from(L0["q"], L0["k_cache"], block_table, max_context_len, partition_tokens)
        given = workspace
        workspace, ws_ptr, ws_bytes = _workspace(self.prob, workspace, L0["q"].device)
        self._made = _MadeForGraph(L0["q"].device, workspace if given is None else None)
        self.workspace = workspace
        self._keep = (layers, block_table, context_lens, arr)
        handle = ctypes.c_void_p()
        rc = load_library().pda_model_step_graph_create(
            ctypes.byref(self.prob), len(layers), arr, block_table.data_ptr(), context_lens.data_ptr(),
            ctypes.c_float(scale), ws_ptr, ws_bytes, ctypes.byref(handle))
        if rc != PDA_OK:
            raise PdaError(rc, "pda_model_step_graph_create")
        self._handle = handle

    def launch(self, stream=None):
        rc = load_library().pda_step_graph_launch(self._handle, self._made.stream_handle(stream))
        if rc != PDA_OK:
            raise PdaError(rc, "pda_step_graph_launch")

    def close(self):
        if getattr(self, "_handle", None) is not None:
            rc = load_library().pda_step_graph_destroy(self._handle)
            self._handle = None
            if rc != PDA_OK:
                raise PdaError(rc, "pda_step_graph_destroy")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class StepGraph:
    """pda_step_graph: append + attention captured once as a HIP graph over
    fixed buffers.  launch() replays it on a stream and reads the buffers'
    current contents.  The tensors are kept alive for the graph's lifetime."""

    def __init__(self, q, k_new, v_new, k_cache, v_cache, block_table, context_lens, scale: float, out=None, *,
                 max_context_len: int, partition_tokens: int = 0, workspace=None):
        import torch

        given = out, workspace
        if out is None:
            out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
        _check_tensors(q, k_cache, v_cache, block_table, context_lens, out)
        _check_new_kv(k_new, v_new, _query_shape(q), k_cache)
        self.prob = _problem_from(q, k_cache, block_table, max_context_len, partition_tokens)
        workspace, ws_ptr, ws_bytes = _workspace(self.prob, workspace, q.device)
        self._made = _MadeForGraph(q.device, out if given[0] is None else None, workspace if given[1] is None else None)
        self.out, self.workspace = out, workspace
        self._keep = (q, k_new, v_new, k_cache, v_cache, block_table, context_lens)
        handle = ctypes.c_void_p()
        rc = load_library().pda_step_graph_create(
            ctypes.byref(self.prob), q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), k_cache.data_ptr(),
            v_cache.data_ptr(), block_table.data_ptr(), context_lens.data_ptr(), ctypes.c_float(scale),
            out.data_ptr(), ws_ptr, ws_bytes, ctypes.byref(handle))
        if rc != PDA_OK:
            raise PdaError(rc, "pda_step_graph_create")
        self._handle = handle

    def launch(self, stream=None):
        rc = load_library().pda_step_graph_launch(self._handle, self._made.stream_handle(stream))
        if rc != PDA_OK:
            raise PdaError(rc, "pda_step_graph_launch")
        return self.out

    def close(self):
        if getattr(self, "_handle", None) is not None:
            rc = load_library().pda_step_graph_destroy(self._handle)
            self._handle = None
            if rc != PDA_OK:
                raise PdaError(rc, "pda_step_graph_destroy")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def pda_logprob_workspace_bytes(rows: int, vocab: int, dtype: int) -> int:
    ws = ctypes.c_size_t()
    rc = load_library().pda_logprob_workspace_bytes(int(rows), int(vocab), int(dtype), ctypes.byref(ws))
    if rc != PDA_OK:
        raise PdaError(rc, "pda_logprob_workspace_bytes")
    return ws.value


def bind_token_logprobs(logits, tokens, inv_temperature: float = 1.0, entropy: bool = True, vocab: int = None,
                        logprobs=None, entropies=None, stream=None, workspace="auto") -> BoundCall:
    """pda_token_logprobs bound to these tensors and the given (else the
    current) stream; calling it returns (logprobs, entropies or None).  The
    arguments are those of pda_token_logprobs; `workspace` is "auto" (a uint8
    tensor of pda_logprob_workspace_bytes, allocated here once), None (one
    workgroup per row) or a caller's uint8 device tensor."""
    import torch

    if logits.dim() != 2 or logits.stride(1) != 1:
        raise ValueError("logits must be [rows][row_stride] with unit element stride")
    if logits.dtype == torch.bfloat16:
        dtype = PDA_DTYPE_BF16
    elif logits.dtype == torch.float32:
        dtype = PDA_DTYPE_F32
    else:
        raise TypeError("logits must be bfloat16 or float32")
    _require("tokens", tokens, torch.int32)
    if not logits.is_cuda:
        raise ValueError("logits must be a device tensor")
    rows = logits.shape[0]
    vocab = logits.shape[1] if vocab is None else int(vocab)
    if tokens.shape != (rows,):
        raise ValueError("tokens must be [rows]")
    if logprobs is None:
        logprobs = _empty((rows,), torch.float32, logits.device, stream)
    if entropy and entropies is None:
        entropies = _empty((rows,), torch.float32, logits.device, stream)
    if isinstance(workspace, str):
        need = pda_logprob_workspace_bytes(rows, vocab, dtype) if vocab >= 1 else 0
        workspace = _empty((need,), torch.uint8, logits.device, stream, result=False) if need > 0 else None
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    args = (rows, vocab, logits.stride(0), dtype, logits.data_ptr(), tokens.data_ptr(),
            ctypes.c_float(inv_temperature), logprobs.data_ptr(), entropies.data_ptr() if entropy else None,
            ws_ptr, ws_bytes, _stream_handle(stream, logits.device))
    keep = (logits, tokens, logprobs, entropies, workspace)
    return BoundCall("pda_token_logprobs", args, keep, (logprobs, entropies if entropy else None))


def pda_token_logprobs(logits, tokens, inv_temperature: float = 1.0, entropy: bool = True, vocab: int = None,
                       logprobs=None, entropies=None, stream=None, workspace="auto"):
    """Log-probability of tokens[r] under softmax(logits[r][:vocab] * inv_temperature),
    and the entropy of that distribution (natural-log units).  logits: a device
    tensor [rows][row_stride] of bf16 or float32 (16-byte aligned rows); tokens
    int32 [rows].  Returns (logprobs fp32 [rows], entropies fp32 [rows] or None)."""
    return bind_token_logprobs(logits, tokens, inv_temperature, entropy, vocab, logprobs, entropies, stream,
                               workspace)()


def pda_decode_shared_prefix(q, k_cache, v_cache, block_table, context_lens, scale: float, group_start,
                             group_prefix_len, out=None, *, max_context_len: int, max_group_size: int,
                             max_prefix_len: int, partition_tokens: int = 0, workspace=None, stream=None):
    """The decode step with each shared-prefix group's prefix attended once for
    all its members.  group_start int32 [num_groups + 1] and group_prefix_len
    int32 [num_groups] are device tensors; max_group_size and max_prefix_len
    are their host bounds (n * G <= 64; groups larger than 64 / (n G) members
    read the prefix once per 64 / (n G) members).  Other arguments
    as pda_decode (q [B][Hq][D], or [B][n][Hq][D] for n new tokens)."""
    import torch

    if out is None:
        out = _empty(q.shape, torch.float32, q.device, stream)
    _check_tensors(q, k_cache, v_cache, block_table, context_lens, out)
    _require("group_start", group_start, torch.int32)
    _require("group_prefix_len", group_prefix_len, torch.int32)
    num_groups = group_prefix_len.shape[0]
    if group_start.shape != (num_groups + 1,):
        raise ValueError("group_start must be [num_groups + 1]")
    prob = _problem_from(q, k_cache, block_table, max_context_len, partition_tokens)
    groups = make_prefix_groups(num_groups, max_group_size, max_prefix_len, group_start, group_prefix_len)
    need = pda_plan_shared_prefix(prob, groups)["workspace_bytes"]
    if workspace is None and need > 0:
        workspace = _empty((need,), torch.uint8, q.device, stream, result=False)
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    rc = load_library().pda_decode_shared_prefix(
        ctypes.byref(prob), ctypes.byref(groups), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
        block_table.data_ptr(), context_lens.data_ptr(), ctypes.c_float(scale), out.data_ptr(), ws_ptr, ws_bytes,
        _stream_handle(stream, q.device))
    if rc != PDA_OK:
        raise PdaError(rc, "pda_decode_shared_prefix")
    return out


def bind_gather_ceiling(block_ids, k_cache, v_cache, workgroups: int, sink=None, stream=None) -> BoundCall:
    """pda_gather_ceiling (include/pda_ceiling.h) bound to these tensors: read
    the K and V tiles of every KV head of the listed physical blocks (device
    int32 [n]) with the attention kernel's loads and no arithmetic."""
    import torch

    _require("block_ids", block_ids, torch.int32)
    _require("k_cache", k_cache, torch.bfloat16)
    _require("v_cache", v_cache, torch.bfloat16)
    if sink is None:
        sink = _empty((4 * workgroups,), torch.int32, k_cache.device, stream)
    NB, Hkv, C, BS, E = k_cache.shape
    args = (int(Hkv), int(C * E), int(NB), k_cache.data_ptr(), v_cache.data_ptr(), block_ids.data_ptr(),
            int(block_ids.numel()), int(workgroups), sink.data_ptr(), _stream_handle(stream, k_cache.device))
    return BoundCall("pda_gather_ceiling", args, (block_ids, k_cache, v_cache, sink), sink)


def bind_stream_ceiling(buf, workgroups: int, sink=None, stream=None) -> BoundCall:
    """pda_stream_ceiling bound to a contiguous device tensor: read all its
    bytes with 16-byte non-temporal loads."""
    import torch

    if not buf.is_cuda or not buf.is_contiguous():
        raise ValueError("buf must be a contiguous device tensor")
    if sink is None:
        sink = _empty((4 * workgroups,), torch.int32, buf.device, stream)
    nbytes = buf.numel() * buf.element_size() // 16 * 16
    args = (buf.data_ptr(), ctypes.c_size_t(nbytes), int(workgroups), sink.data_ptr(),
            _stream_handle(stream, buf.device))
    return BoundCall("pda_stream_ceiling", args, (buf, sink), sink)


# ---- the 8-bit KV cache and rotary positions (include/pda_fp8.h) ----

class DeviceCall(BoundCall):
    """A BoundCall that runs with its tensors' device current, whichever is
    current where it is called."""

    def __init__(self, fn_name, args, keep, device, result=None):
        super().__init__(fn_name, args, keep, result)
        import torch

        self._index = device.index if device.index is not None else torch.cuda.current_device()
        self._current, self._device = torch.cuda.current_device, torch.cuda.device

    def __call__(self):
        if self._current() != self._index:
            with self._device(self._index):
                return super().__call__()
        return super().__call__()


def _same_device(*tensors):
    devices = {t.device for t in tensors if t is not None}
    if len(devices) != 1:
        raise ValueError(f"tensors on different devices: {sorted(map(str, devices))}")
    return devices.pop()


def _zeros_like(t, stream):
    """Zeros of t's shape for a call on `stream`, filled on it too."""
    return _cleared(_empty(t.shape, t.dtype, t.device, stream), stream)


def _cleared(t, stream):
    """t filled with zeros on `stream` (None: the current one)."""
    import torch

    if stream is None:
        return t.zero_()
    with torch.cuda.stream(_as_stream(stream, t.device)):
        return t.zero_()


def _check_fp8_cache(k_cache, v_cache, kv_scale):
    """(num_blocks, Hkv, D) of an 8-bit cache."""
    import torch

    for name, t, dt in (("k_cache", k_cache, torch.float8_e4m3fn), ("v_cache", v_cache, torch.float8_e4m3fn),
                        ("kv_scale", kv_scale, torch.uint8)):
        _require(name, t, dt)
    if k_cache.dim() != 7 or tuple(k_cache.shape[3:]) != (4, 16, 2, 8):
        raise ValueError("k_cache must be [num_blocks][Hkv][D/64][4][16][2][8]")
    NB, Hkv, D = k_cache.shape[0], k_cache.shape[1], 64 * k_cache.shape[2]
    if tuple(v_cache.shape) != (NB, Hkv, 2, 4, D // 8, 2, 8):
        raise ValueError(f"v_cache must be [num_blocks][Hkv][2][4][D/8][2][8] = {(NB, Hkv, 2, 4, D // 8, 2, 8)}")
    if tuple(kv_scale.shape) != (NB, Hkv, 2, 16):
        raise ValueError(f"kv_scale must be [num_blocks][Hkv][2][16] = {(NB, Hkv, 2, 16)}")
    return NB, Hkv, D


def _check_paged(block_table, context_lens, B):
    import torch

    _require("block_table", block_table, torch.int32)
    _require("context_lens", context_lens, torch.int32)
    if block_table.dim() != 2 or block_table.shape[0] != B or context_lens.shape != (B,):
        raise ValueError("block_table [B][max_blocks], context_lens [B]")


def make_fp8_cache(num_blocks: int, num_kv_heads: int, head_dim: int, device="cuda"):
    """An empty 8-bit cache: (k_cache, v_cache, kv_scale), all zero."""
    import torch

    z = lambda *shape: torch.zeros(shape, dtype=torch.uint8, device=device)
    return (z(num_blocks, num_kv_heads, head_dim // 64, 4, 16, 2, 8).view(torch.float8_e4m3fn),
            z(num_blocks, num_kv_heads, 2, 4, head_dim // 8, 2, 8).view(torch.float8_e4m3fn),
            z(num_blocks, num_kv_heads, 2, 16))


def pda_rotary_inv_freq(rotary_dim: int, base: float = 10000.0, kind: int = PDA_ROTARY_PLAIN, factor: float = 1.0,
                        original_len: float = 0.0, low: float = 0.0, high: float = 0.0):
    """(inv_freq, magnitude): the rotary_dim / 2 frequencies base^(-2i / rotary_dim)
    scaled for long contexts as `kind` says (include/pda_fp8.h), as a float64
    numpy array, and the factor on the rotated elements."""
    import torch  # noqa: F401  (before the library: its HIP runtime is the one to share)

    inv_freq = np.empty(max(int(rotary_dim), 0) // 2, dtype=np.float64)
    scaling = pda_rotary_scaling(int(kind), float(factor), float(original_len), float(low), float(high))
    magnitude = ctypes.c_float()
    rc = load_library().pda_rotary_inv_freq(int(rotary_dim), float(base), ctypes.byref(scaling), inv_freq.ctypes.data,
                                            ctypes.byref(magnitude))
    if rc != PDA_OK:
        raise PdaError(rc, "pda_rotary_inv_freq")
    return inv_freq, magnitude.value


def make_rotary(inv_freq, interleaved: bool = False, backward: bool = False, magnitude: float = 1.0) -> pda_rotary:
    """A rotary embedding of the first 2 * len(inv_freq) elements of every head
    row; inv_freq: float64 device tensor (it is kept alive by the result)."""
    import torch

    _require("inv_freq", inv_freq, torch.float64)
    if inv_freq.dim() != 1:
        raise ValueError("inv_freq must be [rotary_dim / 2]")
    r = pda_rotary(2 * inv_freq.shape[0], int(bool(interleaved)), int(bool(backward)), float(magnitude),
                   inv_freq.data_ptr())
    r.tensor = inv_freq
    return r


def _token_rows(name, t, dtype):
    """Token stride of rows [T][H][D] whose heads are contiguous."""
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    T, H, D = t.shape
    if t.numel() and (t.stride(2) != 1 or (H > 1 and t.stride(1) != D)):
        raise ValueError(f"{name} must be [T][H][D] with the heads of a token contiguous")
    return t.stride(0) if T > 1 else H * D  # (the stride of a single token is free)


def bind_rotary_apply(q, positions, rotary: pda_rotary, k=None, q_out=None, k_out=None, stream=None) -> DeviceCall:
    """pda_rotary_apply bound to these tensors and the given (else the current)
    stream; calling it returns (q_out, k_out).  q [T][Hq][D] and k [T][Hkv][D]
    are bf16 or float32 with any token stride; the outputs are allocated when
    not given, and may be the inputs (in place).  positions int32 [T], negative:
    padding, left alone."""
    import torch

    if q.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError("q must be bfloat16 or float32")
    if q.dim() != 3 or (k is not None and (k.dim() != 3 or k.shape[0] != q.shape[0] or k.shape[2] != q.shape[2])):
        raise ValueError("q [T][Hq][D], k [T][Hkv][D]")
    if k is None and k_out is not None:
        raise ValueError("k_out without k")
    if q.shape[0] > 0x7fffffff:
        raise ValueError("more than 2^31 - 1 tokens")
    _require("positions", positions, torch.int32)
    if positions.shape != (q.shape[0],):
        raise ValueError("positions must be [T]")
    # (padding rows are not written: an output made here holds zeros there)
    q_out = _zeros_like(q, stream) if q_out is None else q_out
    if k is not None and k_out is None:
        k_out = _zeros_like(k, stream)
    if q_out.shape != q.shape or (k is not None and k_out.shape != k.shape):
        raise ValueError("the outputs must have the inputs' shapes")
    device = _same_device(q, q_out, k, k_out, positions, rotary.tensor)
    T, Hq, D = q.shape
    rows = [q.data_ptr(), _token_rows("q", q, q.dtype), q_out.data_ptr(), _token_rows("q_out", q_out, q.dtype)]
    if k is not None:
        rows += [k.data_ptr(), _token_rows("k", k, q.dtype), k_out.data_ptr(), _token_rows("k_out", k_out, q.dtype)]
    else:
        rows += [None, 0, None, 0]
    dtype = PDA_DTYPE_BF16 if q.dtype == torch.bfloat16 else PDA_DTYPE_F32
    args = (ctypes.byref(rotary), T, Hq, 0 if k is None else k.shape[1], D, dtype, positions.data_ptr(), *rows,
            _stream_handle(stream, device))
    return DeviceCall("pda_rotary_apply", args, (rotary, q, q_out, k, k_out, positions), device, (q_out, k_out))


def pda_rotary_apply(q, positions, rotary: pda_rotary, k=None, q_out=None, k_out=None, stream=None):
    """Rotary positions of q (and k) rows; returns (q_out, k_out or None).  See
    bind_rotary_apply."""
    call = bind_rotary_apply(q, positions, rotary, k, q_out, k_out, stream)
    result = call()
    _hold(stream, *result)
    return result


def bind_append_kv_fp8(k_new, v_new, block_table, context_lens, k_cache, v_cache, kv_scale, *, max_context_len: int,
                       rotary: pda_rotary = None, q=None, q_out=None, num_q_heads: int = None,
                       stream=None) -> DeviceCall:
    """pda_append_kv_fp8 bound to these tensors and the given (else the current)
    stream: k_new/v_new bf16 [B][n][Hkv][D] quantised and stored at positions
    L - n .. L - 1 of the 8-bit cache (make_fp8_cache); with `rotary` the keys are
    rotated first, and q (bf16 [B][n][Hq][D] or, for n = 1, [B][Hq][D]) into q_out
    (allocated when not given; may be q).  Calling it returns q_out (None without
    q)."""
    import torch

    NB, Hkv, D = _check_fp8_cache(k_cache, v_cache, kv_scale)
    if k_new.dim() != 4:
        raise ValueError("k_new must be [B][n][Hkv][D]")
    B, n = k_new.shape[:2]
    _check_paged(block_table, context_lens, B)
    for name, t in (("k_new", k_new), ("v_new", v_new)):
        _require(name, t, torch.bfloat16)
        if tuple(t.shape) != (B, n, Hkv, D):
            raise ValueError(f"k_new and v_new must be [B][n][Hkv][D] = {(B, n, Hkv, D)}")
    if q is None and q_out is not None:
        raise ValueError("q_out without q")
    Hq = Hkv if num_q_heads is None else num_q_heads
    if q is not None:
        if rotary is None:
            raise ValueError("q is rotated here: give `rotary`")
        _require("q", q, torch.bfloat16)
        if _query_shape(q)[:2] != (B, n) or q.shape[-1] != D:
            raise ValueError("q must be [B][n][Hq][D]")
        Hq = q.shape[-2]
        if q_out is None:
            q_out = _zeros_like(q, stream)
        _require("q_out", q_out, torch.bfloat16)
        if q_out.shape != q.shape:
            raise ValueError("q_out must have the shape of q")
    device = _same_device(k_new, v_new, block_table, context_lens, k_cache, v_cache, kv_scale, q, q_out,
                          rotary.tensor if rotary is not None else None)
    if n == 0:
        raise ValueError("at least one new token")
    prob = make_problem(B, Hq, Hkv, D, NB, block_table.shape[1], max_context_len, 0, 16, n)
    ptr = lambda t: t.data_ptr() if t is not None else None
    args = (ctypes.byref(prob), ctypes.byref(rotary) if rotary is not None else None, ptr(q), ptr(q_out),
            k_new.data_ptr(), v_new.data_ptr(), block_table.data_ptr(), context_lens.data_ptr(), k_cache.data_ptr(),
            v_cache.data_ptr(), kv_scale.data_ptr(), _stream_handle(stream, device))
    keep = (prob, rotary, q, q_out, k_new, v_new, block_table, context_lens, k_cache, v_cache, kv_scale)
    return DeviceCall("pda_append_kv_fp8", args, keep, device, q_out)


def pda_append_kv_fp8(k_new, v_new, block_table, context_lens, k_cache, v_cache, kv_scale, *, max_context_len: int,
                      rotary: pda_rotary = None, q=None, q_out=None, num_q_heads: int = None, stream=None):
    """The new tokens' K/V rows (rotated, when `rotary` is given) quantised and
    stored in the 8-bit cache, in place; returns the rotated queries (None without
    q).  See bind_append_kv_fp8."""
    result = bind_append_kv_fp8(k_new, v_new, block_table, context_lens, k_cache, v_cache, kv_scale,
                                max_context_len=max_context_len, rotary=rotary, q=q, q_out=q_out,
                                num_q_heads=num_q_heads, stream=stream)()
    _hold(stream, result)
    return result


def pda_plan_fp8(prob: pda_problem) -> dict:
    """The plan of pda_decode_fp8: partition_tokens, num_partitions, workspace_bytes."""
    import torch  # noqa: F401  (before the library: its HIP runtime is the one to share)

    info = pda_plan_info()
    rc = load_library().pda_plan_fp8(ctypes.byref(prob), ctypes.byref(info))
    if rc != PDA_OK:
        raise PdaError(rc, "pda_plan_fp8")
    return info.as_dict()


def bind_decode_fp8(q, k_cache, v_cache, kv_scale, block_table, context_lens, scale: float, out=None, *,
                    max_context_len: int, partition_tokens: int = 0, workspace=None, stream=None) -> DeviceCall:
    """pda_decode_fp8 bound to these tensors and the given (else the current)
    stream: the attention of bind_decode over an 8-bit cache (make_fp8_cache).
    `workspace` (uint8, pda_plan_fp8's workspace_bytes) is allocated here when not
    given."""
    import torch

    NB, Hkv, D = _check_fp8_cache(k_cache, v_cache, kv_scale)
    _require("q", q, torch.bfloat16)
    B, n, Hq, Dq = _query_shape(q)
    if Dq != D:
        raise ValueError("q and the caches disagree on the head size")
    if n == 0:
        raise ValueError("at least one new token")
    _check_paged(block_table, context_lens, B)
    if out is None:
        out = _empty(q.shape, torch.float32, q.device, stream)
    _require("out", out, torch.float32)
    if out.shape != q.shape:
        raise ValueError("out must have the shape of q")
    device = _same_device(q, k_cache, v_cache, kv_scale, block_table, context_lens, out, workspace)
    prob = make_problem(B, Hq, Hkv, D, NB, block_table.shape[1], max_context_len, partition_tokens, 16, n)
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    need = pda_plan_fp8(prob)["workspace_bytes"]
    if workspace is None and need > 0:
        workspace = _empty((need,), torch.uint8, device, stream, result=False)
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    args = (ctypes.byref(prob), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), kv_scale.data_ptr(),
            block_table.data_ptr(), context_lens.data_ptr(), ctypes.c_float(scale), out.data_ptr(), ws_ptr, ws_bytes,
            _stream_handle(stream, device))
    keep = (prob, q, k_cache, v_cache, kv_scale, block_table, context_lens, out, workspace)
    call = DeviceCall("pda_decode_fp8", args, keep, device, out)
    call.workspace = workspace
    return call


def pda_decode_fp8(q, k_cache, v_cache, kv_scale, block_table, context_lens, scale: float, out=None, *,
                   max_context_len: int, partition_tokens: int = 0, workspace=None, stream=None):
    """One attention step over an 8-bit cache; the other arguments are those of
    pda_decode.  Returns out (fp32, shaped like q)."""
    call = bind_decode_fp8(q, k_cache, v_cache, kv_scale, block_table, context_lens, scale, out,
                           max_context_len=max_context_len, partition_tokens=partition_tokens, workspace=workspace,
                           stream=stream)
    result = call()
    _hold(stream, result, call.workspace)
    return result


def bind_read_kv_fp8(k_cache, v_cache, kv_scale, block_table, context_lens, row_start, k_out, v_out, *,
                     max_context_len: int, first_token=None, stream=None) -> DeviceCall:
    """pda_read_kv_fp8 bound to these tensors and the given (else the current)
    stream: tokens first_token[b], ... (from 0 without it) of every sequence into
    rows row_start[b] .. row_start[b + 1] - 1 of k_out and v_out (bf16
    [rows][Hkv][D]).  Calling it returns (k_out, v_out)."""
    import torch

    NB, Hkv, D = _check_fp8_cache(k_cache, v_cache, kv_scale)
    B = block_table.shape[0]
    _check_paged(block_table, context_lens, B)
    _require("row_start", row_start, torch.int32)
    if row_start.shape != (B + 1,):
        raise ValueError("row_start must be [B + 1]")
    if first_token is not None:
        _require("first_token", first_token, torch.int32)
        if first_token.shape != (B,):
            raise ValueError("first_token must be [B]")
    _require("k_out", k_out, torch.bfloat16)
    _require("v_out", v_out, torch.bfloat16)
    if k_out.dim() != 3 or tuple(k_out.shape[1:]) != (Hkv, D) or v_out.shape != k_out.shape:
        raise ValueError("k_out and v_out must be [rows][Hkv][D]")
    device = _same_device(k_cache, v_cache, kv_scale, block_table, context_lens, row_start, first_token, k_out, v_out)
    prob = make_problem(B, Hkv, Hkv, D, NB, block_table.shape[1], max_context_len)
    args = (ctypes.byref(prob), k_cache.data_ptr(), v_cache.data_ptr(), kv_scale.data_ptr(), block_table.data_ptr(),
            context_lens.data_ptr(), first_token.data_ptr() if first_token is not None else None, row_start.data_ptr(),
            k_out.shape[0], k_out.data_ptr(), v_out.data_ptr(), _stream_handle(stream, device))
    keep = (prob, k_cache, v_cache, kv_scale, block_table, context_lens, first_token, row_start, k_out, v_out)
    return DeviceCall("pda_read_kv_fp8", args, keep, device, (k_out, v_out))


def pda_read_kv_fp8(k_cache, v_cache, kv_scale, block_table, context_lens, row_start, k_out, v_out, *,
                    max_context_len: int, first_token=None, stream=None):
    """Rows of the 8-bit cache back as contiguous bf16.  See bind_read_kv_fp8."""
    return bind_read_kv_fp8(k_cache, v_cache, kv_scale, block_table, context_lens, row_start, k_out, v_out,
                            max_context_len=max_context_len, first_token=first_token, stream=stream)()


# ---- head norms, rotary positions with several axes, the append through a slot map
# (include/pda_norm_rotary.h) ----

def make_head_norm(q_weight=None, k_weight=None, eps: float = 1e-6, weight_offset: float = 0.0) -> pda_head_norm:
    """The norms of query and key heads: x / sqrt(mean x^2 + eps) * (weight +
    weight_offset).  Weights are bf16 or float32 device tensors [D], both of one type; None:
    no weights.  The result keeps them alive."""
    import torch

    given = [w for w in (q_weight, k_weight) if w is not None]
    for w in given:
        if w.dtype not in (torch.bfloat16, torch.float32) or w.dtype != given[0].dtype:
            raise TypeError("the weights must be bfloat16 or float32, both the same")
        _require("weight", w, w.dtype)
        if w.dim() != 1:
            raise ValueError("the weights must be [D]")
    f32 = bool(given) and given[0].dtype == torch.float32
    norm = pda_head_norm(float(eps), float(weight_offset), PDA_DTYPE_F32 if f32 else PDA_DTYPE_BF16,
                         q_weight.data_ptr() if q_weight is not None else None,
                         k_weight.data_ptr() if k_weight is not None else None)
    norm.tensors = (q_weight, k_weight)
    return norm


def make_rotary_axes(axis_of_pair, num_axes: int) -> pda_rotary_axes:
    """Positions on several axes: pair i turns by the position on axis
    axis_of_pair[i] (uint8 device tensor [rotary_dim / 2], kept alive by the result)."""
    import torch

    _require("axis_of_pair", axis_of_pair, torch.uint8)
    if axis_of_pair.dim() != 1:
        raise ValueError("axis_of_pair must be [rotary_dim / 2]")
    axes = pda_rotary_axes(int(num_axes), axis_of_pair.data_ptr(), 0)
    axes.tensor = axis_of_pair
    return axes


def _head_call(positions, T, D, norm, rotary, axes):
    """Checks what the calls below share; returns (pointers to norm, rotary and axes,
    their tensors, what has to stay alive)."""
    import torch

    if T > 0x7fffffff:
        raise ValueError("more than 2^31 - 1 tokens")
    if positions.dtype != torch.int32:
        raise TypeError(f"positions must be torch.int32, got {positions.dtype}")
    if not positions.is_cuda:
        raise ValueError("positions must be a device tensor")
    tensors = [positions]
    if norm is not None:
        for w in norm.tensors:
            if w is not None and w.shape != (D,):
                raise ValueError(f"the norms' weights must be [{D}]")
        tensors += [w for w in norm.tensors if w is not None]
    if rotary is not None:
        tensors.append(rotary.tensor)
    if axes is None:
        if positions.shape != (T,) or not positions.is_contiguous():
            raise ValueError("positions must be [T], contiguous")
    else:
        if rotary is None:
            raise ValueError("axes without rotary")
        if axes.tensor.shape != rotary.tensor.shape:
            raise ValueError("axis_of_pair must be [rotary_dim / 2]")
        if positions.shape != (axes.num_axes, T) or (T > 1 and positions.stride(1) != 1):
            raise ValueError("positions must be [num_axes][T]")
        tensors.append(axes.tensor)
        # (this call's own copy: the stride is that of its positions; that of a single axis is free)
        axes = pda_rotary_axes(axes.num_axes, axes.axis_of_pair, positions.stride(0) if axes.num_axes > 1 else T)
    ref = lambda x: ctypes.byref(x) if x is not None else None
    return [ref(norm), ref(rotary), ref(axes)], tensors, (norm, rotary, axes, positions, tensors)


def _head_rows(q, k):
    import torch

    if q.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError("q must be bfloat16 or float32")
    if q.dim() != 3 or (k is not None and (k.dim() != 3 or k.shape[0] != q.shape[0] or k.shape[2] != q.shape[2])):
        raise ValueError("q [T][Hq][D], k [T][Hkv][D]")
    return PDA_DTYPE_BF16 if q.dtype == torch.bfloat16 else PDA_DTYPE_F32


def _row_args(pairs):
    """Pointers and token strides of (name, rows or None, dtype), ..."""
    out = []
    for name, t, dtype in pairs:
        out += [None, 0] if t is None else [t.data_ptr(), _token_rows(name, t, dtype)]
    return out


def bind_norm_rotary(q, positions, k=None, norm: pda_head_norm = None, rotary: pda_rotary = None,
                     axes: pda_rotary_axes = None, q_out=None, k_out=None, stream=None) -> DeviceCall:
    """pda_norm_rotary bound to these tensors and the given (else the current)
    stream; calling it returns (q_out, k_out).  q [T][Hq][D] and k [T][Hkv][D] are
    bf16 or float32 with any token stride; the outputs are allocated when not
    given, and may be the inputs (in place).  positions int32 [T], with `axes`
    [num_axes][T]; negative (on the first axis): padding, left alone."""
    dtype = _head_rows(q, k)
    if k is None and k_out is not None:
        raise ValueError("k_out without k")
    # (padding rows are not written: an output made here holds zeros there)
    q_out = _zeros_like(q, stream) if q_out is None else q_out
    if k is not None and k_out is None:
        k_out = _zeros_like(k, stream)
    if q_out.shape != q.shape or (k is not None and k_out.shape != k.shape):
        raise ValueError("the outputs must have the inputs' shapes")
    T, Hq, D = q.shape
    heads, tensors, keep = _head_call(positions, T, D, norm, rotary, axes)
    device = _same_device(q, q_out, k, k_out, *tensors)
    rows = _row_args([("q", q, q.dtype), ("q_out", q_out, q.dtype), ("k", k, q.dtype), ("k_out", k_out, q.dtype)])
    args = (*heads, T, Hq, 0 if k is None else k.shape[1], D, dtype, positions.data_ptr(), *rows,
            _stream_handle(stream, device))
    return DeviceCall("pda_norm_rotary", args, (keep, q, q_out, k, k_out), device, (q_out, k_out))


def pda_norm_rotary(q, positions, k=None, norm: pda_head_norm = None, rotary: pda_rotary = None,
                    axes: pda_rotary_axes = None, q_out=None, k_out=None, stream=None):
    """Norms and rotary positions of q (and k) rows in one pass; returns (q_out, k_out
    or None).  See bind_norm_rotary."""
    result = bind_norm_rotary(q, positions, k, norm, rotary, axes, q_out, k_out, stream)()
    _hold(stream, *result)
    return result


def pda_norm_rotary_workspace_bytes(num_tokens: int, num_q_heads: int, num_kv_heads: int, head_dim: int) -> int:
    import torch  # noqa: F401  (before the library: its HIP runtime is the one to share)

    ws = ctypes.c_size_t()
    rc = load_library().pda_norm_rotary_workspace_bytes(int(num_tokens), int(num_q_heads), int(num_kv_heads),
                                                        int(head_dim), ctypes.byref(ws))
    if rc != PDA_OK:
        raise PdaError(rc, "pda_norm_rotary_workspace_bytes")
    return ws.value


def _given_workspace(workspace, need, device, stream):
    """(workspace, pointer, bytes): the caller's, or one made here."""
    import torch

    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    if workspace is None and need > 0:
        workspace = _empty((need,), torch.uint8, device, stream, result=False)
    if workspace is None:
        return None, None, 0
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def bind_norm_rotary_backward(q, q_grad, positions, k=None, k_grad=None, norm: pda_head_norm = None,
                              rotary: pda_rotary = None, axes: pda_rotary_axes = None, dq=None, dk=None,
                              dq_weight=None, dk_weight=None, workspace=None, stream=None) -> DeviceCall:
    """pda_norm_rotary_backward bound to these tensors and the given (else the current)
    stream: q and k are the inputs of pda_norm_rotary, q_grad and k_grad the
    gradients of its outputs, `rotary` the forward's.  Calling it returns (dq, dk,
    dq_weight, dk_weight); they are allocated when not given (the weights' gradients, float32
    [D], for the weights that `norm` has).  dq may be q or q_grad, dk k or k_grad."""
    import torch

    dtype = _head_rows(q, k)
    if norm is None:
        raise ValueError("norm must be given (the gradient of the rotation alone: pda_norm_rotary with a backward rotary)")
    if (k is None) != (k_grad is None) or (k is None and (dk is not None or dk_weight is not None)):
        raise ValueError("k and k_grad go together")
    T, Hq, D = q.shape
    dq = _zeros_like(q, stream) if dq is None else dq
    if k is not None and dk is None:
        dk = _zeros_like(k, stream)
    for t, like in ((q_grad, q), (dq, q), (k_grad, k), (dk, k)):
        if t is not None and t.shape != like.shape:
            raise ValueError("gradients must have the rows' shapes")
    if dq_weight is None and norm.tensors[0] is not None:
        dq_weight = _empty((D,), torch.float32, q.device, stream)
    if k is not None and dk_weight is None and norm.tensors[1] is not None:
        dk_weight = _empty((D,), torch.float32, q.device, stream)
    for name, t in (("dq_weight", dq_weight), ("dk_weight", dk_weight)):
        if t is not None:
            _require(name, t, torch.float32)
            if t.shape != (D,):
                raise ValueError(f"{name} must be [{D}]")
    heads, tensors, keep = _head_call(positions, T, D, norm, rotary, axes)
    device = _same_device(q, q_grad, dq, k, k_grad, dk, dq_weight, dk_weight, workspace, *tensors)
    Hkv = 0 if k is None else k.shape[1]
    workspace, ws_ptr, ws_bytes = _given_workspace(workspace, pda_norm_rotary_workspace_bytes(T, Hq, Hkv, D), device, stream)
    rows = _row_args([("q", q, q.dtype), ("q_grad", q_grad, q.dtype), ("dq", dq, q.dtype), ("k", k, q.dtype),
                      ("k_grad", k_grad, q.dtype), ("dk", dk, q.dtype)])
    ptr = lambda t: t.data_ptr() if t is not None else None
    args = (*heads, T, Hq, Hkv, D, dtype, positions.data_ptr(), *rows, ptr(dq_weight), ptr(dk_weight), ws_ptr, ws_bytes,
            _stream_handle(stream, device))
    call = DeviceCall("pda_norm_rotary_backward", args, (keep, q, q_grad, k, k_grad, workspace), device,
                      (dq, dk, dq_weight, dk_weight))
    call.workspace = workspace
    return call


def pda_norm_rotary_backward(q, q_grad, positions, k=None, k_grad=None, norm: pda_head_norm = None,
                             rotary: pda_rotary = None, axes: pda_rotary_axes = None, dq=None, dk=None,
                             dq_weight=None, dk_weight=None, workspace=None, stream=None):
    """The gradient of pda_norm_rotary; returns (dq, dk, dq_weight, dk_weight).  See
    bind_norm_rotary_backward."""
    call = bind_norm_rotary_backward(q, q_grad, positions, k, k_grad, norm, rotary, axes, dq, dk, dq_weight, dk_weight,
                                     workspace, stream)
    result = call()
    _hold(stream, *result, call.workspace)
    return result


def bind_norm_rotary_append(q, k, v, positions, slots, k_cache, v_cache, norm: pda_head_norm = None,
                            rotary: pda_rotary = None, axes: pda_rotary_axes = None, q_out=None,
                            stream=None) -> DeviceCall:
    """pda_norm_rotary_append bound to these tensors and the given (else the current)
    stream: k and v bf16 [T][Hkv][D] (k normed and rotated first) stored at slots[t] =
    16 * block + place of the paged cache (k_cache, v_cache as in pda_decode), q bf16 [T][Hq][D] (or
    None) normed and rotated into q_out (allocated when not given; may be q).  Calling it
    returns q_out (None without q)."""
    import torch

    for name, t in (("k_cache", k_cache), ("v_cache", v_cache)):
        _require(name, t, torch.bfloat16)
    if k_cache.dim() != 5 or tuple(k_cache.shape[3:]) != (16, 8):
        raise ValueError("k_cache must be [num_blocks][Hkv][D/8][16][8]")
    NB, Hkv, C = k_cache.shape[:3]
    if tuple(v_cache.shape) != (NB, Hkv, 16, 8 * C):
        raise ValueError("v_cache must be [num_blocks][Hkv][16][D]")
    for name, t in (("k", k), ("v", v), ("q", q)):
        if t is not None and (t.dim() != 3 or t.shape[0] != k.shape[0] or t.shape[2] != 8 * C):
            raise ValueError(f"{name} must be [T][heads][{8 * C}]")
    if k.shape[1] != Hkv or v.shape[1] != Hkv:
        raise ValueError("k, v and the caches disagree on the heads")
    if q is None and q_out is not None:
        raise ValueError("q_out without q")
    if q is not None and norm is None and rotary is None:
        raise ValueError("q without norm and rotary has nothing to be done to it")
    if q is not None:
        q_out = _zeros_like(q, stream) if q_out is None else q_out
        if q_out.shape != q.shape:
            raise ValueError("q_out must have the shape of q")
    T, _, D = k.shape
    _require("slots", slots, torch.int32)
    if slots.shape != (T,):
        raise ValueError("slots must be [T]")
    heads, tensors, keep = _head_call(positions, T, D, norm, rotary, axes)
    device = _same_device(q, q_out, k, v, slots, k_cache, v_cache, *tensors)
    bf = torch.bfloat16
    rows = _row_args([("q", q, bf), ("q_out", q_out, bf), ("k", k, bf), ("v", v, bf)])
    args = (*heads, T, 0 if q is None else q.shape[1], Hkv, D, NB, positions.data_ptr(), slots.data_ptr(), *rows,
            k_cache.data_ptr(), v_cache.data_ptr(), _stream_handle(stream, device))
    return DeviceCall("pda_norm_rotary_append", args, (keep, q, q_out, k, v, slots, k_cache, v_cache), device, q_out)


def pda_norm_rotary_append(q, k, v, positions, slots, k_cache, v_cache, norm: pda_head_norm = None,
                           rotary: pda_rotary = None, axes: pda_rotary_axes = None, q_out=None, stream=None):
    """Norms and rotary positions of packed tokens, their keys and values stored in the
    paged cache; returns q_out (None without q).  See bind_norm_rotary_append."""
    result = bind_norm_rotary_append(q, k, v, positions, slots, k_cache, v_cache, norm, rotary, axes, q_out, stream)()
    _hold(stream, result)
    return result


# ---- attention with a sliding window and sinks (include/pda_window.h) ----

def pda_plan_window(prob: pda_problem, window: int, sinks: int = 0) -> dict:
    """The plan of pda_decode_window: partition_tokens, num_partitions, workspace_bytes."""
    import torch  # noqa: F401  (before the library: its HIP runtime is the one to share)

    info, w = pda_plan_info(), pda_window(int(window), int(sinks))
    rc = load_library().pda_plan_window(ctypes.byref(prob), ctypes.byref(w), ctypes.byref(info))
    if rc != PDA_OK:
        raise PdaError(rc, "pda_plan_window")
    return info.as_dict()


def bind_decode_window(q, k_cache, v_cache, block_table, context_lens, scale: float, out=None, *, window: int,
                       sinks: int = 0, max_context_len: int, partition_tokens: int = 0, workspace=None,
                       stream=None) -> DeviceCall:
    """pda_decode_window bound to these tensors and the given (else the current) stream:
    the attention of bind_decode, of new tokens that see the last `window` tokens up to
    their own, and the first `sinks`.  The other arguments are those of bind_decode
    (`workspace`: pda_plan_window's workspace_bytes)."""
    import torch

    if out is None:
        out = _empty(q.shape, torch.float32, q.device, stream)
    if q.dim() == 4 and q.shape[1] == 0:
        raise ValueError("at least one new token")
    prob = _problem_from(q, k_cache, block_table, max_context_len, partition_tokens)
    _check_tensors(q, k_cache, v_cache, block_table, context_lens, out)
    device = _same_device(q, k_cache, v_cache, block_table, context_lens, out, workspace)
    need = pda_plan_window(prob, window, sinks)["workspace_bytes"]
    workspace, ws_ptr, ws_bytes = _given_workspace(workspace, need, device, stream)
    w = pda_window(int(window), int(sinks))
    args = (ctypes.byref(prob), ctypes.byref(w), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
            block_table.data_ptr(), context_lens.data_ptr(), ctypes.c_float(scale), out.data_ptr(), ws_ptr, ws_bytes,
            _stream_handle(stream, device))
    keep = (prob, w, q, k_cache, v_cache, block_table, context_lens, out, workspace)
    call = DeviceCall("pda_decode_window", args, keep, device, out)
    call.workspace = workspace
    return call


def pda_decode_window(q, k_cache, v_cache, block_table, context_lens, scale: float, out=None, *, window: int,
                      sinks: int = 0, max_context_len: int, partition_tokens: int = 0, workspace=None, stream=None):
    """One attention step with a sliding window and sinks; returns out (fp32, shaped like
    q).  See bind_decode_window."""
    call = bind_decode_window(q, k_cache, v_cache, block_table, context_lens, scale, out, window=window, sinks=sinks,
                              max_context_len=max_context_len, partition_tokens=partition_tokens, workspace=workspace,
                              stream=stream)
    result = call()
    _hold(stream, result, call.workspace)
    return result


# ---- block tables and slot maps on the GPU (include/pda_blocks.h) ----

def make_block_pool(block_table, held, free_blocks, counts) -> pda_block_pool:
    """A block pool of these int32 device tensors: block_table [num_seqs][max_blocks],
    held [num_seqs], free_blocks [num_blocks] and counts [2] (include/pda_blocks.h); they are kept
    alive by the result (`tensors`) and changed in place by pda_blocks_resize."""
    import torch

    for name, t in (("block_table", block_table), ("held", held), ("free_blocks", free_blocks), ("counts", counts)):
        _require(name, t, torch.int32)
    if block_table.dim() != 2 or held.shape != (block_table.shape[0],) or free_blocks.dim() != 1 or counts.shape != (2,):
        raise ValueError("block_table [num_seqs][max_blocks], held [num_seqs], free_blocks [num_blocks], counts [2]")
    pool = pda_block_pool(block_table.shape[0], free_blocks.shape[0], block_table.shape[1], block_table.data_ptr(),
                          held.data_ptr(), free_blocks.data_ptr(), counts.data_ptr())
    pool.tensors = (block_table, held, free_blocks, counts)
    return pool


def new_block_pool(num_seqs: int, num_blocks: int, max_blocks_per_seq: int, device="cuda") -> pda_block_pool:
    """A pool whose rows hold nothing (entries -1) and whose blocks are all free,
    block 0 on top of the stack."""
    import torch

    i32 = dict(dtype=torch.int32, device=device)
    return make_block_pool(torch.full((num_seqs, max_blocks_per_seq), -1, **i32), torch.zeros(num_seqs, **i32),
                           torch.arange(num_blocks - 1, -1, -1, **i32), torch.tensor([num_blocks, 0], **i32))


def _token_map(num_seqs, row_start, positions, slots):
    """(pda_token_rows or None, its tensors) of a slot map's tensors."""
    import torch

    given = [t for t in (positions, slots) if t is not None]
    if not given:
        if row_start is not None:
            raise ValueError("row_start without positions or slots")
        return None, ()
    n = given[0].shape[0] if given[0].dim() == 1 else -1
    for name, t in (("positions", positions), ("slots", slots)):
        if t is not None:
            _require(name, t, torch.int32)
            if t.shape != (n,):
                raise ValueError("positions and slots must be [num_rows], both the same")
    if n > 0x7fffffff:
        raise ValueError("more than 2^31 - 1 rows")
    if row_start is not None:
        _require("row_start", row_start, torch.int32)
        if row_start.shape != (num_seqs + 1,):
            raise ValueError("row_start must be [num_seqs + 1]")
    ptr = lambda t: t.data_ptr() if t is not None else None
    return pda_token_rows(n, ptr(row_start), ptr(positions), ptr(slots)), (row_start, positions, slots)


def _check_lens(context_lens, num_seqs):
    import torch

    _require("context_lens", context_lens, torch.int32)
    if context_lens.shape != (num_seqs,):
        raise ValueError("context_lens must be [num_seqs]")


def bind_blocks_resize(pool: pda_block_pool, context_lens, row_start=None, positions=None, slots=None, workspace=None,
                       stream=None) -> DeviceCall:
    """pda_blocks_resize bound to a pool (make_block_pool), lengths int32 [num_seqs] and the given
    (else the current) stream: every row grown or shrunk to hold its length.  With positions
    and/or slots (int32 [num_rows]) the slot map of the new tokens is written to them: row_start int32
    [num_seqs + 1] says whose they are, None: the same number of every sequence.  `workspace`: uint8 zeros
    of pda_blocks_workspace_bytes, allocated here when not given.  Calling it returns
    (block_table, positions, slots).  Where blocks may run short, attention takes the lengths
    torch.where(16 * held < context_lens, 0, context_lens): a row that was not granted its blocks names
    others' in the entries that it does not hold."""
    import torch

    _check_lens(context_lens, pool.num_seqs)
    rows, tensors = _token_map(pool.num_seqs, row_start, positions, slots)
    device = _same_device(*pool.tensors, context_lens, workspace, *tensors)
    ws = ctypes.c_size_t()
    rc = load_library().pda_blocks_workspace_bytes(ctypes.byref(pool), ctypes.byref(ws))
    if rc != PDA_OK:
        raise PdaError(rc, "pda_blocks_workspace_bytes")
    if workspace is None and ws.value > 0:
        workspace = _cleared(_empty((ws.value,), torch.uint8, device, stream, result=False), stream)
    workspace, ws_ptr, ws_bytes = _given_workspace(workspace, ws.value, device, stream)
    args = (ctypes.byref(pool), context_lens.data_ptr(), ctypes.byref(rows) if rows is not None else None, ws_ptr,
            ws_bytes, _stream_handle(stream, device))
    call = DeviceCall("pda_blocks_resize", args, (pool, context_lens, rows, tensors, workspace), device,
                      (pool.tensors[0], positions, slots))
    call.workspace = workspace
    return call


def pda_blocks_resize(pool: pda_block_pool, context_lens, row_start=None, positions=None, slots=None, workspace=None,
                      stream=None):
    """Resizes a pool's rows for these lengths, in place, and writes the slot map of the
    new tokens; returns (block_table, positions, slots).  See bind_blocks_resize."""
    call = bind_blocks_resize(pool, context_lens, row_start, positions, slots, workspace, stream)
    result = call()
    _hold(stream, call.workspace)
    return result


def bind_slot_map(block_table, context_lens, num_blocks: int, row_start=None, positions=None, slots=None,
                  stream=None) -> DeviceCall:
    """pda_slot_map bound to these tensors and the given (else the current) stream: the
    positions and slots of the new tokens of a block table however it was made.  Calling it returns
    (positions, slots)."""
    import torch

    _require("block_table", block_table, torch.int32)
    if block_table.dim() != 2:
        raise ValueError("block_table must be [num_seqs][max_blocks]")
    B, width = block_table.shape
    _check_lens(context_lens, B)
    rows, tensors = _token_map(B, row_start, positions, slots)
    if rows is None:
        raise ValueError("positions or slots must be given")
    device = _same_device(block_table, context_lens, *tensors)
    args = (B, int(num_blocks), width, block_table.data_ptr(), context_lens.data_ptr(), ctypes.byref(rows),
            _stream_handle(stream, device))
    return DeviceCall("pda_slot_map", args, (block_table, context_lens, rows, tensors), device, (positions, slots))


def pda_slot_map(block_table, context_lens, num_blocks: int, row_start=None, positions=None, slots=None, stream=None):
    """Positions and slots of new tokens; returns (positions, slots).  See bind_slot_map."""
    return bind_slot_map(block_table, context_lens, num_blocks, row_start, positions, slots, stream)()
