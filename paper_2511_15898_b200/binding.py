"""ctypes binding of libgr_b200.so.

Argument marshalling only: every step of the path runs in the CUDA kernels behind
the C interface (include/gr.h).  The low-level functions carry the C names and take
raw device pointers; `solve`, `verify` and `read_rule` accept torch CUDA tensors and
pass their data pointers and the current stream.  There is no CPU fallback: without
the compiled library or without a CUDA device these functions raise.
"""
from __future__ import annotations

import array
import ctypes as C
import dataclasses
import importlib
import os
from typing import Optional, Tuple

import torch

GR_F32, GR_BF16 = 0, 1
GR_F16, GR_Q4 = 2, 3
GR_OK, GR_NOT_CONVERGED, GR_SUPPORT_TOO_LARGE, GR_BAD_LOGITS, GR_DRAFT_OUT_OF_SUPPORT, GR_STALE_PARAMS = range(6)
GR_MAX_SUPPORT, GR_MAX_DRAFTS = 128, 32
GR_STATIC_MAX_BATCH = 256
GR_PARTIAL_RULE = 6
GR_NO_BLOCKS, GR_ROW_FULL, GR_BAD_ROW = 8, 9, 10
GR_MAX_BEAMS, GR_MAX_SELECT = 32, 128
GR_MAX_GIVEN, GR_MAX_HEADS, GR_MAX_DIM, GR_MAX_DIM_Q4 = 64, 1024, 512, 256
_NULL = -2                 # a required pointer is NULL

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libgr_b200.so")
_lib = None
_entry = {}                # addresses of entry points, for _tensors


def _load_tensors():
    """The compiled module beside the library, or None: then every call goes the way in Python.  (With the library and not with the
    package, so that a process that only imports the package neither maps it nor misses one that is built later.)"""
    importlib.invalidate_caches()
    try:
        from . import _tensors as module
    except ImportError:
        return None
    return module if getattr(module, "torch_version", None) == torch.__version__ else None


def __getattr__(name):
    if name == "_tensors":               # (before the library is loaded)
        return _load_tensors()
    raise AttributeError(name)


class GrError(RuntimeError):
    pass


class Options(C.Structure):
    _fields_ = [("tol", C.c_double), ("max_iters", C.c_int), ("quad_step", C.c_double),
                ("scan_done_event", C.c_void_p), ("force_robust", C.c_int), ("tau", C.c_double)]

    def __init__(self, tol: float = 3e-7, max_iters: int = 40, quad_step: float = 0.4, scan_done_event=None,
                 force_robust: int = 0, tau: float = 0.0):
        super().__init__(tol, max_iters, quad_step, scan_done_event, force_robust, tau)


class StateLayout(C.Structure):
    """gr_state_layout: where the pieces of a state lie, in bytes."""
    _fields_ = ([(n, C.c_int) for n in ("batch", "beams_in", "beams_out", "parts")]
                + [(n, C.c_longlong) for n in ("src_group", "src_beam", "src_part", "dst_group", "dst_beam", "dst_part",
                                               "part_bytes", "token_bytes")])


class CacheLayout(C.Structure):
    """gr_cache_layout: where a cache keeps a slot's heads (strides in elements; of a 4-bit cache block_stride alone, in bytes)."""
    _fields_ = ([(n, C.c_int) for n in ("format", "heads", "dim", "block_size", "num_blocks")]
                + [(n, C.c_longlong) for n in ("block_stride", "token_stride", "head_stride")])


class CacheTokens(C.Structure):
    """gr_cache_tokens: new tokens' keys, values and queries (strides in elements)."""
    _fields_ = ([(n, C.c_void_p) for n in ("k", "v", "q", "q_out")] + [(n, C.c_int) for n in ("dtype", "q_heads")]
                + [(n, C.c_longlong) for n in ("k_token", "k_head", "v_token", "v_head", "q_token", "q_head", "out_token", "out_head")])


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """dlopen the compiled library (built by paper_2511_15898_b200.build); raises if it is missing."""
    global _lib
    global _tensors
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise GrError(f"{_LIB_PATH} is missing: build it with `python -m paper_2511_15898_b200.build`")
    lib = C.CDLL(_LIB_PATH)
    vp, ip, fp, dp = C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p
    lib.gr_params_bytes.restype = C.c_size_t
    lib.gr_params_bytes.argtypes = [C.c_int] * 4
    lib.gr_workspace_bytes.restype = C.c_size_t
    lib.gr_workspace_bytes.argtypes = [C.c_int] * 4
    lib.gr_solve.restype = C.c_int
    lib.gr_solve.argtypes = [vp, vp, C.c_int, C.c_int, C.c_int, C.c_int, C.c_float, C.c_float, C.c_int,
                             C.POINTER(Options), vp, vp, fp, ip, vp]
    lib.gr_solve_static.restype = C.c_int
    lib.gr_solve_static.argtypes = [vp, vp, C.c_int, C.c_int, C.c_int, C.c_int, C.c_float, C.c_float, C.c_int,
                                    C.POINTER(Options), vp, fp, ip, vp]
    lib.gr_solve_verify.restype = C.c_int
    lib.gr_solve_verify.argtypes = [vp, vp, C.c_int, C.c_int, C.c_int, C.c_int, C.c_float, C.c_float, C.c_int,
                                    C.POINTER(Options), ip, fp, vp, vp, fp, ip, vp, ip, vp]
    lib.gr_alpha_star.restype = C.c_int
    lib.gr_alpha_star.argtypes = [vp, vp, C.c_int, C.c_int, ip, C.c_int, C.c_int, C.c_float, C.c_float, C.c_int, vp,
                                  fp, ip, vp]
    lib.gr_verify.restype = C.c_int
    lib.gr_verify.argtypes = [vp, ip, fp, C.c_int, ip, vp, ip, vp]
    lib.gr_read_rule.restype = C.c_int
    lib.gr_read_rule.argtypes = [vp, C.c_int, C.c_int, ip, ip, dp, dp, dp, dp, vp]
    lib.gr_read_slice.restype = C.c_int
    lib.gr_read_slice.argtypes = [vp, ip, C.c_int, C.c_int, ip, dp, dp, ip, vp]
    lib.gr_beam_workspace_bytes.restype = C.c_size_t
    lib.gr_beam_workspace_bytes.argtypes = [C.c_int] * 4
    lib.gr_beam_select.restype = C.c_int
    lib.gr_beam_select.argtypes = [vp, C.c_int, C.c_int, C.c_longlong, C.c_int, C.c_int, C.c_float, fp, ip, vp, C.c_int,
                                   C.c_float, C.c_int, vp, ip, ip, fp, ip, vp, ip, vp]
    lib.gr_reorder_states.restype = C.c_int
    lib.gr_reorder_states.argtypes = [vp, vp, C.c_int, C.POINTER(StateLayout), ip, ip, vp]
    lib.gr_block_workspace_bytes.restype = C.c_size_t
    lib.gr_block_workspace_bytes.argtypes = [C.c_int] * 2
    lib.gr_block_plan.restype = C.c_int
    lib.gr_block_plan.argtypes = [ip, C.c_int, C.c_int, C.c_int, C.c_int, ip, ip, C.c_int, ip, ip, ip, C.c_int, vp, vp, ip,
                                  ip, ip, ip, ip, vp]
    lib.gr_copy_blocks.restype = C.c_int
    lib.gr_copy_blocks.argtypes = [vp, C.c_int, C.c_int, C.c_longlong, C.c_longlong, ip, ip, C.c_int, vp]
    lib.gr_cache_append.restype = C.c_int
    lib.gr_cache_append.argtypes = [vp, vp, C.POINTER(CacheLayout), C.POINTER(CacheTokens), C.c_int, vp, ip, dp, C.c_int, C.c_int, vp]
    lib.gr_cache_read.restype = C.c_int
    lib.gr_cache_read.argtypes = [vp, vp, C.POINTER(CacheLayout), vp, C.c_int, C.c_int, vp, C.c_longlong, C.c_longlong, vp,
                                  C.c_longlong, C.c_longlong, vp]
    lib.gr_attend_workspace_bytes.restype = C.c_size_t
    lib.gr_attend_workspace_bytes.argtypes = [C.c_int] * 5
    lib.gr_cache_attend.restype = C.c_int
    lib.gr_cache_attend.argtypes = [vp, C.c_int, C.c_int, C.c_longlong, C.c_longlong, vp, C.POINTER(CacheLayout), ip, C.c_int, C.c_int, ip,
                                    ip, C.c_int, C.c_float, C.c_int, vp, vp, C.c_longlong, C.c_longlong, ip, vp]
    lib.gr_token_logprobs.restype = C.c_int
    lib.gr_token_logprobs.argtypes = [vp, C.c_int, C.c_int, C.c_longlong, C.c_int, C.c_float, ip, C.c_int, C.c_int, fp, fp, ip, fp, ip, vp]
    lib.gr_strerror.restype = C.c_char_p
    lib.gr_strerror.argtypes = [C.c_int]
    _entry.update({n: C.cast(getattr(lib, n), C.c_void_p).value
                   for n in ("gr_beam_select", "gr_reorder_states", "gr_block_plan", "gr_copy_blocks", "gr_cache_append", "gr_cache_read",
                             "gr_cache_attend", "gr_attend_workspace_bytes", "gr_token_logprobs")})
    _lib = lib
    if "_tensors" not in globals():
        _tensors = _load_tensors()
    return lib


# ---------------------------------------------------------------- C names, raw pointers

def gr_params_bytes(V: int, n: int, topk: int, batch: int) -> int:
    return int(load_library().gr_params_bytes(V, n, topk, batch))


def gr_workspace_bytes(V: int, n: int, topk: int, batch: int) -> int:
    return int(load_library().gr_workspace_bytes(V, n, topk, batch))


def gr_strerror(code: int) -> str:
    return load_library().gr_strerror(int(code)).decode()


def gr_solve(q_logits: int, p_logits: int, dtype: int, V: int, n: int, topk: int, temp_target: float,
             temp_draft: float, batch: int, opt: Optional[Options], params: int, workspace: int, alpha_star: int,
             status: int, stream: int) -> int:
    return int(load_library().gr_solve(q_logits, p_logits, dtype, V, n, topk, temp_target, temp_draft, batch,
                                       C.byref(opt) if opt is not None else None, params, workspace, alpha_star,
                                       status, stream))


def gr_solve_static(q_logits: int, p_logits: int, dtype: int, V: int, n: int, topk: int, temp_target: float,
                    temp_draft: float, batch: int, opt: Optional[Options], params: int, alpha_star: int, status: int,
                    stream: int) -> int:
    """gr_solve with the scratch inside the library (at most GR_STATIC_MAX_BATCH instances): for callers that
    must not allocate device memory.  Calls that overlap on the GPU share that scratch and race."""
    return int(load_library().gr_solve_static(q_logits, p_logits, dtype, V, n, topk, temp_target, temp_draft, batch,
                                              C.byref(opt) if opt is not None else None, params, alpha_star, status,
                                              stream))


def gr_solve_verify(q_logits: int, p_logits: int, dtype: int, V: int, n: int, topk: int, temp_target: float,
                    temp_draft: float, batch: int, opt: Optional[Options], draft_tokens: int, uniforms: int,
                    params: int, workspace: int, alpha_star: int, out_token: int, out_accepted: int, status: int,
                    stream: int) -> int:
    return int(load_library().gr_solve_verify(q_logits, p_logits, dtype, V, n, topk, temp_target, temp_draft, batch,
                                              C.byref(opt) if opt is not None else None, draft_tokens, uniforms,
                                              params, workspace, alpha_star, out_token, out_accepted, status, stream))


def gr_alpha_star(q_logits: int, p_logits: int, dtype: int, V: int, n_list, topk: int, temp_target: float,
                  temp_draft: float, batch: int, workspace: int, alpha_star: int, status: int, stream: int) -> int:
    ns = (C.c_int * len(n_list))(*[int(x) for x in n_list])
    return int(load_library().gr_alpha_star(q_logits, p_logits, dtype, V, ns, len(n_list), topk, temp_target,
                                            temp_draft, batch, workspace, alpha_star, status, stream))


def gr_verify(params: int, draft_tokens: int, uniforms: int, batch: int, out_token: int, out_accepted: int,
              status: int, stream: int) -> int:
    return int(load_library().gr_verify(params, draft_tokens, uniforms, batch, out_token, out_accepted, status,
                                        stream))


def gr_read_rule(params: int, batch: int, kcap: int, ids: int, block: int, w: int, resid: int, flow: int,
                 header: int, stream: int) -> int:
    return int(load_library().gr_read_rule(params, batch, kcap, ids, block, w, resid, flow, header, stream))


def gr_read_slice(params: int, draft_tokens: int, batch: int, n: int, U: int, pi: int, rho: int, status: int,
                  stream: int) -> int:
    return int(load_library().gr_read_slice(params, draft_tokens, batch, n, U, pi, rho, status, stream))


def gr_beam_workspace_bytes(V: int, beams: int, select: int, batch: int) -> int:
    return int(load_library().gr_beam_workspace_bytes(V, beams, select, batch))


def gr_beam_select(logits: int, dtype: int, V: int, ld: int, beams: int, batch: int, temperature: float, scores: int,
                   lengths: int, done: int, eos: int, length_penalty: float, select: int, workspace: int, out_token: int,
                   out_parent: int, out_score: int, out_length: int, out_done: int, status: int, stream: int) -> int:
    return int(load_library().gr_beam_select(logits, dtype, V, ld, beams, batch, temperature, scores, lengths, done, eos,
                                             length_penalty, select, workspace, out_token, out_parent, out_score,
                                             out_length, out_done, status, stream))


def gr_reorder_states(src, dst, layout: Optional[StateLayout], parents: int, lengths: int, stream: int) -> int:
    """src, dst: sequences of device addresses (or bytes that hold them, 64 bits each)."""
    if len(src) != len(dst):
        raise GrError("src and dst: one address each for every state")
    a = src if isinstance(src, bytes) else array.array("Q", src).tobytes()
    b = dst if isinstance(dst, bytes) else array.array("Q", dst).tobytes()
    return load_library().gr_reorder_states(a, b, len(a) // 8, C.byref(layout) if layout is not None else None, parents,
                                            lengths, stream)


def gr_block_workspace_bytes(rows: int, num_blocks: int) -> int:
    return int(load_library().gr_block_workspace_bytes(rows, num_blocks))


def gr_block_plan(table: int, rows: int, width: int, beams: int, block_size: int, lengths: int, refs: int,
                  num_blocks: int, parents: int, keep: int, append: int, max_tokens: int, workspace: int, slots: int,
                  positions: int, offsets: int, copy_src: int, copy_dst: int, status: int, stream: int) -> int:
    return int(load_library().gr_block_plan(table, rows, width, beams, block_size, lengths, refs, num_blocks, parents,
                                            keep, append, max_tokens, workspace, slots, positions, offsets, copy_src,
                                            copy_dst, status, stream))


def gr_copy_blocks(caches, num_blocks: int, block_stride: int, block_bytes: int, copy_src: int, copy_dst: int,
                   pairs: int, stream: int) -> int:
    """caches: a sequence of device addresses (or bytes that hold them, 64 bits each)."""
    a = caches if isinstance(caches, bytes) else array.array("Q", caches).tobytes()
    return load_library().gr_copy_blocks(a, len(a) // 8, num_blocks, block_stride, block_bytes, copy_src, copy_dst, pairs,
                                         stream)


def gr_cache_append(keys: int, values: int, layout: Optional[CacheLayout], tokens_in: Optional[CacheTokens], tokens: int, slots: int,
                    positions: int, frequencies: int, rot: int, interleaved: int, stream: int) -> int:
    return load_library().gr_cache_append(keys, values, C.byref(layout) if layout is not None else None,
                                          C.byref(tokens_in) if tokens_in is not None else None, tokens, slots, positions,
                                          frequencies, rot, interleaved, stream)


def gr_cache_read(keys: int, values: int, layout: Optional[CacheLayout], slots: int, tokens: int, dtype: int, k: int, k_token: int,
                  k_head: int, v: int, v_token: int, v_head: int, stream: int) -> int:
    return load_library().gr_cache_read(keys, values, C.byref(layout) if layout is not None else None, slots, tokens, dtype, k,
                                        k_token, k_head, v, v_token, v_head, stream)


def gr_attend_workspace_bytes(heads: int, q_heads: int, dim: int, rows: int, tokens: int) -> int:
    return int(load_library().gr_attend_workspace_bytes(heads, q_heads, dim, rows, tokens))


def gr_cache_attend(q: int, dtype: int, q_heads: int, q_token: int, q_head: int, cache: int, layout: Optional[CacheLayout], table: int,
                    width: int, rows: int, offsets: int, positions: int, tokens: int, scale: float, window: int, workspace: int, out: int,
                    out_token: int, out_head: int, status: int, stream: int) -> int:
    return load_library().gr_cache_attend(q, dtype, q_heads, q_token, q_head, cache, C.byref(layout) if layout is not None else None,
                                          table, width, rows, offsets, positions, tokens, scale, window, workspace, out, out_token,
                                          out_head, status, stream)


def gr_token_logprobs(logits: int, dtype: int, V: int, ld: int, rows: int, temperature: float, tokens: int, given: int, top: int,
                      logprob: int, entropy: int, top_token: int, top_logprob: int, status: int, stream: int) -> int:
    return load_library().gr_token_logprobs(logits, dtype, V, ld, rows, temperature, tokens, given, top, logprob, entropy, top_token,
                                            top_logprob, status, stream)


# ---------------------------------------------------------------- torch tensors

def _check(rc: int, what: str):
    if rc != 0:
        raise GrError(f"{what}: {gr_strerror(rc)} ({rc})")


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return GR_F32
    if t.dtype == torch.bfloat16:
        return GR_BF16
    raise GrError("logits must be float32 or bfloat16")


def _stream() -> int:
    return int(torch.cuda.current_stream().cuda_stream)


def _need_cuda(*ts):
    for t in ts:
        if not (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous()):
            raise GrError("expected contiguous CUDA tensors")


@dataclasses.dataclass
class Solved:
    """Device-side result of gr_solve: the opaque params block and the per-instance outputs."""
    V: int
    n: int
    topk: int
    batch: int
    params: torch.Tensor       # uint8, opaque
    workspace: torch.Tensor    # uint8, scratch
    alpha_star: torch.Tensor   # [B] float32
    status: torch.Tensor       # [B] int32
    q_logits: torch.Tensor     # kept alive: gr_verify re-reads one chunk of a row on the resample branch


def solve(q_logits: torch.Tensor, p_logits: torch.Tensor, n: int, topk: int, temp_target: float = 1.0,
          temp_draft: float = 1.0, opt: Optional[Options] = None, out: Optional[Solved] = None) -> Solved:
    """gr_solve on torch CUDA tensors ([B, V] float32 or bfloat16), on the current stream."""
    _need_cuda(q_logits, p_logits)
    if q_logits.shape != p_logits.shape or q_logits.dim() != 2 or q_logits.dtype != p_logits.dtype:
        raise GrError("q_logits and p_logits must be [B, V] tensors of one dtype")
    B, V = q_logits.shape
    dev = q_logits.device
    if out is None or out.batch != B or out.V != V or out.n != n or out.topk != topk:
        pbytes = gr_params_bytes(V, n, topk, B)
        wbytes = gr_workspace_bytes(V, n, topk, B)
        if pbytes == 0 or wbytes == 0:
            raise GrError("invalid shape")
        out = Solved(V, n, topk, B,
                     torch.empty(pbytes, dtype=torch.uint8, device=dev),
                     torch.empty(wbytes, dtype=torch.uint8, device=dev),
                     torch.empty(B, dtype=torch.float32, device=dev),
                     torch.empty(B, dtype=torch.int32, device=dev), q_logits)
    out.q_logits = q_logits
    rc = gr_solve(q_logits.data_ptr(), p_logits.data_ptr(), _dtype_code(q_logits), V, n, topk, temp_target,
                  temp_draft, B, opt, out.params.data_ptr(), out.workspace.data_ptr(), out.alpha_star.data_ptr(),
                  out.status.data_ptr(), _stream())
    _check(rc, "gr_solve")
    return out


@dataclasses.dataclass
class Verified:
    token: torch.Tensor      # [B] int32
    accepted: torch.Tensor   # [B] uint8
    status: torch.Tensor     # [B] int32


def verify(solved: Solved, draft_tokens: torch.Tensor, uniforms: torch.Tensor,
           out: Optional[Verified] = None) -> Verified:
    """gr_verify on torch CUDA tensors: draft_tokens [B, n] int32, uniforms [B, 2] float32."""
    _need_cuda(draft_tokens, uniforms)
    B = solved.batch
    if draft_tokens.shape != (B, solved.n) or draft_tokens.dtype != torch.int32:
        raise GrError("draft_tokens must be [B, n] int32")
    if uniforms.shape != (B, 2) or uniforms.dtype != torch.float32:
        raise GrError("uniforms must be [B, 2] float32")
    dev = draft_tokens.device
    if out is None or out.token.shape[0] != B:
        out = Verified(torch.empty(B, dtype=torch.int32, device=dev), torch.empty(B, dtype=torch.uint8, device=dev),
                       torch.empty(B, dtype=torch.int32, device=dev))
    rc = gr_verify(solved.params.data_ptr(), draft_tokens.data_ptr(), uniforms.data_ptr(), B, out.token.data_ptr(),
                   out.accepted.data_ptr(), out.status.data_ptr(), _stream())
    _check(rc, "gr_verify")
    return out


def alpha_star(q_logits: torch.Tensor, p_logits: torch.Tensor, n_list, topk: int, temp_target: float = 1.0,
               temp_draft: float = 1.0) -> Tuple[torch.Tensor, torch.Tensor]:
    """gr_alpha_star on torch CUDA tensors: ([B, len(n_list)] float32 optimal acceptances, [B] int32 status)."""
    _need_cuda(q_logits, p_logits)
    if q_logits.shape != p_logits.shape or q_logits.dim() != 2 or q_logits.dtype != p_logits.dtype:
        raise GrError("q_logits and p_logits must be [B, V] tensors of one dtype")
    B, V = q_logits.shape
    dev = q_logits.device
    wbytes = gr_workspace_bytes(V, 1, topk, B)
    if wbytes == 0:
        raise GrError("invalid shape")
    ws = torch.empty(wbytes, dtype=torch.uint8, device=dev)
    out = torch.empty((B, len(n_list)), dtype=torch.float32, device=dev)
    st = torch.empty(B, dtype=torch.int32, device=dev)
    rc = gr_alpha_star(q_logits.data_ptr(), p_logits.data_ptr(), _dtype_code(q_logits), V, n_list, topk, temp_target,
                       temp_draft, B, ws.data_ptr(), out.data_ptr(), st.data_ptr(), _stream())
    _check(rc, "gr_alpha_star")
    return out, st


def solve_verify(q_logits: torch.Tensor, p_logits: torch.Tensor, draft_tokens: torch.Tensor, uniforms: torch.Tensor,
                 topk: int, temp_target: float = 1.0, temp_draft: float = 1.0, opt: Optional[Options] = None,
                 out: Optional[Tuple[Solved, Verified]] = None) -> Tuple[Solved, Verified]:
    """gr_solve_verify on torch CUDA tensors: one call, the solve kernel finishes every instance with its draw.
    The returned Solved carries alpha* and the params block (partial where a system was skipped); the Verified's
    status is what gr_verify would report."""
    _need_cuda(q_logits, p_logits, draft_tokens, uniforms)
    if q_logits.shape != p_logits.shape or q_logits.dim() != 2 or q_logits.dtype != p_logits.dtype:
        raise GrError("q_logits and p_logits must be [B, V] tensors of one dtype")
    B, V = q_logits.shape
    if draft_tokens.dim() != 2 or draft_tokens.shape[0] != B or draft_tokens.dtype != torch.int32:
        raise GrError("draft_tokens must be [B, n] int32")
    n = int(draft_tokens.shape[1])
    if uniforms.shape != (B, 2) or uniforms.dtype != torch.float32:
        raise GrError("uniforms must be [B, 2] float32")
    dev = q_logits.device
    sv, vf = out if out is not None else (None, None)
    if sv is None or sv.batch != B or sv.V != V or sv.n != n or sv.topk != topk:
        pbytes = gr_params_bytes(V, n, topk, B)
        wbytes = gr_workspace_bytes(V, n, topk, B)
        if pbytes == 0 or wbytes == 0:
            raise GrError("invalid shape")
        sv = Solved(V, n, topk, B, torch.empty(pbytes, dtype=torch.uint8, device=dev),
                    torch.empty(wbytes, dtype=torch.uint8, device=dev),
                    torch.empty(B, dtype=torch.float32, device=dev),
                    torch.empty(B, dtype=torch.int32, device=dev), q_logits)
        vf = None
    if vf is None or vf.token.shape[0] != B:
        vf = Verified(torch.empty(B, dtype=torch.int32, device=dev), torch.empty(B, dtype=torch.uint8, device=dev),
                      sv.status)
    sv.q_logits = q_logits
    vf.status = sv.status
    rc = gr_solve_verify(q_logits.data_ptr(), p_logits.data_ptr(), _dtype_code(q_logits), V, n, topk, temp_target,
                         temp_draft, B, opt, draft_tokens.data_ptr(), uniforms.data_ptr(), sv.params.data_ptr(),
                         sv.workspace.data_ptr(), sv.alpha_star.data_ptr(), vf.token.data_ptr(),
                         vf.accepted.data_ptr(), sv.status.data_ptr(), _stream())
    _check(rc, "gr_solve_verify")
    return sv, vf


@dataclasses.dataclass
class Rule:
    """The verification rule copied out of a params block (host tensors), support in ratio order."""
    ids: torch.Tensor     # [B, kcap] int32, -1 padded
    block: torch.Tensor   # [B, kcap] int32: -1 on H*, else block number from the lowest ratio; -2 padding
    w: torch.Tensor       # [B, kcap] float64 exp(alpha)
    resid: torch.Tensor   # [B, kcap] float64 outer residual
    flow: torch.Tensor    # [B, kcap] float64 p_i
    k: torch.Tensor       # [B]
    jstar: torch.Tensor
    nblocks: torch.Tensor
    alpha_star: torch.Tensor   # [B] float64
    gnorm: torch.Tensor
    iters: torch.Tensor        # gradient evaluations spent
    lse_target: torch.Tensor
    status: torch.Tensor
    gnorm_predicted: torch.Tensor = None   # [B] bool: the norm of some system was predicted from its last Newton step


def read_rule(solved: Solved) -> Rule:
    B = solved.batch
    kfull = solved.V if (solved.topk <= 0 or solved.topk >= solved.V) else solved.topk
    kcap = max(1, min(kfull, GR_MAX_SUPPORT))
    dev = solved.params.device
    ids = torch.empty(B, kcap, dtype=torch.int32, device=dev)
    blk = torch.empty(B, kcap, dtype=torch.int32, device=dev)
    w = torch.empty(B, kcap, dtype=torch.float64, device=dev)
    r = torch.empty(B, kcap, dtype=torch.float64, device=dev)
    p = torch.empty(B, kcap, dtype=torch.float64, device=dev)
    hd = torch.empty(B, 8, dtype=torch.float64, device=dev)
    rc = gr_read_rule(solved.params.data_ptr(), B, kcap, ids.data_ptr(), blk.data_ptr(), w.data_ptr(), r.data_ptr(),
                      p.data_ptr(), hd.data_ptr(), _stream())
    _check(rc, "gr_read_rule")
    hd = hd.cpu()
    return Rule(ids.cpu(), blk.cpu(), w.cpu(), r.cpu(), p.cpu(), hd[:, 0].long(), hd[:, 1].long(), hd[:, 2].long(),
                hd[:, 3], hd[:, 4], hd[:, 5].long() & 0xffff, hd[:, 6], hd[:, 7].long(), (hd[:, 5].long() >> 16) & 1 == 1)


@dataclasses.dataclass
class Slice:
    """pi(.|omega) per instance as the verification code computes it (host tensors)."""
    U: torch.Tensor        # [B, n] int32: drafted token s, -1 for a repeat
    pi: torch.Tensor       # [B, n] float64
    rho: torch.Tensor      # [B] float64 mass of the resample segment
    status: torch.Tensor   # [B] int32


def read_slice(solved: Solved, draft_tokens: torch.Tensor) -> Slice:
    """gr_read_slice on torch CUDA tensors."""
    _need_cuda(draft_tokens)
    B, n = solved.batch, solved.n
    if draft_tokens.shape != (B, n) or draft_tokens.dtype != torch.int32:
        raise GrError("draft_tokens must be [B, n] int32")
    dev = draft_tokens.device
    U = torch.empty(B, n, dtype=torch.int32, device=dev)
    pi = torch.empty(B, n, dtype=torch.float64, device=dev)
    rho = torch.empty(B, dtype=torch.float64, device=dev)
    st = torch.empty(B, dtype=torch.int32, device=dev)
    rc = gr_read_slice(solved.params.data_ptr(), draft_tokens.data_ptr(), B, n, U.data_ptr(), pi.data_ptr(),
                       rho.data_ptr(), st.data_ptr(), _stream())
    _check(rc, "gr_read_slice")
    return Slice(U.cpu(), pi.cpu(), rho.cpu(), st.cpu())


def solve_verify_host(q_logits: torch.Tensor, p_logits: torch.Tensor, draft_tokens: torch.Tensor,
                      uniforms: torch.Tensor, n: int, topk: int, temp_target: float = 1.0, temp_draft: float = 1.0,
                      opt: Optional[Options] = None, device="cuda:0", state: Optional[dict] = None):
    """The whole path for HOST tensors (pinned or pageable): copies the inputs to the device, runs gr_solve and
    gr_verify on the current stream and copies token / accepted / alpha* back.  `state` (a dict the caller keeps)
    lets repeated calls reuse the device buffers."""
    st = state if state is not None else {}
    dev = torch.device(device)

    def dev_buf(name, src):
        buf = st.get(name)
        if buf is None or buf.shape != src.shape or buf.dtype != src.dtype:
            buf = torch.empty(src.shape, dtype=src.dtype, device=dev)
            st[name] = buf
        buf.copy_(src, non_blocking=True)
        return buf

    q = dev_buf("q", q_logits); p = dev_buf("p", p_logits)
    tk = dev_buf("tk", draft_tokens); un = dev_buf("un", uniforms)
    sv = st["solved"] = solve(q, p, n, topk, temp_target, temp_draft, opt, st.get("solved"))
    v = st["verified"] = verify(sv, tk, un, st.get("verified"))
    # the four results in one copy (four separate ones, each with its own synchronisation, took 25 us more)
    B = sv.batch
    out = torch.cat([t.view(torch.uint8) for t in (v.token, sv.alpha_star, v.status, v.accepted)]).cpu()
    token, alpha, status = (out[4 * B * i:4 * B * (i + 1)] for i in range(3))
    return token.view(torch.int32), out[12 * B:], alpha.view(torch.float32), status.view(torch.int32)


# ---------------------------------------------------------------- around the decoding step

def _need(t, what: str, dtype, shape=None, device=None, optional: bool = False):
    """The address of a contiguous CUDA tensor of this type, shape and device (0 for None where that is allowed)."""
    if t is None and optional:
        return 0
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous()) or t.dtype is not dtype:
        raise GrError(f"{what}: expected a contiguous CUDA tensor of {dtype}")
    if shape is not None and t.shape != shape:
        raise GrError(f"{what}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if device is not None and t.device != device:
        raise GrError(f"{what}: on {t.device}, the other tensors on {device}")
    return t.data_ptr()


def _fits(what: str, *numbers):
    """Refuses numbers beyond the 32 bits that the C call takes (ctypes would cut them to their low bits)."""
    for n in numbers:
        if not -(1 << 31) <= n < 1 << 31:
            raise GrError(f"{what}: {n} is beyond 32 bits")


# (the handle alone: the public call makes a Stream object around it, 3 us)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: int(torch.cuda.current_stream(index).cuda_stream))


def _short(way: str, name: str, *args):
    """The call of entry point `name` by the short way, where that is open: True when it was made."""
    if _lib is None:
        load_library()
    if _tensors is None:
        return False
    rc = getattr(_tensors, way)(_entry[name], *args)
    if rc is None:
        return False
    if rc != 0:
        _check(rc, name)
    return True


def _starts(at: int, dims) -> torch.Tensor:
    """Where the pieces of a tensor begin, in order: dims are (number, bytes from one to the next)."""
    out = torch.tensor([at])
    for n, step in dims:
        out = (out.view(-1, 1) + torch.arange(n if step else min(n, 1)) * step).view(-1)
    return out.sort().values


def _share_bytes(a, b) -> bool:
    """Whether a tensor of `a` shares a byte with one of `b`: lists of (list it came from, address, dims, bytes of a piece).  (Those of one
    list are the C call's to look at.)"""
    every = []
    for side, tensors in enumerate((a, b)):
        for run, at, dims, size in tensors:
            if size and all(n for n, _ in dims):
                every.append((at, at + size + sum(step * (n - 1) for n, step in dims), side, run, dims, size))
    every.sort(key=lambda e: e[:2])
    within = []                            # those that may reach what follows
    for e in every:
        within = [o for o in within if o[1] > e[0]]
        for o in within:
            if o[3] == e[3] or (o[2] == e[2] and a is not b):
                continue
            # one lies within the other: piece by piece
            if any(torch.Size(n for n, _ in t[4]).numel() > 1 << 24 for t in (o, e)):
                raise GrError("tensors of different layouts within one another have too many pieces to tell them apart")
            p, q = _starts(o[0], o[4]), _starts(e[0], e[4])
            before = torch.searchsorted(p, q + e[5]) - 1              # the last piece of one that begins before the other's ends
            if bool(((before >= 0) & (p[before.clamp(min=0)] + o[5] > q)).any()):
                return True
        within.append(e)
    return False


def _call(dev: torch.device, what: str, function, *args):
    """A C entry point with the tensors' device current and that device's current stream."""
    if torch.cuda.current_device() == dev.index:
        rc = function(*args, _raw_stream(dev.index))
    else:
        with torch.cuda.device(dev):
            rc = function(*args, _raw_stream(dev.index))
    if rc != 0:
        _check(rc, what)


@dataclasses.dataclass
class Beams:
    """Result of beam_select: the best continuations of each group, best first (token and parent -1: none left)."""
    token: torch.Tensor      # [B, select] int32
    parent: torch.Tensor     # [B, select] int32
    score: torch.Tensor      # [B, select] float32
    length: torch.Tensor     # [B, select] int32 (zeros after a call without lengths)
    done: torch.Tensor       # [B, select] bool
    status: torch.Tensor     # [B] int32
    workspace: torch.Tensor  # uint8, scratch
    shape: tuple             # (B, beams, V, select)
    counted: bool = False    # whether a call has written lengths


def beam_select(logits: torch.Tensor, scores: torch.Tensor, select: Optional[int] = None, temperature: float = 1.0,
                lengths: Optional[torch.Tensor] = None, done: Optional[torch.Tensor] = None, eos: int = -1,
                length_penalty: float = 0.0, out: Optional[Beams] = None) -> Beams:
    """gr_beam_select on torch CUDA tensors: logits [B, beams, V] float32 or bfloat16 (rows at any one distance, elements
    next to one another), scores [B, beams] float32, lengths [B, beams] int32, done [B, beams] bool or uint8.  `select`
    defaults to the number of beams; temperature and length_penalty are rounded to float32, as the C call takes them.  `out`: a result of an earlier call of the same shape, written again (it must not
    be read from by this call: scores, lengths and done are other tensors)."""
    if not (isinstance(logits, torch.Tensor) and logits.is_cuda and logits.dim() == 3):
        raise GrError("logits must be a [B, beams, V] CUDA tensor")
    if (out is not None and out.shape == (*logits.shape, logits.shape[1] if select is None else select)
            and _short("select", "gr_beam_select", logits, scores, out.shape[3], temperature, lengths, done, eos, length_penalty,
                       out.workspace, out.token, out.parent, out.score, out.length, out.done, out.status)):
        return _with_lengths(out, lengths)
    B, W, V = logits.shape
    dev, code = logits.device, _dtype_code(logits)
    step = logits.stride()
    ld = step[1] if W > 1 else step[0] if B > 1 else V
    if ((V > 1 and step[2] != 1) or (B > 1 and W > 1 and step[0] != W * ld) or ld < V) and logits.numel() > 0:
        raise GrError("logits: the rows must be apart by one distance, their elements next to one another")
    K = W if select is None else int(select)
    _fits("beam_select", B, V, K, eos)
    rows = (B, W)
    a_scores = _need(scores, "scores", torch.float32, rows, dev)
    a_lengths = _need(lengths, "lengths", torch.int32, rows, dev, optional=True)
    kind = torch.uint8 if done is not None and done.dtype is torch.uint8 else torch.bool
    a_done = _need(done, "done", kind, rows, dev, optional=True)
    if out is None or out.shape != (B, W, V, K) or out.token.device != dev:
        wbytes = gr_beam_workspace_bytes(V, W, K, B)
        if wbytes == 0:
            raise GrError("invalid shape")
        out = Beams(torch.empty(B, K, dtype=torch.int32, device=dev), torch.empty(B, K, dtype=torch.int32, device=dev),
                    torch.empty(B, K, dtype=torch.float32, device=dev), torch.zeros(B, K, dtype=torch.int32, device=dev),
                    torch.empty(B, K, dtype=torch.bool, device=dev), torch.empty(B, dtype=torch.int32, device=dev),
                    torch.empty(wbytes, dtype=torch.uint8, device=dev), (B, W, V, K))
    a_score, a_length, a_fin = out.score.data_ptr(), out.length.data_ptr(), out.done.data_ptr()
    if B > 0 and (a_scores == a_score or a_lengths == a_length or a_done == a_fin):
        raise GrError("scores, lengths or done is a tensor of `out`, which this call writes")
    _call(dev, "gr_beam_select", load_library().gr_beam_select, logits.data_ptr(), code, V, max(ld, V), W, B, temperature,
          a_scores, a_lengths, a_done, eos, length_penalty, K, out.workspace.data_ptr(), out.token.data_ptr(),
          out.parent.data_ptr(), a_score, a_length if lengths is not None else 0, a_fin, out.status.data_ptr())
    return _with_lengths(out, lengths)


def _with_lengths(out: Beams, lengths) -> Beams:
    # (a call without lengths writes none: what an earlier one left is taken away.  Once counted always counted, as a captured call may
    # write lengths again at any time.)
    if lengths is not None:
        out.counted = True
    elif out.counted:
        out.length.zero_()
    return out


def _state_layout(x: torch.Tensor, token_dim: Optional[int]):
    """(parts, bytes between parts, bytes of a part, bytes of a token) of the states in x [B, beams, ...]."""
    e = x.element_size()
    shape, stride = list(x.shape), list(x.stride())
    at = 2 if token_dim is None else token_dim
    part = 1
    for d in range(x.dim() - 1, at - 1, -1):
        if shape[d] > 1 and stride[d] != part:
            raise GrError("states: the dimensions from the tokens on must lie next to one another")
        part *= shape[d]
    parts, step = 1, 0
    for d in range(at - 1, 1, -1):
        if shape[d] == 1:
            continue
        if parts > 1 and stride[d] != step * parts:
            raise GrError("states: the dimensions before the tokens must have one distance between their pieces")
        step = stride[d] if parts == 1 else step
        parts *= shape[d]
    tokens = 1 if token_dim is None else shape[token_dim]
    return parts, step * e, part * e, part // tokens * e if tokens else e


def reorder_states(states, parents: torch.Tensor, lengths: Optional[torch.Tensor] = None,
                   token_dim: Optional[int] = None, out=None):
    """gr_reorder_states on torch CUDA tensors: `states` is a list of tensors [B, beams, ...] (of any types and layouts),
    parents [B, chosen] int32.  In place, with chosen <= beams, unless `out` (a list of tensors [B, chosen, ...]) is
    given, which must not meet the states in memory.  Tensors that share a byte with one another are refused.  With lengths [B, beams] int32 the dimension `token_dim` of the
    states counts tokens, of which each parent's first lengths[b, parent] are copied.  Returns `out` or `states`."""
    if _short("reorder", "gr_reorder_states", states, parents, lengths, token_dim, out):
        return states if out is None else out
    states = list(states)
    to = states if out is None else list(out)
    if len(to) != len(states):
        raise GrError("out: one tensor for each of the states")
    if not states:
        return to
    if not isinstance(parents, torch.Tensor) or parents.dim() != 2:
        raise GrError("parents must be a [B, chosen] CUDA tensor of torch.int32")
    a_parents = _need(parents, "parents", torch.int32)
    B, chosen = parents.shape
    dev = parents.device
    if (lengths is None) != (token_dim is None):
        raise GrError("lengths and token_dim go together")
    if not isinstance(states[0], torch.Tensor) or states[0].dim() < 2:
        raise GrError("states must be CUDA tensors [B, beams, ...] on the device of parents")
    W = states[0].shape[1]
    a_lengths = _need(lengths, "lengths", torch.int32, (B, W), dev, optional=True)
    # runs of tensors of one layout: (layout, addresses of states and outs)
    runs = []

    def layout_of(x, y):
        shape, step, step_y = x.shape, x.stride(), y.stride()
        if x.device != dev or not x.is_cuda:
            raise GrError("states must be CUDA tensors [B, beams, ...] on the device of parents")
        if x.dim() < 2 or shape[0] != B or shape[1] != W:
            raise GrError("states must be [B, beams, ...], of one number of beams")
        if token_dim is not None and not 2 <= token_dim < x.dim():
            raise GrError("token_dim must be a dimension behind the beams")
        if y is not x and (y.shape != (B, chosen) + tuple(shape[2:]) or y.dtype is not x.dtype or y.device != dev):
            raise GrError("out must hold tensors [B, chosen, ...] like the states")
        parts, part_step, part, token = _state_layout(x, token_dim)
        _fits("states", B, parts)
        part_step_y = part_step if y is x else _state_layout(y, token_dim)[1]
        e = x.element_size()
        return StateLayout(B, W, chosen, parts, step[0] * e if B > 1 else 0, step[1] * e if W > 1 else 0, part_step,
                           step_y[0] * e if B > 1 else 0, step_y[1] * e if y.shape[1] > 1 else 0,
                           part_step_y, part, token)

    last = None
    for x, y in zip(states, to):
        if not isinstance(x, torch.Tensor) or not isinstance(y, torch.Tensor):
            raise GrError("states must be CUDA tensors [B, beams, ...] on the device of parents")
        kind = (x.shape, x.stride(), x.dtype, x.device, y.shape, y.stride(), y.dtype, y.device)
        if kind != last:
            last = kind
            runs.append((layout_of(x, y), [], []))
        runs[-1][1].append(x.data_ptr())
        runs[-1][2].append(y.data_ptr())
    if len(runs) > 1:
        # nothing is launched before every call is known to be taken (without parents the C call looks at the rest and answers so)
        mine, theirs = [], []
        for run, (t, at, at_y) in enumerate(runs):
            if chosen > 0 and t.part_bytes > 0:
                rc = gr_reorder_states(at, at_y, t, 0, a_lengths, 0)
                if out is not None and at[0] == at_y[0]:
                    raise GrError("out shares memory with the states")
                if rc not in (GR_OK, _NULL):
                    _check(rc, "gr_reorder_states")
                theirs += [(run, p, ((B, t.src_group), (W, t.src_beam), (t.parts, t.src_part)), t.part_bytes) for p in at]
                mine += [(run, p, ((B, t.dst_group), (W if out is None else chosen, t.dst_beam), (t.parts, t.dst_part)), t.part_bytes) for p in at_y]
        if _share_bytes(mine, mine):
            raise GrError("two of the tensors share memory")
        if out is not None and _share_bytes(mine, theirs):
            raise GrError("out shares memory with the states")
    for layout, at, at_y in runs:
        if chosen > 0 and layout.part_bytes > 0:
            _call(dev, "gr_reorder_states", gr_reorder_states, at, at_y, layout, a_parents, a_lengths)
    return to


@dataclasses.dataclass
class BlockTables:
    """Block tables of a paged cache: row r's token t lies in block table[r, t // block_size] at t % block_size; refs[i]
    rows hold block i.  Rows come in groups of `beams`."""
    table: torch.Tensor      # [rows, width] int32, -1 where no block is held
    lengths: torch.Tensor    # [rows] int32 tokens
    refs: torch.Tensor       # [num_blocks] int32
    block_size: int
    beams: int = 1

    @staticmethod
    def empty(rows: int, width: int, num_blocks: int, block_size: int, beams: int = 1, device="cuda") -> "BlockTables":
        return BlockTables(torch.full((rows, width), -1, dtype=torch.int32, device=device),
                           torch.zeros(rows, dtype=torch.int32, device=device),
                           torch.zeros(num_blocks, dtype=torch.int32, device=device), block_size, beams)


@dataclasses.dataclass
class BlockPlan:
    """Result of block_plan: where the appended tokens go, and which blocks are to be copied before they are written."""
    slots: torch.Tensor      # [max_tokens] int64, -1 behind the last token
    positions: torch.Tensor  # [max_tokens] int32
    offsets: torch.Tensor    # [rows + 1] int32
    copy_src: torch.Tensor   # [rows] int32, -1: nothing to copy
    copy_dst: torch.Tensor   # [rows] int32
    status: torch.Tensor     # [rows] int32
    workspace: torch.Tensor  # uint8, scratch
    shape: tuple             # (rows, num_blocks, max_tokens)


def block_plan(tables: BlockTables, append: torch.Tensor, max_tokens: int, keep: Optional[torch.Tensor] = None,
               parents: Optional[torch.Tensor] = None, out: Optional[BlockPlan] = None) -> BlockPlan:
    """gr_block_plan on torch CUDA tensors: `tables` is updated in place; append, keep [rows] int32, parents [rows] or
    [rows / beams, beams] int32 (row numbers within the group, as beam_select returns them).  keep may be tables.lengths itself."""
    if (out is not None and isinstance(tables.table, torch.Tensor) and isinstance(tables.refs, torch.Tensor)
            and out.shape == (*tables.table.shape[:1], *tables.refs.shape, max_tokens)
            and _short("plan", "gr_block_plan", tables.table, tables.lengths, tables.refs, tables.block_size, tables.beams, append,
                       max_tokens, keep, parents, out.workspace, out.slots, out.positions, out.offsets, out.copy_src,
                       out.copy_dst, out.status)):
        return out
    if not isinstance(tables.table, torch.Tensor) or tables.table.dim() != 2:
        raise GrError("table must be a [rows, width] CUDA tensor of torch.int32")
    R, width = tables.table.shape
    dev, i32 = tables.table.device, torch.int32
    a_table = _need(tables.table, "table", i32)
    a_lengths = _need(tables.lengths, "lengths", i32, (R,), dev)
    N = int(tables.refs.numel())
    a_refs = _need(tables.refs, "refs", i32, (N,), dev)
    a_append = _need(append, "append", i32, (R,), dev)
    a_keep = _need(keep, "keep", i32, (R,), dev, optional=True)
    a_parents = _need(parents, "parents", i32, None, dev, optional=True)
    if parents is not None and parents.shape != (R,):
        if tables.beams < 1 or parents.shape != (R // tables.beams, tables.beams):
            raise GrError("parents must be [rows] or [rows / beams, beams]")
    _fits("block_plan", R, width, N, tables.beams, tables.block_size, max_tokens)
    if out is None or out.shape != (R, N, max_tokens) or out.slots.device != dev:
        wbytes = gr_block_workspace_bytes(R, N)
        if wbytes == 0 or max_tokens < 0:
            raise GrError("invalid shape")
        out = BlockPlan(torch.empty(max_tokens, dtype=torch.int64, device=dev),
                        torch.empty(max_tokens, dtype=i32, device=dev), torch.empty(R + 1, dtype=i32, device=dev),
                        torch.empty(R, dtype=i32, device=dev), torch.empty(R, dtype=i32, device=dev),
                        torch.empty(R, dtype=i32, device=dev), torch.empty(wbytes, dtype=torch.uint8, device=dev),
                        (R, N, max_tokens))
    _call(dev, "gr_block_plan", load_library().gr_block_plan, a_table, R, width, tables.beams, tables.block_size,
          a_lengths, a_refs, N, a_parents, a_keep, a_append, max_tokens, out.workspace.data_ptr(), out.slots.data_ptr(),
          out.positions.data_ptr(), out.offsets.data_ptr(), out.copy_src.data_ptr(), out.copy_dst.data_ptr(),
          out.status.data_ptr())
    return out


def copy_blocks(caches, copy_src: torch.Tensor, copy_dst: torch.Tensor) -> None:
    """gr_copy_blocks on torch CUDA tensors: `caches` is a list of tensors [num_blocks, ...] whose blocks are contiguous,
    copy_src and copy_dst [pairs] int32 as block_plan returns them.  Caches that share a byte with one another are refused."""
    if _short("copy", "gr_copy_blocks", caches, copy_src, copy_dst):
        return
    caches = list(caches)
    if not caches:
        return
    if not isinstance(copy_src, torch.Tensor) or copy_src.dim() != 1:
        raise GrError("copy_src must be a [pairs] CUDA tensor of torch.int32")
    dev = copy_src.device
    a_src = _need(copy_src, "copy_src", torch.int32)
    a_dst = _need(copy_dst, "copy_dst", torch.int32, copy_src.shape, dev)
    # runs of caches of one layout: (blocks, bytes from one to the next, bytes, addresses)
    runs = []

    def layout_of(x):
        if x.device != dev or x.dim() < 1:
            raise GrError("caches must be CUDA tensors [num_blocks, ...] on the device of copy_src")
        shape, step = x.shape, x.stride()
        per = x.numel() // shape[0] if shape[0] else 0
        if per and (not x[0].is_contiguous() or (shape[0] > 1 and step[0] < per)):
            raise GrError("caches: a block's elements must lie next to one another, and the blocks apart")
        e = x.element_size()
        _fits("caches", shape[0], copy_src.shape[0])
        return shape[0], (step[0] if shape[0] > 1 else per) * e, per * e

    last = None
    for x in caches:
        if not isinstance(x, torch.Tensor):
            raise GrError("caches must be CUDA tensors [num_blocks, ...] on the device of copy_src")
        kind = (x.shape, x.stride(), x.dtype, x.device)
        if kind != last:
            last = kind
            runs.append(layout_of(x) + ([],))
        runs[-1][3].append(x.data_ptr())
    if len(runs) > 1:
        # (as for states: nothing is launched before every call is known to be taken)
        every = []
        for run, (blocks, stride, size, at) in enumerate(runs):
            rc = gr_copy_blocks(at, blocks, stride, size, 0, 0, copy_src.shape[0], 0)
            if rc not in (GR_OK, _NULL):
                _check(rc, "gr_copy_blocks")
            every += [(run, p, ((blocks, stride),), size) for p in at]
        if _share_bytes(every, every):
            raise GrError("two of the caches share memory")
    for blocks, stride, size, at in runs:
        if size > 0:
            _call(dev, "gr_copy_blocks", gr_copy_blocks, at, blocks, stride, size, a_src, a_dst, copy_src.shape[0])


# ---------------------------------------------------------------- filling and reading a paged cache

_CODES = {torch.float32: GR_F32, torch.bfloat16: GR_BF16, torch.float16: GR_F16}


@dataclasses.dataclass
class KVCache:
    """A layer's keys and values in blocks, slot z at z % block_size of block z // block_size.  In 16 or 32 bits keys and values are
    [num_blocks, block_size, heads, dim], apart by any strides; in 4 bits `keys` holds both, [num_blocks, heads, block_size / 8, 9 dim]
    bytes (gr.h says where what is)."""
    keys: torch.Tensor
    values: Optional[torch.Tensor]
    block_size: int
    heads: int
    dim: int

    @staticmethod
    def empty(num_blocks: int, block_size: int, heads: int, dim: int, dtype=torch.bfloat16, device="cuda") -> "KVCache":
        """Zeros, of type float32, bfloat16 or float16; uint8: in 4 bits."""
        if dtype is torch.uint8:
            if block_size % 8 or dim % 32:
                raise GrError("a cache in 4 bits has blocks of a multiple of 8 tokens and heads of a multiple of 32 dims")
            return KVCache(torch.zeros(num_blocks, heads, block_size // 8, 9 * dim, dtype=dtype, device=device), None, block_size, heads, dim)
        if dtype not in _CODES:
            raise GrError("a cache is of float32, bfloat16 or float16, or in 4 bits (uint8)")
        shape = (num_blocks, block_size, heads, dim)
        return KVCache(torch.zeros(shape, dtype=dtype, device=device), torch.zeros(shape, dtype=dtype, device=device), block_size, heads, dim)

    def tensors(self):
        """What copy_blocks copies of it."""
        return [self.keys] if self.values is None else [self.keys, self.values]


def _cache(cache: KVCache):
    """(address of the keys, address of the values, layout) of a cache."""
    k, v = cache.keys, cache.values
    if not (isinstance(k, torch.Tensor) and k.is_cuda and k.dim() == 4):
        raise GrError("cache: keys must be a CUDA tensor of four dimensions")
    bs, H, D = cache.block_size, cache.heads, cache.dim
    _fits("cache", k.shape[0], bs, H, D)
    step = k.stride()
    if k.dtype is torch.uint8:
        if v is not None or k.shape[1:] != (H, bs // 8, 9 * D) or bs % 8 or D % 32:
            raise GrError("cache: in 4 bits keys is [num_blocks, heads, block_size / 8, 9 dim] and values None")
        if k.numel() and not k[0].is_contiguous():
            raise GrError("cache: a block's bytes must lie next to one another")
        block = H * (bs // 8) * 9 * D
        return k.data_ptr(), 0, CacheLayout(GR_Q4, H, D, bs, k.shape[0], step[0] if k.shape[0] > 1 else block, 0, 0)
    if k.dtype not in _CODES:
        raise GrError("cache: keys and values are float32, bfloat16 or float16, or uint8 in 4 bits")
    if not isinstance(v, torch.Tensor) or v.shape != k.shape or v.dtype is not k.dtype or v.device != k.device or v.stride() != step:
        raise GrError("cache: keys and values must be alike")
    if k.shape[1:] != (bs, H, D) or (D > 1 and step[3] != 1):
        raise GrError("cache: keys and values are [num_blocks, block_size, heads, dim], a head's elements next to one another")
    return k.data_ptr(), v.data_ptr(), CacheLayout(_CODES[k.dtype], H, D, bs, k.shape[0], step[0], step[1], step[2])


def _rows(t, what: str, shape, dtype, device):
    """(address, distance of tokens, distance of heads) of a [tokens, heads, dim] tensor."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dim() != 3 or t.dtype is not dtype or t.device != device:
        raise GrError(f"{what}: expected a [tokens, heads, dim] CUDA tensor of {dtype} on {device}")
    if t.shape != shape:
        raise GrError(f"{what}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    step = t.stride()
    if shape[2] > 1 and step[2] != 1:
        raise GrError(f"{what}: a head's elements must lie next to one another")
    return t.data_ptr(), step[0], step[1]


def cache_append(cache: KVCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, positions: Optional[torch.Tensor] = None,
                 frequencies: Optional[torch.Tensor] = None, interleaved: bool = False, q: Optional[torch.Tensor] = None,
                 q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """gr_cache_append on torch CUDA tensors: k, v [tokens, heads, dim] of float32, bfloat16 or float16 go to slots [tokens] int64 (-1:
    nowhere) of the cache, as block_plan gives them.  With frequencies [rot / 2] float64 and positions [tokens] int32 the first rot dims of
    keys and queries are rotated: pairs (c, c + rot / 2), or (2 c, 2 c + 1) if interleaved.  q [tokens, any heads, dim]: queries to be rotated into q_out,
    which may be q itself (default: a new tensor, zeros where positions are negative).  Returns q_out."""
    if _short("append", "gr_cache_append", cache.keys, cache.values, cache.block_size, cache.heads, cache.dim, k, v, slots, positions, frequencies,
              interleaved, q, q_out):
        return q_out
    a_keys, a_values, layout = _cache(cache)
    dev = cache.keys.device
    if not isinstance(k, torch.Tensor) or k.dim() != 3 or k.dtype not in _CODES:
        raise GrError("k must be a [tokens, heads, dim] CUDA tensor of float32, bfloat16 or float16")
    T, dt = k.shape[0], k.dtype
    _fits("cache_append", T)
    shape = (T, cache.heads, cache.dim)
    k_at, v_at = _rows(k, "k", shape, dt, dev), _rows(v, "v", shape, dt, dev)
    a_slots = _need(slots, "slots", torch.int64, (T,), dev)
    rot = 0
    if frequencies is not None:
        if positions is None:
            raise GrError("frequencies and positions go together")
        if not isinstance(frequencies, torch.Tensor) or frequencies.dim() != 1 or 2 * frequencies.numel() > cache.dim:
            raise GrError("frequencies must be [rot / 2], with rot at most the heads' dim")
        rot = 2 * frequencies.numel()
    a_freq = _need(frequencies, "frequencies", torch.float64, None, dev, optional=True)
    a_pos = _need(positions, "positions", torch.int32, (T,), dev, optional=True)
    q_at = out_at = (0, 0, 0)
    heads = 0
    if q is not None:
        if not isinstance(q, torch.Tensor) or q.dim() != 3:
            raise GrError("q must be a [tokens, heads, dim] CUDA tensor")
        heads = q.shape[1]
        shape = (T, heads, cache.dim)
        q_at = _rows(q, "q", shape, dt, dev)
        if q_out is None:
            q_out = torch.zeros(shape, dtype=dt, device=dev)
        out_at = _rows(q_out, "q_out", shape, dt, dev)
    elif q_out is not None:
        raise GrError("q_out without q")
    tokens_in = CacheTokens(k_at[0], v_at[0], q_at[0], out_at[0], _CODES[dt], heads, *k_at[1:], *v_at[1:], *q_at[1:], *out_at[1:])
    _call(dev, "gr_cache_append", gr_cache_append, a_keys, a_values, layout, tokens_in, T, a_slots, a_pos, a_freq, rot, int(interleaved))
    return q_out


def cache_read(cache: KVCache, slots: torch.Tensor, dtype=torch.bfloat16, out=None):
    """gr_cache_read on torch CUDA tensors: keys and values [tokens, heads, dim] of slots [tokens] int64 (zeros for a slot outside the
    cache), of float32, bfloat16 or float16.  `out`: a pair of such tensors, to be written."""
    if _lib is None:
        load_library()
    if _tensors is not None and (out is None or len(out) == 2):
        got = _tensors.read(_entry["gr_cache_read"], cache.keys, cache.values, cache.block_size, cache.heads, cache.dim, slots, dtype,
                            *(out if out is not None else (None, None)))
        if isinstance(got, tuple):
            return got
        if got is not None:
            _check(got, "gr_cache_read")
    a_keys, a_values, layout = _cache(cache)
    dev = cache.keys.device
    if not isinstance(slots, torch.Tensor) or slots.dim() != 1:
        raise GrError("slots must be a [tokens] CUDA tensor of torch.int64")
    a_slots = _need(slots, "slots", torch.int64, None, dev)
    shape = (slots.shape[0], cache.heads, cache.dim)
    _fits("cache_read", shape[0])
    if out is None:
        if dtype not in _CODES:
            raise GrError("cache_read gives float32, bfloat16 or float16")
        out = tuple(torch.empty(shape, dtype=dtype, device=dev) for _ in range(2))
    k, v = out
    if not isinstance(k, torch.Tensor) or k.dtype not in _CODES:
        raise GrError("cache_read gives float32, bfloat16 or float16")
    k_at, v_at = _rows(k, "out", shape, k.dtype, dev), _rows(v, "out", shape, k.dtype, dev)
    _call(dev, "gr_cache_read", gr_cache_read, a_keys, a_values, layout, a_slots, shape[0], _CODES[k.dtype], *k_at, *v_at)
    return k, v


@dataclasses.dataclass
class Attended:
    """Result of cache_attend."""
    out: torch.Tensor        # [tokens, heads, dim], of the queries' type
    status: torch.Tensor     # [rows] int32
    workspace: torch.Tensor  # uint8, scratch
    shape: tuple             # (tokens, heads, dim, rows, heads of the cache, type)


def cache_attend(q: torch.Tensor, cache: KVCache, table: torch.Tensor, offsets: torch.Tensor, positions: torch.Tensor,
                 scale: Optional[float] = None, window: int = 0, out: Optional[Attended] = None) -> Attended:
    """gr_cache_attend on torch CUDA tensors: queries q [tokens, heads, dim] bfloat16 or float16 (a multiple of the cache's heads), a cache in 4
    bits, the rows' block table [rows, width] int32, and, as block_plan returns them, offsets [rows + 1] (row r's queries are
    offsets[r] .. offsets[r + 1] - 1) and positions [tokens] int32.  `scale` defaults to dim ** -0.5; with a window a query sees that many
    tokens, itself the last.  The kernel is chosen by tokens / rows: fastest without room behind the last row's tokens, and with prompts in a call of their own.
    `out`: a result of an earlier call of the same shape, written again; what lies behind the last row's tokens stays."""
    if (out is not None and out.shape[4] == cache.heads
            and _short("attend", "gr_cache_attend", q, cache.keys, cache.values, cache.block_size, cache.heads, cache.dim, table, offsets, positions,
                       scale, window, out.workspace, out.out, out.status, _entry.get("gr_attend_workspace_bytes"))):
        return out
    a_cache, _, layout = _cache(cache)
    if layout.format != GR_Q4:
        raise GrError("cache_attend wants a cache in 4 bits")
    dev = cache.keys.device
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or q.dtype not in (torch.bfloat16, torch.float16):
        raise GrError("q must be a [tokens, heads, dim] CUDA tensor of bfloat16 or float16")
    T, Hq, D = q.shape
    q_at = _rows(q, "q", (T, Hq, cache.dim), q.dtype, dev)
    if not isinstance(table, torch.Tensor) or table.dim() != 2:
        raise GrError("table must be a [rows, width] CUDA tensor of torch.int32")
    R, width = table.shape
    a_table = _need(table, "table", torch.int32, None, dev)
    a_off = _need(offsets, "offsets", torch.int32, (R + 1,), dev)
    a_pos = _need(positions, "positions", torch.int32, (T,), dev)
    _fits("cache_attend", T, Hq, R, width, window)
    shape = (T, Hq, D, R, cache.heads, q.dtype)
    wbytes = gr_attend_workspace_bytes(cache.heads, Hq, D, R, T)
    if wbytes == 0:
        raise GrError("invalid shape")
    if out is None or out.shape != shape or out.out.device != dev:
        out = Attended(torch.zeros(T, Hq, D, dtype=q.dtype, device=dev), torch.empty(R, dtype=torch.int32, device=dev),
                       torch.empty(wbytes, dtype=torch.uint8, device=dev), shape)
    out_at = _rows(out.out, "out", q.shape, q.dtype, dev)
    a_ws, a_status = _need(out.workspace, "out.workspace", torch.uint8, None, dev), _need(out.status, "out.status", torch.int32, (R,), dev)
    if out.workspace.numel() < wbytes:
        raise GrError(f"out.workspace: {wbytes} bytes are needed")
    _call(dev, "gr_cache_attend", gr_cache_attend, q_at[0], _CODES[q.dtype], Hq, *q_at[1:], a_cache, layout, a_table, width, R, a_off, a_pos,
          T, D ** -0.5 if scale is None else scale, window, a_ws, *out_at, a_status)
    return out


# ---------------------------------------------------------------- log probabilities

@dataclasses.dataclass
class Logprobs:
    """Result of token_logprobs."""
    logprob: torch.Tensor      # [rows, given] float32
    entropy: torch.Tensor      # [rows] float32
    top_token: torch.Tensor    # [rows, top] int32, -1: none left
    top_logprob: torch.Tensor  # [rows, top] float32
    status: torch.Tensor       # [rows] int32
    shape: tuple               # (rows, given, top)


def token_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, top: int = 0, temperature: float = 1.0,
                   out: Optional[Logprobs] = None) -> Logprobs:
    """gr_token_logprobs on torch CUDA tensors: logits [rows, V] float32 or bfloat16 (rows at any one distance, elements next to one another), tokens
    [rows, given] or [rows] int32 (None: none).  The temperature is rounded to float32, as the C call takes it.  `out`: a result of an earlier call of
    the same shape, written again."""
    if (out is not None and out.shape[2] == top
            and _short("logprobs", "gr_token_logprobs", logits, tokens, top, temperature, out.logprob, out.entropy, out.top_token, out.top_logprob,
                       out.status)):
        return out
    if not (isinstance(logits, torch.Tensor) and logits.is_cuda and logits.dim() == 2):
        raise GrError("logits must be a [rows, V] CUDA tensor")
    R, V = logits.shape
    dev, code = logits.device, _dtype_code(logits)
    step = logits.stride()
    ld = step[0] if R > 1 else V
    if logits.numel() > 0 and ((V > 1 and step[1] != 1) or ld < V):
        raise GrError("logits: the rows must not overlap, their elements lie next to one another")
    if tokens is not None and isinstance(tokens, torch.Tensor) and tokens.dim() == 1:
        tokens = tokens.view(-1, 1) if tokens.is_contiguous() else tokens.unsqueeze(1)
    if tokens is not None and (not isinstance(tokens, torch.Tensor) or tokens.dim() != 2 or tokens.shape[0] != R):
        raise GrError("tokens must be [rows, given] or [rows] int32")
    given = 0 if tokens is None else tokens.shape[1]
    a_tokens = _need(tokens, "tokens", torch.int32, None, dev, optional=True)
    _fits("token_logprobs", R, V, given, top)
    if out is None or out.shape != (R, given, top) or out.status.device != dev:
        if top < 0:
            raise GrError("top must not be negative")
        f32, i32 = dict(dtype=torch.float32, device=dev), dict(dtype=torch.int32, device=dev)
        out = Logprobs(torch.empty(R, given, **f32), torch.empty(R, **f32), torch.empty(R, top, **i32), torch.empty(R, top, **f32),
                       torch.empty(R, **i32), (R, given, top))
    own = [_need(getattr(out, n), f"out.{n}", kind, size, dev)
           for n, kind, size in (("logprob", torch.float32, (R, given)), ("entropy", torch.float32, (R,)), ("top_token", torch.int32, (R, top)),
                                 ("top_logprob", torch.float32, (R, top)), ("status", torch.int32, (R,)))]
    if R > 0 and a_tokens and a_tokens == out.top_token.data_ptr() and top > 0:
        raise GrError("tokens is a tensor of `out`, which this call writes")
    _call(dev, "gr_token_logprobs", load_library().gr_token_logprobs, logits.data_ptr(), code, V, max(ld, V), R, temperature, a_tokens, given, top,
          *own)
    return out
