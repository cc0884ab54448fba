"""ctypes binding of ``libvideoscan.so`` -- argument marshalling only.

The functions keep the C names (``vs_create_stream``, ``vs_frame_prefill``,
``vs_decode_step``, ``vs_bank_state`` ...).  :class:`StreamBatch` is a convenience
wrapper that owns the torch tensors the library borrows (weights, workspace) and turns
tensors into pointers; every step of the method runs inside the library's CUDA kernels.
There is no fallback: if the shared library is missing, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
import threading
from typing import List, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "lib", "libvideoscan.so")

VS_OK = 0
VS_ERR_INVALID_ARG = -1
VS_ERR_STATE = -2
VS_ERR_CAPACITY = -3
VS_ERR_CUDA = -4
VS_ERR_DEVICE_TIMEOUT = -5
VS_ERR_UNSUPPORTED = -6
VS_ERR_BOUNDS = -7
VS_MAX_BATCH = 64

EXPORTS = ["vs_workspace_bytes", "vs_create_stream", "vs_frame_prefill", "vs_frame_prefill_chunk", "vs_bank_forward", "vs_decode_step",
           "vs_lm_head", "vs_end_turn", "vs_bank_state", "vs_last_step_kv", "vs_poison_scratch",
           "vs_destroy_stream", "vs_status_string", "vs_reset_stream", "vs_profile_enable",
           "vs_profile_read", "vs_kernel_class_name", "vs_evict_choose_static", "vs_rope_axes", "vs_cache_write", "vs_cache_read",
           "vs_cache_attention_bytes", "vs_cache_attention", "vs_token_logprobs"]
VS_STATIC_MAX_BANK = 4096
VS_N_KERNEL_CLASSES = 10
VS_MAX_AXES = 4
VS_MAX_TOP = 32
VS_CACHE_PAGE = 64
VS_CACHE_MAX_SEQS = 1024


class VsConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "max_tokens_per_frame",
        "max_prefix", "max_text", "max_step_tokens", "bank_capacity", "n_streams", "agg_mode",
        "evict_policy", "use_rmsnorm", "residual")] + [
        ("rope_theta", C.c_float), ("rms_eps", C.c_float), ("device", C.c_int32),
        ("evict_log_capacity", C.c_int32), ("out_dtype", C.c_int32),
        ("max_chunk_frames", C.c_int32), ("d_ff", C.c_int32), ("vocab", C.c_int32)]


class VsWeights(C.Structure):
    _fields_ = [("w_qkv", C.POINTER(C.c_void_p)), ("b_qkv", C.POINTER(C.c_void_p)),
                ("norm_w", C.POINTER(C.c_void_p)), ("w_o", C.POINTER(C.c_void_p)), ("w_gate", C.POINTER(C.c_void_p)),
                ("w_up", C.POINTER(C.c_void_p)), ("w_down", C.POINTER(C.c_void_p)), ("norm2_w", C.POINTER(C.c_void_p)),
                ("w_lm", C.c_void_p), ("norm_f_w", C.c_void_p)]


class VsBankInfo(C.Structure):
    _fields_ = [("count", C.c_int32), ("capacity", C.c_int32), ("frames_seen", C.c_int64),
                ("evictions", C.c_int64), ("next_pos", C.c_int64), ("prefix_len", C.c_int64),
                ("text_len", C.c_int64), ("last_victim_frame", C.c_int32),
                ("device_status", C.c_int32), ("persistent_bytes", C.c_uint64),
                ("workspace_bytes", C.c_uint64)]


class VsCache(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k", "v", "k_scale", "v_scale")] + [
        (n, C.c_int32) for n in ("n_pages", "n_kv_heads", "head_dim", "device")]


# The argument blocks of the stand-alone operators, packed in one go: a call of one row is bound by the host.  Field by field as in the header.
VS_ROPE = struct.Struct("3P5qd12i")
VS_CACHE_ROWS = struct.Struct("3P4i2P4q2i")
VS_CACHE_QUERIES = struct.Struct("3P4i4PQ4q4ifi")
VS_SCORES = struct.Struct("7Pq6i")


class VsError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {status_string(code)} ({code})")
        self.code = code


_lib = None


def load_library(path: Optional[str] = None) -> C.CDLL:
    """Loads the CUDA library; raises if it has not been built (there is no other path)."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise FileNotFoundError(
            f"{p} is missing: build it with `python -m paper_2503_09387_b200.build` "
            "(the library is the only implementation; nothing falls back to the CPU)")
    lib = C.CDLL(p)
    vp, i32, i32p = C.c_void_p, C.c_int32, C.POINTER(C.c_int32)
    lib.vs_workspace_bytes.argtypes = [C.POINTER(VsConfig), C.POINTER(C.c_size_t)]
    lib.vs_create_stream.argtypes = [C.POINTER(VsConfig), C.POINTER(VsWeights), vp, C.c_size_t, C.POINTER(vp)]
    lib.vs_frame_prefill.argtypes = [vp, i32p, i32, vp, i32, vp, vp, vp]
    lib.vs_frame_prefill_chunk.argtypes = [vp, i32, vp, i32, i32, vp, vp]
    lib.vs_bank_forward.argtypes = [vp, i32, vp, vp]
    lib.vs_decode_step.argtypes = [vp, i32p, i32, vp, i32, vp, vp]
    lib.vs_end_turn.argtypes = [vp, i32p, i32]
    lib.vs_lm_head.argtypes = [vp, vp, i32, vp, vp, vp]
    lib.vs_bank_state.argtypes = [vp, i32, C.POINTER(VsBankInfo), i32p, C.POINTER(C.c_int64), i32p,
                                  i32p, i32, i32p, vp, i32, vp, vp]
    lib.vs_last_step_kv.argtypes = [vp, vp, vp, i32]
    lib.vs_poison_scratch.argtypes = [vp, vp]
    lib.vs_destroy_stream.argtypes = [vp]
    lib.vs_status_string.argtypes = [C.c_int]
    lib.vs_status_string.restype = C.c_char_p
    lib.vs_reset_stream.argtypes = [vp, i32p, i32, vp]
    lib.vs_profile_enable.argtypes = [vp, i32, i32]
    lib.vs_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
    lib.vs_evict_choose_static.argtypes = [vp, vp, i32, i32, i32, vp, vp]
    block = C.c_char_p                                                  # (a packed argument block)
    lib.vs_rope_axes.argtypes = [block, vp]
    lib.vs_cache_write.argtypes = lib.vs_cache_read.argtypes = lib.vs_cache_attention.argtypes = [C.POINTER(VsCache), block, vp]
    lib.vs_cache_attention_bytes.argtypes = [i32, C.POINTER(C.c_size_t)]
    lib.vs_token_logprobs.argtypes = [block, vp]
    lib.vs_kernel_class_name.argtypes = [i32]
    lib.vs_kernel_class_name.restype = C.c_char_p
    for name in EXPORTS:
        if name not in ("vs_status_string", "vs_kernel_class_name"):
            getattr(lib, name).restype = C.c_int
    if path is None:
        _lib = lib
    return lib


def status_string(code: int) -> str:
    return load_library().vs_status_string(code).decode()


def _check(code: int, what: str) -> None:
    if code != VS_OK:
        raise VsError(code, what)


_id_arrays = {n: C.c_int32 * n for n in range(65)}       # (making the type takes longer than filling an array of it)


def _ids(stream_ids: Sequence[int]):
    n = len(stream_ids)
    return (_id_arrays.get(n) or C.c_int32 * n)(*stream_ids), n


# ---- C-named entry points (thin) ----------------------------------------------------------
def vs_workspace_bytes(cfg: VsConfig) -> int:
    out = C.c_size_t(0)
    _check(load_library().vs_workspace_bytes(C.byref(cfg), C.byref(out)), "vs_workspace_bytes")
    return int(out.value)


def vs_create_stream(cfg: VsConfig, w_ptrs: List[int], b_ptrs: Optional[List[Optional[int]]],
                     g_ptrs: Optional[List[Optional[int]]], workspace_ptr: int, workspace_bytes: int,
                     block_ptrs: Optional[dict] = None, lm_ptrs: Optional[Sequence[Optional[int]]] = None) -> int:
    """block_ptrs (full decoder block, cfg.d_ff > 0): {"w_o", "w_gate", "w_up", "w_down": [L pointers], "norm2_w": [L] or None}.
    lm_ptrs (language-model head, cfg.vocab > 0): (w_lm pointer, final-norm gain pointer or None)."""
    L = cfg.n_layers
    arr = lambda ptrs: C.cast((C.c_void_p * L)(*[p or None for p in ptrs]), C.POINTER(C.c_void_p)) if ptrs is not None else None
    keep = [arr(w_ptrs), arr(b_ptrs), arr(g_ptrs)]
    for name in ("w_o", "w_gate", "w_up", "w_down", "norm2_w"):
        keep.append(arr(block_ptrs.get(name)) if block_ptrs else None)
    ws = VsWeights(*keep, (lm_ptrs[0] if lm_ptrs else None), (lm_ptrs[1] if lm_ptrs else None) or None)
    handle = C.c_void_p(None)
    _check(load_library().vs_create_stream(C.byref(cfg), C.byref(ws), workspace_ptr, workspace_bytes,
                                           C.byref(handle)), "vs_create_stream")
    return handle.value


def vs_frame_prefill(handle: int, stream_ids: Sequence[int], hidden_ptr: int, N: int,
                     carrier_override_ptr: Optional[int], out_ptr: Optional[int], cuda_stream: int = 0) -> None:
    ids, n = _ids(stream_ids)
    _check(load_library().vs_frame_prefill(handle, ids, n, hidden_ptr, N, carrier_override_ptr or None,
                                           out_ptr or None, cuda_stream or None), "vs_frame_prefill")


def vs_lm_head(handle: int, hidden_ptr: int, rows: int, logits_ptr: int, next_token_ptr: Optional[int],
               cuda_stream: Optional[int] = None) -> None:
    _check(load_library().vs_lm_head(handle, hidden_ptr, rows, logits_ptr, next_token_ptr or None, cuda_stream or None),
           "vs_lm_head")


def vs_bank_forward(handle: int, stream_id: int, out_ptr: int, cuda_stream: Optional[int] = None) -> None:
    _check(load_library().vs_bank_forward(handle, stream_id, out_ptr, cuda_stream or None), "vs_bank_forward")


def vs_frame_prefill_chunk(handle: int, stream_id: int, hidden_ptr: int, F: int, N: int,
                           out_ptr: Optional[int] = None, cuda_stream: Optional[int] = None) -> None:
    _check(load_library().vs_frame_prefill_chunk(handle, stream_id, hidden_ptr, F, N, out_ptr or None,
                                                 cuda_stream or None), "vs_frame_prefill_chunk")


def vs_decode_step(handle: int, stream_ids: Sequence[int], hidden_ptr: int, T: int, out_ptr: int,
                   cuda_stream: int = 0) -> None:
    ids, n = _ids(stream_ids)
    _check(load_library().vs_decode_step(handle, ids, n, hidden_ptr, T, out_ptr, cuda_stream or None),
           "vs_decode_step")


def vs_end_turn(handle: int, stream_ids: Sequence[int]) -> None:
    ids, n = _ids(stream_ids)
    _check(load_library().vs_end_turn(handle, ids, n), "vs_end_turn")


def vs_reset_stream(handle: int, stream_ids: Sequence[int], cuda_stream: int = 0) -> None:
    ids, n = _ids(stream_ids)
    _check(load_library().vs_reset_stream(handle, ids, n, cuda_stream or None), "vs_reset_stream")


def vs_profile_enable(handle: int, on: bool, max_launches: int = 0) -> None:
    _check(load_library().vs_profile_enable(handle, 1 if on else 0, max_launches), "vs_profile_enable")


def vs_profile_read(handle: int) -> dict:
    """{class name: (summed ms of timed launches, timed launches, all launches)} since the last read."""
    lib = load_library()
    ms = (C.c_double * VS_N_KERNEL_CLASSES)()
    timed = (C.c_int64 * VS_N_KERNEL_CLASSES)()
    launches = (C.c_int64 * VS_N_KERNEL_CLASSES)()
    _check(lib.vs_profile_read(handle, ms, timed, launches), "vs_profile_read")
    return {lib.vs_kernel_class_name(k).decode(): (ms[k], int(timed[k]), int(launches[k]))
            for k in range(VS_N_KERNEL_CLASSES)}


def vs_evict_choose_static(bank_emb_ptr: int, incoming_ptr: int, count: int, d_model: int, policy: int,
                           victim_out_ptr: int, cuda_stream: int = 0) -> None:
    """Enqueues the allocation-free eviction decision; the result lands in the int32 at victim_out_ptr."""
    _check(load_library().vs_evict_choose_static(bank_emb_ptr, incoming_ptr, count, d_model, policy,
                                                 victim_out_ptr, cuda_stream or None), "vs_evict_choose_static")


def vs_destroy_stream(handle: int) -> None:
    _check(load_library().vs_destroy_stream(handle), "vs_destroy_stream")


def vs_poison_scratch(handle: int, cuda_stream: int = 0) -> None:
    _check(load_library().vs_poison_scratch(handle, cuda_stream or None), "vs_poison_scratch")


def vs_bank_state(handle: int, stream_id: int, cfg: VsConfig, layer: Optional[int] = None,
                  want_emb: bool = False) -> dict:
    """Synchronises and returns the bank of one stream in temporal order (numpy arrays;
    bf16 tensors as uint16 bit patterns)."""
    lib = load_library()
    M = max(cfg.bank_capacity, 1)
    info = VsBankInfo()
    frame_ids = np.zeros(M, dtype=np.int32)
    positions = np.zeros(M, dtype=np.int64)
    slots = np.zeros(M, dtype=np.int32)
    cap = max(cfg.evict_log_capacity, 1)
    log = np.zeros((cap, 2), dtype=np.int32)
    log_n = C.c_int32(0)
    emb = np.zeros((M, cfg.d_model), dtype=np.uint16) if want_emb else None
    k = v = None
    if layer is not None:
        k = np.zeros((M, cfg.n_kv_heads, cfg.head_dim), dtype=np.uint16)
        v = np.zeros_like(k)
    p = lambda a: a.ctypes.data_as(C.c_void_p) if a is not None else None
    code = lib.vs_bank_state(handle, stream_id, C.byref(info),
                             frame_ids.ctypes.data_as(C.POINTER(C.c_int32)),
                             positions.ctypes.data_as(C.POINTER(C.c_int64)),
                             slots.ctypes.data_as(C.POINTER(C.c_int32)),
                             log.ctypes.data_as(C.POINTER(C.c_int32)), cap, C.byref(log_n),
                             p(emb), layer if layer is not None else 0, p(k), p(v))
    _check(code, "vs_bank_state")
    n = info.count
    res = dict(count=n, capacity=info.capacity, frames_seen=info.frames_seen, evictions=info.evictions,
               next_pos=info.next_pos, prefix_len=info.prefix_len, text_len=info.text_len,
               last_victim_frame=info.last_victim_frame, device_status=info.device_status,
               persistent_bytes=info.persistent_bytes, workspace_bytes=info.workspace_bytes,
               frame_ids=frame_ids[:n].copy(), positions=positions[:n].copy(), slots=slots[:n].copy(),
               evict_log=log[:log_n.value].copy())
    if emb is not None:
        res["emb"] = emb[:n].copy()
    if k is not None:
        res["k"] = k[:n].copy()
        res["v"] = v[:n].copy()
    return res


def vs_last_step_kv(handle: int, rows: int, n_kv_heads: int, head_dim: int):
    k = np.zeros((rows, n_kv_heads * head_dim), dtype=np.uint16)
    v = np.zeros_like(k)
    _check(load_library().vs_last_step_kv(handle, k.ctypes.data_as(C.c_void_p), v.ctypes.data_as(C.c_void_p), rows),
           "vs_last_step_kv")
    return k, v


# ---- stand-alone operators on torch tensors ------------------------------------------------------
_torch = None
_raw_stream = None


def _need_torch():
    global _torch, _raw_stream
    if _torch is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (      # (not part of torch's public API)
            lambda i: torch.cuda.current_stream(i).cuda_stream)
        _torch = torch
    return _torch


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _dtype_code(dtype, what: str) -> int:
    if dtype is _torch.bfloat16:
        return 0
    _need(dtype is _torch.float32, what)
    return 1


def _capturing(index: int) -> bool:
    """Whether what is enqueued on the current stream of GPU ``index`` goes into a graph."""
    if _torch.cuda.current_device() == index:
        return _torch.cuda.is_current_stream_capturing()
    with _torch.cuda.device(index):
        return _torch.cuda.is_current_stream_capturing()


def _on_gpu(t, what: str) -> int:
    index = t.get_device()
    _need(index >= 0, what)
    return index


def rope_axes(x, positions, sections, theta: float = 1.0e6, interleaved: bool = False, inverse: bool = False, out=None):
    """Rotary positions with several axes: ``x`` [rows, heads, head_dim] (bf16 or fp32, any row and head stride of whole 16
    bytes) turned by ``positions`` int64 [n_axes, rows]; ``sections``: pairs of each axis, head_dim / 2 in all.  ``out``:
    where to (``x`` itself turns in place); a new tensor if None.  Returns ``out``."""
    torch = _need_torch()
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    shape, step, pos_shape, pos_step, n = x.shape, x.stride(), positions.shape, positions.stride(), len(sections)
    _need(len(shape) == 3 and pos_shape == (n, shape[0]), "rope_axes: x [rows, heads, head_dim] and positions [n_axes, rows] wanted")
    _need(1 <= n <= VS_MAX_AXES, "rope_axes: 1 to 4 axes")
    _need(positions.dtype is torch.int64 and (pos_step[1] == 1 or shape[0] <= 1), "rope_axes: positions int64, rows side by side")
    out_step = step if out is x else out.stride()
    _need(out is x or out.shape == shape and out.dtype is x.dtype, "rope_axes: out like x")
    _need(step[2] == 1 and out_step[2] == 1, "rope_axes: the elements of a head side by side")
    code, index = _dtype_code(x.dtype, "rope_axes: bf16 or fp32 wanted"), _on_gpu(x, "rope_axes: tensors on a GPU wanted")
    _need(positions.get_device() == index and out.get_device() == index, "rope_axes: tensors on one GPU wanted")
    block = VS_ROPE.pack(x.data_ptr(), out.data_ptr(), positions.data_ptr(), step[0], step[1], out_step[0], out_step[1], pos_step[0], theta,
                         code, shape[0], shape[1], shape[2], n, interleaved, inverse, index, *sections, *((0,) * (VS_MAX_AXES - n)))
    _check(load_library().vs_rope_axes(block, _raw_stream(index)), "vs_rope_axes")
    return out


def token_logprobs(logits, tokens=None, top: int = 0, out=None):
    """What rows of ``logits`` [rows, vocab] (fp32 or bf16) say about ``tokens`` int32 [rows] (None: nothing is asked):
    (logprob fp32 [rows], entropy fp32 [rows], rank int32 [rows], top_index int32 [rows, top], top_logprob fp32 [rows, top]);
    ``out``: such a tuple to write to."""
    torch = _need_torch()
    shape, step = logits.shape, logits.stride()
    _need(len(shape) == 2 and (step[1] == 1 or shape[1] == 1), "token_logprobs: logits [rows, vocab], a row's side by side")
    rows, vocab = shape
    code, index = _dtype_code(logits.dtype, "token_logprobs: fp32 or bf16 wanted"), _on_gpu(logits, "token_logprobs: tensors on a GPU wanted")
    asked = tokens is not None
    if asked:
        _need(tokens.dtype is torch.int32 and tokens.shape == (rows,) and tokens.is_contiguous() and tokens.get_device() == index,
              "token_logprobs: tokens int32 [rows]")
    if out is None:
        new = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=logits.device)
        out = (new(rows, torch.float32), new(rows, torch.float32), new(rows, torch.int32), new((rows, top), torch.int32),
               new((rows, top), torch.float32))
    else:
        for t, n, dtype in zip(out, (rows, rows, rows, rows * top, rows * top), (torch.float32, torch.float32, torch.int32, torch.int32, torch.float32)):
            _need(t.numel() == n and t.dtype is dtype and t.is_contiguous() and t.get_device() == index, "token_logprobs: out as described")
    lp, entropy, rank, best, best_lp = out
    if not asked:
        lp.zero_()
        rank.fill_(-1)
    block = VS_SCORES.pack(logits.data_ptr(), tokens.data_ptr() if asked else 0, lp.data_ptr() if asked else 0, entropy.data_ptr(),
                           rank.data_ptr() if asked else 0, best.data_ptr(), best_lp.data_ptr(), step[0], code, rows, vocab, top, index, 0)
    _check(load_library().vs_token_logprobs(block, _raw_stream(index)), "vs_token_logprobs")
    return out


class PageCache:
    """A paged cache of 8-bit keys and values over the caller's tensors: ``k``, ``v`` float8_e4m3fn [n_pages, n_kv_heads, 64,
    head_dim], ``k_scale``, ``v_scale`` fp32 [n_pages, n_kv_heads].  ``page_table`` int32 [n_seqs, table_width], ``start`` /
    ``lengths`` int32 [n_seqs] and ``row_offsets`` int32 [n_seqs + 1] (None: the same number of rows for each sequence) are device
    tensors, read when the kernels run.  All methods only enqueue work on the current torch stream."""

    def __init__(self, k, v, k_scale, v_scale):
        torch = _need_torch()
        _need(k.dim() == 4 and k.shape[2] == VS_CACHE_PAGE and v.shape == k.shape and k_scale.shape == k.shape[:2] and v_scale.shape == k.shape[:2],
              "PageCache: k, v [n_pages, n_kv_heads, 64, head_dim] and scales [n_pages, n_kv_heads] wanted")
        _need(k.dtype == v.dtype == torch.float8_e4m3fn and k_scale.dtype == v_scale.dtype == torch.float32, "PageCache: e4m3 codes, fp32 scales")
        _need(all(t.is_contiguous() for t in (k, v, k_scale, v_scale)), "PageCache: contiguous tensors wanted")
        self.device_index = _on_gpu(k, "PageCache: tensors on a GPU wanted")
        _need(all(t.get_device() == self.device_index for t in (v, k_scale, v_scale)), "PageCache: tensors on one GPU wanted")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.n_kv_heads, _, self.head_dim = k.shape
        self._cache = VsCache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), self.n_pages, self.n_kv_heads,
                              self.head_dim, self.device_index)
        self._workspaces = {}
        self._attending = threading.Lock()           # a call is several launches, and two calls' may not mix on one workspace

    @classmethod
    def empty(cls, n_pages: int, n_kv_heads: int, head_dim: int, device=0) -> "PageCache":
        """A cache of its own, all zeros."""
        torch = _need_torch()
        dev = torch.device("cuda", device)
        codes = lambda: torch.zeros((n_pages, n_kv_heads, VS_CACHE_PAGE, head_dim), dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
        scales = lambda: torch.zeros((n_pages, n_kv_heads), dtype=torch.float32, device=dev)
        return cls(codes(), codes(), scales(), scales())

    def _seqs(self, page_table, tokens, row_offsets):
        """Pointers and sizes of a call's sequences, checked."""
        i32, index, shape = _torch.int32, self.device_index, page_table.shape
        _need(len(shape) == 2 and page_table.dtype is i32 and page_table.is_contiguous() and page_table.get_device() == index,
              "PageCache: page_table int32 [n_seqs, table_width], on the cache's GPU")
        n, width = shape
        _need(tokens.numel() == n and tokens.dtype is i32 and tokens.is_contiguous() and tokens.get_device() == index,
              "PageCache: start / lengths int32 [n_seqs], on the cache's GPU")
        if row_offsets is None:
            return page_table.data_ptr(), tokens.data_ptr(), 0, n, width
        _need(row_offsets.numel() == n + 1 and row_offsets.dtype is i32 and row_offsets.is_contiguous() and row_offsets.get_device() == index,
              "PageCache: row_offsets int32 [n_seqs + 1], on the cache's GPU")
        return page_table.data_ptr(), tokens.data_ptr(), row_offsets.data_ptr(), n, width

    def _kv(self, page_table, start, k, v, row_offsets):
        shape, ks, vs, dtype = k.shape, k.stride(), v.stride(), k.dtype
        _need(len(shape) == 3 and v.shape == shape and shape[1] == self.n_kv_heads and shape[2] == self.head_dim and v.dtype is dtype,
              "PageCache: k, v [n_rows, n_kv_heads, head_dim] wanted")
        _need(ks[2] == 1 and vs[2] == 1, "PageCache: the elements of a head side by side")
        _need(k.get_device() == self.device_index and v.get_device() == self.device_index, "PageCache: k, v on the cache's GPU")
        return VS_CACHE_ROWS.pack(*self._seqs(page_table, start, row_offsets), shape[0], 0, k.data_ptr(), v.data_ptr(), ks[0], ks[1], vs[0], vs[1],
                                  _dtype_code(dtype, "PageCache: rows of bf16 or fp32 wanted"), 0)

    def write(self, page_table, start, k, v, row_offsets=None):
        """Appends rows [n_rows, n_kv_heads, head_dim] (bf16 or fp32): sequence i's from its token ``start[i]`` on."""
        _check(load_library().vs_cache_write(self._cache, self._kv(page_table, start, k, v, row_offsets), _raw_stream(self.device_index)),
               "vs_cache_write")

    def read(self, page_table, start, k, v, row_offsets=None):
        """Reads rows back into k, v [n_rows, n_kv_heads, head_dim] (bf16 or fp32); returns them."""
        _check(load_library().vs_cache_read(self._cache, self._kv(page_table, start, k, v, row_offsets), _raw_stream(self.device_index)),
               "vs_cache_read")
        return k, v

    def workspace(self):
        """A workspace for ``attend``; two calls that may overlap (graphs replayed side by side) need one each."""
        workspace = self._new_workspace()
        workspace[:256].zero_()
        return workspace

    def _new_workspace(self):
        out = C.c_size_t(0)
        _check(load_library().vs_cache_attention_bytes(self.head_dim, C.byref(out)), "vs_cache_attention_bytes")
        return _torch.empty(out.value, dtype=_torch.uint8, device=self.k.device)

    def attend_status(self) -> int:
        """0, or VS_ERR_DEVICE_TIMEOUT if a wait of an ``attend`` with one of the cache's own workspaces ever ran out.  Synchronises."""
        return min([int(w[:4].view(_torch.int32).item()) for w in self._workspaces.values()], default=VS_OK)

    def attend(self, page_table, lengths, q, out=None, lse=None, row_offsets=None, scale=None, causal=True, window=0, workspace=None,
               out_dtype=None):
        """Attention of q bf16 [n_rows, n_q_heads, head_dim] over each sequence's ``lengths[i]`` tokens, its rows counted in.
        -> (out [n_rows, n_q_heads, head_dim], lse fp32 [n_rows, n_q_heads]).  ``causal`` hides what lies behind a row, ``window`` > 0 what lies
        ``window`` tokens or more ahead of it.  ``out_dtype``: of a new ``out``, bf16 or fp32.  Without
        ``workspace`` the cache keeps one for every stream it is used on; a call that is captured takes one from the graph's own memory, so
        that graphs replayed side by side share none (its status is then nobody's to read).  Several host threads may call it, on one stream too."""
        torch, index = _torch, self.device_index
        shape, step = q.shape, q.stride()
        _need(len(shape) == 3 and q.dtype is torch.bfloat16 and shape[2] == self.head_dim and step[2] == 1 and q.get_device() == index,
              "attend: q bf16 [n_rows, n_q_heads, head_dim], on the cache's GPU")
        n_rows, n_heads, head_dim = shape
        if out is None:
            out = torch.empty(shape, dtype=out_dtype or torch.bfloat16, device=q.device)
        if lse is None:
            lse = torch.empty((n_rows, n_heads), dtype=torch.float32, device=q.device)
        out_step = out.stride()
        _need(out.shape == shape and out_step[2] == 1 and out.get_device() == index, "attend: out like q")
        _need(lse.numel() == n_rows * n_heads and lse.dtype is torch.float32 and lse.is_contiguous() and lse.get_device() == index,
              "attend: lse fp32 [n_rows, n_q_heads]")
        seqs = self._seqs(page_table, lengths, row_offsets)
        code = _dtype_code(out.dtype, "attend: out of bf16 or fp32 wanted")
        _need(workspace is None or workspace.is_contiguous() and workspace.get_device() == index, "attend: a workspace on the cache's GPU")
        stream = _raw_stream(index)
        with self._attending:
            if workspace is None:
                if _capturing(index):
                    workspace = self._new_workspace()
                else:
                    workspace = self._workspaces.get(stream)
                    if workspace is None:
                        workspace = self._workspaces[stream] = self.workspace()
            block = VS_CACHE_QUERIES.pack(*seqs, n_rows, 0, q.data_ptr(), out.data_ptr(), lse.data_ptr(), workspace.data_ptr(), workspace.nbytes,
                                          step[0], step[1], out_step[0], out_step[1], n_heads, causal, window, code,
                                          head_dim ** -0.5 if scale is None else scale, 0)
            _check(load_library().vs_cache_attention(self._cache, block, stream), "vs_cache_attention")
        return out, lse


# ---- convenience wrapper: owns the borrowed tensors -------------------------------------------
class StreamBatch:
    """A handle plus the device tensors it borrows.  ``weights`` are torch bf16 CUDA tensors
    [E_out, d_model] per layer.  All methods take / return torch CUDA tensors and only enqueue
    work on the current torch stream."""

    def __init__(self, cfg: VsConfig, weights, biases=None, norm_weights=None, block=None, lm=None):
        # block (cfg.d_ff > 0): {"w_o", "w_gate", "w_up", "w_down": [L device tensors], "norm2_w": [L] or None}
        # lm (cfg.vocab > 0): (w_lm [vocab, d_model] device tensor, final-norm gain [d_model] or None)
        import torch
        self.torch = torch
        self.cfg = cfg
        self.device = torch.device("cuda", cfg.device)
        self.device_index = int(cfg.device)
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # (not part of torch's public API)
        self.weights = [w.contiguous() for w in weights]
        self.biases = biases
        self.norm_weights = norm_weights
        self.block = block
        self.lm = lm
        nbytes = vs_workspace_bytes(cfg)
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = self.workspace.data_ptr()
        self._ws_ptr = (base + 255) // 256 * 256
        self.workspace_bytes = nbytes
        self.handle = vs_create_stream(
            cfg, [w.data_ptr() for w in self.weights],
            [b.data_ptr() if b is not None else None for b in biases] if biases is not None else None,
            [g.data_ptr() if g is not None else None for g in norm_weights] if norm_weights is not None else None,
            self._ws_ptr, nbytes,
            {k: ([t.data_ptr() if t is not None else None for t in v] if v is not None else None) for k, v in block.items()}
            if block else None,
            (lm[0].data_ptr(), lm[1].data_ptr() if lm[1] is not None else None) if lm else None)
        self.out_width = cfg.n_q_heads * cfg.head_dim
        self.out_torch_dtype = torch.float32 if cfg.out_dtype == 1 else torch.bfloat16

    def _stream(self) -> int:
        # without the Stream object where this torch has the call: a token step of one layer is bound by the host
        if self._raw_stream is not None:
            return self._raw_stream(self.device_index)
        return self.torch.cuda.current_stream(self.device).cuda_stream

    def lm_head(self, hidden, logits=None, want_token=True):
        """hidden: [rows, d_model] of the handle's output dtype -> (logits fp32 [rows, vocab], next tokens int32 [rows] or None)."""
        rows = hidden.shape[0]
        assert hidden.is_contiguous() and hidden.dtype == self.out_torch_dtype and hidden.numel() == rows * self.cfg.d_model
        if logits is None:
            logits = self.torch.empty((rows, self.cfg.vocab), dtype=self.torch.float32, device=self.device)
        token = self.torch.empty((rows,), dtype=self.torch.int32, device=self.device) if want_token else None
        vs_lm_head(self.handle, hidden.data_ptr(), rows, logits.data_ptr(), token.data_ptr() if want_token else None, self._stream())
        return logits, token

    def lm_score(self, hidden, tokens, top=0, logits=None):
        """What the language-model head says about given answer tokens: ``lm_head`` of hidden [rows, d_model], then
        ``token_logprobs`` of its logits for tokens int32 [rows] -> (logprob, entropy, rank, top_index, top_logprob)."""
        logits, _ = self.lm_head(hidden, logits, want_token=False)
        return token_logprobs(logits, tokens, top=top)

    def frame_prefill(self, stream_ids, hidden, carrier_override=None, out=None, want_out=True):
        n = len(stream_ids)
        N = hidden.shape[-2]
        assert hidden.is_contiguous() and hidden.numel() == n * N * self.cfg.d_model
        if out is None and want_out:
            out = self.torch.empty((n, N + 1, self.out_width), dtype=self.out_torch_dtype, device=self.device)
        vs_frame_prefill(self.handle, stream_ids, hidden.data_ptr(), N,
                         carrier_override.data_ptr() if carrier_override is not None else None,
                         out.data_ptr() if out is not None else None, self._stream())
        return out

    def frame_prefill_chunk(self, stream_id, hidden, out=None, want_out=True):
        """hidden: [F][N][d] of one stream."""
        F, N = hidden.shape[0], hidden.shape[1]
        assert hidden.is_contiguous() and hidden.numel() == F * N * self.cfg.d_model
        if out is None and want_out:
            out = self.torch.empty((F, N + 1, self.out_width), dtype=self.out_torch_dtype, device=self.device)
        vs_frame_prefill_chunk(self.handle, stream_id, hidden.data_ptr(), F, N,
                               out.data_ptr() if out is not None else None, self._stream())
        return out

    def bank_forward(self, stream_id, count):
        """Carriers-only forward of one stream's bank; `count` = carriers in it."""
        out = self.torch.empty((count, self.out_width), dtype=self.out_torch_dtype, device=self.device)
        vs_bank_forward(self.handle, stream_id, out.data_ptr(), self._stream())
        return out

    def decode_step(self, stream_ids, hidden, out=None):
        n = len(stream_ids)
        T = hidden.shape[-2]
        assert hidden.is_contiguous() and hidden.numel() == n * T * self.cfg.d_model
        if out is None:
            out = self.torch.empty((n, T, self.out_width), dtype=self.out_torch_dtype, device=self.device)
        vs_decode_step(self.handle, stream_ids, hidden.data_ptr(), T, out.data_ptr(), self._stream())
        return out

    def end_turn(self, stream_ids):
        vs_end_turn(self.handle, stream_ids)

    def bank_state(self, stream_id=0, layer=None, want_emb=False):
        return vs_bank_state(self.handle, stream_id, self.cfg, layer, want_emb)

    def last_step_kv(self, rows):
        return vs_last_step_kv(self.handle, rows, self.cfg.n_kv_heads, self.cfg.head_dim)

    def reset(self, stream_ids):
        vs_reset_stream(self.handle, stream_ids, self._stream())

    def profile_enable(self, on, max_launches=0):
        vs_profile_enable(self.handle, on, max_launches)

    def profile_read(self):
        return vs_profile_read(self.handle)

    def poison_scratch(self):
        vs_poison_scratch(self.handle, self._stream())

    def close(self):
        if self.handle:
            vs_destroy_stream(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def make_config(n_layers, d_model, n_q_heads, n_kv_heads, head_dim, max_tokens_per_frame, max_prefix,
                max_text, bank_capacity, n_streams=1, max_step_tokens=64, agg_mode=0, evict_policy=0,
                use_rmsnorm=0, residual=0, rope_theta=1.0e6, rms_eps=1.0e-6, device=0,
                evict_log_capacity=4096, out_dtype=1, max_chunk_frames=1, d_ff=0, vocab=0) -> VsConfig:
    return VsConfig(n_layers, d_model, n_q_heads, n_kv_heads, head_dim, max_tokens_per_frame, max_prefix,
                    max_text, max_step_tokens, bank_capacity, n_streams, agg_mode, evict_policy, use_rmsnorm,
                    residual, rope_theta, rms_eps, device, evict_log_capacity, out_dtype, max_chunk_frames, d_ff, vocab)
