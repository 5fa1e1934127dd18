"""ctypes binding of libgbmla.so (``include/gbmla.h``).

Argument marshalling only: every function here forwards torch tensors' device
pointers, sizes and the current CUDA stream to the C entry point of the same
name and raises ``MlaError`` on a non-OK status.  All compute happens in the
library's kernels.  PyTorch supplies device memory and streams.
"""
from __future__ import annotations

import ctypes
import os
import threading
from dataclasses import dataclass
from typing import Optional

import torch

from . import build as _build

MLA_OK, MLA_ERR_INVALID_ARG, MLA_ERR_UNSUPPORTED, MLA_ERR_CUDA, MLA_ERR_DEVICE_BOUNDS, MLA_ERR_DEVICE_TIMEOUT = range(6)
SPLIT_TILE = 128
EXPORTS = ("mla_workspace_size", "mla_cache_append", "mla_project_append", "mla_acceptance_stats",
           "mla_gqa_append", "mla_gqa_workspace_size", "mla_gqa_decode_attn", "mla_gqa_project", "mla_gqa_out_proj",
           "mla_gqa_prompt_append", "mla_gqa_prompt_workspace_size", "mla_gqa_prompt_attn", "mla_gqa_prompt_out_proj",
           "mla_token_logprobs", "mla_pages_workspace_size", "mla_pages_release", "mla_pages_reserve",
           "mla_pages_fork", "mla_pages_compact", "mla_e2e_loss", "mla_absorb_q", "mla_decode_attn", "mla_combine",
           "mla_out_proj", "mla_decode_step", "mla_check_status", "mla_selftest_wait_timeout",
           "mla_selftest_wait_looks",
           "mla_decode_attn_noalloc", "mla_reload_tuning", "mla_status_str", "mla_last_error")


class MlaError(RuntimeError):
    def __init__(self, where: str, code: int, name: str):
        super().__init__(f"{where}: {name}")
        self.code = code
        self.name = name


class MlaDims(ctypes.Structure):
    _fields_ = [("num_heads", ctypes.c_int32), ("num_kv_groups", ctypes.c_int32), ("d_nope", ctypes.c_int32),
                ("d_rope", ctypes.c_int32), ("d_v", ctypes.c_int32), ("rank", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("sm_scale", ctypes.c_float), ("rope_style", ctypes.c_int32),
                ("rope_base", ctypes.c_float)]


class MlaGqaDims(ctypes.Structure):
    _fields_ = [("num_heads", ctypes.c_int32), ("num_kv_groups", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("sm_scale", ctypes.c_float), ("rope_style", ctypes.c_int32), ("rope_base", ctypes.c_float)]


class MlaCache(ctypes.Structure):
    _fields_ = [("c_kv", ctypes.c_void_p), ("k_rope", ctypes.c_void_p), ("c_tok_stride", ctypes.c_int64),
                ("r_tok_stride", ctypes.c_int64), ("c_blk_stride", ctypes.c_int64), ("r_blk_stride", ctypes.c_int64),
                ("block_table", ctypes.c_void_p), ("bt_stride", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("capacity", ctypes.c_int32)]


class MlaPagePool(ctypes.Structure):
    _fields_ = [("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("num_rows", ctypes.c_int32), ("bt_stride", ctypes.c_int32), ("refs", ctypes.c_void_p),
                ("block_table", ctypes.c_void_p)]


_lock = threading.Lock()
_lib = None


def library_path() -> str:
    return _build.LIB


def lib(auto_build: bool = True):
    """The loaded library (built first if missing or stale and ``auto_build``)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            # GBMLA_LIBRARY selects another build of the library
            path = os.environ.get("GBMLA_LIBRARY") or (_build.build() if auto_build else _build.LIB)
            if not os.path.exists(path):
                raise RuntimeError(f"libgbmla.so is missing at {path}; run paper_2607_27269_gb300.build.build()")
            L = ctypes.CDLL(path)
            vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
            P = ctypes.POINTER
            L.mla_status_str.restype = ctypes.c_char_p
            L.mla_status_str.argtypes = [ctypes.c_int]
            L.mla_workspace_size.argtypes = [P(MlaDims), i32, i32, i32, i32, P(sz), P(sz), P(i32)]
            L.mla_cache_append.argtypes = [P(MlaDims), P(MlaCache), i32, i32, vp, vp, vp, vp]
            L.mla_project_append.argtypes = [P(MlaDims), P(MlaCache), i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
            L.mla_absorb_q.argtypes = [P(MlaDims), i32, i32, vp, vp, vp, vp, vp, vp]
            L.mla_acceptance_stats.argtypes = [i32, i32, i32, vp, vp, i64, vp, vp, vp, vp, vp]
            L.mla_gqa_append.argtypes = [P(MlaGqaDims), P(MlaCache), i32, i32, vp, vp, vp, vp]
            L.mla_gqa_project.argtypes = [P(MlaGqaDims), i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
            L.mla_gqa_out_proj.argtypes = [P(MlaGqaDims), i32, i32, i32, vp, vp, vp, vp]
            L.mla_e2e_loss.argtypes = [i32, i32, vp, vp, vp, vp, vp]
            L.mla_gqa_prompt_append.argtypes = [P(MlaGqaDims), P(MlaCache), i32, i32, vp, vp, vp, i64, vp, i64, vp, i64,
                                                vp, i64, vp]
            L.mla_gqa_prompt_workspace_size.argtypes = [P(MlaGqaDims), i32, i32, i32, i32, P(sz), P(sz), P(i32)]
            L.mla_gqa_prompt_attn.argtypes = [P(MlaGqaDims), P(MlaCache), i32, i32, vp, vp, i32, vp, i64, i32, vp, vp,
                                              vp, vp, vp]
            L.mla_gqa_prompt_out_proj.argtypes = [P(MlaGqaDims), i32, i32, vp, vp, vp, vp]
            L.mla_token_logprobs.argtypes = [i32, i32, i32, vp, i64, vp, i32, vp, vp, vp, vp, vp, vp]
            L.mla_pages_workspace_size.argtypes = [P(MlaPagePool), P(sz)]
            L.mla_pages_release.argtypes = [P(MlaPagePool), i32, vp, vp, vp]
            L.mla_pages_reserve.argtypes = [P(MlaPagePool), i32, vp, vp, vp, vp]
            L.mla_pages_fork.argtypes = [P(MlaPagePool), i32, P(MlaCache), i32, i32, i32, vp, vp, vp, vp, vp]
            L.mla_pages_compact.argtypes = [P(MlaPagePool), i32, P(MlaCache), i32, i32, vp, vp]
            L.mla_gqa_workspace_size.argtypes = [P(MlaGqaDims), i32, i32, i32, i32, P(sz), P(sz), P(i32)]
            L.mla_gqa_decode_attn.argtypes = [P(MlaGqaDims), P(MlaCache), i32, i32, vp, i32, vp, i32, vp, vp, vp, vp,
                                              vp]
            L.mla_decode_attn.argtypes = [P(MlaDims), P(MlaCache), i32, i32, vp, i32, vp, i32, vp, vp, vp]
            L.mla_combine.argtypes = [P(MlaDims), i32, i32, i32, vp, i32, vp, vp, vp, vp, vp]
            L.mla_out_proj.argtypes = [P(MlaDims), i32, i32, vp, vp, vp, vp, vp, vp]
            L.mla_decode_step.argtypes = [P(MlaDims), P(MlaCache), i32, i32, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp,
                                          i32, vp, vp, vp, vp, vp, vp, vp, vp]
            L.mla_check_status.argtypes = [vp]
            L.mla_selftest_wait_timeout.argtypes = [i64, vp]
            L.mla_selftest_wait_looks.argtypes = [vp, vp]
            L.mla_decode_attn_noalloc.argtypes = [P(MlaDims), P(MlaCache), i32, i32, vp, i32, vp, i32, vp, vp, vp]
            L.mla_last_error.restype = ctypes.c_char_p
            L.mla_last_error.argtypes = []
            for name in EXPORTS[:-3]:
                getattr(L, name).restype = ctypes.c_int
            L.mla_reload_tuning.restype = None
            L.mla_reload_tuning.argtypes = []
            _lib = L
        return _lib


def reload_tuning() -> None:
    """Re-read the GBMLA_* testing variables (mla_reload_tuning)."""
    lib().mla_reload_tuning()


def status_name(code: int) -> str:
    return lib().mla_status_str(code).decode()


def _check(where: str, code: int):
    if code != MLA_OK:
        name = status_name(code)
        if code == MLA_ERR_CUDA:
            name += f" ({lib().mla_last_error().decode()})"
        raise MlaError(where, code, name)


# The current stream's handle without a torch.cuda.Stream around it (0.2 us a
# call instead of 2.9, of the 15 us a one-launch call took on the host).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None and _raw_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_raw_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _new_on(stream):
    """torch.empty for what a call writes on ``stream``: in that stream's memory, since a block of the current stream's
    may still be in use by work queued there, and is handed out again there when its tensor goes."""
    if stream is None:
        return torch.empty
    on = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(_stream(stream))

    def new(*shape, **kw):
        with torch.cuda.stream(on):
            return torch.empty(*shape, **kw)

    return new


def _p(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    if not t.is_cuda:
        raise ValueError("tensor must live on the GPU")
    raise ValueError("tensor must be contiguous")


@dataclass
class Dims:
    num_heads: int
    num_kv_groups: int
    d_nope: int
    d_rope: int
    d_v: int
    rank: int
    hidden: int = 0
    sm_scale: float = 1.0
    rope_style: int = 0
    rope_base: float = 10000.0

    def c(self) -> MlaDims:
        return MlaDims(self.num_heads, self.num_kv_groups, self.d_nope, self.d_rope, self.d_v, self.rank,
                       self.hidden, self.sm_scale, self.rope_style, self.rope_base)


@dataclass
class Cache:
    """Device cache: ``c_kv`` [blocks, block_tokens, r] and ``k_rope``
    [blocks, block_tokens, d_rope] bf16 (or strided views of one fused
    buffer), blocks = sequences (contiguous) or pages (paged)."""
    c_kv: torch.Tensor
    k_rope: torch.Tensor
    capacity: int
    block_table: Optional[torch.Tensor] = None
    page_size: int = 0
    num_pages: int = 0

    def c(self) -> MlaCache:
        c, k = self.c_kv, self.k_rope
        cs, ks = c.stride(), k.stride()
        for t, s in ((c, cs), (k, ks)):
            if not t.is_cuda or t.dtype != torch.bfloat16 or len(s) != 3 or s[2] != 1:
                raise ValueError("cache tensors must be 3-d bf16 CUDA tensors with unit inner stride")
        bt = self.block_table
        return MlaCache(c.data_ptr(), k.data_ptr(), cs[1], ks[1], cs[0], ks[0],
                        _p(bt), 0 if bt is None else bt.shape[1], self.page_size, self.num_pages, self.capacity)


def workspace_size(dims: Dims, batch: int, q_len: int, max_kv_len: int, num_splits: int = 0):
    """(o_part_bytes, lse_part_bytes, num_splits_used)."""
    ob, lb, s = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_int32()
    _check("mla_workspace_size", lib().mla_workspace_size(ctypes.byref(dims.c()), batch, q_len, max_kv_len,
                                                          num_splits, ctypes.byref(ob), ctypes.byref(lb),
                                                          ctypes.byref(s)))
    return ob.value, lb.value, s.value


def cache_append(dims: Dims, cache: Cache, c_new: torch.Tensor, kr_new: torch.Tensor, start_pos: torch.Tensor,
                 stream=None):
    batch, n_new = c_new.shape[0], c_new.shape[1]
    _check("mla_cache_append", lib().mla_cache_append(ctypes.byref(dims.c()), ctypes.byref(cache.c()), batch, n_new,
                                                      _p(c_new), _p(kr_new), _p(start_pos), _stream(stream)))


def project_append(dims: Dims, cache: Cache, h: torch.Tensor, w_dkv: torch.Tensor, w_kr: torch.Tensor,
                   w_q: Optional[torch.Tensor], start_pos: torch.Tensor, q_nope: Optional[torch.Tensor] = None,
                   q_pe: Optional[torch.Tensor] = None, stream=None):
    """h [B, n, hidden] -> cache rows at start_pos + k and, with ``w_q``, the
    query parts q_nope [B, n, H, d_nope] / q_pe [B, n, H, d_rope]."""
    batch, n_new = h.shape[0], h.shape[1]
    _check("mla_project_append", lib().mla_project_append(ctypes.byref(dims.c()), ctypes.byref(cache.c()), batch,
                                                          n_new, _p(h), _p(w_dkv), _p(w_kr), _p(w_q),
                                                          _p(start_pos), _p(q_nope), _p(q_pe), _stream(stream)))


@dataclass
class GqaDims:
    """Shape of an original GQA layer (key and value width head_dim)."""
    num_heads: int
    num_kv_groups: int
    head_dim: int
    sm_scale: float
    rope_style: int = 0
    rope_base: float = 10000.0

    def c(self) -> MlaGqaDims:
        return MlaGqaDims(self.num_heads, self.num_kv_groups, self.head_dim, self.sm_scale, self.rope_style,
                          self.rope_base)


def gqa_append(dims: GqaDims, cache: Cache, k_new: torch.Tensor, v_new: torch.Tensor, start_pos: torch.Tensor,
               stream=None):
    """k_new / v_new [B, n, G, head_dim] into the GQA cache (keys in cache.k_rope, values in cache.c_kv)."""
    batch, n_new = k_new.shape[0], k_new.shape[1]
    _check("mla_gqa_append", lib().mla_gqa_append(ctypes.byref(dims.c()), ctypes.byref(cache.c()), batch, n_new,
                                                  _p(k_new), _p(v_new), _p(start_pos), _stream(stream)))


def gqa_workspace_size(dims: GqaDims, batch: int, q_len: int, max_kv_len: int, num_splits: int = 0):
    ob, lb, s = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_int32()
    _check("mla_gqa_workspace_size", lib().mla_gqa_workspace_size(ctypes.byref(dims.c()), batch, q_len, max_kv_len,
                                                                  num_splits, ctypes.byref(ob), ctypes.byref(lb),
                                                                  ctypes.byref(s)))
    return ob.value, lb.value, s.value


class GqaStep:
    """GQA decode attention with its partial buffers allocated once:
    o [B, q_len, H, head_dim] fp32, lse [B, q_len, H]."""

    def __init__(self, dims: GqaDims, cache: Cache, batch: int, q_len: int, max_kv_len: int, num_splits: int = 0):
        self.dims, self.cache, self.batch, self.q_len, self.max_kv_len = dims, cache, batch, q_len, max_kv_len
        dev = cache.c_kv.device
        ob, lb, self.num_splits = gqa_workspace_size(dims, batch, q_len, max_kv_len, num_splits)
        G, hpg, d = dims.num_kv_groups, dims.num_heads // dims.num_kv_groups, dims.head_dim
        self.o_part = torch.empty(max(ob // 4, 1), dtype=torch.float32, device=dev)
        self.lse_part = torch.empty(max(lb // 4, 1), dtype=torch.float32, device=dev)
        self.o = torch.empty(batch, q_len, dims.num_heads, d, dtype=torch.float32, device=dev)
        self.lse = torch.empty(batch, q_len, dims.num_heads, dtype=torch.float32, device=dev)

    def __call__(self, q: torch.Tensor, kv_len: torch.Tensor, stream=None):
        _check("mla_gqa_decode_attn", lib().mla_gqa_decode_attn(
            ctypes.byref(self.dims.c()), ctypes.byref(self.cache.c()), self.batch, self.q_len, _p(kv_len),
            self.max_kv_len, _p(q), self.num_splits, _p(self.o_part), _p(self.lse_part), _p(self.o), _p(self.lse),
            _stream(stream)))
        return self.o


def gqa_project(dims: GqaDims, h: torch.Tensor, w_q, w_k, w_v, q, k_new, v_new, stream=None):
    """q [B, n, H, d], k_new / v_new [B, n, G, d] = h [B, n, D] times W_Q^T, W_K^T, W_V^T (bf16)."""
    batch, n_new, hidden = h.shape
    _check("mla_gqa_project", lib().mla_gqa_project(ctypes.byref(dims.c()), batch, n_new, hidden, _p(h), _p(w_q),
                                                    _p(w_k), _p(w_v), _p(q), _p(k_new), _p(v_new), _stream(stream)))


def gqa_out_proj(dims: GqaDims, o: torch.Tensor, w_o: torch.Tensor, out: torch.Tensor, stream=None):
    """out [B, q, D] = W_O concat_h o (o fp32 [B, q, H, d])."""
    batch, q_len = o.shape[:2]
    _check("mla_gqa_out_proj", lib().mla_gqa_out_proj(ctypes.byref(dims.c()), batch, q_len, w_o.shape[0], _p(o),
                                                      _p(w_o), _p(out), _stream(stream)))


def _rows(t: Optional[torch.Tensor], heads: int, width: int, total: Optional[int] = None):
    """(pointer, token stride) of packed rows [total, heads, width]: bf16, heads and their entries dense."""
    if t is None:
        return None, 0
    shape = t.shape
    if not t.is_cuda or t.dtype != torch.bfloat16 or len(shape) != 3 or shape[1] != heads or shape[2] != width:
        raise ValueError(f"packed rows must be bf16 CUDA tensors [total, {heads}, {width}]")
    if total is not None and shape[0] != total:
        raise ValueError("packed rows must share their token count")
    s = t.stride()
    if s[2] != 1 or (heads > 1 and s[1] != width):
        raise ValueError("packed rows must have dense heads (only the token stride is free)")
    return t.data_ptr(), s[0] if shape[0] > 1 else (heads * width + 7) // 8 * 8


def gqa_prompt_append(dims: GqaDims, cache: Cache, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor,
                      cu_seqlens: torch.Tensor, start_pos: torch.Tensor, q_rot: Optional[torch.Tensor] = None,
                      stream=None):
    """Packed prompts (k / v [total, G, head_dim], q [total, H, head_dim] or None; token strides are free) at
    positions start_pos[b] + i into the GQA cache; the rotated queries go to ``q_rot`` (may be ``q``)."""
    total, batch = k.shape[0], start_pos.shape[0]
    if cu_seqlens.shape[0] != batch + 1:
        raise ValueError("cu_seqlens holds one entry more than start_pos")
    H, G, d = dims.num_heads, dims.num_kv_groups, dims.head_dim
    _check("mla_gqa_prompt_append", lib().mla_gqa_prompt_append(
        ctypes.byref(dims.c()), ctypes.byref(cache.c()), batch, total, _i32(cu_seqlens), _i32(start_pos),
        *_rows(q, H, d, total), *_rows(k, G, d), *_rows(v, G, d, total), *_rows(q_rot, H, d, total), _stream(stream)))


def _i32(t: Optional[torch.Tensor]):
    if t is not None and t.dtype != torch.int32:
        raise ValueError("lengths, positions and indices must be int32")
    return _p(t)


def _room(t: torch.Tensor, rows: int, width: int, dtype: torch.dtype, device: torch.device):
    """A caller's tensor holds what a call writes: rows of `width` entries (0: nothing), one behind the other."""
    if width == 0:
        return
    if t.dtype != dtype or t.device != device:
        raise ValueError(f"outputs must be {dtype} tensors on {device}")
    if t.numel() < rows * width or (t.dim() > 1 and t.shape[-1] != width) or not t.is_contiguous():
        raise ValueError(f"outputs must be contiguous and hold {rows} rows of {width}")


def gqa_prompt_workspace_size(dims: GqaDims, batch: int, total: int, max_kv_len: int, num_splits: int = 0):
    """(o_part_bytes, lse_part_bytes, num_splits_used)."""
    ob, lb, s = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_int32()
    _check("mla_gqa_prompt_workspace_size", lib().mla_gqa_prompt_workspace_size(
        ctypes.byref(dims.c()), batch, total, max_kv_len, num_splits, ctypes.byref(ob), ctypes.byref(lb),
        ctypes.byref(s)))
    return ob.value, lb.value, s.value


class GqaPrompt:
    """Whole prompts of an original GQA layer: packed ragged sequences of up to
    ``batch`` sequences and ``max_tokens`` tokens a call, with every buffer
    allocated once (the rotated queries', the projections' and each hidden
    width's at their first use, in the memory of that call's stream) and kept as
    long as the handle, which has to outlive the work queued with it.  The cache's
    tensors are those that it has at each call.  ``append`` writes a call's keys and values to the cache and
    rotates its queries, ``attend`` runs the causal attention over the cache
    (o [total, H, head_dim] bf16, ``lse`` [total, H]), ``__call__`` both, and
    ``from_hidden`` the whole layer from hidden states to its output
    projection."""

    def __init__(self, dims: GqaDims, cache: Cache, batch: int, max_tokens: int, max_kv_len: int, num_splits: int = 0):
        self.dims, self.cache, self.batch, self.max_tokens = dims, cache, batch, max_tokens
        self.max_kv_len, self.num_splits = max_kv_len, num_splits
        dev = cache.c_kv.device
        H, d = dims.num_heads, dims.head_dim
        ob, lb, _ = gqa_prompt_workspace_size(dims, batch, max_tokens, max_kv_len, num_splits)
        self._o_part = torch.empty(ob // 4, dtype=torch.float32, device=dev) if ob else None
        self._lse_part = torch.empty(lb // 4, dtype=torch.float32, device=dev) if lb else None
        self._parts = _p(self._o_part), _p(self._lse_part)
        self._o = torch.empty(max_tokens, H, d, dtype=torch.bfloat16, device=dev)
        self._lse = torch.empty(max_tokens, H, dtype=torch.float32, device=dev)
        self._q = self._proj = None
        self._outs = {}  # of from_hidden, by hidden width
        self._views = 0, self._o[:0], self._lse[:0]  # of the last call's length
        self.lse = self._views[2]
        self._layer = self._marshalled()

    def _marshalled(self):
        """The layer's descriptors, and what of the cache they were made from."""
        c = self.cache
        structs = self.dims.c(), c.c()
        return (*map(ctypes.byref, structs), c.c_kv, c.k_rope, c.block_table, c.capacity, c.num_pages, c.page_size, structs)

    def _refs(self):
        """The descriptors, made anew where the cache has changed."""
        c = self.cache
        dims, cache, c_kv, k_rope, table, capacity, pages, size, _ = self._layer
        if (c.c_kv is not c_kv or c.k_rope is not k_rope or c.block_table is not table or c.capacity != capacity
                or c.num_pages != pages or c.page_size != size):
            self._layer = dims, cache, *_ = self._marshalled()
        return dims, cache

    def _sizes(self, total: int, batch: int):
        if total > self.max_tokens or batch > self.batch:
            raise ValueError(f"{total} tokens of {batch} sequences: this handle holds {self.max_tokens} of {self.batch}")

    def append(self, q, k, v, cu_seqlens, start_pos, q_rot=None, stream=None):
        """The packed prompts' entries into the cache; returns the rotated queries (in ``q_rot``, else in a buffer
        of this handle)."""
        total, batch = k.size(0), start_pos.size(0)
        self._sizes(total, batch)
        if cu_seqlens.size(0) != batch + 1:
            raise ValueError("cu_seqlens holds one entry more than start_pos")
        d = self.dims
        H, G, w = d.num_heads, d.num_kv_groups, d.head_dim
        if q is not None and q_rot is None:
            if self._q is None:
                self._q = _new_on(stream)(self.max_tokens, H, w, dtype=torch.bfloat16, device=k.device)
            q_rot = self._q[:total]
        _check("mla_gqa_prompt_append", lib().mla_gqa_prompt_append(
            *self._refs(), batch, total, _i32(cu_seqlens), _i32(start_pos), *_rows(q, H, w, total),
            *_rows(k, G, w), *_rows(v, G, w, total), *_rows(q_rot, H, w, total), _stream(stream)))
        return q_rot

    def attend(self, q_rot, cu_seqlens, kv_len, stream=None):
        """Attention of the rotated queries over the cache: o [total, H, head_dim]; the log-sum-exps are ``lse``."""
        total, batch = q_rot.size(0), kv_len.size(0)
        self._sizes(total, batch)
        if cu_seqlens.size(0) != batch + 1:
            raise ValueError("cu_seqlens holds one entry more than kv_len")
        q, stride = _rows(q_rot, self.dims.num_heads, self.dims.head_dim)
        if self._views[0] != total:
            self._views = total, self._o[:total], self._lse[:total]
        _, o, self.lse = self._views
        _check("mla_gqa_prompt_attn", lib().mla_gqa_prompt_attn(
            *self._refs(), batch, total, _i32(cu_seqlens), _i32(kv_len), self.max_kv_len, q, stride, self.num_splits,
            *self._parts, o.data_ptr(), self.lse.data_ptr(), _stream(stream)))
        return o

    def __call__(self, q, k, v, cu_seqlens, start_pos, kv_len, stream=None):
        return self.attend(self.append(q, k, v, cu_seqlens, start_pos, stream=stream), cu_seqlens, kv_len, stream)

    def from_hidden(self, h, w_q, w_k, w_v, w_o, cu_seqlens, start_pos, kv_len, stream=None):
        """The layer on packed hidden states h [total, hidden]: projections, append, attention, output projection;
        out [total, hidden] bf16."""
        d, (total, hidden) = self.dims, h.shape
        self._sizes(total, kv_len.shape[0])
        if self._proj is None or hidden not in self._outs:
            new = lambda *s: _new_on(stream)(self.max_tokens, *s, dtype=torch.bfloat16, device=h.device)
            if self._proj is None:
                self._proj = (new(d.num_heads, d.head_dim), *(new(d.num_kv_groups, d.head_dim) for _ in range(2)))
            if hidden not in self._outs:
                self._outs[hidden] = new(hidden)
        q, k, v = (t[:total] for t in self._proj)
        gqa_project(d, h[None], w_q, w_k, w_v, q, k, v, stream)
        o = self.attend(self.append(q, k, v, cu_seqlens, start_pos, q, stream), cu_seqlens, kv_len, stream)
        return gqa_prompt_out_proj(d, o, w_o, self._outs[hidden][:total], stream)


def gqa_prompt_out_proj(dims: GqaDims, o: torch.Tensor, w_o: torch.Tensor, out: torch.Tensor, stream=None):
    """out [total, D] = W_O concat_h o (o bf16 [total, H, head_dim], as GqaPrompt gives it)."""
    H, d = dims.num_heads, dims.head_dim
    if o.dtype != torch.bfloat16 or tuple(o.shape[1:]) != (H, d):
        raise ValueError(f"o must be bf16 [total, {H}, {d}]")
    if w_o.dtype != torch.bfloat16 or w_o.dim() != 2 or w_o.shape[1] != H * d:
        raise ValueError(f"w_o must be bf16 [hidden, {H * d}]")
    _room(out, o.shape[0], w_o.shape[0], torch.bfloat16, o.device)
    _check("mla_gqa_prompt_out_proj", lib().mla_gqa_prompt_out_proj(ctypes.byref(dims.c()), o.shape[0], w_o.shape[0],
                                                                    _p(o), _p(w_o), _p(out), _stream(stream)))
    return out


def token_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor], n_top: int = 0,
                   logprob: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                   top_index: Optional[torch.Tensor] = None, top_logprob: Optional[torch.Tensor] = None,
                   lse: Optional[torch.Tensor] = None, stream=None):
    """logits [rows, vocab] (fp32 or bf16, any row stride) -> the log probability of each row's token (int32; None: not
    asked for), the entropy, and the indices and log probabilities of the n_top likeliest tokens, written into the given
    device tensors (fp32 but for the int32 indices, of rows entries or rows x n_top at least; allocated if None; ``lse``
    only if given)."""
    if logits.dtype not in (torch.float32, torch.bfloat16) or logits.dim() != 2 or not logits.is_cuda:
        raise ValueError("logits must be a 2-d fp32 or bf16 CUDA tensor")
    rows, vocab = logits.shape
    if logits.stride(1) != 1 and vocab > 1:
        raise ValueError("logits must have unit inner stride")
    dev = logits.device
    if tokens is not None and (tokens.shape[0] != rows or tokens.device != dev):
        raise ValueError("tokens holds one entry per row, on the logits' device")
    for t in (logprob, entropy, lse):
        if t is not None:
            _room(t, rows, 1, torch.float32, dev)
    if top_index is not None:
        _room(top_index, rows, n_top, torch.int32, dev)
    if top_logprob is not None:
        _room(top_logprob, rows, n_top, torch.float32, dev)
    new = _new_on(stream)
    if logprob is None and tokens is not None:
        logprob = new(rows, dtype=torch.float32, device=dev)
    entropy = new(rows, dtype=torch.float32, device=dev) if entropy is None else entropy
    top_index = new(rows, n_top, dtype=torch.int32, device=dev) if top_index is None else top_index
    top_logprob = new(rows, n_top, dtype=torch.float32, device=dev) if top_logprob is None else top_logprob
    _check("mla_token_logprobs", lib().mla_token_logprobs(
        rows, vocab, 0 if logits.dtype == torch.float32 else 1, logits.data_ptr(),
        logits.stride(0) if rows > 1 else vocab, _i32(tokens), n_top, _p(logprob), _p(entropy), _p(lse), _i32(top_index),
        _p(top_logprob), _stream(stream)))
    return logprob, entropy, top_index, top_logprob


class PagePool:
    """The pages of one or several paged caches (a model's layers) that share a
    block table: ``block_table`` [rows, entries] int32 (-1: no page; the tensor
    the caches carry), ``refs`` [pages] int32 (entries that hold a page; 0:
    free), ``groups`` table rows per sequence (G of the original GQA caches, 1
    of the latent cache).  All tensors are those that the pool and its
    caches have at each call.  Sequences and lengths are int32 device tensors; all
    work is on the device, in stream order."""

    def __init__(self, caches, block_table: torch.Tensor, refs: torch.Tensor, groups: int = 1):
        self.caches, self.block_table, self.refs, self.groups = list(caches), block_table, refs, groups
        self._ws = []  # (the last one is in use; work on those before may still be queued)
        self._marshal()

    def _marshal(self):
        """The descriptors of the pool and its caches, and what they were made from."""
        table, refs = self.block_table, self.refs
        if not self.caches or table.dim() != 2:
            raise ValueError("a pool has at least one cache and a 2-d block table")
        c = self.caches[0]
        widths = c.c_kv.shape[2], c.k_rope.shape[2]
        if any((x.c_kv.shape[2], x.k_rope.shape[2]) != widths for x in self.caches):
            raise ValueError("the caches of a pool have the same widths")
        if any(t.shape[0] < x.num_pages or t.shape[1] < x.page_size for x in self.caches for t in (x.c_kv, x.k_rope)):
            raise ValueError("a cache holds num_pages pages of page_size tokens")
        self._c = MlaPagePool(refs.shape[0], c.page_size, self.groups, table.shape[0], table.shape[1], _i32(refs),
                              _i32(table))
        self._structs = (MlaCache * len(self.caches))(*(x.c() for x in self.caches))
        size = ctypes.c_size_t()
        _check("mla_pages_workspace_size", lib().mla_pages_workspace_size(ctypes.byref(self._c), ctypes.byref(size)))
        if not self._ws or self._ws[-1].numel() < size.value // 4:
            self._ws.append(torch.empty(size.value // 4, dtype=torch.int32, device=refs.device))
        self._ref, self._ws_p = ctypes.byref(self._c), self._ws[-1].data_ptr()
        self._cache_args = len(self.caches), self._structs, *widths
        self._of = table, refs, [t for x in self.caches for t in (x.c_kv, x.k_rope)]

    def _pool(self):
        """The pool's descriptor, made anew where its table or counts are other tensors."""
        if self.block_table is not self._of[0] or self.refs is not self._of[1]:
            self._marshal()
        return self._ref

    def _layers(self):
        """The caches' descriptors, made anew where their tensors are others."""
        now = [t for x in self.caches for t in (x.c_kv, x.k_rope)]
        if len(now) != len(self._of[2]) or any(a is not b for a, b in zip(now, self._of[2])):
            self._marshal()
        return self._cache_args

    def _lists(self, first, *more):
        shape = first.shape
        for t in more:
            if t.shape != shape:
                raise ValueError("sequences and lengths share their count")
        return (shape[0], _i32(first), *map(_i32, more))

    def release(self, sequences: torch.Tensor, lens: torch.Tensor, stream=None):
        """Give back the pages past the first lens[i] tokens of each sequence."""
        _check("mla_pages_release", lib().mla_pages_release(self._pool(), *self._lists(sequences, lens), _stream(stream)))

    def reserve(self, sequences: torch.Tensor, lens: torch.Tensor, stream=None):
        """Pages for the first lens[i] tokens of each sequence."""
        _check("mla_pages_reserve", lib().mla_pages_reserve(self._pool(), *self._lists(sequences, lens), self._ws_p,
                                                            _stream(stream)))

    def fork(self, parents: torch.Tensor, children: torch.Tensor, lens: torch.Tensor, stream=None):
        """children[i] becomes a copy of the first lens[i] tokens of parents[i]: full pages shared, a partial last
        page copied."""
        _check("mla_pages_fork", lib().mla_pages_fork(self._pool(), *self._layers(),
                                                      *self._lists(parents, children, lens), self._ws_p,
                                                      _stream(stream)))

    def compact(self, stream=None):
        """Move the pages in use to the low end of the pool."""
        _check("mla_pages_compact", lib().mla_pages_compact(self._pool(), *self._layers(), self._ws_p,
                                                            _stream(stream)))


def e2e_loss(a_mla: torch.Tensor, a_orig: torch.Tensor, mask: Optional[torch.Tensor] = None,
             loss: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """E2E functional-reconstruction loss forward (masked MSE of the two blocks'
    post-W_O outputs, bf16 [.., D]); returns a one-element fp32 device tensor."""
    hidden = a_mla.shape[-1]
    rows = a_mla.numel() // hidden
    loss = _new_on(stream)(1, dtype=torch.float32, device=a_mla.device) if loss is None else loss
    _check("mla_e2e_loss", lib().mla_e2e_loss(rows, hidden, _p(a_mla), _p(a_orig), _p(mask), _p(loss),
                                              _stream(stream)))
    return loss


class E2EForward:
    """Forward of the E2E functional-reconstruction loss (Sec. 4.1) on one
    chunk of calibration hidden states: the converted MLA layer (projection
    into its latent cache, absorbed attention, W_UV, W_O) and the original GQA
    layer (its projections, cache append, attention, the same frozen W_O) run
    on the same h, and their post-W_O outputs meet in the masked MSE.  Every
    buffer is allocated once here."""

    def __init__(self, mla_step: "DecodeStep", gqa_dims: GqaDims, gqa_cache: Cache, hidden: int):
        self.mla = mla_step
        b, q = mla_step.batch, mla_step.q_len
        dev = mla_step.q_abs.device
        self.gqa_dims = gqa_dims
        self.gqa = GqaStep(gqa_dims, gqa_cache, b, q, mla_step.max_kv_len)
        d, H, G = gqa_dims.head_dim, gqa_dims.num_heads, gqa_dims.num_kv_groups
        self.q = torch.empty(b, q, H, d, dtype=torch.bfloat16, device=dev)
        self.k_new = torch.empty(b, q, G, d, dtype=torch.bfloat16, device=dev)
        self.v_new = torch.empty(b, q, G, d, dtype=torch.bfloat16, device=dev)
        self.out_orig = torch.empty(b, q, hidden, dtype=torch.bfloat16, device=dev)
        self.loss = torch.empty(1, dtype=torch.float32, device=dev)

    def __call__(self, h, mla_w, gqa_w, w_o, start_pos, kv_len, mask=None, stream=None):
        """mla_w = (w_dkv, w_kr, w_q, w_uk, w_uv), gqa_w = (w_q, w_k, w_v); returns the loss tensor."""
        w_dkv, w_kr, w_qm, w_uk, w_uv = mla_w
        out_mla = self.mla.from_hidden(h, w_dkv, w_kr, w_qm, start_pos, kv_len, w_uk, w_uv, w_o, stream=stream)
        gqa_project(self.gqa_dims, h, *gqa_w, self.q, self.k_new, self.v_new, stream)
        gqa_append(self.gqa_dims, self.gqa.cache, self.k_new, self.v_new, start_pos, stream)
        o = self.gqa(self.q, kv_len, stream)
        gqa_out_proj(self.gqa_dims, o, w_o, self.out_orig, stream)
        return e2e_loss(out_mla, self.out_orig, mask, self.loss, stream)


def acceptance_stats(draft: torch.Tensor, target: torch.Tensor, alpha: Optional[torch.Tensor] = None,
                     argmax_draft: Optional[torch.Tensor] = None, argmax_target: Optional[torch.Tensor] = None,
                     greedy: Optional[torch.Tensor] = None, stream=None):
    """draft / target logits [rows, vocab] (fp32 or bf16, same dtype) -> the
    per-row overlap alpha_sample (fp32), the two argmaxes and greedy agreement
    (int32), written into the given device tensors (allocated if None)."""
    if draft.dtype != target.dtype or draft.dtype not in (torch.float32, torch.bfloat16) or draft.shape != target.shape:
        raise ValueError("draft and target logits must share a shape and be fp32 or bf16")
    rows, vocab = draft.shape
    if draft.stride() != target.stride() or draft.stride(1) != 1 or not draft.is_cuda or not target.is_cuda:
        raise ValueError("logits must be CUDA tensors with unit inner stride and equal row strides")
    row_stride = draft.stride(0) if rows > 1 else vocab
    dev = draft.device
    new = _new_on(stream)
    alpha = new(rows, dtype=torch.float32, device=dev) if alpha is None else alpha
    argmax_draft = new(rows, dtype=torch.int32, device=dev) if argmax_draft is None else argmax_draft
    argmax_target = new(rows, dtype=torch.int32, device=dev) if argmax_target is None else argmax_target
    greedy = new(rows, dtype=torch.int32, device=dev) if greedy is None else greedy
    _check("mla_acceptance_stats", lib().mla_acceptance_stats(rows, vocab, 0 if draft.dtype == torch.float32 else 1,
                                                              draft.data_ptr(), target.data_ptr(), row_stride,
                                                              _p(alpha),
                                                              _p(argmax_draft), _p(argmax_target), _p(greedy),
                                                              _stream(stream)))
    return alpha, argmax_draft, argmax_target, greedy


def absorb_q(dims: Dims, q_nope: torch.Tensor, q_pe: torch.Tensor, kv_len: torch.Tensor, w_uk: torch.Tensor,
             q_abs: torch.Tensor, stream=None):
    batch, q_len = q_nope.shape[0], q_nope.shape[1]
    _check("mla_absorb_q", lib().mla_absorb_q(ctypes.byref(dims.c()), batch, q_len, _p(q_nope), _p(q_pe),
                                              _p(kv_len), _p(w_uk), _p(q_abs), _stream(stream)))


def decode_attn(dims: Dims, cache: Cache, kv_len: torch.Tensor, max_kv_len: int, q_abs: torch.Tensor,
                o_part: torch.Tensor, lse_part: torch.Tensor, num_splits: int = 0, stream=None):
    batch, q_len = q_abs.shape[0], q_abs.shape[1]
    _check("mla_decode_attn", lib().mla_decode_attn(ctypes.byref(dims.c()), ctypes.byref(cache.c()), batch, q_len,
                                                    _p(kv_len), max_kv_len, _p(q_abs), num_splits, _p(o_part),
                                                    _p(lse_part), _stream(stream)))


def combine(dims: Dims, batch: int, q_len: int, kv_len: torch.Tensor, max_kv_len: int, o_part: torch.Tensor,
            lse_part: torch.Tensor, o_lat: torch.Tensor, lse: Optional[torch.Tensor] = None, num_splits: int = 0,
            stream=None):
    _check("mla_combine", lib().mla_combine(ctypes.byref(dims.c()), batch, q_len, num_splits, _p(kv_len), max_kv_len,
                                            _p(o_part), _p(lse_part), _p(o_lat), _p(lse), _stream(stream)))


def out_proj(dims: Dims, o_lat: torch.Tensor, w_uv: torch.Tensor, w_o: Optional[torch.Tensor], o: torch.Tensor,
             out: Optional[torch.Tensor], stream=None):
    batch, q_len = o_lat.shape[0], o_lat.shape[1]
    _check("mla_out_proj", lib().mla_out_proj(ctypes.byref(dims.c()), batch, q_len, _p(o_lat), _p(w_uv), _p(w_o),
                                              _p(o), _p(out), _stream(stream)))


def decode_attn_noalloc(dims: Dims, cache: Cache, kv_len: torch.Tensor, max_kv_len: int, q_abs: torch.Tensor,
                        o_lat: torch.Tensor, lse: Optional[torch.Tensor] = None, num_splits: int = 0, stream=None):
    """Attention core and combine with the library's static scratch (for callers
    that cannot allocate device memory): writes o_lat and lse directly."""
    batch, q_len = q_abs.shape[0], q_abs.shape[1]
    _check("mla_decode_attn_noalloc",
           lib().mla_decode_attn_noalloc(ctypes.byref(dims.c()), ctypes.byref(cache.c()), batch, q_len, _p(kv_len),
                                         max_kv_len, _p(q_abs), num_splits, _p(o_lat), _p(lse), _stream(stream)))


def check_status(stream=None) -> int:
    """Synchronise the stream and return (and clear) the device status code."""
    return lib().mla_check_status(_stream(stream))


def selftest_wait_timeout(limit_ns: int, stream=None):
    _check("mla_selftest_wait_timeout", lib().mla_selftest_wait_timeout(int(limit_ns), _stream(stream)))


def selftest_wait_looks(elapsed_ns: Optional[torch.Tensor] = None, stream=None):
    """1000 looks at an mbarrier that nothing signals (MLA_ERR_DEVICE_TIMEOUT afterwards); their time into the given
    int64 device tensor."""
    if elapsed_ns is not None and (elapsed_ns.dtype != torch.int64 or elapsed_ns.numel() < 1):
        raise ValueError("elapsed_ns must be int64 and hold one entry")
    _check("mla_selftest_wait_looks", lib().mla_selftest_wait_looks(_p(elapsed_ns), _stream(stream)))


class DecodeStep:
    """One decode step of an MLA layer (mla_decode_step: the five entry points
    in one call), with every intermediate buffer allocated once (by PyTorch)
    up front: append -> absorb -> split-KV attention -> combine -> up/out
    projection (or, through ``from_hidden``, projection -> absorb -> ...).

    ``graph=True`` replays the step as a CUDA graph: the first call with a
    given set of input tensors (their addresses) runs the step once and
    captures it, later calls with the same tensors replay the capture, on the
    current stream (or ``stream``, a ``torch.cuda.Stream``).  A serving loop
    that refills fixed input buffers pays one graph launch per step instead of
    the launches of every kernel."""

    def __init__(self, dims: Dims, cache: Cache, batch: int, q_len: int, max_kv_len: int, num_splits: int = 0,
                 device=None, graph: bool = False):
        self.graph = graph
        self._graphs = {}
        self.dims, self.cache = dims, cache
        self.batch, self.q_len, self.max_kv_len = batch, q_len, max_kv_len
        dev = device or cache.c_kv.device
        ob, lb, s = workspace_size(dims, batch, q_len, max_kv_len, num_splits)
        self.num_splits = s
        H, r, dr = dims.num_heads, dims.rank, dims.d_rope
        slots = max(ob // 4 // max(q_len * H * r, 1), 1)
        self.q_abs = torch.empty(batch, q_len, H, r + dr, dtype=torch.bfloat16, device=dev)
        self.o_part = torch.empty(slots, q_len, H, r, dtype=torch.float32, device=dev)
        self.lse_part = torch.empty(slots, q_len, H, dtype=torch.float32, device=dev)
        self.o_lat = torch.empty(batch, q_len, H, r, dtype=torch.float32, device=dev)
        self.lse = torch.empty(batch, q_len, H, dtype=torch.float32, device=dev)
        self.o = torch.empty(batch, q_len, H, dims.d_v, dtype=torch.bfloat16, device=dev)
        self.out = (torch.empty(batch, q_len, dims.hidden, dtype=torch.bfloat16, device=dev)
                    if dims.hidden else None)

    def __call__(self, q_nope, q_pe, kv_len, w_uk, w_uv, w_o=None, c_new=None, kr_new=None, start_pos=None,
                 stream=None):
        args = (q_nope, q_pe, kv_len, w_uk, w_uv, w_o, c_new, kr_new, start_pos)
        if not self.graph:
            return self._launch(*args, stream=stream)
        if stream is not None and not isinstance(stream, torch.cuda.Stream):
            raise ValueError("graph mode takes a torch.cuda.Stream (or None)")
        key = tuple(0 if t is None else t.data_ptr() for t in args)
        entry = self._graphs.get(key)
        if entry is None:
            self._launch(*args, stream=stream)  # the library's per-device set-up runs outside the capture
            g = torch.cuda.CUDAGraph()
            side = torch.cuda.Stream()
            side.wait_stream(stream or torch.cuda.current_stream())
            with torch.cuda.graph(g, stream=side):
                self._launch(*args)
            (stream or torch.cuda.current_stream()).wait_stream(side)
            entry = self._graphs[key] = (g, args)  # the tensors stay referenced while the graph lives
        if stream is None:
            entry[0].replay()
        else:
            with torch.cuda.stream(stream):
                entry[0].replay()
        return self.out if (self.dims.hidden and w_o is not None) else self.o

    def _launch(self, q_nope, q_pe, kv_len, w_uk, w_uv, w_o=None, c_new=None, kr_new=None, start_pos=None,
                stream=None):
        # the layer's descriptors and the step's own buffers are fixed: marshal
        # them once, so that a step costs the five library calls and little else
        if getattr(self, "_fixed", None) is None:
            self._structs = (self.dims.c(), self.cache.c())  # kept alive for the references below
            self._fixed = (ctypes.byref(self._structs[0]), ctypes.byref(self._structs[1]), self.q_abs.data_ptr(),
                           self.o_part.data_ptr(), self.lse_part.data_ptr(), self.o_lat.data_ptr(),
                           self.lse.data_ptr(), self.o.data_ptr(),
                           self.out.data_ptr() if self.out is not None else None)
        dims, cache, qa, op, lp, ol, ls, o, out = self._fixed
        d, L, sp = self.dims, lib(), _stream(stream)
        if c_new is not None and c_new.shape[1] != self.q_len:
            raise ValueError("c_new must hold q_len new entries per sequence")
        with_o = d.hidden and w_o is not None
        # the whole step in one library call (append, absorption, attention, combine, projections)
        _check("mla_decode_step", L.mla_decode_step(dims, cache, self.batch, self.q_len, _p(c_new), _p(kr_new),
                                                    _p(start_pos), _p(q_nope), _p(q_pe), _p(kv_len), self.max_kv_len,
                                                    _p(w_uk), _p(w_uv), _p(w_o) if with_o else None,
                                                    self.num_splits, qa, op, lp, ol, ls, o,
                                                    out if with_o else None, sp))
        return self.out if with_o else self.o

    def from_hidden(self, h, w_dkv, w_kr, w_q, start_pos, kv_len, w_uk, w_uv, w_o=None, stream=None):
        """The step fed by hidden states h [B, q_len, hidden]: the projection
        writes the cache rows and the queries (kept in ``self.q_nope`` /
        ``self.q_pe``), then absorption, attention, combine and projections."""
        d = self.dims
        if getattr(self, "q_nope", None) is None:
            dev = h.device
            self.q_nope = torch.empty(self.batch, self.q_len, d.num_heads, d.d_nope, dtype=torch.bfloat16, device=dev)
            self.q_pe = torch.empty(self.batch, self.q_len, d.num_heads, d.d_rope, dtype=torch.bfloat16, device=dev)
        project_append(d, self.cache, h, w_dkv, w_kr, w_q, start_pos, self.q_nope, self.q_pe, stream)
        return self(self.q_nope, self.q_pe, kv_len, w_uk, w_uv, w_o, stream=stream)


@dataclass
class DeviceWorkload:
    """A workload's tensors on the GPU plus its Dims and Cache descriptors."""
    dims: Dims
    cache: Cache
    batch: int
    q_len: int
    max_kv_len: int
    kv_len: torch.Tensor
    start_pos: torch.Tensor
    w_uk: torch.Tensor
    w_uv: torch.Tensor
    w_o: Optional[torch.Tensor]
    q_nope: torch.Tensor
    q_pe: torch.Tensor
    c_new: torch.Tensor
    kr_new: torch.Tensor


def to_device(w, device="cuda") -> DeviceWorkload:
    """Copy a ``workloads.Workload`` to the GPU (plain host-to-device copies)."""
    s = w.shape
    dims = Dims(s.num_heads, s.num_kv_groups, s.d_nope, s.d_rope, s.d_v, s.rank, s.hidden, s.sm_scale,
                s.rope_style, s.rope_base)
    put = lambda t: None if t is None else t.to(device)
    bt = put(w.block_table)
    cache = Cache(put(w.c_kv), put(w.k_rope), w.capacity, bt, s.page_size if s.paged else 0, w.num_pages)
    batch, q_len = w.kv_len.numel(), w.q_nope.shape[1]
    return DeviceWorkload(dims, cache, batch, q_len, int(w.kv_len.max()) if batch else q_len, put(w.kv_len),
                          put(w.start_pos), put(w.w_uk), put(w.w_uv), put(w.w_o), put(w.q_nope), put(w.q_pe),
                          put(w.c_new), put(w.kr_new))
