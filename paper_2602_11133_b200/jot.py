"""ctypes binding of libjot.so: argument marshalling only.

Every step of the JoT denoising path runs inside the CUDA library; this module turns torch tensors
into raw device pointers, checks dtypes/shapes, and raises on any non-zero status.  There is no
fallback: if the library is missing or fails to load, importing the binding's functions raises.
"""
from __future__ import annotations

import array
import ctypes as C
import dataclasses
import functools
import math
import os
import struct
from typing import List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libjot.so")

EXPORTS = [
    "jot_status_string", "jot_last_cuda_error", "jot_workspace_bytes", "jot_init_model", "jot_free_model",
    "jot_denoise_step", "jot_lm_head_stats", "jot_accept_freeze", "jot_generate", "jot_gemm_bf16",
    "jot_launch_count", "jot_profile", "jot_profile_read", "jot_gemm_bf16_noalloc",
    "jot_selftest_wait_expiry", "jot_kv_cache_bytes", "jot_attach_kv_cache", "jot_denoise_step_cached",
    "jot_max_active_rows", "jot_lm_head_partition", "jot_set_sync", "jot_read_status",
    "jot_lm_head_stats_slice", "jot_merge_stats", "jot_head_norm_rope", "jot_kv_write", "jot_kv_copy_pages",
    "jot_paged_attention", "jot_paged_attention_workspace_bytes", "jot_kv_pages_workspace_bytes", "jot_attach_kv_pages",
]

NOALLOC_SCRATCH_BYTES = 16 << 20

PROF_CLASSES = ["embed", "rmsnorm", "gemm_qkv", "rope", "attention", "gemm_o", "gemm_gate_up", "gemm_down", "rows",
                "lm_head", "merge", "accept"]


class JotError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = _lib().jot_status_string(status).decode()
        cuda = _lib().jot_last_cuda_error()
        super().__init__(f"{where}: {msg} (status {status}, cuda error {cuda})")


GATE_RATIO, GATE_MAXPROB, GATE_GLOBAL_GAP = 0, 1, 2
SCHEDULE_FIXED, SCHEDULE_FRACTIONAL = 0, 1


class Params(C.Structure):
    """tau_max, tau_min, gamma, D of Algorithm 1; eps of Eq. 4."""
    _fields_ = [("tau_max", C.c_float), ("tau_min", C.c_float), ("gamma", C.c_float), ("D", C.c_int32),
                ("eps", C.c_float), ("schedule_after_exit", C.c_int32), ("gate", C.c_int32),
                ("prob_threshold", C.c_float), ("gap_threshold", C.c_float), ("schedule", C.c_int32)]

    def __init__(self, tau_max=90.0, tau_min=1.0, gamma=0.5, D=8, eps=1e-12, schedule_after_exit=0, gate=0,
                 prob_threshold=0.9, gap_threshold=5.0, schedule=0):
        super().__init__(tau_max, tau_min, gamma, D, eps, schedule_after_exit, gate, prob_threshold, gap_threshold,
                         schedule)


class ModelConfig(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("d_ff", C.c_int32), ("vocab", C.c_int32), ("mask_id", C.c_int32),
                ("rope_theta", C.c_float), ("rms_eps", C.c_float)]


class _Weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("lm_head", C.c_void_p), ("final_norm", C.c_void_p),
                ("attn_norm", C.POINTER(C.c_void_p)), ("wqkv", C.POINTER(C.c_void_p)), ("wo", C.POINTER(C.c_void_p)),
                ("mlp_norm", C.POINTER(C.c_void_p)), ("w_gate_up", C.POINTER(C.c_void_p)),
                ("w_down", C.POINTER(C.c_void_p))]


class Sampling(C.Structure):
    """Sampling-based finalisation: temperature > 0 draws each active row's token from softmax(l / T)."""
    _fields_ = [("temperature", C.c_float), ("seed", C.c_uint64), ("step", C.c_int32)]


class GenConfig(C.Structure):
    _fields_ = [("gen_len", C.c_int32), ("steps", C.c_int32), ("block_len", C.c_int32),
                ("exclude_mask_token", C.c_int32), ("compact_finished", C.c_int32), ("use_cuda_graph", C.c_int32),
                ("temperature", C.c_float), ("seed_lo", C.c_uint32), ("seed_hi", C.c_uint32), ("kv_cache", C.c_int32)]


class _Trace(C.Structure):
    _fields_ = [("exit_step", C.c_void_p), ("exit_reason", C.c_void_p), ("mean_ratio", C.c_void_p),
                ("n_candidates", C.c_void_p)]


# The small structs of the paged calls as packed bytes (native sizes and alignment): a ctypes.Structure takes a microsecond to fill, three or
# four of them a third of a short call.
_pack_pages = struct.Struct("PPqqqqiiiiii").pack     # jot_kv_pages: k, v, strides of layers (k, v) and pages (k, v), layers, pages, heads, page size, head_dim, dtype
_pack_rope = struct.Struct("Piif4x").pack            # jot_rope: inv_freq, rotary_dim, interleaved, magnitude
_pack_heads = struct.Struct("PqqPqqPi4x").pack       # jot_heads: in, strides (row, head), out, strides, gain, n_heads


@dataclasses.dataclass
class Trace:
    """Optional per-position / per-step record of a generation (device tensors)."""
    exit_step: torch.Tensor        # [B, L] int16: 1-based step of the sequence that finalised the position
    exit_reason: torch.Tensor      # [B, L] uint8: bit 0 early exit, bit 1 transfer schedule
    mean_ratio: torch.Tensor       # [steps, B] float32: mean confidence ratio over the step's candidates
    n_candidates: torch.Tensor     # [steps, B] int32


_LIB = None


def _lib():
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2602_11133_b200.build` "
                               "(there is no CPU or PyTorch fallback)")
        lib = C.CDLL(LIB_PATH)
        lib.jot_status_string.restype = C.c_char_p
        lib.jot_status_string.argtypes = [C.c_int]
        lib.jot_last_cuda_error.restype = C.c_int
        lib.jot_workspace_bytes.restype = C.c_size_t
        lib.jot_workspace_bytes.argtypes = [C.POINTER(ModelConfig), C.c_int, C.c_int]
        lib.jot_init_model.argtypes = [C.POINTER(ModelConfig), C.POINTER(_Weights), C.c_int, C.c_int, C.c_void_p,
                                       C.c_size_t, C.POINTER(C.c_void_p)]
        lib.jot_free_model.argtypes = [C.c_void_p]
        step_args = [C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                     C.c_void_p, C.c_void_p, C.POINTER(Sampling), C.c_void_p, C.c_void_p]
        lib.jot_denoise_step.argtypes = [C.c_void_p, C.c_void_p] + step_args
        lib.jot_lm_head_stats.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p] + step_args
        lib.jot_lm_head_stats_slice.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int,
                                                C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p,
                                                C.c_void_p, C.POINTER(Sampling), C.c_void_p, C.c_void_p]
        lib.jot_merge_stats.argtypes = [C.c_int] + [C.c_void_p] * 13
        lib.jot_kv_cache_bytes.restype = C.c_size_t
        lib.jot_kv_cache_bytes.argtypes = [C.POINTER(ModelConfig), C.c_int, C.c_int]
        lib.jot_attach_kv_cache.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t]
        lib.jot_denoise_step_cached.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int,
                                                C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                                C.c_void_p, C.POINTER(Sampling), C.c_void_p, C.c_void_p]
        lib.jot_accept_freeze.argtypes = [C.POINTER(Params), C.c_int, C.c_int32, C.c_void_p, C.c_int, C.c_int, C.c_int,
                                          C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                          C.c_void_p, C.c_void_p, C.c_int, C.c_void_p]
        lib.jot_generate.argtypes = [C.c_void_p, C.POINTER(Params), C.c_int, C.POINTER(GenConfig), C.c_void_p, C.c_int,
                                     C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(C.c_int32),
                                     C.POINTER(C.c_int32), C.POINTER(_Trace), C.c_void_p]
        lib.jot_gemm_bf16.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int,
                                      C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        lib.jot_gemm_bf16_noalloc.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int,
                                              C.c_void_p, C.c_void_p]
        lib.jot_launch_count.restype = C.c_int64
        lib.jot_selftest_wait_expiry.argtypes = [C.c_void_p, C.c_uint64, C.c_void_p]
        lib.jot_max_active_rows.argtypes = [C.c_int]
        lib.jot_lm_head_partition.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int), C.POINTER(C.c_int)]
        lib.jot_set_sync.argtypes = [C.c_void_p, C.c_int]
        lib.jot_read_status.argtypes = [C.c_void_p, C.c_void_p]
        lib.jot_profile.argtypes = [C.c_void_p, C.c_int]
        lib.jot_profile_read.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int64), C.c_int]
        heads = rope = pages = C.c_void_p        # structs, or bytes packed as they are
        lib.jot_head_norm_rope.argtypes = [heads, heads, rope, C.c_int, C.c_int, C.c_int, C.c_float, C.c_void_p,
                                           heads, pages, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.jot_kv_write.argtypes = [pages, C.c_int, C.c_int, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_int64,
                                     C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.jot_kv_copy_pages.argtypes = [pages, C.c_int, C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.c_void_p]
        lib.jot_kv_pages_workspace_bytes.restype = C.c_size_t
        lib.jot_kv_pages_workspace_bytes.argtypes = [C.POINTER(ModelConfig), C.c_int, C.c_int]
        lib.jot_attach_kv_pages.argtypes = [C.c_void_p, pages, C.c_void_p, C.c_int64, C.c_int, C.c_void_p, C.c_size_t]
        lib.jot_paged_attention_workspace_bytes.restype = C.c_size_t
        lib.jot_paged_attention_workspace_bytes.argtypes = [C.c_int] * 4
        lib.jot_paged_attention.argtypes = ([C.c_void_p, C.c_int64, C.c_int64, C.c_int64] * 2 + [C.c_void_p] + [C.c_int] * 3
                                            + [pages, C.c_int, C.c_void_p, C.c_int64, C.c_int, C.c_void_p, C.c_float,
                                               C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p])
        _LIB = lib
    return _LIB


def _check(status: int, where: str):
    if status != 0:
        raise JotError(status, where)


def _ptr(t: Optional[torch.Tensor], dtype, name: str) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name}: expected a contiguous CUDA tensor of {dtype}, got {t.dtype} on {t.device}")
    return t.data_ptr()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _sampling_args(sampling, out, B, L, device):
    """(pointer to the descriptor or None, device pointer of the sampled-token array or None)."""
    if sampling is None or not sampling.temperature > 0:
        return None, None
    if out.sampled is None:
        out.sampled = torch.zeros(B, L, dtype=torch.int32, device=device)
    return C.byref(sampling), _ptr(out.sampled, torch.int32, "sampled")


def max_active_rows(n_sms: int) -> int:
    return int(_lib().jot_max_active_rows(n_sms))


def lm_head_partition(active_rows: int, n_ctas: int, vocab_tiles: int, pair_mode: bool):
    """(row blocks, vocabulary chunks per row block) of the LM-head schedule; host arithmetic only."""
    n_rb, n_ch = C.c_int(0), C.c_int(0)
    _check(_lib().jot_lm_head_partition(active_rows, n_ctas, vocab_tiles, int(pair_mode), C.byref(n_rb), C.byref(n_ch)),
           "jot_lm_head_partition")
    return n_rb.value, n_ch.value


def launch_count() -> int:
    return int(_lib().jot_launch_count())


@dataclasses.dataclass
class Stats:
    """Per-position softmax statistics, each [B, L]; only active rows are written."""
    top1: torch.Tensor
    top2: torch.Tensor
    sumexp: torch.Tensor
    argmax: torch.Tensor
    sampled: Optional[torch.Tensor] = None      # [B, L] int32, written when sampling is on

    @staticmethod
    def empty(B: int, L: int, device) -> "Stats":
        return Stats(torch.zeros(B, L, dtype=torch.float32, device=device),
                     torch.zeros(B, L, dtype=torch.float32, device=device),
                     torch.ones(B, L, dtype=torch.float32, device=device),
                     torch.zeros(B, L, dtype=torch.int32, device=device))


class Model:
    """Owner of the device workspace and the library's model handle.  Weights are borrowed."""

    def __init__(self, geometry, weights: dict, max_batch: int, max_seq: int):
        g = geometry
        self.geometry = g
        self.cfg = ModelConfig(len(weights["layers"]), g.d_model, g.n_q_heads, g.n_kv_heads, g.head_dim, g.d_ff,
                               g.vocab, g.mask_id, g.rope_theta, g.rms_eps)
        self.weights = weights           # keep the tensors alive
        self.max_batch, self.max_seq = max_batch, max_seq
        lib = _lib()
        nbytes = lib.jot_workspace_bytes(C.byref(self.cfg), max_batch, max_seq)
        if nbytes == 0:
            raise JotError(-2, "jot_workspace_bytes")
        dev = weights["lm_head"].device
        self.workspace = torch.empty(nbytes + 1024, dtype=torch.uint8, device=dev)
        base = (self.workspace.data_ptr() + 1023) // 1024 * 1024
        nl = self.cfg.n_layers
        arr = lambda key: (C.c_void_p * max(nl, 1))(*[_ptr(lw[key], torch.bfloat16, key) for lw in weights["layers"]])
        self._arrays = [arr(k) for k in ("attn_norm", "wqkv", "wo", "mlp_norm", "w_gate_up", "w_down")]
        w = _Weights(_ptr(weights["embed"], torch.bfloat16, "embed"), _ptr(weights["lm_head"], torch.bfloat16, "lm_head"),
                     _ptr(weights["final_norm"], torch.bfloat16, "final_norm"),
                     *[C.cast(a, C.POINTER(C.c_void_p)) for a in self._arrays])
        handle = C.c_void_p()
        torch.cuda.current_stream(dev).synchronize()         # kernels queued on it may still write what is the workspace's memory now
        _check(lib.jot_init_model(C.byref(self.cfg), C.byref(w), max_batch, max_seq, base, nbytes, C.byref(handle)),
               "jot_init_model")
        self.handle = handle
        self.kv_cache = None

    def close(self):
        if getattr(self, "handle", None):
            _lib().jot_free_model(self.handle)
            self.handle = None
        self.kv_cache = None

    # ---- block-wise KV cache -----------------------------------------------------------------------
    def attach_kv_cache(self) -> int:
        """Allocate the cache for (max_batch, max_seq) and hand it to the library; returns its size in bytes."""
        nbytes = _lib().jot_kv_cache_bytes(C.byref(self.cfg), self.max_batch, self.max_seq)
        if nbytes == 0:
            raise JotError(-2, "jot_kv_cache_bytes")
        self.kv_cache = torch.empty(nbytes + 1024, dtype=torch.uint8, device=self.workspace.device)
        base = (self.kv_cache.data_ptr() + 1023) // 1024 * 1024
        _check(_lib().jot_attach_kv_cache(self.handle, base, nbytes), "jot_attach_kv_cache")
        return int(nbytes)

    def detach_kv_cache(self) -> None:
        _check(_lib().jot_attach_kv_cache(self.handle, None, 0), "jot_attach_kv_cache")
        self.kv_cache = None

    def attach_kv_pages(self, pages: "KVPages", page_table: torch.Tensor) -> None:
        """The block-wise cache in the caller's pages: page_table [max_batch, max_pages] int32, read by every pass (it may
        change between them).  Takes the place of an attached contiguous cache; detach_kv_cache detaches it."""
        dev = self.workspace.device
        if pages.device != dev or page_table.device != dev or page_table.dtype != torch.int32 or page_table.dim() != 2 or (
                page_table.shape[1] > 1 and page_table.stride(1) != 1):
            raise TypeError(f"attach_kv_pages: expected pages and an int32 table with contiguous rows on {dev}")
        if page_table.shape[0] < self.max_batch:
            raise ValueError(f"attach_kv_pages: the table has {page_table.shape[0]} rows, the model takes {self.max_batch} sequences")
        nbytes = _lib().jot_kv_pages_workspace_bytes(C.byref(self.cfg), self.max_batch, self.max_seq)
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        torch.cuda.current_stream(dev).synchronize()         # kernels queued on it may still write what is the workspace's memory now
        _check(_lib().jot_attach_kv_pages(self.handle, pages._packed, page_table.data_ptr(), page_table.stride(0), page_table.shape[1],
                                          workspace.data_ptr(), nbytes), "jot_attach_kv_pages")
        self.kv_cache = (pages, page_table, workspace)       # keep them alive

    def denoise_step_cached(self, tokens: torch.Tensor, blk_lo: int, blk_hi: int, refresh: bool,
                            out: Optional["Stats"] = None, exclude_mask_token: bool = True,
                            bump_id: Optional[torch.Tensor] = None, bump_val: Optional[torch.Tensor] = None,
                            sampling: Optional[Sampling] = None) -> "Stats":
        B, L = tokens.shape
        out = out or Stats.empty(B, L, tokens.device)
        sp, d_sampled = _sampling_args(sampling, out, B, L, tokens.device)
        _check(_lib().jot_denoise_step_cached(self.handle, _ptr(tokens, torch.int32, "tokens"), B, L, blk_lo, blk_hi,
                                              int(refresh), int(exclude_mask_token), _ptr(bump_id, torch.int32, "bump_id"),
                                              _ptr(bump_val, torch.float32, "bump_val"), out.top1.data_ptr(),
                                              out.top2.data_ptr(), out.sumexp.data_ptr(), out.argmax.data_ptr(), sp,
                                              d_sampled, _stream()),
               "jot_denoise_step_cached")
        return out

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_sync(self, sync: bool) -> None:
        """sync=False: the single-step calls return once their kernels are enqueued; read_status() asks later."""
        _check(_lib().jot_set_sync(self.handle, int(sync)), "jot_set_sync")

    def read_status(self) -> None:
        """Synchronise the current stream and raise if a kernel reported a failure since the last read."""
        _check(_lib().jot_read_status(self.handle, _stream()), "jot_read_status")

    def profile(self, enable: bool) -> None:
        """Start (and clear) or stop per-kernel-class event timing."""
        _check(_lib().jot_profile(self.handle, int(enable)), "jot_profile")

    def profile_read(self) -> dict:
        """{class: (milliseconds, spans)} accumulated since profile(True)."""
        n = len(PROF_CLASSES)
        ms, cnt = (C.c_double * n)(), (C.c_int64 * n)()
        _check(_lib().jot_profile_read(self.handle, ms, cnt, n), "jot_profile_read")
        return {name: (ms[i], int(cnt[i])) for i, name in enumerate(PROF_CLASSES)}

    # ---- one step -------------------------------------------------------------------------------
    def denoise_step(self, tokens: torch.Tensor, blk_lo: int, blk_hi: int, out: Optional[Stats] = None,
                     exclude_mask_token: bool = True, bump_id: Optional[torch.Tensor] = None,
                     bump_val: Optional[torch.Tensor] = None, sampling: Optional[Sampling] = None) -> Stats:
        B, L = tokens.shape
        out = out or Stats.empty(B, L, tokens.device)
        sp, d_sampled = _sampling_args(sampling, out, B, L, tokens.device)
        _check(_lib().jot_denoise_step(self.handle, _ptr(tokens, torch.int32, "tokens"), B, L, blk_lo, blk_hi,
                                       int(exclude_mask_token), _ptr(bump_id, torch.int32, "bump_id"),
                                       _ptr(bump_val, torch.float32, "bump_val"), out.top1.data_ptr(),
                                       out.top2.data_ptr(), out.sumexp.data_ptr(), out.argmax.data_ptr(), sp,
                                       d_sampled, _stream()),
               "jot_denoise_step")
        return out

    def lm_head_stats(self, hidden: torch.Tensor, tokens: torch.Tensor, blk_lo: int, blk_hi: int,
                      out: Optional[Stats] = None, exclude_mask_token: bool = True,
                      bump_id: Optional[torch.Tensor] = None, bump_val: Optional[torch.Tensor] = None,
                      sampling: Optional[Sampling] = None) -> Stats:
        B, L = tokens.shape
        if hidden.shape != (B * L, self.cfg.d_model):
            raise ValueError("hidden must be [B*L, d_model]")
        out = out or Stats.empty(B, L, tokens.device)
        sp, d_sampled = _sampling_args(sampling, out, B, L, tokens.device)
        _check(_lib().jot_lm_head_stats(self.handle, _ptr(hidden, torch.bfloat16, "hidden"),
                                        _ptr(tokens, torch.int32, "tokens"), B, L, blk_lo, blk_hi,
                                        int(exclude_mask_token), _ptr(bump_id, torch.int32, "bump_id"),
                                        _ptr(bump_val, torch.float32, "bump_val"), out.top1.data_ptr(),
                                        out.top2.data_ptr(), out.sumexp.data_ptr(), out.argmax.data_ptr(), sp,
                                        d_sampled, _stream()),
               "jot_lm_head_stats")
        return out

    def lm_head_stats_slice(self, hidden: torch.Tensor, tokens: torch.Tensor, blk_lo: int, blk_hi: int, v_lo: int,
                            v_hi: int, out: Optional[Stats] = None, exclude_mask_token: bool = True,
                            bump_id: Optional[torch.Tensor] = None, bump_val: Optional[torch.Tensor] = None) -> Stats:
        """Statistics of the active rows over the vocabulary slice [v_lo, v_hi) only (one rank's share of a
        vocabulary-parallel head)."""
        B, L = tokens.shape
        if hidden.shape != (B * L, self.cfg.d_model):
            raise ValueError("hidden must be [B*L, d_model]")
        out = out or Stats.empty(B, L, tokens.device)
        _check(_lib().jot_lm_head_stats_slice(self.handle, _ptr(hidden, torch.bfloat16, "hidden"),
                                              _ptr(tokens, torch.int32, "tokens"), B, L, blk_lo, blk_hi,
                                              int(exclude_mask_token), _ptr(bump_id, torch.int32, "bump_id"),
                                              _ptr(bump_val, torch.float32, "bump_val"), v_lo, v_hi, out.top1.data_ptr(),
                                              out.top2.data_ptr(), out.sumexp.data_ptr(), out.argmax.data_ptr(), None,
                                              None, _stream()),
               "jot_lm_head_stats_slice")
        return out

    # ---- Algorithm 1 ----------------------------------------------------------------------------
    def generate(self, prompt: torch.Tensor, gen_len: int, steps: int, params, block_len: Optional[int] = None,
                 exclude_mask_token: bool = True, bump_id: Optional[torch.Tensor] = None,
                 bump_val: Optional[torch.Tensor] = None, compact_finished: bool = True, use_cuda_graph: bool = False,
                 temperature: float = 0.0, seed: int = 0, trace: bool = False, kv_cache: bool = False):
        """Returns (tokens [B, P+gen_len] int32 on device, steps_used list[int], forward_passes int), and a
        Trace as a fourth element when trace is set."""
        B, P = prompt.shape
        per_seq = isinstance(params, (list, tuple))
        if per_seq:
            if len(params) != B:
                raise ValueError("need one Params per sequence")
            parr = (Params * B)(*params)
        else:
            parr = (Params * 1)(params)
        gen = GenConfig(gen_len, steps, block_len or gen_len, int(exclude_mask_token), int(compact_finished),
                        int(use_cuda_graph), float(temperature), seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF,
                        int(kv_cache))
        out = torch.empty(B, P + gen_len, dtype=torch.int32, device=prompt.device)
        used = (C.c_int32 * B)()
        passes = C.c_int32(0)
        tr, tr_arg = None, None
        if trace:
            dev = prompt.device
            tr = Trace(torch.empty(B, P + gen_len, dtype=torch.int16, device=dev),
                       torch.empty(B, P + gen_len, dtype=torch.uint8, device=dev),
                       torch.empty(steps, B, dtype=torch.float32, device=dev),
                       torch.empty(steps, B, dtype=torch.int32, device=dev))
            tr_arg = C.byref(_Trace(tr.exit_step.data_ptr(), tr.exit_reason.data_ptr(), tr.mean_ratio.data_ptr(),
                                    tr.n_candidates.data_ptr()))
        _check(_lib().jot_generate(self.handle, parr, int(per_seq), C.byref(gen), _ptr(prompt, torch.int32, "prompt"), B,
                                   P, _ptr(bump_id, torch.int32, "bump_id"), _ptr(bump_val, torch.float32, "bump_val"),
                                   out.data_ptr(), used, C.byref(passes), tr_arg, _stream()), "jot_generate")
        if trace:
            return out, list(used), int(passes.value), tr
        return out, list(used), int(passes.value)


def accept_freeze(params, mask_id: int, tokens: torch.Tensor, blk_lo: int, blk_hi: int, k_transfer: int,
                  stats: Stats, n_masked: Optional[torch.Tensor] = None, exit_reason: Optional[torch.Tensor] = None,
                  exit_step: Optional[torch.Tensor] = None, step_index: int = 0) -> None:
    """In-place acceptance / freeze update of tokens [B, L] (Section 4.1, Algorithm 1).
    params: one Params for the whole batch, or a list of B (one per sequence)."""
    B, L = tokens.shape
    per_seq = isinstance(params, (list, tuple))
    if per_seq:
        if len(params) != B:
            raise ValueError("need one Params per sequence")
        parr = (Params * B)(*params)
    else:
        parr = (Params * 1)(params)
    _check(_lib().jot_accept_freeze(parr, int(per_seq), mask_id, _ptr(tokens, torch.int32, "tokens"), B, L, blk_lo,
                                    blk_hi, k_transfer, _ptr(stats.top1, torch.float32, "top1"),
                                    _ptr(stats.top2, torch.float32, "top2"), _ptr(stats.sumexp, torch.float32, "sumexp"),
                                    _ptr(stats.argmax, torch.int32, "argmax"), _ptr(n_masked, torch.int32, "n_masked"),
                                    _ptr(exit_reason, torch.uint8, "exit_reason"),
                                    _ptr(exit_step, torch.int16, "exit_step"), step_index, _stream()),
           "jot_accept_freeze")


def merge_stats(a: Stats, b: Stats, out: Optional[Stats] = None) -> Stats:
    """Statistics of the same positions over two disjoint vocabulary slices -> over their union (device kernel)."""
    out = out or Stats(torch.empty_like(a.top1), torch.empty_like(a.top2), torch.empty_like(a.sumexp),
                       torch.empty_like(a.argmax))
    n = a.top1.numel()
    args = []
    for s in (a, b, out):
        args += [_ptr(s.top1, torch.float32, "top1"), _ptr(s.top2, torch.float32, "top2"),
                 _ptr(s.sumexp, torch.float32, "sumexp"), _ptr(s.argmax, torch.int32, "argmax")]
    _check(_lib().jot_merge_stats(n, *args, _stream()), "jot_merge_stats")
    return out


def gemm_bf16(a: torch.Tensor, w: torch.Tensor, residual: Optional[torch.Tensor] = None,
              out: Optional[torch.Tensor] = None, scratch: Optional[torch.Tensor] = None) -> torch.Tensor:
    """out[M, N] = a[M, K] @ w[N, K]^T (+ residual), bf16 in/out, fp32 accumulate.
    scratch: optional float32 CUDA tensor the kernel may use for split-K partial sums."""
    M, K = a.shape
    N = w.shape[0]
    out = torch.empty(M, N, dtype=torch.bfloat16, device=a.device) if out is None else out
    status = torch.zeros(1, dtype=torch.int32, device=a.device)
    _check(_lib().jot_gemm_bf16(_ptr(a, torch.bfloat16, "a"), _ptr(w, torch.bfloat16, "w"),
                                _ptr(residual, torch.bfloat16, "residual"), _ptr(out, torch.bfloat16, "out"), M, N, K,
                                _ptr(scratch, torch.float32, "scratch"), scratch.numel() * 4 if scratch is not None else 0,
                                status.data_ptr(), _stream()), "jot_gemm_bf16")
    if int(status.item()) != 0:
        raise JotError(-5, "jot_gemm_bf16")
    return out


def gemm_bf16_noalloc(a: torch.Tensor, w: torch.Tensor, residual: Optional[torch.Tensor], out: torch.Tensor,
                      status: torch.Tensor) -> torch.Tensor:
    """out[M, N] = a[M, K] @ w[N, K]^T (+ residual) through the entry point that never allocates.

    For callers that may not create device memory (a serving loop with a fixed memory plan, a plugin that
    only gets buffers handed to it): the split-K scratch is a fixed 16 MiB array inside the library, so
    4 * M * N * 4 bytes must fit in it.  `out` and the int32 `status` word are the caller's, too; this
    wrapper creates no tensor.  Calls share the array: keep them on one stream."""
    M, K = a.shape
    N = w.shape[0]
    _check(_lib().jot_gemm_bf16_noalloc(_ptr(a, torch.bfloat16, "a"), _ptr(w, torch.bfloat16, "w"),
                                        _ptr(residual, torch.bfloat16, "residual"), _ptr(out, torch.bfloat16, "out"),
                                        M, N, K, _ptr(status, torch.int32, "status"), _stream()),
           "jot_gemm_bf16_noalloc")
    return out


def selftest_wait_expiry(limit_ns: int = 20_000_000) -> int:
    """Run the bounded-wait self test; returns the status word the kernel wrote (1 = the wait gave up)."""
    status = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    _check(_lib().jot_selftest_wait_expiry(status.data_ptr(), limit_ns, _stream()), "jot_selftest_wait_expiry")
    return int(status.item())


# ---- decoding over a paged key-value cache -----------------------------------------------------------------------------
_ELEMENTS = {torch.bfloat16: 0, torch.float16: 1}     # JOT_BF16, JOT_FP16
STATUS_BAD_INDEX = 6                                    # what a status word becomes: a slot, page or length outside the pages


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _launch(device, where: str, fn, *args) -> None:
    """fn(*args, stream) on the current stream of the tensors' own device, whichever device is current."""
    index = device.index
    if index == torch.cuda.current_device():
        status = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, _raw_stream(index))
    if status != 0:
        raise JotError(status, where)


def _int_ptr(t: Optional[torch.Tensor], name: str, device, n: int) -> Optional[int]:
    """Pointer of an int32 tensor [n] on the device (None for None)."""
    if t is None:
        return None
    if t.dtype != torch.int32 or t.device != device or not t.is_contiguous():
        raise TypeError(f"{name}: expected a contiguous int32 tensor on {device}, got {t.dtype} on {t.device}")
    if t.dim() != 1 or t.numel() != n:
        raise ValueError(f"{name}: expected shape ({n},), got {tuple(t.shape)}")
    return t.data_ptr()


def _element_strides(t: torch.Tensor, name: str, dtype, device, shape):
    """Strides of a tensor of the given shape, element type and device whose last dimension is contiguous."""
    strides = t.stride()
    if t.dtype != dtype or t.device != device or len(strides) != len(shape) or (strides[-1] != 1 and shape[-1] > 1):
        raise TypeError(f"{name}: expected a {len(shape)}-D {dtype} tensor on {device} whose last dimension is contiguous, got "
                        f"{t.dim()}-D {t.dtype} on {t.device} with strides {strides}")
    if t.shape != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    return strides


class KVPages:
    """The pages of a key-value cache: k and v [n_layers, n_pages, n_kv_heads, page_size, head_dim], bf16 or fp16.  A page
    (its last three dimensions) is contiguous; layers and pages may lie at any stride that is a multiple of 8 elements, so
    that k and v may be two halves of one tensor.  The tensors are borrowed and written in place."""

    __slots__ = ("k", "v", "device", "dtype", "n_layers", "n_pages", "n_kv_heads", "page_size", "head_dim", "_packed")

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        shape, ks, vs, device, dtype = k.shape, k.stride(), v.stride(), k.device, k.dtype
        if len(shape) != 5 or v.shape != shape or v.dtype != dtype or dtype not in _ELEMENTS or device.type != "cuda" or v.device != device:
            raise TypeError("KVPages: k and v must be CUDA tensors [n_layers, n_pages, n_kv_heads, page_size, head_dim] of one "
                            "shape and device, bf16 or fp16")
        n_layers, n_pages, n_kv_heads, page_size, head_dim = shape
        inner = (page_size * head_dim, head_dim, 1)
        for st in (ks, vs):
            if st[2:] != inner and any(n > 1 and x != y for n, x, y in zip(shape[2:], st[2:], inner)):
                raise TypeError("KVPages: the last three dimensions must be contiguous")
        self.k, self.v, self.device, self.dtype = k, v, device, dtype
        self.n_layers, self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = shape
        self._packed = _pack_pages(k.data_ptr(), v.data_ptr(), ks[0], vs[0], ks[1], vs[1], n_layers, n_pages, n_kv_heads, page_size, head_dim,
                                   _ELEMENTS[dtype])

    @staticmethod
    def empty(n_layers: int, n_pages: int, n_kv_heads: int, page_size: int, head_dim: int, dtype=torch.bfloat16,
              device="cuda") -> "KVPages":
        shape = (n_layers, n_pages, n_kv_heads, page_size, head_dim)
        return KVPages(torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device))


@dataclasses.dataclass
class Rope:
    """A position rotation: inv_freq [rotary_dim / 2] (fp32, on the device, any long-context scaling already in it), pairs
    (i, i + rotary_dim / 2) or neighbours, cos and sin times `magnitude`."""
    inv_freq: torch.Tensor
    interleaved: bool = False
    magnitude: float = 1.0


def rope_frequencies(rotary_dim: int, theta: float, factor: float = 1.0, original_len: Optional[int] = None,
                     low_turns: float = 1.0, high_turns: float = 4.0, device="cuda") -> torch.Tensor:
    """Frequencies theta^(-2 i / rotary_dim) of a rotation, made in float64 and rounded to float32.

    For contexts `factor` times as long as the model was trained on: without original_len every frequency is divided by
    the factor (positions interpolated); with it, pairs that make at least high_turns turns over original_len positions keep
    their frequency, pairs that make at most low_turns are divided by the factor, and in between the two are blended
    linearly in the number of turns."""
    if rotary_dim <= 0 or rotary_dim % 2 or not theta > 0 or not factor > 0:
        raise ValueError("rope_frequencies: rotary_dim must be positive and even, theta and factor positive")
    f = float(theta) ** (-2.0 * torch.arange(rotary_dim // 2, dtype=torch.float64) / rotary_dim)
    keep = torch.zeros_like(f)
    if original_len is not None:
        if not high_turns > low_turns:
            raise ValueError("rope_frequencies: high_turns must exceed low_turns")
        keep = ((original_len * f / (2.0 * math.pi) - low_turns) / (high_turns - low_turns)).clamp(0.0, 1.0)
    return (f * (keep + (1.0 - keep) / factor)).to(torch.float32).to(device)


def _heads(x: torch.Tensor, out: Optional[torch.Tensor], gain: Optional[torch.Tensor], name: str, device, dtype, rows: int, hd: int,
           fresh: bool = False) -> bytes:
    """A packed jot_heads.  fresh: out was made here, like x."""
    n = x.shape[1]
    shape = (rows, n, hd)
    xs = _element_strides(x, name, dtype, device, shape)
    outs = (0, 0) if out is None else out.stride() if fresh else _element_strides(out, name + "_out", dtype, device, shape)
    if gain is not None and (gain.dtype != dtype or gain.device != device or gain.dim() != 1 or gain.numel() != hd or not gain.is_contiguous()):
        raise TypeError(f"{name}_gain: expected a contiguous {dtype} tensor [{hd}] on {device}")
    return _pack_heads(x.data_ptr(), xs[0], xs[1], 0 if out is None else out.data_ptr(), outs[0], outs[1], 0 if gain is None else gain.data_ptr(), n)


def head_norm_rope(q: torch.Tensor, k: Optional[torch.Tensor], positions: torch.Tensor, rope: Rope,
                   q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None, eps: float = 1e-6, *,
                   q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None,
                   v: Optional[torch.Tensor] = None, pages: Optional[KVPages] = None, layer: int = 0,
                   slots: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """Norm of every head of q [rows, heads, head_dim] and k (where a gain is given), then the rotation by positions [rows]
    (int32), in one pass.  Returns (q_out, k_out): new tensors unless given (q itself: in place).  With pages, k's results and
    v go to `layer` of the pages at slots [rows] = page * page_size + offset (int32), and k_out is None.  A row with a
    negative position, and the pages of a row with a negative slot, stay as they were."""
    device, dtype = q.device, q.dtype
    if dtype not in _ELEMENTS or q.dim() != 3 or device.type != "cuda":
        raise TypeError(f"q: expected a 3-D bf16 or fp16 CUDA tensor, got {q.dim()}-D {dtype} on {device}")
    if k is not None and k.dim() != 3 or v is not None and v.dim() != 3:
        raise TypeError("head_norm_rope: expected 3-D k and v")
    rows, _, hd = q.shape
    f = rope.inv_freq
    if f.dtype != torch.float32 or f.device != device or f.dim() != 1 or not f.is_contiguous():
        raise TypeError(f"rope.inv_freq: expected a contiguous 1-D float32 tensor on {device}")
    hk = hv = ref = None
    fresh_q, fresh_k = q_out is None, k_out is None
    if fresh_q:
        q_out = torch.empty_like(q)
    if pages is None:
        if v is not None or slots is not None:
            raise ValueError("head_norm_rope: v and slots go with pages")
        if k is not None:
            if k_out is None:
                k_out = torch.empty_like(k)
            hk = _heads(k, k_out, k_gain, "k", device, dtype, rows, hd, fresh_k)
    else:
        if k is None or v is None or slots is None or k_out is not None:
            raise ValueError("head_norm_rope: pages need k, v and slots, and take the place of k_out")
        if pages.device != device:
            raise TypeError(f"pages: expected on {device}, got {pages.device}")
        ref = pages._packed
        hk = _heads(k, None, k_gain, "k", device, dtype, rows, hd)
        hv = _heads(v, None, None, "v", device, dtype, rows, hd)
    _launch(device, "jot_head_norm_rope", _lib().jot_head_norm_rope, _heads(q, q_out, q_gain, "q", device, dtype, rows, hd, fresh_q), hk,
            _pack_rope(f.data_ptr(), 2 * f.numel(), rope.interleaved, rope.magnitude), _ELEMENTS[dtype], rows, hd, eps,
            _int_ptr(positions, "positions", device, rows), hv, ref, layer, _int_ptr(slots, "slots", device, rows),
            _int_ptr(status, "status", device, 1))
    return q_out, k_out


def kv_write(pages: KVPages, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, layer: int = 0,
             status: Optional[torch.Tensor] = None) -> None:
    """Rows k, v [rows, n_kv_heads, head_dim] into `layer` of the pages at slots [rows] (int32; negative: skipped).  Slots must
    differ from each other."""
    device, rows = pages.device, k.shape[0]
    shape = (rows, pages.n_kv_heads, pages.head_dim)
    ks, vs = _element_strides(k, "k", pages.dtype, device, shape), _element_strides(v, "v", pages.dtype, device, shape)
    _launch(device, "jot_kv_write", _lib().jot_kv_write, pages._packed, layer, rows, k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1],
            _int_ptr(slots, "slots", device, rows), _int_ptr(status, "status", device, 1))


def kv_copy_pages(pages: KVPages, src: Sequence[int], dst: Sequence[int]) -> None:
    """Page src[i] onto page dst[i], in every layer.  src and dst are lists on the host; no page twice in dst, none in both."""
    if len(src) != len(dst):
        raise ValueError("kv_copy_pages: src and dst differ in length")
    n = len(src)
    src, dst = array.array("i", src), array.array("i", dst)      # refuses what is no 32-bit integer
    pair = C.c_int32 * n
    _launch(pages.device, "jot_kv_copy_pages", _lib().jot_kv_copy_pages, pages._packed, n, pair.from_buffer(src) if n else None,
            pair.from_buffer(dst) if n else None)


@functools.lru_cache(maxsize=None)
def paged_attention_workspace_bytes(T: int, n_q_heads: int, n_kv_heads: int, head_dim: int) -> int:
    """Device bytes a paged_attention call of T rows a sequence needs, whatever the batch and the lengths (0: unsupported)."""
    return int(_lib().jot_paged_attention_workspace_bytes(T, n_q_heads, n_kv_heads, head_dim))


def paged_attention(q: torch.Tensor, pages: KVPages, page_table: torch.Tensor, lens: torch.Tensor, layer: int = 0,
                    scale: Optional[float] = None, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of q [B, T, n_q_heads, head_dim] over the first lens[b] keys of each sequence, which lie in the pages of
    `layer` that page_table [B, max_pages] names (both int32).  Bidirectional: every row sees every key.  scale defaults to
    head_dim^-0.5; lse [B, T, n_q_heads] (fp32, optional) receives the logarithm of the sum of exponentials.  A length of 0
    gives zeros and -inf, a negative one leaves its sequence's rows of out and lse as they were.

    workspace: optional uint8 tensor of paged_attention_workspace_bytes(); calls that may overlap need one each."""
    device, shape = pages.device, q.shape
    if len(shape) != 4 or shape[3] != pages.head_dim:
        raise ValueError(f"q: expected [B, T, n_q_heads, {pages.head_dim}], got {tuple(shape)}")
    B, T, nq, hd = shape
    qs = _element_strides(q, "q", pages.dtype, device, shape)
    if out is None:
        out = torch.empty_like(q)
        outs = out.stride()
    else:
        outs = _element_strides(out, "out", pages.dtype, device, shape)
    if lse is not None and (lse.dtype != torch.float32 or lse.device != device or lse.shape != shape[:3] or not lse.is_contiguous()):
        raise TypeError(f"lse: expected a contiguous float32 tensor {tuple(shape[:3])} on {device}")
    table = page_table.shape
    if page_table.dtype != torch.int32 or page_table.device != device or len(table) != 2 or table[0] != B or (
            table[1] > 1 and page_table.stride(1) != 1):
        raise TypeError(f"page_table: expected an int32 tensor [{B}, max_pages] on {device} with contiguous rows")
    if workspace is None:
        workspace = torch.empty(paged_attention_workspace_bytes(T, nq, pages.n_kv_heads, hd), dtype=torch.uint8, device=device)
    elif workspace.dtype != torch.uint8 or workspace.device != device or not workspace.is_contiguous():
        raise TypeError(f"workspace: expected a contiguous uint8 tensor on {device}")
    _launch(device, "jot_paged_attention", _lib().jot_paged_attention, q.data_ptr(), qs[0], qs[1], qs[2], out.data_ptr(), outs[0], outs[1], outs[2],
            None if lse is None else lse.data_ptr(), B, T, nq, pages._packed, layer, page_table.data_ptr(), page_table.stride(0), table[1],
            _int_ptr(lens, "lens", device, B), hd ** -0.5 if scale is None else scale, workspace.data_ptr(), workspace.numel(),
            _int_ptr(status, "status", device, 1))
    return out
