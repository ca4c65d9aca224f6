"""Thin Python binding of the C-ABI CUDA library (``include/ngc.h``).

Argument marshalling only: torch tensors provide device memory and the current
CUDA stream, every step of the path runs inside the library's kernels.  There
is no CPU fallback: importing this module without the built library raises,
and so does every call made without a CUDA device.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libngc_b200.so")

F32, BF16 = 0, 1
LISTS_SHARED, LISTS_PER_LAYER, LISTS_PER_LAYER_KVHEAD = 0, 1, 2
OP_SCORE, OP_SAMPLE, OP_LOGPROB, OP_COMPACT, OP_DECODE, OP_SCORE_BACKWARD, OP_TREE_ATTN = range(7)

DEV_STATUS = {0: "ok", 1: "bad counts", 2: "NaN logit", 3: "bad kept list", 4: "strip full",
              5: "lists disagree", 6: "timeout", 7: "index out of bounds (bounds-checking build)", 8: "bad drafted tree or path",
              9: "numbers that are no probabilities, or have no finite positive sum", 10: "bad fork source", 11: "bad page-table entry",
              12: "pool has too few free pages", 13: "slot outside the pool"}

EXPORTS = ["ngc_version", "ngc_strerror", "ngc_last_cuda_error", "ngc_workspace_bytes", "ngc_decode_splits", "ngc_score_evict", "ngc_score_evict_launches",
           "ngc_sample_evict", "ngc_evict_logprob", "ngc_evict_logprob_backward", "ngc_compact_kv", "ngc_decode_attn_ragged",
           "ngc_decode_attn_ragged_static", "ngc_evict_pages", "ngc_decode_attn_paged", "ngc_score_evict_paged", "ngc_replay_visibility", "ngc_score_evict_backward", "ngc_replay_attn", "ngc_replay_attn_variant", "ngc_selftest_bounded_wait",
           "ngc_tree_attn", "ngc_tree_attn_paged", "ngc_tree_attn_launches", "ngc_verify_draft", "ngc_commit_draft", "ngc_commit_draft_paged",
           "ngc_fork_kv", "ngc_fork_pages", "ngc_pool_update", "ngc_latent_write", "ngc_latent_decode", "ngc_latent_decode_workspace_bytes",
           "ngc_latent_replay_attn", "ngc_latent_replay_attn_backward", "ngc_latent_replay_workspace_bytes"]
STATIC_SCRATCH_BYTES = 8 << 20
TREE_MAX_NODES = 128


class NgcError(RuntimeError):
    pass


class CacheDesc(C.Structure):
    """Mirror of ``ngc_cache``."""
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("seq_off", C.c_void_p), ("lens", C.c_void_p),
                ("rows", C.c_int64), ("L", C.c_int32), ("B", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32),
                ("d", C.c_int32), ("dtype", C.c_int32), ("max_len", C.c_int32), ("lens_lists", C.c_int32)]


class PagedCacheDesc(C.Structure):
    """Mirror of ``ngc_paged_cache``."""
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_table", C.c_void_p), ("lens", C.c_void_p),
                ("L", C.c_int32), ("B", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("d", C.c_int32),
                ("dtype", C.c_int32), ("page", C.c_int32), ("pages_cap", C.c_int32), ("lists", C.c_int32),
                ("lens_per_list", C.c_int32)]


class LatentPoolDesc(C.Structure):
    """Mirror of ``ngc_latent_pool``."""
    _fields_ = [("rows", C.c_void_p), ("page_table", C.c_void_p), ("page_used", C.c_void_p), ("lens", C.c_void_p),
                ("L", C.c_int32), ("B", C.c_int32), ("d_latent", C.c_int32), ("d_rope", C.c_int32), ("dtype", C.c_int32),
                ("page", C.c_int32), ("pages_cap", C.c_int32), ("n_pages", C.c_int32), ("lists", C.c_int32)]


class LatentSeqsDesc(C.Structure):
    """Mirror of ``ngc_latent_seqs``."""
    _fields_ = [("seq_off", C.c_void_p), ("lens", C.c_void_p), ("rows", C.c_int64), ("L", C.c_int32), ("B", C.c_int32),
                ("H", C.c_int32), ("d_nope", C.c_int32), ("d_v", C.c_int32), ("d_rope", C.c_int32), ("dtype", C.c_int32),
                ("max_len", C.c_int32)]


def _load(path: str = LIB_PATH):
    if not os.path.exists(path):
        raise ImportError(
            f"{path} is missing: build it with `python -m paper_2604_18002_b200.build` "
            "(there is no CPU fallback)")
    lib = C.CDLL(path)
    vp, i32, u32, u64, sz = C.c_void_p, C.c_int, C.c_uint32, C.c_uint64, C.c_size_t
    lib.ngc_version.restype = i32
    lib.ngc_strerror.restype = C.c_char_p
    lib.ngc_strerror.argtypes = [i32]
    lib.ngc_last_cuda_error.restype = i32
    lib.ngc_workspace_bytes.restype = sz
    lib.ngc_workspace_bytes.argtypes = [i32, C.POINTER(CacheDesc), i32, i32, i32]
    lib.ngc_decode_splits.restype = i32
    lib.ngc_decode_splits.argtypes = [C.POINTER(CacheDesc), i32]
    lib.ngc_score_evict_launches.restype = i32
    lib.ngc_score_evict_launches.argtypes = [C.POINTER(CacheDesc), i32]
    lib.ngc_score_evict.restype = i32
    lib.ngc_score_evict.argtypes = [C.POINTER(CacheDesc), vp, i32, i32, i32, i32, vp, i32, vp, vp, sz, vp, vp]
    lib.ngc_sample_evict.restype = i32
    lib.ngc_sample_evict.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, u64, u64, u32, i32, vp, vp, vp, vp, sz, vp, vp]
    lib.ngc_evict_logprob.restype = i32
    lib.ngc_evict_logprob.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, sz, vp, vp]
    lib.ngc_evict_logprob_backward.restype = i32
    lib.ngc_evict_logprob_backward.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, sz, vp, vp]
    lib.ngc_compact_kv.restype = i32
    lib.ngc_compact_kv.argtypes = [C.POINTER(CacheDesc), vp, vp, i32, i32, i32, vp, vp]
    lib.ngc_decode_attn_ragged.restype = i32
    lib.ngc_decode_attn_ragged.argtypes = [C.POINTER(CacheDesc), vp, vp, vp, i32, i32, C.c_float, vp, i32, vp, sz, vp, vp]
    lib.ngc_decode_attn_ragged_static.restype = i32
    lib.ngc_decode_attn_ragged_static.argtypes = [C.POINTER(CacheDesc), vp, vp, vp, i32, i32, C.c_float, vp, i32, vp, vp]
    lib.ngc_score_evict_paged.restype = i32
    lib.ngc_score_evict_paged.argtypes = [C.POINTER(PagedCacheDesc), vp, i32, i32, vp, i32, vp, vp, sz, vp, vp]
    lib.ngc_score_evict_backward.restype = i32
    lib.ngc_score_evict_backward.argtypes = [C.POINTER(CacheDesc), vp, i32, i32, i32, i32, vp, vp, i32, vp, vp, vp, sz, vp, vp]
    lib.ngc_replay_attn.restype = i32
    lib.ngc_replay_attn.argtypes = [C.POINTER(CacheDesc), vp, i32, vp, vp, vp, i32, i32, i32, C.c_float, vp, i32, vp, vp]
    lib.ngc_replay_attn_variant.restype = i32
    lib.ngc_replay_attn_variant.argtypes = [C.POINTER(CacheDesc), vp, i32, vp, vp, vp, i32, i32, i32, C.c_float, vp, i32, i32, vp, vp]
    lib.ngc_replay_visibility.restype = i32
    lib.ngc_replay_visibility.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp]
    lib.ngc_selftest_bounded_wait.restype = i32
    lib.ngc_selftest_bounded_wait.argtypes = [u32, vp, vp, vp]
    lib.ngc_evict_pages.restype = i32
    lib.ngc_evict_pages.argtypes = [C.POINTER(PagedCacheDesc), vp, vp, i32, vp, vp]
    lib.ngc_decode_attn_paged.restype = i32
    lib.ngc_decode_attn_paged.argtypes = [C.POINTER(PagedCacheDesc), vp, vp, vp, i32, i32, C.c_float, vp, i32, vp, sz, vp, vp]
    tree = [vp, vp, vp, vp, vp, i32, i32, i32, C.c_float, vp, i32, vp, sz, vp, vp]
    lib.ngc_tree_attn.restype = i32
    lib.ngc_tree_attn.argtypes = [C.POINTER(CacheDesc)] + tree
    lib.ngc_tree_attn_paged.restype = i32
    lib.ngc_tree_attn_paged.argtypes = [C.POINTER(PagedCacheDesc)] + tree
    lib.ngc_tree_attn_launches.restype = i32
    lib.ngc_tree_attn_launches.argtypes = [C.POINTER(CacheDesc), i32, i32]
    lib.ngc_verify_draft.restype = i32
    lib.ngc_verify_draft.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp]
    lib.ngc_commit_draft.restype = i32
    lib.ngc_commit_draft.argtypes = [C.POINTER(CacheDesc), vp, vp, vp, vp, i32, vp, vp]
    lib.ngc_commit_draft_paged.restype = i32
    lib.ngc_commit_draft_paged.argtypes = [C.POINTER(PagedCacheDesc), vp, vp, vp, vp, i32, vp, vp]
    lib.ngc_fork_kv.restype = i32
    lib.ngc_fork_kv.argtypes = [C.POINTER(CacheDesc), vp, vp, vp]
    lib.ngc_fork_pages.restype = i32
    lib.ngc_fork_pages.argtypes = [C.POINTER(PagedCacheDesc), vp, vp, vp]
    lib.ngc_pool_update.restype = i32
    lib.ngc_pool_update.argtypes = [C.POINTER(LatentPoolDesc), vp, vp, i32, vp, vp, i32, vp, vp, vp]
    lib.ngc_latent_write.restype = i32
    lib.ngc_latent_write.argtypes = [C.POINTER(LatentPoolDesc), vp, i32, vp, vp, i32, i32, vp, vp]
    lib.ngc_latent_decode.restype = i32
    lib.ngc_latent_decode.argtypes = [C.POINTER(LatentPoolDesc), vp, vp, i32, i32, i32, C.c_float, vp, i32, vp, sz, vp, vp]
    lib.ngc_latent_decode_workspace_bytes.restype = sz
    lib.ngc_latent_decode_workspace_bytes.argtypes = [C.POINTER(LatentPoolDesc), i32]
    replay = [C.POINTER(LatentSeqsDesc), vp, vp, vp, vp, vp, vp, i32, i32, i32, C.c_float, vp, i32, vp]
    lib.ngc_latent_replay_attn.restype = i32
    lib.ngc_latent_replay_attn.argtypes = replay + [vp, sz, vp, vp]
    lib.ngc_latent_replay_attn_backward.restype = i32
    lib.ngc_latent_replay_attn_backward.argtypes = replay + [vp, vp, vp, vp, vp, sz, vp, vp]
    lib.ngc_latent_replay_workspace_bytes.restype = sz
    lib.ngc_latent_replay_workspace_bytes.argtypes = [C.POINTER(LatentSeqsDesc), i32, i32, i32]
    return lib


lib = _load()


@contextlib.contextmanager
def use_library(path: str):
    """Route every call of this module to another build of the library (the bounds-checking or the
    NVTX build) for the duration of the block."""
    global lib
    saved, lib = lib, _load(path)
    try:
        yield lib
    finally:
        lib = saved


def _check(rc: int, what: str):
    if rc != 0:
        msg = lib.ngc_strerror(rc).decode()
        if rc == -4:
            msg += f" (cudaError {lib.ngc_last_cuda_error()})"
        raise NgcError(f"{what}: {msg}")


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise NgcError("device tensors required: the library has no CPU path")
    if not t.is_contiguous():
        raise NgcError("contiguous tensors required")
    return t.data_ptr()


# Argument checks of the drafted-token calls.  A draft step is a handful of calls per layer, a few microseconds each on
# the GPU, so the checks are written to cost little: one pass per tensor that ends in its address.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_I32, _F32, _I64, _U8 = torch.int32, torch.float32, torch.int64, torch.uint8


def _refuse(what: str, name: str, t: torch.Tensor, shape, dtype, index: int):
    if t.shape != shape or t.dtype is not dtype:
        raise NgcError(f"{what}: {name} must be {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    if not t.is_contiguous():
        raise NgcError(f"{what}: {name} must be contiguous")
    raise NgcError(f"{what}: {name} is on {t.device}, the call's other tensors on " + ("the host" if index < 0 else f"cuda:{index}"))


def _arg(what: str, name: str, t: Optional[torch.Tensor], shape, dtype, index: int):
    """Address of a contiguous tensor of that shape and type on device ``index`` (-1: host); None for None."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index or not t.is_contiguous():
        _refuse(what, name, t, shape, dtype, index)
    return t.data_ptr()


def _launch_stream(what: str, index: int):
    """The current stream of the device that the tensors are on, which must be the current one (the library launches there)."""
    if index < 0:
        raise NgcError(f"{what}: device tensors required: the library has no CPU path")
    if index != torch.cuda.current_device():
        raise NgcError(f"{what}: tensors on cuda:{index}, but the current device is {torch.cuda.current_device()}")
    return _raw_stream(index) if _raw_stream is not None else torch.cuda.current_stream(index).cuda_stream


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise NgcError(f"unsupported cache dtype {t.dtype}")


def lists_G(lists: int, L: int, Hkv: int) -> int:
    return 1 if lists == LISTS_SHARED else (L if lists == LISTS_PER_LAYER else L * Hkv)


@dataclass
class NgcCache:
    """Device K/V cache plus the host-side numbers the launches need."""
    k: torch.Tensor        # [L][Hkv][R][d]
    v: torch.Tensor
    seq_off: torch.Tensor  # int64 [B+1], device
    lens: torch.Tensor     # int32 [B] (or [B][G] with lens_lists != 0), device
    Hq: int
    max_len: int           # host bound on lens (any value >= max(lens) at call time)
    lens_lists: int = 0    # 0: one length per sequence; LISTS_PER_LAYER / _KVHEAD: one per (sequence, list)

    def desc(self, extra_len: int = 0) -> CacheDesc:
        L, Hkv, R, d = self.k.shape
        if self.lens_lists:
            assert tuple(self.lens.shape) == (self.seq_off.shape[0] - 1, lists_G(self.lens_lists, L, Hkv))
        return CacheDesc(_ptr(self.k), _ptr(self.v), _ptr(self.seq_off), _ptr(self.lens), R, L,
                         self.seq_off.shape[0] - 1, self.Hq, Hkv, d, _dtype_code(self.k), self.max_len + extra_len,
                         self.lens_lists)

    @property
    def L(self):
        return self.k.shape[0]

    @property
    def B(self):
        return self.seq_off.shape[0] - 1

    @property
    def Hkv(self):
        return self.k.shape[1]

    @property
    def d(self):
        return self.k.shape[3]


def version() -> int:
    return lib.ngc_version()


def workspace_bytes(op: int, cache: Optional[NgcCache] = None, G: int = 1, n_max: int = 0, k_max: int = 0,
                    B: Optional[int] = None) -> int:
    if cache is not None:
        d = cache.desc(1)
    else:
        d = CacheDesc(None, None, None, None, 0, 1, B or 1, 1, 1, 128, BF16, 0)
    return int(lib.ngc_workspace_bytes(op, C.byref(d), G, n_max, k_max))


def decode_splits(cache: NgcCache, layers: Optional[int] = None, append: bool = True) -> int:
    d = cache.desc(1 if append else 0)
    return int(lib.ngc_decode_splits(C.byref(d), cache.L if layers is None else layers))


def score_launches(cache: NgcCache, w: int) -> int:
    """Kernels one ngc_score_evict call enqueues (launch counting)."""
    d = cache.desc()
    return int(lib.ngc_score_evict_launches(C.byref(d), w))


def alloc_workspace(nbytes: int, device="cuda") -> Optional[torch.Tensor]:
    if nbytes == 0:
        return None
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def new_status(device="cuda") -> torch.Tensor:
    return torch.zeros(1, dtype=torch.int32, device=device)


def ngc_score_evict(cache: NgcCache, q_recent: torch.Tensor, block: int, lists: int, logits: torch.Tensor,
                    log_transform: int = 0, ws: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                    n_units_out: Optional[torch.Tensor] = None):
    """q_recent [L][B][Hq][w][d] -> logits [B][G][n_max] fp32 (in place); n_units_out int32 [B] (optional):
    the unit count per sequence to hand to the sampler."""
    w = q_recent.shape[3]
    n_max = logits.shape[2]
    d = cache.desc()
    rc = lib.ngc_score_evict(C.byref(d), _ptr(q_recent), w, block, lists, log_transform, _ptr(logits), n_max,
                             _ptr(n_units_out), _ptr(ws), 0 if ws is None else ws.numel(), _ptr(status), _stream())
    _check(rc, "ngc_score_evict")


def ngc_sample_evict(logits: torch.Tensor, n: torch.Tensor, n_protect: Optional[torch.Tensor], budget: torch.Tensor,
                     seed: int, rnd: int, kept_order: torch.Tensor, kept_sorted: torch.Tensor,
                     keep_mask: Optional[torch.Tensor] = None, greedy: int = 0, list_base: int = 0,
                     ws: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    B, G, n_max = logits.shape
    k_max = kept_order.shape[2]
    rc = lib.ngc_sample_evict(_ptr(logits), _ptr(n), _ptr(n_protect), _ptr(budget), B, G, n_max, k_max,
                              seed, rnd, list_base, greedy, _ptr(kept_order), _ptr(kept_sorted), _ptr(keep_mask),
                              _ptr(ws), 0 if ws is None else ws.numel(), _ptr(status), _stream())
    _check(rc, "ngc_sample_evict")


def ngc_evict_logprob(logits: torch.Tensor, n: torch.Tensor, n_protect: Optional[torch.Tensor], budget: torch.Tensor,
                      kept_order: torch.Tensor, logp: torch.Tensor, status: Optional[torch.Tensor] = None):
    """logits [NB][B][G][n_max] (or [B][G][n_max]); logp fp64 [NB][B][G]."""
    if logits.dim() == 3:
        NB = 1
        B, G, n_max = logits.shape
    else:
        NB, B, G, n_max = logits.shape
    k_max = kept_order.shape[-1]
    rc = lib.ngc_evict_logprob(_ptr(logits), _ptr(n), _ptr(n_protect), _ptr(budget), _ptr(kept_order),
                               NB, B, G, n_max, k_max, _ptr(logp), None, 0, _ptr(status), _stream())
    _check(rc, "ngc_evict_logprob")


def ngc_evict_logprob_backward(logits: torch.Tensor, n: torch.Tensor, n_protect: Optional[torch.Tensor], budget: torch.Tensor,
                               kept_order: torch.Tensor, grad_logits: torch.Tensor, grad_logp: Optional[torch.Tensor] = None,
                               status: Optional[torch.Tensor] = None):
    """grad_logits fp32, same shape as logits; grad_logp fp64 [NB][B][G] or None (= ones)."""
    if logits.dim() == 3:
        NB = 1
        B, G, n_max = logits.shape
    else:
        NB, B, G, n_max = logits.shape
    k_max = kept_order.shape[-1]
    rc = lib.ngc_evict_logprob_backward(_ptr(logits), _ptr(n), _ptr(n_protect), _ptr(budget), _ptr(kept_order), _ptr(grad_logp),
                                        NB, B, G, n_max, k_max, _ptr(grad_logits), None, 0, _ptr(status), _stream())
    _check(rc, "ngc_evict_logprob_backward")


def ngc_compact_kv(cache: NgcCache, kept_sorted: torch.Tensor, budget: torch.Tensor, lists: int, block: int = 1,
                   status: Optional[torch.Tensor] = None):
    d = cache.desc()
    rc = lib.ngc_compact_kv(C.byref(d), _ptr(kept_sorted), _ptr(budget), kept_sorted.shape[2], lists, block,
                            _ptr(status), _stream())
    _check(rc, "ngc_compact_kv")


def ngc_decode_attn_ragged(cache: NgcCache, q: torch.Tensor, out: torch.Tensor, new_k: Optional[torch.Tensor] = None,
                           new_v: Optional[torch.Tensor] = None, layer_begin: int = 0, layer_end: Optional[int] = None,
                           scale: Optional[float] = None, ws: Optional[torch.Tensor] = None,
                           status: Optional[torch.Tensor] = None):
    if layer_end is None:
        layer_end = cache.L
    if scale is None:
        scale = 1.0 / (cache.d ** 0.5)
    d = cache.desc(1 if new_k is not None else 0)
    rc = lib.ngc_decode_attn_ragged(C.byref(d), _ptr(q), _ptr(new_k), _ptr(new_v), layer_begin, layer_end,
                                    scale, _ptr(out), _dtype_code(out), _ptr(ws), 0 if ws is None else ws.numel(),
                                    _ptr(status), _stream())
    _check(rc, "ngc_decode_attn_ragged")


def ngc_decode_attn_ragged_static(cache: NgcCache, q: torch.Tensor, out: torch.Tensor, new_k: Optional[torch.Tensor] = None,
                                  new_v: Optional[torch.Tensor] = None, layer_begin: int = 0,
                                  layer_end: Optional[int] = None, scale: Optional[float] = None,
                                  status: Optional[torch.Tensor] = None):
    """Decode attention for callers that cannot supply device scratch memory: the split partials
    live in an array built into the library (``STATIC_SCRATCH_BYTES``), nothing is allocated.
    Keep calls stream-ordered (they share the array); make the first call on a device outside
    any stream capture (it looks the array's address up).  Raises when the launch would need
    more scratch than the array holds."""
    if layer_end is None:
        layer_end = cache.L
    if scale is None:
        scale = 1.0 / (cache.d ** 0.5)
    d = cache.desc(1 if new_k is not None else 0)
    rc = lib.ngc_decode_attn_ragged_static(C.byref(d), _ptr(q), _ptr(new_k), _ptr(new_v), layer_begin, layer_end,
                                           scale, _ptr(out), _dtype_code(out), _ptr(status), _stream())
    _check(rc, "ngc_decode_attn_ragged_static")


@dataclass
class NgcPagedCache:
    """Paged device K/V cache: one eviction unit = one page; eviction edits ``page_table`` only."""
    k: torch.Tensor           # [L][Hkv][B * pages_cap][page][d] bf16
    v: torch.Tensor
    page_table: torch.Tensor  # int32 [B][G][pages_cap], each row a permutation of 0..pages_cap-1
    lens: torch.Tensor        # int32 [B], or [B][G] (a length per list)
    Hq: int
    lists: int

    def desc(self) -> PagedCacheDesc:
        L, Hkv, n_pages, page, d = self.k.shape
        B, G, pages_cap = self.page_table.shape
        assert n_pages == B * pages_cap and G == lists_G(self.lists, L, Hkv)
        return PagedCacheDesc(_ptr(self.k), _ptr(self.v), _ptr(self.page_table), _ptr(self.lens), L, B, self.Hq, Hkv, d,
                              _dtype_code(self.k), page, pages_cap, self.lists, 1 if self.lens.dim() == 2 else 0)

    def as_contiguous_desc(self) -> "NgcCache":
        """Shape-only view for workspace sizing (same L, B, Hq, Hkv)."""
        L, Hkv, n_pages, page, d = self.k.shape
        B, _, pages_cap = self.page_table.shape
        flat = self.k.view(L, Hkv, n_pages * page, d)
        return NgcCache(flat, flat, torch.zeros(B + 1, dtype=torch.int64, device=self.k.device), self.lens, self.Hq, pages_cap * page)


def ngc_evict_pages(cache: NgcPagedCache, kept_sorted: torch.Tensor, budget: torch.Tensor, status: Optional[torch.Tensor] = None):
    d = cache.desc()
    rc = lib.ngc_evict_pages(C.byref(d), _ptr(kept_sorted), _ptr(budget), kept_sorted.shape[2], _ptr(status), _stream())
    _check(rc, "ngc_evict_pages")


def ngc_decode_attn_paged(cache: NgcPagedCache, q: torch.Tensor, out: torch.Tensor, new_k: Optional[torch.Tensor] = None,
                          new_v: Optional[torch.Tensor] = None, layer_begin: int = 0, layer_end: Optional[int] = None,
                          scale: Optional[float] = None, ws: Optional[torch.Tensor] = None,
                          status: Optional[torch.Tensor] = None):
    L, d = cache.k.shape[0], cache.k.shape[4]
    if layer_end is None:
        layer_end = L
    if scale is None:
        scale = 1.0 / (d ** 0.5)
    desc = cache.desc()
    rc = lib.ngc_decode_attn_paged(C.byref(desc), _ptr(q), _ptr(new_k), _ptr(new_v), layer_begin, layer_end, scale,
                                   _ptr(out), _dtype_code(out), _ptr(ws), 0 if ws is None else ws.numel(), _ptr(status), _stream())
    _check(rc, "ngc_decode_attn_paged")


def ngc_score_evict_paged(cache: NgcPagedCache, q_recent: torch.Tensor, logits: torch.Tensor, log_transform: int = 0,
                          ws: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                          n_units_out: Optional[torch.Tensor] = None):
    """q_recent [L][B][Hq][w][d] -> logits [B][G][n_max] fp32 (units = pages)."""
    d = cache.desc()
    rc = lib.ngc_score_evict_paged(C.byref(d), _ptr(q_recent), q_recent.shape[3], log_transform, _ptr(logits), logits.shape[2],
                                   _ptr(n_units_out), _ptr(ws), 0 if ws is None else ws.numel(), _ptr(status), _stream())
    _check(rc, "ngc_score_evict_paged")


def ngc_replay_visibility(kept_sorted: torch.Tensor, budget: torch.Tensor, alive_before: torch.Tensor, total_before: torch.Tensor,
                          block: int, alive_max: int, alive_pos: torch.Tensor, alive_count: torch.Tensor,
                          status: Optional[torch.Tensor] = None):
    """kept_sorted [R][B][G][k_max] -> alive_pos [R][B][G][k_max*block], alive_count [R][B][G] (int32)."""
    R, B, G, k_max = kept_sorted.shape
    rc = lib.ngc_replay_visibility(_ptr(kept_sorted), _ptr(budget), _ptr(alive_before), _ptr(total_before), R, B, G, k_max, block,
                                   alive_max, 1 if alive_before.dim() == 3 else 0, _ptr(alive_pos), _ptr(alive_count), _ptr(status),
                                   _stream())
    _check(rc, "ngc_replay_visibility")


def ngc_score_evict_backward(cache: NgcCache, q_recent: torch.Tensor, block: int, lists: int, grad_logits: torch.Tensor,
                             grad_q_recent: torch.Tensor, grad_k: torch.Tensor, logits: Optional[torch.Tensor] = None,
                             log_transform: int = 0, ws: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """grad_logits [B][G][n_max] fp32 -> grad_q_recent fp32 (shape of q_recent), grad_k (shape and dtype of cache.k)."""
    d = cache.desc()
    rc = lib.ngc_score_evict_backward(C.byref(d), _ptr(q_recent), q_recent.shape[3], block, lists, log_transform, _ptr(logits),
                                      _ptr(grad_logits), grad_logits.shape[2], _ptr(grad_q_recent), _ptr(grad_k),
                                      _ptr(ws), 0 if ws is None else ws.numel(), _ptr(status), _stream())
    _check(rc, "ngc_score_evict_backward")


def tree_attn_launches(cache: NgcCache, N: int, layers: Optional[int] = None) -> int:
    """Kernels one ngc_tree_attn call over ``layers`` layers enqueues (launch counting)."""
    d = cache.desc()
    return int(lib.ngc_tree_attn_launches(C.byref(d), cache.L if layers is None else layers, N))


def _view(what: str, cache):
    """Checks a cache's own tensors; (descriptor, L, B, Hkv, d, dtype, device index)."""
    k, lens = cache.k, cache.lens
    shape, dt, index = k.shape, k.dtype, k.get_device()
    kp, vp = _arg(what, "k", k, shape, dt, index), _arg(what, "v", cache.v, shape, dt, index)
    if isinstance(cache, NgcPagedCache):
        L, Hkv, n_pages, page, d = shape
        table = cache.page_table
        B, G, cap = table.shape
        if n_pages != B * cap or G != lists_G(cache.lists, L, Hkv):
            raise NgcError(f"{what}: page_table {tuple(table.shape)} does not fit k {tuple(shape)} and the lists")
        per = lens.dim() == 2
        desc = PagedCacheDesc(kp, vp, _arg(what, "page_table", table, table.shape, _I32, index),
                              _arg(what, "lens", lens, (B, G) if per else (B,), _I32, index), L, B, cache.Hq, Hkv, d, _dtype_code(k), page, cap,
                              cache.lists, 1 if per else 0)
    else:
        L, Hkv, R, d = shape
        B, per = cache.seq_off.shape[0] - 1, cache.lens_lists
        desc = CacheDesc(kp, vp, _arg(what, "seq_off", cache.seq_off, (B + 1,), _I64, index),
                         _arg(what, "lens", lens, (B, lists_G(per, L, Hkv)) if per else (B,), _I32, index), R, L, B, cache.Hq, Hkv, d,
                         _dtype_code(k), cache.max_len, per)
    return desc, L, B, Hkv, d, dt, index


def _tree_attn(what, call, cache, q, tree_k, tree_v, parent, out, n_nodes, layer_begin, layer_end, scale, ws, status):
    desc, L, B, Hkv, d, dt, index = _view(what, cache)
    N = parent.shape[-1]
    heads, rows = (L, B, cache.Hq, N, d), (L, B, Hkv, N, d)
    args = (_arg(what, "q", q, heads, dt, index), _arg(what, "tree_k", tree_k, rows, dt, index), _arg(what, "tree_v", tree_v, rows, dt, index),
            _arg(what, "parent", parent, (B, N), _I32, index), _arg(what, "n_nodes", n_nodes, (B,), _I32, index), N, layer_begin,
            L if layer_end is None else layer_end, d ** -0.5 if scale is None else scale, _arg(what, "out", out, heads, out.dtype, index),
            _dtype_code(out), None if ws is None else _arg(what, "ws", ws, ws.shape, _U8, index), 0 if ws is None else ws.numel(),
            _arg(what, "status", status, (1,), _I32, index))
    _check(call(C.byref(desc), *args, _launch_stream(what, index)), what)


def ngc_tree_attn(cache: NgcCache, q: torch.Tensor, tree_k: torch.Tensor, tree_v: torch.Tensor, parent: torch.Tensor,
                  out: torch.Tensor, n_nodes: Optional[torch.Tensor] = None, layer_begin: int = 0, layer_end: Optional[int] = None,
                  scale: Optional[float] = None, ws: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """Attention for a tree of drafted tokens over the cache: q, out [L][B][Hq][N][d]; tree_k, tree_v [L][B][Hkv][N][d];
    parent int32 [B][N]; n_nodes int32 [B] or None (= N).  ``ws``: workspace_bytes(OP_TREE_ATTN, cache, n_max=N)."""
    _tree_attn("ngc_tree_attn", lib.ngc_tree_attn, cache, q, tree_k, tree_v, parent, out, n_nodes, layer_begin, layer_end, scale, ws, status)


def ngc_tree_attn_paged(cache: NgcPagedCache, q: torch.Tensor, tree_k: torch.Tensor, tree_v: torch.Tensor, parent: torch.Tensor,
                        out: torch.Tensor, n_nodes: Optional[torch.Tensor] = None, layer_begin: int = 0,
                        layer_end: Optional[int] = None, scale: Optional[float] = None, ws: Optional[torch.Tensor] = None,
                        status: Optional[torch.Tensor] = None):
    """ngc_tree_attn over a paged cache (``ws``: workspace_bytes(OP_TREE_ATTN, cache.as_contiguous_desc(), n_max=N))."""
    _tree_attn("ngc_tree_attn_paged", lib.ngc_tree_attn_paged, cache, q, tree_k, tree_v, parent, out, n_nodes, layer_begin, layer_end,
               scale, ws, status)


def ngc_verify_draft(tokens: torch.Tensor, parent: torch.Tensor, target_probs: torch.Tensor, uniforms: Optional[torch.Tensor],
                     path: torch.Tensor, n_path: torch.Tensor, next_token: torch.Tensor, draft_probs: Optional[torch.Tensor] = None,
                     n_nodes: Optional[torch.Tensor] = None, greedy: int = 0, status: Optional[torch.Tensor] = None):
    """Walk of a drafted tree: target_probs, draft_probs fp32 [B][N][vocab]; tokens, parent, path int32 [B][N]; uniforms
    fp32 [B][N] (entry 0: the final draw); n_path, next_token int32 [B]."""
    B, N, V = target_probs.shape
    what, index, probs = "ngc_verify_draft", target_probs.get_device(), (B, N, V)
    args = (_arg(what, "tokens", tokens, (B, N), _I32, index), _arg(what, "parent", parent, (B, N), _I32, index),
            _arg(what, "n_nodes", n_nodes, (B,), _I32, index), _arg(what, "target_probs", target_probs, probs, _F32, index),
            _arg(what, "draft_probs", draft_probs, probs, _F32, index), _arg(what, "uniforms", uniforms, (B, N), _F32, index), B, N, V, greedy,
            _arg(what, "path", path, (B, N), _I32, index), _arg(what, "n_path", n_path, (B,), _I32, index),
            _arg(what, "next_token", next_token, (B,), _I32, index), _arg(what, "status", status, (1,), _I32, index))
    _check(lib.ngc_verify_draft(*args, _launch_stream(what, index)), what)


def _commit_draft(what, call, cache, tree_k, tree_v, path, n_path, status):
    desc, L, B, Hkv, d, dt, index = _view(what, cache)
    N = path.shape[-1]
    rows = (L, B, Hkv, N, d)
    args = (_arg(what, "tree_k", tree_k, rows, dt, index), _arg(what, "tree_v", tree_v, rows, dt, index),
            _arg(what, "path", path, (B, N), _I32, index), _arg(what, "n_path", n_path, (B,), _I32, index), N,
            _arg(what, "status", status, (1,), _I32, index))
    _check(call(C.byref(desc), *args, _launch_stream(what, index)), what)


def ngc_commit_draft(cache: NgcCache, tree_k: torch.Tensor, tree_v: torch.Tensor, path: torch.Tensor, n_path: torch.Tensor,
                     status: Optional[torch.Tensor] = None):
    """Appends the accepted nodes' rows of tree_k / tree_v [L][B][Hkv][N][d] to the cache; lens grows by n_path."""
    _commit_draft("ngc_commit_draft", lib.ngc_commit_draft, cache, tree_k, tree_v, path, n_path, status)


def ngc_commit_draft_paged(cache: NgcPagedCache, tree_k: torch.Tensor, tree_v: torch.Tensor, path: torch.Tensor,
                           n_path: torch.Tensor, status: Optional[torch.Tensor] = None):
    _commit_draft("ngc_commit_draft_paged", lib.ngc_commit_draft_paged, cache, tree_k, tree_v, path, n_path, status)


def _fork(what, call, cache, src_of, status):
    desc, _, B, _, _, _, index = _view(what, cache)
    args = (_arg(what, "src_of", src_of, (B,), _I32, index), _arg(what, "status", status, (1,), _I32, index))
    _check(call(C.byref(desc), *args, _launch_stream(what, index)), what)


def ngc_fork_kv(cache: NgcCache, src_of: torch.Tensor, status: Optional[torch.Tensor] = None):
    """Sequence b becomes a copy of sequence src_of[b] (int32 [B]; -1 or b itself: left alone)."""
    _fork("ngc_fork_kv", lib.ngc_fork_kv, cache, src_of, status)


def ngc_fork_pages(cache: NgcPagedCache, src_of: torch.Tensor, status: Optional[torch.Tensor] = None):
    """ngc_fork_kv on a paged cache: the source's pages are copied into b's own."""
    _fork("ngc_fork_pages", lib.ngc_fork_pages, cache, src_of, status)


# ---------------------------------------------------------------- latent attention

@dataclass
class NgcLatentPool:
    """Rows of a latent cache in pages of a common pool (any page may serve any sequence) and the pool's books."""
    rows: torch.Tensor        # [L][n_pages][page][d_latent + d_rope] bf16
    page_table: torch.Tensor  # int32 [B][G][pages_cap], -1: no page
    page_used: torch.Tensor   # uint8 [G][n_pages], 0: free
    lens: torch.Tensor        # int32 [B][G]
    d_latent: int
    lists: int = LISTS_SHARED

    @property
    def L(self):
        return self.rows.shape[0]

    @property
    def B(self):
        return self.page_table.shape[0]

    @property
    def d_rope(self):
        return self.rows.shape[3] - self.d_latent


def new_latent_pool(L: int, B: int, d_latent: int, d_rope: int, n_pages: int, pages_cap: int, page: int = 64, lists: int = LISTS_SHARED,
                    device="cuda") -> NgcLatentPool:
    """An empty pool: ``n_pages`` pages in every layer for ``B`` sequences of up to ``pages_cap`` pages."""
    G = lists_G(lists, L, 1)
    return NgcLatentPool(torch.empty((L, n_pages, page, d_latent + d_rope), dtype=torch.bfloat16, device=device),
                         torch.full((B, G, pages_cap), -1, dtype=_I32, device=device), torch.zeros((G, n_pages), dtype=_U8, device=device),
                         torch.zeros((B, G), dtype=_I32, device=device), d_latent, lists)


def _pool_view(what: str, pool: NgcLatentPool):
    """Checks a pool's own tensors; (descriptor, L, B, G, d_rope, device index)."""
    rows, table, used, lens = pool.rows, pool.page_table, pool.page_used, pool.lens
    index = rows.get_device()
    L, n_pages, page, width = rows.shape
    B, G, cap = table.shape
    if G != lists_G(pool.lists, L, 1):
        raise NgcError(f"{what}: page_table {tuple(table.shape)} does not fit rows {tuple(rows.shape)} and the lists")
    if not (rows.dtype is torch.bfloat16 and table.dtype is _I32 and used.dtype is _U8 and lens.dtype is _I32 and used.shape == (G, n_pages)
            and lens.shape == (B, G) and table.get_device() == used.get_device() == lens.get_device() == index and rows.is_contiguous()
            and table.is_contiguous() and used.is_contiguous() and lens.is_contiguous()):
        for name, t, shape, dtype in (("rows", rows, rows.shape, torch.bfloat16), ("page_table", table, table.shape, _I32),
                                      ("page_used", used, (G, n_pages), _U8), ("lens", lens, (B, G), _I32)):
            _arg(what, name, t, shape, dtype, index)
    desc = LatentPoolDesc(rows.data_ptr(), table.data_ptr(), used.data_ptr(), lens.data_ptr(), L, B, pool.d_latent, width - pool.d_latent, BF16,
                          page, cap, n_pages, pool.lists)
    return desc, L, B, G, width - pool.d_latent, index


def ngc_pool_update(pool: NgcLatentPool, n_new: torch.Tensor, slots: torch.Tensor, first: torch.Tensor, kept_sorted: Optional[torch.Tensor] = None,
                    budget: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """The pool's books for the next step: eviction (``kept_sorted`` int32 [B][G][k_max], ``budget`` int32 [B], -1: none), finished
    sequences (``n_new[b]`` = -1), pages for ``n_new[b]`` tokens each, and their ``slots`` int32 [G][n_slots]; ``first`` int32 [B+1]."""
    what = "ngc_pool_update"
    desc, _, B, G, _, index = _pool_view(what, pool)
    k_max = 0 if kept_sorted is None else kept_sorted.shape[-1]
    args = (_arg(what, "kept_sorted", kept_sorted, (B, G, k_max), _I32, index), _arg(what, "budget", budget, (B,), _I32, index), k_max,
            _arg(what, "n_new", n_new, (B,), _I32, index), _arg(what, "slots", slots, (G, slots.shape[-1]), _I32, index), slots.shape[-1],
            _arg(what, "first", first, (B + 1,), _I32, index), _arg(what, "status", status, (1,), _I32, index))
    _check(lib.ngc_pool_update(C.byref(desc), *args, _launch_stream(what, index)), what)


def ngc_latent_write(pool: NgcLatentPool, slots: torch.Tensor, latent: torch.Tensor, rope: torch.Tensor, layer_begin: int = 0,
                     layer_end: Optional[int] = None, status: Optional[torch.Tensor] = None):
    """Rows (latent [L][n_slots][d_latent] | rope [L][n_slots][d_rope]) to their ``slots`` [G][n_slots]; slot -1: no row."""
    what = "ngc_latent_write"
    desc, L, _, G, d_rope, index = _pool_view(what, pool)
    n = slots.shape[-1]
    args = (_arg(what, "slots", slots, (G, n), _I32, index), n, _arg(what, "latent", latent, (L, n, pool.d_latent), torch.bfloat16, index),
            _arg(what, "rope", rope, (L, n, d_rope), torch.bfloat16, index), layer_begin, L if layer_end is None else layer_end,
            _arg(what, "status", status, (1,), _I32, index))
    _check(lib.ngc_latent_write(C.byref(desc), *args, _launch_stream(what, index)), what)


def latent_decode_workspace_bytes(pool: NgcLatentPool, H: int) -> int:
    desc = _pool_view("latent_decode_workspace_bytes", pool)[0]
    return int(lib.ngc_latent_decode_workspace_bytes(C.byref(desc), H))


def ngc_latent_decode(pool: NgcLatentPool, q_latent: torch.Tensor, q_rope: torch.Tensor, out: torch.Tensor, scale: float, layer_begin: int = 0,
                      layer_end: Optional[int] = None, ws: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """Absorbed latent attention of one token per sequence: q_latent, out [L][B][H][d_latent]; q_rope [L][B][H][d_rope].  ``scale``:
    one over the root of the EXPANDED key's width.  ``ws``: latent_decode_workspace_bytes(pool, H)."""
    what = "ngc_latent_decode"
    desc, L, B, _, d_rope, index = _pool_view(what, pool)
    H = q_latent.shape[2]
    heads = (L, B, H, pool.d_latent)
    args = (_arg(what, "q_latent", q_latent, heads, torch.bfloat16, index), _arg(what, "q_rope", q_rope, (L, B, H, d_rope), torch.bfloat16, index), H,
            layer_begin, L if layer_end is None else layer_end, scale, _arg(what, "out", out, heads, out.dtype, index), _dtype_code(out),
            None if ws is None else _arg(what, "ws", ws, ws.shape, _U8, index), 0 if ws is None else ws.numel(),
            _arg(what, "status", status, (1,), _I32, index))
    _check(lib.ngc_latent_decode(C.byref(desc), *args, _launch_stream(what, index)), what)


@dataclass
class NgcLatentSeqs:
    """Whole sequences in token-major rows: sequence b owns rows seq_off[b] .. seq_off[b+1], the first lens[b] are tokens."""
    seq_off: torch.Tensor  # int64 [B+1], device; seq_off[B] = rows
    lens: torch.Tensor     # int32 [B], device
    max_len: int           # host bound on lens


def _seqs_view(what: str, seqs: NgcLatentSeqs, q: torch.Tensor, kv: torch.Tensor):
    """Descriptor of a call on whole sequences; (descriptor, L, rows, H, d_rope, B, device index)."""
    index = q.get_device()
    L, rows, H, width = q.shape
    B = seqs.lens.shape[0]
    desc = LatentSeqsDesc(_arg(what, "seq_off", seqs.seq_off, (B + 1,), _I64, index), _arg(what, "lens", seqs.lens, (B,), _I32, index), rows, L, B, H,
                          128, 128, width - 128, BF16, seqs.max_len)
    return desc, L, rows, H, width - 128, B, index


def latent_replay_workspace_bytes(seqs: NgcLatentSeqs, q: torch.Tensor, kv: torch.Tensor, lists: int = LISTS_SHARED, n_rounds: int = 1,
                                  backward: bool = False) -> int:
    """Workspace of ngc_latent_replay_attn (or its gradient) for queries and keys of these shapes; ``n_rounds`` 0: causal."""
    desc = _seqs_view("latent_replay_workspace_bytes", seqs, q, kv)[0]
    return int(lib.ngc_latent_replay_workspace_bytes(C.byref(desc), lists, n_rounds, int(backward)))


def _replay_args(what, seqs, q, kv, k_rope, out, lse, alive_pos, alive_count, total_before, lists, scale):
    desc, L, rows, H, d_rope, B, index = _seqs_view(what, seqs, q, kv)
    bf16, G = torch.bfloat16, lists_G(lists, L, 1)
    R, kt = (0, 0) if alive_pos is None else (alive_pos.shape[0], alive_pos.shape[-1])
    args = (_arg(what, "q", q, (L, rows, H, 128 + d_rope), bf16, index), _arg(what, "kv", kv, (L, rows, H, 256), bf16, index),
            _arg(what, "k_rope", k_rope, (L, rows, d_rope), bf16, index), _arg(what, "alive_pos", alive_pos, (R, B, G, kt), _I32, index),
            _arg(what, "alive_count", alive_count, (R, B, G), _I32, index), _arg(what, "total_before", total_before, (R, B), _I32, index), R, kt,
            lists, (128 + d_rope) ** -0.5 if scale is None else scale, _arg(what, "out", out, (L, rows, H, 128), out.dtype, index),
            _dtype_code(out), _arg(what, "lse", lse, (L, H, rows), _F32, index))
    return desc, args, index


def _ws(what, ws, index):
    return (None, 0) if ws is None else (_arg(what, "ws", ws, ws.shape, _U8, index), ws.numel())


def ngc_latent_replay_attn(seqs: NgcLatentSeqs, q: torch.Tensor, kv: torch.Tensor, k_rope: torch.Tensor, out: torch.Tensor,
                           lse: Optional[torch.Tensor] = None, alive_pos: Optional[torch.Tensor] = None, alive_count: Optional[torch.Tensor] = None,
                           total_before: Optional[torch.Tensor] = None, lists: int = LISTS_SHARED, scale: Optional[float] = None,
                           ws: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """Expanded latent attention of whole sequences under their history of evictions (none: causal).  q [L][rows][H][128 + d_rope],
    kv [L][rows][H][128 + 128], k_rope [L][rows][d_rope] (shared by the heads), out [L][rows][H][128], lse fp32 [L][H][rows]."""
    what = "ngc_latent_replay_attn"
    desc, args, index = _replay_args(what, seqs, q, kv, k_rope, out, lse, alive_pos, alive_count, total_before, lists, scale)
    rc = lib.ngc_latent_replay_attn(C.byref(desc), *args, *_ws(what, ws, index), _arg(what, "status", status, (1,), _I32, index),
                                    _launch_stream(what, index))
    _check(rc, what)


def ngc_latent_replay_attn_backward(seqs: NgcLatentSeqs, q: torch.Tensor, kv: torch.Tensor, k_rope: torch.Tensor, out: torch.Tensor, lse: torch.Tensor,
                                    grad_out: torch.Tensor, grad_q: torch.Tensor, grad_kv: torch.Tensor, grad_k_rope: torch.Tensor,
                                    alive_pos: Optional[torch.Tensor] = None, alive_count: Optional[torch.Tensor] = None,
                                    total_before: Optional[torch.Tensor] = None, lists: int = LISTS_SHARED, scale: Optional[float] = None,
                                    ws: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """Gradient of ngc_latent_replay_attn from grad_out (bf16, shape of out): grad_q, grad_kv, grad_k_rope in shape and type of q, kv,
    k_rope; ``out`` and ``lse`` are the forward call's."""
    what = "ngc_latent_replay_attn_backward"
    desc, args, index = _replay_args(what, seqs, q, kv, k_rope, out, lse, alive_pos, alive_count, total_before, lists, scale)
    bf16 = torch.bfloat16
    grads = (_arg(what, "grad_out", grad_out, out.shape, bf16, index), _arg(what, "grad_q", grad_q, q.shape, bf16, index),
             _arg(what, "grad_kv", grad_kv, kv.shape, bf16, index), _arg(what, "grad_k_rope", grad_k_rope, k_rope.shape, bf16, index))
    rc = lib.ngc_latent_replay_attn_backward(C.byref(desc), *args, *grads, *_ws(what, ws, index), _arg(what, "status", status, (1,), _I32, index),
                                             _launch_stream(what, index))
    _check(rc, what)


REPLAY_ATTN_AUTO, REPLAY_ATTN_MMA_SYNC, REPLAY_ATTN_TCGEN05 = 0, 1, 2


def ngc_replay_attn(cache: NgcCache, q: torch.Tensor, out: torch.Tensor, alive_pos: Optional[torch.Tensor] = None,
                    alive_count: Optional[torch.Tensor] = None, total_before: Optional[torch.Tensor] = None,
                    lists: int = LISTS_SHARED, scale: Optional[float] = None, status: Optional[torch.Tensor] = None,
                    variant: Optional[int] = None):
    """q, out [L][B][Hq][t_max][d]; cache holds the full sequences (lens = total tokens).  ``variant`` picks the device
    path (REPLAY_ATTN_*) through ngc_replay_attn_variant; None calls ngc_replay_attn itself."""
    t_max = q.shape[3]
    if scale is None:
        scale = 1.0 / (cache.d ** 0.5)
    n_rounds = 0 if alive_pos is None else alive_pos.shape[0]
    kt_max = 0 if alive_pos is None else alive_pos.shape[3]
    d = cache.desc()
    if variant is None:
        rc = lib.ngc_replay_attn(C.byref(d), _ptr(q), t_max, _ptr(alive_pos), _ptr(alive_count), _ptr(total_before), n_rounds, kt_max,
                                 lists, scale, _ptr(out), _dtype_code(out), _ptr(status), _stream())
    else:
        rc = lib.ngc_replay_attn_variant(C.byref(d), _ptr(q), t_max, _ptr(alive_pos), _ptr(alive_count), _ptr(total_before), n_rounds,
                                         kt_max, lists, scale, _ptr(out), _dtype_code(out), variant, _ptr(status), _stream())
    _check(rc, "ngc_replay_attn")


def ngc_selftest_bounded_wait(limit_us: int, status: torch.Tensor, waited_ns: Optional[torch.Tensor] = None):
    """One warp waits at most ``limit_us`` microseconds on a barrier that never completes; ``status`` becomes the
    timeout code and the call returns normally (diagnostic of the kernels' bounded waits)."""
    rc = lib.ngc_selftest_bounded_wait(limit_us, _ptr(status), _ptr(waited_ns), _stream())
    _check(rc, "ngc_selftest_bounded_wait")
