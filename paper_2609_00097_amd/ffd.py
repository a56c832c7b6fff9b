"""Thin Python binding of libffd.so (ctypes). Argument marshalling only: every step of the decode
path runs in the library's HIP kernels. PyTorch supplies device memory and the current stream.

If the library is not built or cannot be loaded, every call raises ``FfdLibraryError``; there is
no CPU fallback.
"""
from __future__ import annotations

import ctypes
import math
import os
import struct

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libffd.so")

HEAD_DIM = 128
BLOCK = 64
MAX_SPLITS = 1024
THUMB_BITS = (2, 4, 8)      # thumbnail depths: 2+8 (the method), 4+8 and 8+8 (App. C)
STATUS = {0: "FFD_OK", 1: "FFD_ERR_INVALID_ARGUMENT", 2: "FFD_ERR_UNSUPPORTED",
          3: "FFD_ERR_WORKSPACE_TOO_SMALL", 4: "FFD_ERR_HIP", 5: "FFD_ERR_SCRATCH_TOO_SMALL"}
NOALLOC_SCRATCH_BYTES = 16 << 20     # FFD_NOALLOC_SCRATCH_BYTES

EXPORTS = ("ffd_quantize_keys", "ffd_append_kv", "ffd_decode_attention", "ffd_decode_attention_ex",
           "ffd_decode_attention_noalloc", "ffd_dense_decode_attention", "ffd_write_kv8", "ffd_read_kv8",
           "ffd_kv8_decode_attention", "ffd_kv8_workspace_bytes", "ffd_shared_prefix_decode_attention",
           "ffd_shared_prefix_workspace_bytes", "ffd_write_paged", "ffd_paged_attention", "ffd_paged_workspace_bytes",
           "ffd_paged_attention_weights", "ffd_evict_paged", "ffd_resolve_splits", "ffd_fused_splits", "ffd_select_kernels", "ffd_dense_resolve_splits",
           "ffd_workspace_bytes", "ffd_dense_workspace_bytes", "ffd_status_string")


class FfdLibraryError(RuntimeError):
    """libffd.so is missing or failed to load."""


class FfdError(RuntimeError):
    """A library call returned an error status."""

    def __init__(self, fn: str, status: int, detail: str):
        super().__init__(f"{fn} -> {detail} ({status})")
        self.status = status


_lib = None
P, I, F, SZ = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
PSEUDO_MAX = {"thumbnail": 0, "refined": 1}     # FFD_PSEUDO_MAX_THUMBNAIL, FFD_PSEUDO_MAX_REFINED


KERNELS = {"auto": 0, "fused": 1, "split": 2}     # FFD_KERNELS_AUTO, _FUSED, _SPLIT


class DecodeExtras(ctypes.Structure):
    """``ffd_decode_extras``: stage events, the pseudo-max output, the pseudo-max source, the
    fixed-budget (top-k) selection and the top-delta kernels."""
    _fields_ = [("stage_events", P), ("m_tilde", P), ("pseudo_max", I), ("top_k", I), ("kernels", I)]


class KvCache(ctypes.Structure):
    """``ffd_kv``: a cache's keys, their absmaxes, its values and theirs (absmaxes None: bf16)."""
    _fields_ = [("k", P), ("k_absmax", P), ("v", P), ("v_absmax", P)]


class PagedCache(ctypes.Structure):
    """``ffd_paged``: pages and the sequences' table of them."""
    _fields_ = [("pages", KvCache), ("page_table", P), ("num_pages", I), ("page", I), ("max_pages", I)]


class Rotation(ctypes.Structure):
    """``ffd_rotation``: the norms' weights and the table of the rotation."""
    _fields_ = [("q_weight", P), ("k_weight", P), ("eps", F), ("table", P), ("rows", I), ("dims", I), ("interleaved", I), ("positions", P)]


class ScoreRules(ctypes.Structure):
    """``ffd_score_rules``: what a score is, and which tokens a query sees."""
    _fields_ = [("softcap", F), ("window", I), ("slopes", P), ("prefix_lens", P)]


def lib() -> ctypes.CDLL:
    """Load libffd.so (once) and declare its signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FfdLibraryError(f"{LIB_PATH} is not built; run paper_2609_00097_amd/build.py")
    try:
        so = ctypes.CDLL(LIB_PATH)
    except OSError as e:
        raise FfdLibraryError(f"cannot load {LIB_PATH}: {e}") from e
    so.ffd_quantize_keys.argtypes = [P, P, P, P, I, I, I, I, I, I, I, P]
    so.ffd_append_kv.argtypes = [P, P, P, P, P, P, P, P, I, I, I, I, I, P]
    so.ffd_decode_attention.argtypes = [P, P, P, P, P, P, I, I, I, I, I, I, I, F, I, I, I, F,
                                        P, P, P, P, SZ, P]
    so.ffd_decode_attention_ex.argtypes = so.ffd_decode_attention.argtypes + [ctypes.POINTER(DecodeExtras)]
    so.ffd_decode_attention_noalloc.argtypes = [P, P, P, P, P, P, I, I, I, I, I, I, I, F, I, I, I, F,
                                                P, P, P, P]
    so.ffd_dense_decode_attention.argtypes = [P, P, P, P, I, I, I, I, I, I, F, P, P, P, SZ, P]
    KV, STRIDES = ctypes.POINTER(KvCache), ctypes.POINTER(ctypes.c_int64)
    so.ffd_write_kv8.argtypes = [P, P, STRIDES, STRIDES, KV, P, P, I, I, I, I, I, P]
    so.ffd_read_kv8.argtypes = [KV, P, P, P, I, I, I, I, I, I, P]
    so.ffd_kv8_decode_attention.argtypes = [P, KV, P, I, I, I, I, I, I, F, P, P, P, SZ, P]
    so.ffd_shared_prefix_decode_attention.argtypes = [P, KV, P, I, KV, P, I, I, I, I, I, I, F, P, P, P, SZ, P]
    so.ffd_shared_prefix_workspace_bytes.argtypes = [I, I, I, I, I, I, I]
    so.ffd_shared_prefix_workspace_bytes.restype = SZ
    # (structures as addresses: the binding packs them, others pass them by ctypes.byref)
    so.ffd_write_paged.argtypes = [P, P, P, P, P, P, P, P, P, P, P, I, I, I, I, I, P]
    so.ffd_paged_attention.argtypes = [P, P, P, P, P, I, I, I, I, I, F, P, P, P, SZ, P]
    so.ffd_paged_workspace_bytes.argtypes = [I, I, I, I, I]
    so.ffd_paged_workspace_bytes.restype = SZ
    so.ffd_paged_attention_weights.argtypes = [P, P, P, P, P, P, I, I, I, I, I, F, I, P, P, P]
    so.ffd_evict_paged.argtypes = [P, P, I, P, P, I, I, I, I, I, P, P, P, P]
    so.ffd_resolve_splits.argtypes = [I, I, I, I]
    so.ffd_fused_splits.argtypes = [I, I, I, I]
    so.ffd_select_kernels.argtypes = [I, I, I, I]
    so.ffd_dense_resolve_splits.argtypes = [I, I, I, I]
    for name in ("ffd_workspace_bytes", "ffd_dense_workspace_bytes", "ffd_kv8_workspace_bytes"):
        getattr(so, name).argtypes = [I, I, I, I, I, I]
        getattr(so, name).restype = SZ
    so.ffd_status_string.argtypes = [I]
    so.ffd_status_string.restype = ctypes.c_char_p
    for name in ("ffd_quantize_keys", "ffd_append_kv", "ffd_decode_attention", "ffd_decode_attention_ex",
                 "ffd_decode_attention_noalloc", "ffd_dense_decode_attention", "ffd_write_kv8", "ffd_read_kv8",
                 "ffd_kv8_decode_attention", "ffd_shared_prefix_decode_attention", "ffd_write_paged", "ffd_paged_attention",
                 "ffd_paged_attention_weights", "ffd_evict_paged", "ffd_resolve_splits", "ffd_fused_splits", "ffd_select_kernels", "ffd_dense_resolve_splits"):
        getattr(so, name).restype = I
    _lib = so
    return so


def _check(fn: str, st: int) -> None:
    if st != 0:
        raise FfdError(fn, st, lib().ffd_status_string(st).decode())


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


# A call's checks, allocations and argument conversion cost more than its kernels at short contexts, so
# each is the cheapest form that keeps its meaning (decode_attention with its defaults: 10 us of host time a
# call with one launch, 18 us in the plain form): the usual tensor passes one expression, and only one that
# does not goes through the checks that name what is wrong.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(t) -> int:
    """The current stream of the tensor's device."""
    if _raw_stream is not None:
        return _raw_stream(t.get_device())
    return torch.cuda.current_stream(t.device).cuda_stream


def _need(t, name, dtype, shape=None):
    if (type(t) is torch.Tensor and t.is_cuda and t.dtype is dtype and t.is_contiguous()
            and (shape is None or t.shape == shape)):
        return
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def resolve_splits(B: int, Hkv: int, Lcap: int, num_splits: int = 0) -> int:
    """The split count that sizes the workspace for this ``num_splits`` (0 = automatic); a given one is also
    the split kernels' refinement workgroups per KV group (automatic: see ``ffd_resolve_splits`` in ffd.h)."""
    return lib().ffd_resolve_splits(B, Hkv, Lcap, num_splits)


def fused_splits(B: int, Hkv: int, Lcap: int, num_splits: int = 0) -> int:
    """Workgroups per KV group of the fused top-delta kernel for this ``num_splits`` (in a batch of 2 to 64
    sequences, which are given workgroups by their lengths, on average at most)."""
    return lib().ffd_fused_splits(B, Hkv, Lcap, num_splits)


def select_kernels(B: int, Hkv: int, Lcap: int, num_splits: int = 0) -> str:
    """The top-delta kernels the automatic choice uses: ``"fused"`` or ``"split"``."""
    k = lib().ffd_select_kernels(B, Hkv, Lcap, num_splits)
    return {1: "fused", 2: "split"}[k]


def dense_resolve_splits(B: int, Hkv: int, Lcap: int, num_splits: int = 0) -> int:
    """Splits a dense call with this ``num_splits`` uses (0 = automatic)."""
    return lib().ffd_dense_resolve_splits(B, Hkv, Lcap, num_splits)


def workspace_bytes(B: int, Hq: int, Hkv: int, Lcap: int, num_splits: int = 0,
                    dense: bool = False) -> int:
    """Bytes for ``decode_attention`` (enough for both entry points), or for the dense one only."""
    fn = lib().ffd_dense_workspace_bytes if dense else lib().ffd_workspace_bytes
    return fn(B, Hq, Hkv, Lcap, HEAD_DIM, num_splits)


def new_workspace(B: int, Hq: int, Hkv: int, Lcap: int, num_splits: int = 0, device="cuda",
                  dense: bool = False):
    """A workspace (one per stream): for ``decode_attention`` and the dense entry point alike, or,
    with ``dense=True``, the smaller one the dense entry point needs."""
    return torch.empty(max(workspace_bytes(B, Hq, Hkv, Lcap, num_splits, dense), 16),
                       dtype=torch.uint8, device=device)


def quantized_shapes(B: int, Hkv: int, Lcap: int, bits: int = 2):
    """Shapes of (codes int32, absmax bf16, resid int8) for a cache of capacity Lcap with a
    ``bits``-bit thumbnail."""
    return ((B, Hkv, Lcap // 64, bits, 64, 4), (B, Hkv, Lcap // 64, 16, 4),
            (B, Hkv, Lcap // 16, 2, 64, 16))


def thumb_bits(codes: torch.Tensor) -> int:
    """The thumbnail depth of a codes tensor ``[B, Hkv, Lcap/64, b, 64, 4]``."""
    shape = codes.shape
    bits = shape[3] if len(shape) == 6 and shape[4] == 64 and shape[5] == 4 else 0
    if bits not in THUMB_BITS:
        raise ValueError(f"codes must be [B, Hkv, Lcap/64, b, 64, 4] with b in {THUMB_BITS}, "
                         f"got {tuple(codes.shape)}")
    return bits


def empty_quantized(B: int, Hkv: int, Lcap: int, device, bits: int = 2):
    sc, sa, sr = quantized_shapes(B, Hkv, Lcap, bits)
    return (torch.empty(sc, dtype=torch.int32, device=device),
            torch.empty(sa, dtype=torch.bfloat16, device=device),
            torch.empty(sr, dtype=torch.int8, device=device))


def _need_quantized(quantized, B, Hkv, Lcap) -> int:
    codes, absmax, resid = quantized
    bits = thumb_bits(codes)
    sc, sa, sr = quantized_shapes(B, Hkv, Lcap, bits)
    _need(codes, "codes", torch.int32, sc)
    _need(absmax, "absmax", torch.bfloat16, sa)
    _need(resid, "resid", torch.int8, sr)
    return bits


def quantize_keys(k: torch.Tensor, t_begin: int = 0, t_end: int | None = None, out=None,
                  bits: int = 2):
    """Split bf16 keys ``[B, Hkv, Lcap, 128]`` into (codes, absmax, resid) for ``[t_begin, t_end)``
    with a ``bits``-bit thumbnail (2, 4 or 8; taken from ``out``'s codes shape when given)."""
    if k.dim() != 4:
        raise ValueError("k must be [B, Hkv, Lcap, 128]")
    B, Hkv, Lcap, D = k.shape
    _need(k, "k", torch.bfloat16)
    t_end = Lcap if t_end is None else t_end
    if out is None:
        if bits not in THUMB_BITS:
            raise ValueError(f"bits must be one of {THUMB_BITS}")
        out = empty_quantized(B, Hkv, Lcap, k.device, bits)
    bits = _need_quantized(out, B, Hkv, Lcap)
    codes, absmax, resid = out
    _check("ffd_quantize_keys", lib().ffd_quantize_keys(
        _ptr(k), _ptr(codes), _ptr(absmax), _ptr(resid), B, Hkv, Lcap, D, bits, t_begin, t_end,
        _stream(k)))
    return codes, absmax, resid


def append_kv(k_new, v_new, quantized, seq_lens, *, k_cache=None, v_cache=None):
    """Append one token per sequence at position ``seq_lens[b]`` (device-side) to the quantized key
    cache ``(codes, absmax, resid)`` and, when given, the bf16 caches ``[B, Hkv, Lcap, 128]``; then
    ``seq_lens[b] += 1`` for every sequence below capacity. ``k_new``/``v_new``: bf16 ``[B, Hkv, 128]``."""
    codes, absmax, resid = quantized
    B, Hkv, D = k_new.shape
    Lcap = codes.shape[2] * 64
    _need(k_new, "k_new", torch.bfloat16)
    _need(v_new, "v_new", torch.bfloat16, (B, Hkv, D))
    _need(seq_lens, "seq_lens", torch.int32, (B,))
    bits = _need_quantized(quantized, B, Hkv, Lcap)
    for t, nm in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        if t is not None:
            _need(t, nm, torch.bfloat16, (B, Hkv, Lcap, D))
    _check("ffd_append_kv", lib().ffd_append_kv(
        _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(codes), _ptr(absmax), _ptr(resid),
        _ptr(seq_lens), B, Hkv, Lcap, D, bits, _stream(k_new)))


def _attn_outputs(q, B, Hq, Lcap, want_lse, want_mask, out, lse, mask):
    plain = type(q) is torch.Tensor and q.shape[-1] == HEAD_DIM     # then q, checked before, has out's shape
    if out is None:
        out = torch.empty_like(q) if plain else torch.empty((B, Hq, HEAD_DIM), dtype=torch.bfloat16, device=q.device)
    if want_lse and lse is None:
        lse = (q.new_empty((B, Hq), dtype=torch.float32) if plain else
               torch.empty((B, Hq), dtype=torch.float32, device=q.device))
    if want_mask and mask is None:
        mask = torch.empty((B, Hq, Lcap // BLOCK), dtype=torch.uint8, device=q.device)
    return out, lse, mask


def decode_attention(q, codes, absmax, resid, v, seq_lens, *, delta: float, n_sink: int = 64,
                     n_local: int = 256, num_splits: int = 0, softmax_scale: float = 0.0,
                     return_lse: bool = True, return_mask: bool = False, workspace=None,
                     out=None, lse=None, mask=None, stage_events=None, m_tilde=None,
                     pseudo_max: str = "thumbnail", top_k: int = 0, kernels: str = "auto"):
    """FFD decode attention. Returns ``(out, lse, mask)`` (lse/mask None unless requested).
    The thumbnail depth is that of ``codes`` (its last dimension is 4 words per bit).

    ``stage_events``: optional four ``torch.cuda.Event`` objects, already recorded once (so that
    they exist), which the library records before the scan kernel, after it, after the refinement
    kernel and after the merge. ``m_tilde``: optional float32 ``[B, Hq]`` receiving each head's
    pseudo-max. ``pseudo_max``: ``"thumbnail"`` (default) or ``"refined"``, the scores of the window
    tokens the pseudo-max is taken over. ``top_k > 0`` replaces the top-delta rule by the fixed
    budget of ``top_k`` blocks per head (largest thumbnail block scores, ties in block order); delta
    and the windows are then unused and ``m_tilde`` must be None. ``kernels``: ``"auto"``,
    ``"fused"`` or ``"split"`` (top-delta's kernels; see ``FFD_KERNELS_*`` in ffd.h)."""
    B, Hq, D = q.shape
    Hkv, Lcap = v.shape[1], v.shape[2]
    _need(q, "q", torch.bfloat16)
    _need(v, "v", torch.bfloat16, (B, Hkv, Lcap, D))
    _need(seq_lens, "seq_lens", torch.int32, (B,))
    bits = _need_quantized((codes, absmax, resid), B, Hkv, Lcap)
    out, lse, mask = _attn_outputs(q, B, Hq, Lcap, return_lse or lse is not None,
                                   return_mask or mask is not None, out, lse, mask)
    if workspace is None:
        workspace = new_workspace(B, Hq, Hkv, Lcap, num_splits, q.device)
    if pseudo_max not in PSEUDO_MAX:
        raise ValueError(f"pseudo_max must be one of {tuple(PSEUDO_MAX)}")
    if m_tilde is not None:
        _need(m_tilde, "m_tilde", torch.float32, (B, Hq))
    ev = None
    if stage_events is not None:
        if len(stage_events) != 4 or any(e.cuda_event == 0 for e in stage_events):
            raise ValueError("stage_events must be four recorded torch.cuda.Event objects")
        ev = (ctypes.c_void_p * 4)(*[e.cuda_event for e in stage_events])
    if kernels not in KERNELS:
        raise ValueError(f"kernels must be one of {tuple(KERNELS)}")
    top_k = int(top_k)
    extras = None               # the library's defaults
    if ev is not None or m_tilde is not None or pseudo_max != "thumbnail" or top_k or kernels != "auto":
        extras = ctypes.byref(DecodeExtras(ctypes.cast(ev, P) if ev is not None else None, _ptr(m_tilde),
                                           PSEUDO_MAX[pseudo_max], top_k, KERNELS[kernels]))
    _check("ffd_decode_attention", lib().ffd_decode_attention_ex(
        _ptr(q), _ptr(codes), _ptr(absmax), _ptr(resid), _ptr(v), _ptr(seq_lens), B, Hq, Hkv, Lcap,
        D, bits, BLOCK, float(delta), n_sink, n_local, num_splits, float(softmax_scale), _ptr(out),
        _ptr(lse), _ptr(mask), _ptr(workspace), workspace.numel() * workspace.element_size(),
        _stream(q), extras))
    return out, lse, mask


def decode_attention_noalloc(q, codes, absmax, resid, v, seq_lens, *, delta: float, n_sink: int = 64,
                             n_local: int = 256, num_splits: int = 0, softmax_scale: float = 0.0,
                             out=None, lse=None, mask=None):
    """``decode_attention`` through ``ffd_decode_attention_noalloc``: the library's fixed device
    scratch stands in for the workspace (no device allocation by the library; calls on one device
    must not overlap in time). ``out`` (and ``lse``/``mask`` when wanted) should be passed in by
    callers that cannot allocate; otherwise they are allocated here. Returns ``(out, lse, mask)``."""
    B, Hq, D = q.shape
    Hkv, Lcap = v.shape[1], v.shape[2]
    _need(q, "q", torch.bfloat16)
    _need(v, "v", torch.bfloat16, (B, Hkv, Lcap, D))
    _need(seq_lens, "seq_lens", torch.int32, (B,))
    bits = _need_quantized((codes, absmax, resid), B, Hkv, Lcap)
    if out is None:
        out = torch.empty((B, Hq, HEAD_DIM), dtype=torch.bfloat16, device=q.device)
    _need(out, "out", torch.bfloat16, (B, Hq, D))
    if lse is not None:
        _need(lse, "lse", torch.float32, (B, Hq))
    if mask is not None:
        _need(mask, "mask", torch.uint8, (B, Hq, Lcap // BLOCK))
    _check("ffd_decode_attention_noalloc", lib().ffd_decode_attention_noalloc(
        _ptr(q), _ptr(codes), _ptr(absmax), _ptr(resid), _ptr(v), _ptr(seq_lens), B, Hq, Hkv, Lcap,
        D, bits, BLOCK, float(delta), n_sink, n_local, num_splits, float(softmax_scale), _ptr(out),
        _ptr(lse), _ptr(mask), _stream(q)))
    return out, lse, mask


def dense_decode_attention(q, k, v, seq_lens, *, num_splits: int = 0, softmax_scale: float = 0.0,
                           return_lse: bool = True, workspace=None, out=None, lse=None):
    """Exact dense decode attention. Returns ``(out, lse)``."""
    B, Hq, D = q.shape
    Hkv, Lcap = k.shape[1], k.shape[2]
    _need(q, "q", torch.bfloat16)
    _need(k, "k", torch.bfloat16, (B, Hkv, Lcap, D))
    _need(v, "v", torch.bfloat16, (B, Hkv, Lcap, D))
    _need(seq_lens, "seq_lens", torch.int32, (B,))
    out, lse, _ = _attn_outputs(q, B, Hq, Lcap, return_lse or lse is not None, False, out, lse, None)
    if workspace is None:
        workspace = new_workspace(B, Hq, Hkv, Lcap, num_splits, q.device, dense=True)
    _check("ffd_dense_decode_attention", lib().ffd_dense_decode_attention(
        _ptr(q), _ptr(k), _ptr(v), _ptr(seq_lens), B, Hq, Hkv, Lcap, D, num_splits,
        float(softmax_scale), _ptr(out), _ptr(lse), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(q)))
    return out, lse


# ---- 8-bit caches and shared prefixes -----------------------------------------------------------------
# An 8-bit cache is (k_codes, k_absmax, v_codes, v_absmax): codes int8 [B, Hkv, Lcap, 128], absmaxes bf16
# [B, Hkv, Lcap]; a bf16 cache (k, v). The calls below run on the device of their tensors, whatever device is
# current, and require all of them there.

def kv8_shapes(B: int, Hkv: int, Lcap: int):
    """Shapes of (k_codes, k_absmax, v_codes, v_absmax) of an 8-bit cache of capacity Lcap."""
    return ((B, Hkv, Lcap, HEAD_DIM), (B, Hkv, Lcap)) * 2


def empty_kv8(B: int, Hkv: int, Lcap: int, device="cuda"):
    """An 8-bit cache with uninitialised contents: (k_codes, k_absmax, v_codes, v_absmax)."""
    return tuple(torch.empty(s, dtype=torch.int8 if len(s) == 4 else torch.bfloat16, device=device)
                 for s in kv8_shapes(B, Hkv, Lcap))


def _need_on(device, t, name, dtype, shape, part=""):
    if (type(t) is torch.Tensor and t.dtype is dtype and t.shape == shape and t.get_device() == device >= 0
            and t.is_contiguous()):
        return                                           # the usual tensor, cheaply; see _need
    name += part
    _need(t, name, dtype, shape)
    if t.get_device() != device:
        raise ValueError(f"{name} must be on cuda:{device}, got {t.device}")


def _launch(name, fn, device, *args):
    """The library call ``fn`` on this device (its launches go to the current one) and on its current stream."""
    stream = _raw_stream(device) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream
    if torch._C._cuda_getDevice() == device:
        st = fn(*args, stream)
    else:
        with torch.cuda.device(device):
            st = fn(*args, stream)
    if st != 0:
        _check(name, st)


def _cache_dims(cache, name, bf16=False):
    """(B, Hkv, Lcap) of a cache, from its keys."""
    if not isinstance(cache, (tuple, list)) or len(cache) not in ((2, 4) if bf16 else (4,)):
        raise ValueError(f"{name} must be (k_codes, k_absmax, v_codes, v_absmax)" + (" or (k, v)" if bf16 else ""))
    if not isinstance(cache[0], torch.Tensor) or cache[0].dim() != 4:
        raise ValueError(f"{name}'s keys must be [B, Hkv, Lcap, {HEAD_DIM}]")
    return tuple(cache[0].shape[:3])


def _kv_cache(cache, name, device, rows):
    """``ffd_kv`` of a cache whose tensors are as they have to be; rows = [B, Hkv, Lcap, 128]."""
    if len(cache) == 2:
        k, v = cache
        _need_on(device, k, name, torch.bfloat16, rows, " k")
        _need_on(device, v, name, torch.bfloat16, rows, " v")
        return KvCache(k.data_ptr(), None, v.data_ptr(), None)
    k, k_absmax, v, v_absmax = cache
    vectors = rows[:3]
    if not (type(k) is type(k_absmax) is type(v) is type(v_absmax) is torch.Tensor       # the usual tensors, cheaply
            and k.dtype is torch.int8 and v.dtype is torch.int8
            and k_absmax.dtype is torch.bfloat16 and v_absmax.dtype is torch.bfloat16
            and k.shape == rows and v.shape == rows and k_absmax.shape == vectors and v_absmax.shape == vectors
            and k.get_device() == k_absmax.get_device() == v.get_device() == v_absmax.get_device() == device >= 0
            and k.is_contiguous() and v.is_contiguous() and k_absmax.is_contiguous() and v_absmax.is_contiguous()):
        _need_on(device, k, name, torch.int8, rows, " k_codes")
        _need_on(device, k_absmax, name, torch.bfloat16, vectors, " k_absmax")
        _need_on(device, v, name, torch.int8, rows, " v_codes")
        _need_on(device, v_absmax, name, torch.bfloat16, vectors, " v_absmax")
    return KvCache(k.data_ptr(), k_absmax.data_ptr(), v.data_ptr(), v_absmax.data_ptr())


_Strides = ctypes.c_int64 * 3


def _strided(t, name, device, shape):
    """The three strides, in elements, of ``t`` as [B, T, Hkv, 128]; None where it is contiguous. Only the dims of a vector
    need to be."""
    if (type(t) is torch.Tensor and t.dtype is torch.bfloat16 and t.shape == shape and t.get_device() == device >= 0
            and t.is_contiguous()):
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype != torch.bfloat16 or t.get_device() != device:
        raise ValueError(f"{name} must be torch.bfloat16 on cuda:{device}, got {t.dtype} on {t.device}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")
    strides = t.stride()
    if strides[-1] != 1:
        raise ValueError(f"{name}'s last dimension must be contiguous")
    # the stride of a dimension of one is never used, and may be anything
    if len(shape) == 3:
        return _Strides(strides[0] if shape[0] > 1 else 0, 0, strides[1] if shape[1] > 1 else 0)
    return _Strides(strides[0] if shape[0] > 1 else 0, strides[1] if shape[1] > 1 else 0, strides[2] if shape[2] > 1 else 0)


def write_kv8(k_new, v_new, cache, start, *, counts=None):
    """Quantize new tokens into the 8-bit ``cache``: token t < ``counts[b]`` of sequence b goes to position
    ``start[b] + t`` (device-side; positions outside the capacity are not written, nor is anything else of the cache).
    ``k_new``/``v_new``: bf16 ``[B, T, Hkv, 128]``, or ``[B, Hkv, 128]`` for one token each, with any strides (slices
    of a projection's output are taken as they are) that are multiples of 8 elements. ``start``, ``counts``: int32
    ``[B]``; without ``counts`` all T. Lengths are the caller's to advance."""
    B, Hkv, Lcap = _cache_dims(cache, "cache")
    device = cache[0].get_device()
    kv = _kv_cache(cache, "cache", device, (B, Hkv, Lcap, HEAD_DIM))
    dims = k_new.dim() if isinstance(k_new, torch.Tensor) else 0
    T = k_new.shape[1] if dims == 4 else 1
    shape = (B, Hkv, HEAD_DIM) if dims == 3 else (B, T, Hkv, HEAD_DIM)
    k_strides, v_strides = _strided(k_new, "k_new", device, shape), _strided(v_new, "v_new", device, shape)
    _need_on(device, start, "start", torch.int32, (B,))
    if counts is not None:
        _need_on(device, counts, "counts", torch.int32, (B,))
    _launch("ffd_write_kv8", lib().ffd_write_kv8, device, k_new.data_ptr(), v_new.data_ptr(), k_strides, v_strides,
            ctypes.byref(kv), start.data_ptr(), _ptr(counts), B, T, Hkv, Lcap, HEAD_DIM)


def read_kv8(cache, t_begin: int = 0, t_end: int | None = None, *, seq_lens=None, out=None):
    """Tokens ``[t_begin, t_end)`` of an 8-bit cache as bf16 ``(k, v)``, each ``[B, Hkv, t_end - t_begin, 128]``;
    with ``seq_lens`` (int32 ``[B]``) the rows of tokens at or behind a sequence's length are zeros."""
    B, Hkv, Lcap = _cache_dims(cache, "cache")
    device = cache[0].get_device()
    kv = _kv_cache(cache, "cache", device, (B, Hkv, Lcap, HEAD_DIM))
    t_end = Lcap if t_end is None else t_end
    if not 0 <= t_begin <= t_end <= Lcap:
        raise ValueError(f"need 0 <= t_begin <= t_end <= {Lcap}, got {t_begin}, {t_end}")
    shape = (B, Hkv, t_end - t_begin, HEAD_DIM)
    if seq_lens is not None:
        _need_on(device, seq_lens, "seq_lens", torch.int32, (B,))
    if out is None:
        k, v = cache[1].new_empty(shape), cache[1].new_empty(shape)
    else:
        k, v = out
        _need_on(device, k, "out k", torch.bfloat16, shape)
        _need_on(device, v, "out v", torch.bfloat16, shape)
    _launch("ffd_read_kv8", lib().ffd_read_kv8, device, ctypes.byref(kv), _ptr(seq_lens), k.data_ptr(), v.data_ptr(), B,
            Hkv, Lcap, HEAD_DIM, t_begin, t_end)
    return k, v


def _dense_arguments(q, cache, name, seq_lens, return_lse, out, lse, bf16):
    """Checks shared by the attentions below; (device, B, Hq, Hkv, Lcap, cache, out, lse)."""
    B, Hkv, Lcap = _cache_dims(cache, name, bf16)
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError(f"q must be [B, Hq, {HEAD_DIM}]")
    Hq, device = q.shape[1], q.get_device()
    _need_on(device, q, "q", torch.bfloat16, (B, Hq, HEAD_DIM))
    kv = _kv_cache(cache, name, device, (B, Hkv, Lcap, HEAD_DIM))
    _need_on(device, seq_lens, "seq_lens", torch.int32, (B,))
    if out is None:
        out = torch.empty_like(q)
    else:
        _need_on(device, out, "out", torch.bfloat16, (B, Hq, HEAD_DIM))
    if lse is not None:
        _need_on(device, lse, "lse", torch.float32, (B, Hq))
    elif return_lse:
        lse = q.new_empty((B, Hq), dtype=torch.float32)
    return device, B, Hq, Hkv, Lcap, kv, out, lse


def _need_workspace(workspace, device):
    """The workspace's bytes."""
    if not isinstance(workspace, torch.Tensor) or workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on cuda:{device}")
    return workspace.nbytes


def kv8_workspace_bytes(B: int, Hq: int, Hkv: int, Lcap: int, num_splits: int = 0) -> int:
    """Bytes for ``kv8_decode_attention``."""
    return lib().ffd_kv8_workspace_bytes(B, Hq, Hkv, Lcap, HEAD_DIM, num_splits)


def new_kv8_workspace(B: int, Hq: int, Hkv: int, Lcap: int, num_splits: int = 0, device="cuda"):
    """A workspace for ``kv8_decode_attention`` (one per stream)."""
    return torch.empty(max(kv8_workspace_bytes(B, Hq, Hkv, Lcap, num_splits), 16), dtype=torch.uint8, device=device)


def kv8_decode_attention(q, cache, seq_lens, *, num_splits: int = 0, softmax_scale: float = 0.0,
                         return_lse: bool = True, workspace=None, out=None, lse=None):
    """Exact dense decode attention over an 8-bit cache: ``dense_decode_attention`` on the values that it stands
    for. Returns ``(out, lse)``. ``workspace``: ``new_kv8_workspace``'s."""
    device, B, Hq, Hkv, Lcap, kv, out, lse = _dense_arguments(q, cache, "cache", seq_lens, return_lse, out, lse, False)
    if workspace is None:
        workspace = new_kv8_workspace(B, Hq, Hkv, Lcap, num_splits, q.device)
    _launch("ffd_kv8_decode_attention", lib().ffd_kv8_decode_attention, device, q.data_ptr(), ctypes.byref(kv),
            seq_lens.data_ptr(), B, Hq, Hkv, Lcap, HEAD_DIM, num_splits, softmax_scale, out.data_ptr(), _ptr(lse),
            workspace.data_ptr(), _need_workspace(workspace, device))
    return out, lse


def shared_prefix_workspace_bytes(B: int, Hq: int, Hkv: int, Pcap: int, Lcap: int, num_splits: int = 0) -> int:
    """Bytes for ``shared_prefix_decode_attention`` with a prefix of capacity Pcap and caches of capacity Lcap."""
    return lib().ffd_shared_prefix_workspace_bytes(B, Hq, Hkv, Pcap, Lcap, HEAD_DIM, num_splits)


def new_shared_prefix_workspace(B: int, Hq: int, Hkv: int, Pcap: int, Lcap: int, num_splits: int = 0, device="cuda"):
    """A workspace for ``shared_prefix_decode_attention`` (one per stream)."""
    return torch.empty(max(shared_prefix_workspace_bytes(B, Hq, Hkv, Pcap, Lcap, num_splits), 16), dtype=torch.uint8,
                       device=device)


def shared_prefix_decode_attention(q, prefix, prefix_lens, cache, seq_lens, *, num_splits: int = 0,
                                   softmax_scale: float = 0.0, return_lse: bool = True, workspace=None, out=None,
                                   lse=None):
    """Exact dense decode attention of a batch whose sequences begin with the same tokens: sequence b attends over the
    first ``prefix_lens[b]`` tokens of ``prefix`` and the ``seq_lens[b]`` tokens of its own ``cache``. The prefix is a
    cache of one sequence (B = 1) and is read once for up to 256 query rows of a KV head. ``prefix`` and ``cache`` are
    each ``(k, v)`` in bf16 or an 8-bit cache; the lengths int32 ``[B]``. Returns ``(out, lse)``."""
    device, B, Hq, Hkv, Lcap, own, out, lse = _dense_arguments(q, cache, "cache", seq_lens, return_lse, out, lse, True)
    Pcap = _cache_dims(prefix, "prefix", True)[2]
    shared = _kv_cache(prefix, "prefix", device, (1, Hkv, Pcap, HEAD_DIM))
    _need_on(device, prefix_lens, "prefix_lens", torch.int32, (B,))
    if workspace is None:
        workspace = new_shared_prefix_workspace(B, Hq, Hkv, Pcap, Lcap, num_splits, q.device)
    _launch("ffd_shared_prefix_decode_attention", lib().ffd_shared_prefix_decode_attention, device, q.data_ptr(),
            ctypes.byref(shared), prefix_lens.data_ptr(), Pcap, ctypes.byref(own), seq_lens.data_ptr(), B, Hq, Hkv, Lcap,
            HEAD_DIM, num_splits, softmax_scale, out.data_ptr(), _ptr(lse), workspace.data_ptr(),
            _need_workspace(workspace, device))
    return out, lse


# ---- paged caches -------------------------------------------------------------------------------------------
# A paged cache is one of the tuples above whose first dimension counts pages and whose third the tokens of a page:
# keys and values [num_pages, Hkv, page, 128] (bf16, or 8 bits with absmaxes [num_pages, Hkv, page]), as empty_kv8(num_pages,
# Hkv, page) and empty_paged make them. page_table int32 [B, max_pages] says where a sequence's pages are; an entry outside
# [0, num_pages) is a page that is not there. A batch's new tokens are rows q_start[b] .. q_start[b + 1] - 1 (int32 [B + 1]) for
# sequence b, the last of its seq_lens[b] tokens (int32 [B]).

def empty_paged(num_pages: int, Hkv: int, page: int, device="cuda"):
    """A bf16 paged cache with uninitialised contents: ``(k, v)``. (For one in 8 bits: ``empty_kv8``.)"""
    return tuple(torch.empty((num_pages, Hkv, page, HEAD_DIM), dtype=torch.bfloat16, device=device) for _ in range(2))


# The structures of these calls, packed as C lays them out: cheaper than ctypes' own, like the single expressions that the
# usual tensors pass (see _need).
_pack_paged = struct.Struct("@5P3i0P").pack
_pack_rotation = struct.Struct("@2Pf0PP3i0PP").pack
_pack_rules = struct.Struct("@fi2P").pack
_pack_strides = struct.Struct("@2q").pack


def _address(t) -> int:
    return 0 if t is None else t.data_ptr()


def _paged(cache, page_table, device):
    """(``ffd_paged``, B, Hkv, page, max_pages) of a cache whose tensors are as they have to be."""
    try:
        if len(cache) == 2:
            k, v = cache
            num_pages, Hkv, page, D = shape = k.shape
            B, max_pages = page_table.shape
            if (k.dtype is torch.bfloat16 and v.dtype is torch.bfloat16 and page_table.dtype is torch.int32 and v.shape == shape and D == HEAD_DIM
                    and k.get_device() == v.get_device() == page_table.get_device() == device >= 0
                    and k.is_contiguous() and v.is_contiguous() and page_table.is_contiguous()):
                return _pack_paged(k.data_ptr(), 0, v.data_ptr(), 0, page_table.data_ptr(), num_pages, page, max_pages), B, Hkv, page, max_pages
    except (AttributeError, TypeError, ValueError):
        pass                                             # named below
    num_pages, Hkv, page = _cache_dims(cache, "cache", True)
    kv = _kv_cache(cache, "cache", device, (num_pages, Hkv, page, HEAD_DIM))
    if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
        raise ValueError("page_table must be [B, max_pages]")
    B, max_pages = page_table.shape
    _need_on(device, page_table, "page_table", torch.int32, (B, max_pages))
    return (_pack_paged(kv.k or 0, kv.k_absmax or 0, kv.v or 0, kv.v_absmax or 0, page_table.data_ptr(), num_pages, page, max_pages),
            B, Hkv, page, max_pages)


def _need_int(x, name):
    if not -1 << 31 <= x < 1 << 31:                      # ctypes would take its low bits
        raise ValueError(f"{name} must fit 32 bits, got {x}")


def _ragged(q_start, seq_lens, device, B):
    try:
        if (q_start.dtype is torch.int32 and seq_lens.dtype is torch.int32 and q_start.shape == (B + 1,) and seq_lens.shape == (B,)
                and q_start.get_device() == seq_lens.get_device() == device and q_start.is_contiguous() and seq_lens.is_contiguous()):
            return
    except AttributeError:
        pass
    _need_on(device, q_start, "q_start", torch.int32, (B + 1,))
    _need_on(device, seq_lens, "seq_lens", torch.int32, (B,))


def _strided_rows(t, name, device, shape):
    """The two strides, in elements, of ``t`` as [T, heads, 128]; None where it is contiguous."""
    try:
        usual = t.dtype is torch.bfloat16 and t.shape == shape and t.get_device() == device >= 0
    except AttributeError:
        usual = False
    if not usual:
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise ValueError(f"{name} must be a CUDA (HIP) tensor")
        if t.dtype != torch.bfloat16 or t.get_device() != device:
            raise ValueError(f"{name} must be torch.bfloat16 on cuda:{device}, got {t.dtype} on {t.device}")
        if t.shape != shape:
            raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")
    if t.is_contiguous():
        return None
    strides = t.stride()
    if strides[2] != 1:
        raise ValueError(f"{name}'s last dimension must be contiguous")
    # the stride of a dimension of one is never used, and may be anything
    return _pack_strides(strides[0] if shape[0] > 1 else 0, strides[1] if shape[1] > 1 else 0)


def write_paged(q, k, v, cache, page_table, q_start, seq_lens, *, q_weight=None, k_weight=None, eps: float = 1e-6, rope=None,
                interleaved: bool = False, positions=None, out=None):
    """The new tokens' keys and values into a paged cache (bf16 or 8 bits), and their queries: each head of ``q`` and ``k``
    is normalised (root mean square, where its weight ``[128]`` is given) and rotated (where ``rope`` is given), in fp32 with
    one rounding. Returns the queries, bf16 ``[T, Hq, 128]`` (None without ``q``).

    ``q`` bf16 ``[T, Hq, 128]`` or None, ``k``, ``v`` ``[T, Hkv, 128]``, with any strides that are multiples of 8 elements
    (slices of a projection's output are taken as they are). ``seq_lens`` counts the new tokens already. ``rope``: fp32
    ``[rows, dims]``, the ``dims / 2`` cosines of a position, then its sines (dims 32, 64, 96 or 128; the other dims are not
    rotated); pairs are ``(i, i + dims / 2)``, or neighbours where ``interleaved``. ``positions``: int32 ``[T]``, the rows
    of ``rope``; without it a token's place in the cache (after an eviction that is not its place in the text)."""
    device = cache[0].get_device() if isinstance(cache, (tuple, list)) and cache and isinstance(cache[0], torch.Tensor) else -1
    paged, B, Hkv, _, _ = _paged(cache, page_table, device)
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError(f"k must be [T, Hkv, {HEAD_DIM}]")
    T, Hq = k.shape[0], Hkv
    k_strides, v_strides = _strided_rows(k, "k", device, (T, Hkv, HEAD_DIM)), _strided_rows(v, "v", device, (T, Hkv, HEAD_DIM))
    q_strides = None
    if q is not None:
        if not isinstance(q, torch.Tensor) or q.dim() != 3:
            raise ValueError(f"q must be [T, Hq, {HEAD_DIM}]")
        Hq = q.shape[1]
        q_strides = _strided_rows(q, "q", device, (T, Hq, HEAD_DIM))
        if out is None:
            out = q.new_empty((T, Hq, HEAD_DIM))
        else:
            _need_on(device, out, "out", torch.bfloat16, (T, Hq, HEAD_DIM))
    elif out is not None or q_weight is not None:
        raise ValueError("out and q_weight need q")
    _ragged(q_start, seq_lens, device, B)
    rows = dims = 0
    if rope is not None:
        if not isinstance(rope, torch.Tensor) or rope.dim() != 2:
            raise ValueError("rope must be [rows, dims]")
        rows, dims = rope.shape
        _need_on(device, rope, "rope", torch.float32, (rows, dims))
    if positions is not None:
        _need_on(device, positions, "positions", torch.int32, (T,))
    for weight, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        if weight is not None:
            _need_on(device, weight, name, torch.bfloat16, (HEAD_DIM,))
    rotation = _pack_rotation(_address(q_weight), _address(k_weight), eps, _address(rope), rows, dims, bool(interleaved), _address(positions))
    _launch("ffd_write_paged", lib().ffd_write_paged, device, _ptr(q), k.data_ptr(), v.data_ptr(), q_strides, k_strides, v_strides,
            _ptr(out), rotation, paged, q_start.data_ptr(), seq_lens.data_ptr(), B, T, Hq, Hkv,
            HEAD_DIM)
    return out


def paged_workspace_bytes(B: int, T: int, Hq: int, Hkv: int) -> int:
    """Bytes for ``paged_attention`` of T new tokens of B sequences."""
    return lib().ffd_paged_workspace_bytes(B, T, Hq, Hkv, HEAD_DIM)


def new_paged_workspace(B: int, T: int, Hq: int, Hkv: int, device="cuda"):
    """A workspace for ``paged_attention`` (one per stream)."""
    return torch.empty(max(paged_workspace_bytes(B, T, Hq, Hkv), 16), dtype=torch.uint8, device=device)


def _chunk_arguments(q, cache, page_table, q_start, seq_lens, softcap, window, slopes, prefix_lens):
    """Checks shared by the calls over new tokens' queries; (device, cache, rules, B, T, Hq, Hkv, Lcap)."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError(f"q must be [T, Hq, {HEAD_DIM}]")
    T, Hq, D = q.shape
    device = q.get_device()
    if not (q.dtype is torch.bfloat16 and D == HEAD_DIM and device >= 0 and q.is_contiguous()):
        _need_on(device, q, "q", torch.bfloat16, (T, Hq, HEAD_DIM))
    paged, B, Hkv, page, max_pages = _paged(cache, page_table, device)
    _ragged(q_start, seq_lens, device, B)
    if slopes is not None:
        _need_on(device, slopes, "slopes", torch.float32, (Hq,))
    if prefix_lens is not None:
        _need_on(device, prefix_lens, "prefix_lens", torch.int32, (B,))
    _need_int(window, "window")
    rules = None
    if softcap or window or slopes is not None or prefix_lens is not None:
        rules = _pack_rules(softcap, window, _address(slopes), _address(prefix_lens))
    return device, paged, rules, B, T, Hq, Hkv, page * max_pages


def paged_attention(q, cache, page_table, q_start, seq_lens, *, softmax_scale: float = 0.0, softcap: float = 0.0, window: int = 0,
                    slopes=None, prefix_lens=None, return_lse: bool = True, workspace=None, out=None, lse=None):
    """Attention of each sequence's new tokens, one or a chunk, over a paged cache that holds them already. ``q``: bf16
    ``[T, Hq, 128]``. Returns ``(out [T, Hq, 128], lse [T, Hq])``.

    The query at place i scores token j with ``softmax_scale`` q.k, then ``softcap tanh(. / softcap)``, then minus ``slopes[head]
    |i - j|`` (fp32 ``[Hq]``), and sees it if ``j <= i`` and, with a ``window``, ``i - j < window``, or if ``j < prefix_lens[b]``
    (int32 ``[B]``). A query that sees nothing gets zeros and ``lse = -inf``. ``workspace``: ``new_paged_workspace``'s."""
    device, paged, rules, B, T, Hq, Hkv, _ = _chunk_arguments(q, cache, page_table, q_start, seq_lens, softcap, window, slopes,
                                                              prefix_lens)
    if out is None:
        out = torch.empty_like(q)
    else:
        _need_on(device, out, "out", torch.bfloat16, (T, Hq, HEAD_DIM))
    if lse is not None:
        _need_on(device, lse, "lse", torch.float32, (T, Hq))
    elif return_lse:
        lse = q.new_empty((T, Hq), dtype=torch.float32)
    if workspace is None:
        workspace = new_paged_workspace(B, T, Hq, Hkv, q.device)
    _launch("ffd_paged_attention", lib().ffd_paged_attention, device, q.data_ptr(), paged, q_start.data_ptr(),
            seq_lens.data_ptr(), rules, B, T, Hq, Hkv, HEAD_DIM, softmax_scale, out.data_ptr(), _ptr(lse), workspace.data_ptr(),
            _need_workspace(workspace, device))
    return out, lse


def paged_attention_weights(q, cache, page_table, q_start, seq_lens, lse, *, softmax_scale: float = 0.0, softcap: float = 0.0,
                            window: int = 0, slopes=None, prefix_lens=None, last: int = 0, previous=None, out=None):
    """The attention weight that each cached token gets from the new ones, summed over the query heads of its KV head: fp32
    ``[B, Hkv, Lcap]``, Lcap the capacity of ``page_table``. ``q`` and the rules are those of the ``paged_attention`` call that
    gave ``lse``; ``last > 0`` counts the last tokens of each sequence only. Tokens that were there before the new ones start from
    ``previous`` (same shape; may be ``out``), the new ones from zero. Entries at and behind a length are left as they were
    (zeros without ``out``)."""
    device, paged, rules, B, T, Hq, Hkv, Lcap = _chunk_arguments(q, cache, page_table, q_start, seq_lens, softcap, window, slopes,
                                                                 prefix_lens)
    _need_on(device, lse, "lse", torch.float32, (T, Hq))
    _need_int(last, "last")
    if previous is not None:
        _need_on(device, previous, "previous", torch.float32, (B, Hkv, Lcap))
    if out is None:
        out = q.new_zeros((B, Hkv, Lcap), dtype=torch.float32)
    else:
        _need_on(device, out, "out", torch.float32, (B, Hkv, Lcap))
    _launch("ffd_paged_attention_weights", lib().ffd_paged_attention_weights, device, _ptr(q), paged,
            q_start.data_ptr(), seq_lens.data_ptr(), rules, _ptr(lse), B, T, Hq, Hkv, HEAD_DIM, softmax_scale, last, _ptr(previous),
            out.data_ptr())
    return out


def evict_paged(cache, page_table, new_table, seq_lens, weights, budget: int, *, recent: int = 0, new_lens=None, kept=None,
                new_weights=None):
    """Keep ``budget`` tokens of each sequence and KV head: the last ``recent`` and the heaviest of the others by ``weights``
    (``[B, Hkv, Lcap]``; equal ones from the lowest place on), in their order, moved to the pages of ``new_table`` (int32
    ``[B, new_max_pages]``, other pages of the same cache). Returns ``(kept, new_lens, new_weights)``: the old places int32
    ``[B, Hkv, budget]`` (-1 behind the last), the lengths int32 ``[B]`` (``new_lens`` may be ``seq_lens``) and the kept weights
    ``[B, Hkv, new_max_pages * page]`` (zeros behind the last, or what a given tensor holds)."""
    device = cache[0].get_device() if isinstance(cache, (tuple, list)) and cache and isinstance(cache[0], torch.Tensor) else -1
    paged, B, Hkv, page, max_pages = _paged(cache, page_table, device)
    if not isinstance(new_table, torch.Tensor) or new_table.dim() != 2:
        raise ValueError("new_table must be [B, new_max_pages]")
    new_max_pages = new_table.shape[1]
    _need_int(budget, "budget")
    _need_int(recent, "recent")
    try:
        usual = (new_table.dtype is torch.int32 and seq_lens.dtype is torch.int32 and weights.dtype is torch.float32
                 and new_table.shape[0] == B and seq_lens.shape == (B,) and weights.shape == (B, Hkv, max_pages * page)
                 and new_table.get_device() == seq_lens.get_device() == weights.get_device() == device
                 and new_table.is_contiguous() and seq_lens.is_contiguous() and weights.is_contiguous())
    except AttributeError:
        usual = False
    if not usual:
        _need_on(device, new_table, "new_table", torch.int32, (B, new_max_pages))
        _need_on(device, seq_lens, "seq_lens", torch.int32, (B,))
        _need_on(device, weights, "weights", torch.float32, (B, Hkv, max_pages * page))
    if new_table.data_ptr() == page_table.data_ptr() and B > 0:
        raise ValueError("new_table must hold other pages than page_table")
    if kept is None:
        kept = page_table.new_empty((B, Hkv, max(budget, 0)))
    else:
        _need_on(device, kept, "kept", torch.int32, (B, Hkv, budget))
    if new_lens is None:
        new_lens = page_table.new_empty((B,))
    else:
        _need_on(device, new_lens, "new_lens", torch.int32, (B,))
    if new_weights is None:
        new_weights = weights.new_zeros((B, Hkv, new_max_pages * page))
    else:
        _need_on(device, new_weights, "new_weights", torch.float32, (B, Hkv, new_max_pages * page))
    _launch("ffd_evict_paged", lib().ffd_evict_paged, device, paged, new_table.data_ptr(), new_max_pages,
            seq_lens.data_ptr(), weights.data_ptr(), B, Hkv, HEAD_DIM, budget, recent, new_lens.data_ptr(), kept.data_ptr(),
            new_weights.data_ptr())
    return kept, new_lens, new_weights


def default_scale() -> float:
    return 1.0 / math.sqrt(HEAD_DIM)
