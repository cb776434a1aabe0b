"""Thin ctypes binding of libjetlong.so (C ABI in include/jetlong.h).

Argument marshalling only: every step of the attention runs in the library's
HIP kernels.  PyTorch supplies device memory and the current stream.  If the
library is not built this module raises -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
import re

HERE = os.path.dirname(os.path.abspath(__file__))
# JETLONG_LIB may name another build of the same library (the host-sanitizer build)
LIB_PATH = os.environ.get("JETLONG_LIB") or os.path.join(HERE, "libjetlong.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "jetlong.h")

JL_OK, JL_ERR_INVALID_ARG, JL_ERR_UNSUPPORTED, JL_ERR_WORKSPACE, JL_ERR_HIP = range(5)
REMOTE_MAPS = {"alias": 0, "freq": 1}  # JL_REMOTE_ALIAS, JL_REMOTE_FREQ
TILE_SKIP, TILE_LOCAL, TILE_REMOTE, TILE_MIXED = range(4)

_lib = None


class JetLongError(RuntimeError):
    def __init__(self, status: int, name: str, detail: str):
        super().__init__("%s (%d): %s" % (name, status, detail))
        self.status = status


def lib() -> ctypes.CDLL:
    """Load libjetlong.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libjetlong.so is not built (run __graft_entry__.build()); "
                               "the HIP library is the only implementation")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, dbl, sz = (ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_double,
                                 ctypes.c_size_t)
        L.jl_status_string.restype = ctypes.c_char_p
        L.jl_status_string.argtypes = [i32]
        L.jl_last_error.restype = ctypes.c_char_p
        L.jl_last_error.argtypes = []
        L.jl_version.restype = i32
        L.jl_version.argtypes = []
        L.jl_group_size.restype = i64
        L.jl_group_size.argtypes = [i64, i64]
        L.jl_bifocal_prefill.restype = i32
        L.jl_bifocal_prefill.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, dbl, i32,
                                         i32, vp]
        L.jl_bifocal_prefill_map.restype = i32
        L.jl_bifocal_prefill_map.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, dbl,
                                             i32, i32, i32, vp]
        L.jl_bifocal_prefill_chunk.restype = i32
        L.jl_bifocal_prefill_chunk.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32,
                                               i32, dbl, i32, i32, vp]
        L.jl_rope_attention_chunk.restype = i32
        L.jl_rope_attention_chunk.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32,
                                              i32, dbl, vp]
        L.jl_bifocal_prefill_chunk_paged.restype = i32
        L.jl_bifocal_prefill_chunk_paged.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, i32,
                                                     i32, i32, i32, i32, i32, dbl, i32, i32, vp]
        L.jl_rope_attention_chunk_paged.restype = i32
        L.jl_rope_attention_chunk_paged.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, i32,
                                                    i32, i32, i32, i32, i32, dbl, vp]
        L.jl_bifocal_prefill_varlen.restype = i32
        L.jl_bifocal_prefill_varlen.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32,
                                                i32, dbl, i32, i32, vp]
        L.jl_bifocal_prefill_varlen_map.restype = i32
        L.jl_bifocal_prefill_varlen_map.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32,
                                                    i32, i32, dbl, i32, i32, i32, vp]
        L.jl_rope_attention_varlen.restype = i32
        L.jl_rope_attention_varlen.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32,
                                               i32, dbl, vp]
        L.jl_decode_map_workspace_bytes.restype = sz
        L.jl_decode_map_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32]
        L.jl_bifocal_decode_map.restype = i32
        L.jl_bifocal_decode_map.argtypes = [vp, vp, vp, vp, i32, vp, i32, i32, i32, i32, dbl,
                                            i32, i32, i32, vp, sz, vp]
        L.jl_rope_attention.restype = i32
        L.jl_rope_attention.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, dbl, vp]
        L.jl_prefill_literal_workspace_bytes.restype = sz
        L.jl_prefill_literal_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
        L.jl_bifocal_prefill_literal.restype = i32
        L.jl_bifocal_prefill_literal.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, dbl,
                                                 i32, i32, vp, sz, vp]
        L.jl_decode_workspace_bytes.restype = sz
        L.jl_decode_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
        L.jl_bifocal_decode.restype = i32
        L.jl_bifocal_decode.argtypes = [vp, vp, vp, vp, i32, vp, i32, i32, i32, i32, dbl, i32, i32,
                                        vp, sz, vp]
        L.jl_bifocal_decode_noalloc.restype = i32
        L.jl_bifocal_decode_noalloc.argtypes = [vp, vp, vp, vp, i32, vp, i32, i32, i32, i32, dbl,
                                                i32, i32, vp]
        L.jl_rope_attention_decode.restype = i32
        L.jl_rope_attention_decode.argtypes = [vp, vp, vp, vp, i32, vp, i32, i32, i32, i32, dbl,
                                               vp, sz, vp]
        L.jl_bifocal_decode_paged.restype = i32
        L.jl_bifocal_decode_paged.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, i32, i32, i32,
                                              i32, dbl, i32, i32, vp, sz, vp]
        L.jl_bifocal_decode_paged_map.restype = i32
        L.jl_bifocal_decode_paged_map.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, i32,
                                                  i32, i32, i32, dbl, i32, i32, i32, vp, sz, vp]
        L.jl_rope_attention_decode_paged.restype = i32
        L.jl_rope_attention_decode_paged.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, i32,
                                                     i32, i32, i32, dbl, vp, sz, vp]
        L.jl_cache8_append.restype = i32
        L.jl_cache8_append.argtypes = [vp, vp, i32, vp, vp, vp, vp, i32, i32, vp]
        L.jl_cache8_read.restype = i32
        L.jl_cache8_read.argtypes = [vp, vp, i32, vp, vp, i32, i32, i32, vp]
        L.jl_decode8_workspace_bytes.restype = sz
        L.jl_decode8_workspace_bytes.argtypes = [i32, i32, i32]
        L.jl_bifocal_decode8.restype = i32
        L.jl_bifocal_decode8.argtypes = [vp, vp, i32, vp, vp, vp, i32, i32, dbl, i32, i32, vp, sz,
                                         vp]
        L.jl_rope_attention_decode8.restype = i32
        L.jl_rope_attention_decode8.argtypes = [vp, vp, i32, vp, vp, vp, i32, i32, dbl, vp, sz, vp]
        L.jl_bifocal_decode8_blocks.restype = i32
        L.jl_bifocal_decode8_blocks.argtypes = [vp, vp, i32, vp, vp, vp, i32, vp, i32, i32, dbl,
                                                i32, i32, vp, sz, vp]
        L.jl_rope_attention_decode8_blocks.restype = i32
        L.jl_rope_attention_decode8_blocks.argtypes = [vp, vp, i32, vp, vp, vp, i32, vp, i32, i32,
                                                       dbl, vp, sz, vp]
        L.jl_bifocal_block_scores8.restype = i32
        L.jl_bifocal_block_scores8.argtypes = [vp, vp, i32, vp, vp, vp, i32, i32, dbl, i32, vp]
        L.jl_rope_block_scores8.restype = i32
        L.jl_rope_block_scores8.argtypes = [vp, vp, i32, vp, vp, vp, i32, i32, dbl, vp]
        L.jl_select_blocks.restype = i32
        L.jl_select_blocks.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, i32, vp]
        L.jl_pages_fork.restype = i32
        L.jl_pages_fork.argtypes = [vp, vp, vp]
        L.jl_pages_reserve.restype = i32
        L.jl_pages_reserve.argtypes = [vp, vp, vp, vp, vp, vp, vp]
        L.jl_pages_compact.restype = i32
        L.jl_pages_compact.argtypes = [vp, vp, vp, vp, vp]
        L.jl_copy_pages.restype = i32
        L.jl_copy_pages.argtypes = [vp, i32, i32, vp, vp, i32, vp]
        L.jl_cache_append.restype = i32
        L.jl_cache_append.argtypes = [vp, vp, i32, i32, vp, i32, vp, vp, vp, vp, vp, i32, i32, i32,
                                      i32, vp]
        L.jl_shared_plan_bytes.restype = sz
        L.jl_shared_plan_bytes.argtypes = [i32, i32, i32, i32]
        L.jl_bifocal_shared_plan.restype = i32
        L.jl_bifocal_shared_plan.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, i32,
                                             i32, vp, sz, vp]
        L.jl_rope_shared_plan.restype = i32
        L.jl_rope_shared_plan.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, sz,
                                          vp]
        L.jl_decode_shared_workspace_bytes.restype = sz
        L.jl_decode_shared_workspace_bytes.argtypes = [i32, i32, i32, i32]
        L.jl_bifocal_decode_shared.restype = i32
        L.jl_bifocal_decode_shared.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, sz, vp, i32, i32,
                                               i32, i32, i32, dbl, i32, i32, vp, sz, vp]
        L.jl_rope_attention_decode_shared.restype = i32
        L.jl_rope_attention_decode_shared.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, sz, vp, i32,
                                                      i32, i32, i32, i32, dbl, vp, sz, vp]
        L.jl_varlen_paged_workspace_bytes.restype = sz
        L.jl_varlen_paged_workspace_bytes.argtypes = [i32] * 7
        L.jl_bifocal_prefill_varlen_paged.restype = i32
        L.jl_bifocal_prefill_varlen_paged.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp,
                                                      i32, i32, i32, i32, i32, dbl, i32, i32, vp, sz,
                                                      vp]
        L.jl_rope_attention_varlen_paged.restype = i32
        L.jl_rope_attention_varlen_paged.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp,
                                                     i32, i32, i32, i32, i32, dbl, vp, sz, vp]
        L.jl_debug_schedule.restype = i32
        L.jl_debug_schedule.argtypes = [vp, i32, vp, i32, i32, vp, vp, vp, vp]
        L.jl_debug_prefill_tiles.restype = i32
        L.jl_debug_prefill_tiles.argtypes = [i32, i32, i32, i32, vp, i64,
                                             ctypes.POINTER(i32), ctypes.POINTER(i32),
                                             ctypes.POINTER(i32), ctypes.POINTER(i32), vp]
        L.jl_debug_prefill_rescale_log2.restype = dbl
        L.jl_debug_prefill_rescale_log2.argtypes = [dbl]
        L.jl_debug_kernel_events.restype = i32
        L.jl_debug_kernel_events.argtypes = [i32, vp, vp]
        L.jl_release_caches.restype = None
        L.jl_release_caches.argtypes = []
        _lib = L
    return _lib


def declared_functions() -> list:
    """Function names declared in include/jetlong.h."""
    src = open(HEADER).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    return sorted(set(re.findall(r"\b(jl_[a-z0-9_]+)\s*\(", src)))


def _check(status: int) -> None:
    if status != JL_OK:
        L = lib()
        raise JetLongError(status, L.jl_status_string(status).decode(),
                           L.jl_last_error().decode())


_torch = None


def _t():
    """The torch module, imported at the first call that takes tensors."""
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _stream(stream):
    """hipStream_t of the given stream, else of the current device's current one."""
    if stream is not None:
        return stream.cuda_stream
    # the raw handle: building a Stream object for it takes 3 us, a fifth of a
    # small decode call's time on the host.  Its entry is not part of torch's
    # public interface, so a torch without it gets the object.
    torch = _t()
    try:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    except AttributeError:
        return torch.cuda.current_stream().cuda_stream


def _dev(t, name, dtype=None, shape=None, device=None):
    """Device pointer of a contiguous CUDA tensor.  The library reads and writes
    through raw pointers, so a caller-supplied output must have exactly the
    shape the call writes (shape), and every tensor must sit on the query's
    device (device)."""
    if not isinstance(t, _t().Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) tensor" % name)
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if shape is not None and t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if device is not None and t.device != device:
        raise ValueError("%s is on %s, the query on %s" % (name, t.device, device))
    return t.data_ptr()


def _bf16(t, name, q, shape=None):
    """A bf16 tensor of the call, on q's device."""
    return _dev(t, name, _t().bfloat16, shape, q.device)


def _f32(t, name, q, shape):
    """An optional fp32 output (None passes a null pointer), on q's device."""
    return None if t is None else _dev(t, name, _t().float32, shape, q.device)


def _i32(t, name, q):
    return _dev(t, name, _t().int32, None, q.device)


def group_size(L: int, w_pretrained: int) -> int:
    return int(lib().jl_group_size(L, w_pretrained))


def _prefill(bifocal, q, k, v, w_pretrained, w_local, rope_theta, out, lse, want_lse, stream,
             remote_map="alias"):
    torch = _t()
    B, L, Hq, D = q.shape
    Hkv = k.shape[2]
    if k.shape != (B, L, Hkv, D) or v.shape != k.shape:
        raise ValueError("k and v must be [B, L, Hkv, D] matching q [B, L, Hq, D]")
    if out is None:
        out = torch.empty_like(q)
    if lse is None and want_lse:
        lse = torch.empty((B, Hq, L), dtype=torch.float32, device=q.device)
    args = [_bf16(q, "q", q), _bf16(k, "k", q), _bf16(v, "v", q),
            _bf16(out, "out", q, q.shape), _f32(lse, "lse", q, (B, Hq, L)), B, Hq, Hkv, L, D,
            float(rope_theta)]
    if bifocal and remote_map != "alias":
        _check(lib().jl_bifocal_prefill_map(*args, int(w_pretrained), int(w_local),
                                            REMOTE_MAPS[remote_map], _stream(stream)))
    elif bifocal:
        _check(lib().jl_bifocal_prefill(*args, int(w_pretrained), int(w_local), _stream(stream)))
    else:
        _check(lib().jl_rope_attention(*args, _stream(stream)))
    return (out, lse) if want_lse else out


def bifocal_prefill(q, k, v, *, w_pretrained: int, w_local: int, rope_theta: float = 1e6,
                    out=None, lse=None, want_lse: bool = False, stream=None,
                    remote_map: str = "alias"):
    """jl_bifocal_prefill: q [B, L, Hq, 128], k/v [B, L, Hkv, 128] raw bf16 -> out bf16.
    remote_map "freq" calls jl_bifocal_prefill_map with JL_REMOTE_FREQ (Sec. 4.5)."""
    if remote_map not in REMOTE_MAPS:
        raise ValueError("remote_map must be one of %s" % sorted(REMOTE_MAPS))
    return _prefill(True, q, k, v, w_pretrained, w_local, rope_theta, out, lse,
                    want_lse or lse is not None, stream, remote_map)


def rope_attention(q, k, v, *, rope_theta: float = 1e6, out=None, lse=None,
                   want_lse: bool = False, stream=None):
    """jl_rope_attention: vanilla causal RoPE attention with the same kernel."""
    return _prefill(False, q, k, v, 1, 0, rope_theta, out, lse, want_lse or lse is not None,
                    stream)


def prefill_chunk(q, k_cache, v_cache, *, q_start: int, w_pretrained: int = 1, w_local: int = 0,
                  rope_theta: float = 1e6, bifocal: bool = True, out=None, lse=None,
                  want_lse: bool = False, stream=None):
    """jl_bifocal_prefill_chunk / jl_rope_attention_chunk: q [B, n, Hq, 128] raw queries at
    positions q_start .. q_start + n - 1 over the raw caches [B, max_len, Hkv, 128]."""
    torch = _t()
    B, n, Hq, D = q.shape
    _, max_len, Hkv, _ = k_cache.shape
    if k_cache.shape != (B, max_len, Hkv, D) or v_cache.shape != k_cache.shape:
        raise ValueError("caches must be [B, max_len, Hkv, D] matching q [B, n, Hq, D]")
    if out is None:
        out = torch.empty_like(q)
    want_lse = want_lse or lse is not None
    if lse is None and want_lse:
        lse = torch.empty((B, Hq, n), dtype=torch.float32, device=q.device)
    args = [_bf16(q, "q", q), _bf16(k_cache, "k_cache", q), _bf16(v_cache, "v_cache", q),
            _bf16(out, "out", q, q.shape), _f32(lse, "lse", q, (B, Hq, n)), B, Hq, Hkv,
            int(q_start), n, max_len, D, float(rope_theta)]
    if bifocal:
        _check(lib().jl_bifocal_prefill_chunk(*args, int(w_pretrained), int(w_local),
                                              _stream(stream)))
    else:
        _check(lib().jl_rope_attention_chunk(*args, _stream(stream)))
    return (out, lse) if want_lse else out


def prefill_chunk_paged(q, k_pages, v_pages, block_table, *, q_start: int,
                        w_pretrained: int = 1, w_local: int = 0, rope_theta: float = 1e6,
                        bifocal: bool = True, out=None, lse=None, want_lse: bool = False,
                        stream=None):
    """jl_bifocal_prefill_chunk_paged / jl_rope_attention_chunk_paged: q [B, n, Hq, 128] raw
    queries at positions q_start .. q_start + n - 1, pools [n_pages, page_size, Hkv, 128] raw,
    block_table int32 [B, max_pages] on the device."""
    torch = _t()
    B, n, Hq, D = q.shape
    n_pages, page_size, Hkv, _ = k_pages.shape
    if k_pages.shape != (n_pages, page_size, Hkv, D) or v_pages.shape != k_pages.shape:
        raise ValueError("page pools must be [n_pages, page_size, Hkv, D]")
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError("block_table must be [B, max_pages]")
    max_pages = block_table.shape[1]
    if out is None:
        out = torch.empty_like(q)
    want_lse = want_lse or lse is not None
    if lse is None and want_lse:
        lse = torch.empty((B, Hq, n), dtype=torch.float32, device=q.device)
    args = [_bf16(q, "q", q), _bf16(k_pages, "k_pages", q), _bf16(v_pages, "v_pages", q),
            _i32(block_table, "block_table", q), max_pages, page_size, n_pages,
            _bf16(out, "out", q, q.shape), _f32(lse, "lse", q, (B, Hq, n)), B, Hq, Hkv,
            int(q_start), n, D, float(rope_theta)]
    if bifocal:
        _check(lib().jl_bifocal_prefill_chunk_paged(*args, int(w_pretrained), int(w_local),
                                                    _stream(stream)))
    else:
        _check(lib().jl_rope_attention_chunk_paged(*args, _stream(stream)))
    return (out, lse) if want_lse else out


def prefill_varlen(q, k, v, cu_seqlens, *, max_seqlen: int, w_pretrained: int = 1,
                   w_local: int = 0, rope_theta: float = 1e6, bifocal: bool = True, out=None,
                   lse=None, want_lse: bool = False, stream=None, remote_map: str = "alias"):
    """jl_bifocal_prefill_varlen / jl_rope_attention_varlen: packed sequences, q [T, Hq, 128],
    k, v [T, Hkv, 128], cu_seqlens int32 [B + 1] on the device; lse is [Hq, T].
    remote_map "freq" calls jl_bifocal_prefill_varlen_map with JL_REMOTE_FREQ (Sec. 4.5)."""
    if remote_map not in REMOTE_MAPS:
        raise ValueError("remote_map must be one of %s" % sorted(REMOTE_MAPS))
    torch = _t()
    T, Hq, D = q.shape
    Hkv = k.shape[1]
    if k.shape != (T, Hkv, D) or v.shape != k.shape:
        raise ValueError("k and v must be [T, Hkv, D] matching q [T, Hq, D]")
    if cu_seqlens.dim() != 1 or cu_seqlens.numel() < 2:
        raise ValueError("cu_seqlens must be [B + 1] with B >= 1")
    B = cu_seqlens.numel() - 1
    if out is None:
        out = torch.empty_like(q)
    want_lse = want_lse or lse is not None
    if lse is None and want_lse:
        lse = torch.empty((Hq, T), dtype=torch.float32, device=q.device)
    args = [_bf16(q, "q", q), _bf16(k, "k", q), _bf16(v, "v", q),
            _bf16(out, "out", q, q.shape), _f32(lse, "lse", q, (Hq, T)),
            _i32(cu_seqlens, "cu_seqlens", q), B, T, int(max_seqlen), Hq, Hkv, D,
            float(rope_theta)]
    if bifocal and remote_map != "alias":
        _check(lib().jl_bifocal_prefill_varlen_map(*args, int(w_pretrained), int(w_local),
                                                   REMOTE_MAPS[remote_map], _stream(stream)))
    elif bifocal:
        _check(lib().jl_bifocal_prefill_varlen(*args, int(w_pretrained), int(w_local),
                                               _stream(stream)))
    else:
        _check(lib().jl_rope_attention_varlen(*args, _stream(stream)))
    return (out, lse) if want_lse else out


def prefill_literal_workspace_bytes(B: int, Hq: int, Hkv: int, L: int,
                                    head_dim: int = 128) -> int:
    return int(lib().jl_prefill_literal_workspace_bytes(B, Hq, Hkv, L, head_dim))


def bifocal_prefill_literal(q, k, v, *, w_pretrained: int, w_local: int, rope_theta: float = 1e6,
                            out=None, lse=None, want_lse: bool = False, workspace=None,
                            stream=None):
    """jl_bifocal_prefill_literal: Eq. (7) as three window passes and a merge.

    Returns out (and lse when asked).  workspace, if given, is a uint8 CUDA
    tensor of at least prefill_literal_workspace_bytes(...) bytes; after the
    call literal_window_states(workspace, ...) views the per-window results.
    """
    torch = _t()
    B, L, Hq, D = q.shape
    Hkv = k.shape[2]
    if k.shape != (B, L, Hkv, D) or v.shape != k.shape:
        raise ValueError("k and v must be [B, L, Hkv, D] matching q [B, L, Hq, D]")
    want_lse = want_lse or lse is not None
    if out is None:
        out = torch.empty_like(q)
    if lse is None and want_lse:
        lse = torch.empty((B, Hq, L), dtype=torch.float32, device=q.device)
    need = prefill_literal_workspace_bytes(B, Hq, Hkv, L, D)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    _check(lib().jl_bifocal_prefill_literal(
        _bf16(q, "q", q), _bf16(k, "k", q), _bf16(v, "v", q), _bf16(out, "out", q, q.shape),
        _f32(lse, "lse", q, (B, Hq, L)), B, Hq, Hkv, L, D, float(rope_theta), int(w_pretrained),
        int(w_local), _dev(workspace, "workspace", device=q.device),
        workspace.numel() * workspace.element_size(), _stream(stream)))
    return (out, lse) if want_lse else out


def literal_window_states(workspace, B: int, Hq: int, L: int, head_dim: int = 128):
    """Views of a literal-prefill workspace: (O [3, B, L, Hq, D] fp32, LSE [3, B, Hq, L] fp32)."""
    torch = _t()
    n_o = 3 * B * L * Hq * head_dim
    f = workspace[: 4 * (n_o + 3 * B * Hq * L)].view(torch.float32)
    return (f[:n_o].view(3, B, L, Hq, head_dim), f[n_o:].view(3, B, Hq, L))


def decode_workspace_bytes(B: int, Hq: int, Hkv: int, max_len: int, head_dim: int = 128) -> int:
    return int(lib().jl_decode_workspace_bytes(B, Hq, Hkv, max_len, head_dim))


def _decode(bifocal, q, k_cache, v_cache, kv_lens, w_pretrained, w_local, rope_theta, out,
            workspace, stream):
    torch = _t()
    B, Hq, D = q.shape
    _, max_len, Hkv, _ = k_cache.shape
    if k_cache.shape != (B, max_len, Hkv, D) or v_cache.shape != k_cache.shape:
        raise ValueError("caches must be [B, max_len, Hkv, D]")
    if kv_lens.shape != (B,):
        raise ValueError("kv_lens must be [B]")
    if out is None:
        out = torch.empty_like(q)
    need = decode_workspace_bytes(B, Hq, Hkv, max_len, D)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
    args = [_bf16(q, "q", q), _bf16(k_cache, "k_cache", q), _bf16(v_cache, "v_cache", q),
            _i32(kv_lens, "kv_lens", q), max_len, _bf16(out, "out", q, q.shape), B, Hq, Hkv, D,
            float(rope_theta)]
    ws = [_dev(workspace, "workspace", device=q.device),
          workspace.numel() * workspace.element_size()]
    if bifocal:
        _check(lib().jl_bifocal_decode(*args, int(w_pretrained), int(w_local), *ws,
                                       _stream(stream)))
    else:
        _check(lib().jl_rope_attention_decode(*args, *ws, _stream(stream)))
    return out


def bifocal_decode_noalloc(q, k_cache, v_cache, kv_lens, *, w_pretrained: int, w_local: int,
                           rope_theta: float = 1e6, out=None, stream=None):
    """jl_bifocal_decode_noalloc: jl_bifocal_decode without a workspace; the library's
    fixed per-device array holds the split states and the cos/sin table."""
    torch = _t()
    B, Hq, D = q.shape
    _, max_len, Hkv, _ = k_cache.shape
    if k_cache.shape != (B, max_len, Hkv, D) or v_cache.shape != k_cache.shape:
        raise ValueError("caches must be [B, max_len, Hkv, D]")
    if kv_lens.shape != (B,):
        raise ValueError("kv_lens must be [B]")
    if out is None:
        out = torch.empty_like(q)
    _check(lib().jl_bifocal_decode_noalloc(
        _bf16(q, "q", q), _bf16(k_cache, "k_cache", q), _bf16(v_cache, "v_cache", q),
        _i32(kv_lens, "kv_lens", q), max_len, _bf16(out, "out", q, q.shape), B, Hq, Hkv, D,
        float(rope_theta),
        int(w_pretrained), int(w_local), _stream(stream)))
    return out


def bifocal_decode(q, k_cache, v_cache, kv_lens, *, w_pretrained: int, w_local: int,
                   rope_theta: float = 1e6, out=None, workspace=None, stream=None,
                   remote_map: str = "alias"):
    """jl_bifocal_decode: q [B, Hq, 128] raw, caches [B, max_len, Hkv, 128] raw, kv_lens int32.
    remote_map "freq" calls jl_bifocal_decode_map with JL_REMOTE_FREQ (Sec. 4.5)."""
    if remote_map == "alias":
        return _decode(True, q, k_cache, v_cache, kv_lens, w_pretrained, w_local, rope_theta,
                       out, workspace, stream)
    torch = _t()
    if remote_map not in REMOTE_MAPS:
        raise ValueError("remote_map must be one of %s" % sorted(REMOTE_MAPS))
    B, Hq, D = q.shape
    _, max_len, Hkv, _ = k_cache.shape
    if k_cache.shape != (B, max_len, Hkv, D) or v_cache.shape != k_cache.shape:
        raise ValueError("caches must be [B, max_len, Hkv, D]")
    if kv_lens.shape != (B,):
        raise ValueError("kv_lens must be [B]")
    if out is None:
        out = torch.empty_like(q)
    need = decode_map_workspace_bytes(B, Hq, Hkv, max_len, D, remote_map)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
    _check(lib().jl_bifocal_decode_map(
        _bf16(q, "q", q), _bf16(k_cache, "k_cache", q), _bf16(v_cache, "v_cache", q),
        _i32(kv_lens, "kv_lens", q), max_len, _bf16(out, "out", q, q.shape), B, Hq, Hkv, D,
        float(rope_theta), int(w_pretrained), int(w_local), REMOTE_MAPS[remote_map],
        _dev(workspace, "workspace", device=q.device),
        workspace.numel() * workspace.element_size(), _stream(stream)))
    return out


def decode_map_workspace_bytes(B: int, Hq: int, Hkv: int, max_len: int, head_dim: int = 128,
                               remote_map: str = "alias") -> int:
    return int(lib().jl_decode_map_workspace_bytes(B, Hq, Hkv, max_len, head_dim,
                                                   REMOTE_MAPS[remote_map]))


def rope_attention_decode(q, k_cache, v_cache, kv_lens, *, rope_theta: float = 1e6, out=None,
                          workspace=None, stream=None):
    """jl_rope_attention_decode: vanilla RoPE decode with the same kernels."""
    return _decode(False, q, k_cache, v_cache, kv_lens, 1, 0, rope_theta, out, workspace, stream)


def decode_paged(q, k_pages, v_pages, block_table, kv_lens, *, w_pretrained: int = 1,
                 w_local: int = 0, rope_theta: float = 1e6, bifocal: bool = True, out=None,
                 workspace=None, stream=None, remote_map: str = "alias"):
    """jl_bifocal_decode_paged / jl_rope_attention_decode_paged: q [B, Hq, 128] raw,
    pools [n_pages, page_size, Hkv, 128] raw, block_table int32 [B, max_pages],
    kv_lens int32 [B].  remote_map "freq" calls jl_bifocal_decode_paged_map with
    JL_REMOTE_FREQ (Sec. 4.5)."""
    torch = _t()
    B, Hq, D = q.shape
    n_pages, page_size, Hkv, _ = k_pages.shape
    if k_pages.shape != (n_pages, page_size, Hkv, D) or v_pages.shape != k_pages.shape:
        raise ValueError("page pools must be [n_pages, page_size, Hkv, D]")
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError("block_table must be [B, max_pages]")
    if kv_lens.shape != (B,):
        raise ValueError("kv_lens must be [B]")
    max_pages = block_table.shape[1]
    if remote_map not in REMOTE_MAPS:
        raise ValueError("remote_map must be one of %s" % sorted(REMOTE_MAPS))
    if out is None:
        out = torch.empty_like(q)
    if remote_map != "alias" and bifocal:
        need = decode_map_workspace_bytes(B, Hq, Hkv, max_pages * page_size, D, remote_map)
    else:
        need = decode_workspace_bytes(B, Hq, Hkv, max_pages * page_size, D)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
    args = [_bf16(q, "q", q), _bf16(k_pages, "k_pages", q), _bf16(v_pages, "v_pages", q),
            _i32(block_table, "block_table", q), max_pages, page_size, n_pages,
            _i32(kv_lens, "kv_lens", q), _bf16(out, "out", q, q.shape), B, Hq, Hkv, D,
            float(rope_theta)]
    ws = [_dev(workspace, "workspace", device=q.device),
          workspace.numel() * workspace.element_size()]
    if bifocal and remote_map != "alias":
        _check(lib().jl_bifocal_decode_paged_map(*args, int(w_pretrained), int(w_local),
                                                 REMOTE_MAPS[remote_map], *ws, _stream(stream)))
    elif bifocal:
        _check(lib().jl_bifocal_decode_paged(*args, int(w_pretrained), int(w_local), *ws,
                                             _stream(stream)))
    else:
        _check(lib().jl_rope_attention_decode_paged(*args, *ws, _stream(stream)))
    return out


# ------------------------------------------------------------- 8-bit cache
BLOCK8 = 64  # tokens of a block: one scale, one mean key, one unit of selection


class _Cache8Struct(ctypes.Structure):  # jl_cache8
    _fields_ = ([(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale", "k_mean")]
                + [(n, ctypes.c_int) for n in ("n_pages", "page_size", "Hkv", "head_dim")])


class Cache8:
    """The pools of an 8-bit cache (jl_cache8): k, v uint8 [n_pages, Hkv, page_size, 128],
    k_scale, v_scale fp32 [n_pages, Hkv, page_size // 64], k_mean bf16 [n_pages, Hkv,
    page_size // 64, 128], contiguous on one device.  cache8_alloc makes an empty one.
    Without a block table page b is sequence b.  The library gets the addresses that the
    tensors have here, so nothing of a Cache8 can be replaced, and a call on one whose tensors
    have moved since (resize_, set_) is refused."""

    def __init__(self, k, v, k_scale, v_scale, k_mean):
        torch = _t()
        if k.dim() != 4:
            raise ValueError("k must be [n_pages, Hkv, page_size, 128]")
        n_pages, Hkv, page_size, D = k.shape
        if page_size % BLOCK8:
            raise ValueError("page_size must be a multiple of %d, got %d" % (BLOCK8, page_size))
        blocks = (n_pages, Hkv, page_size // BLOCK8)
        ptrs = [_dev(k, "k", torch.uint8), _dev(v, "v", torch.uint8, k.shape, k.device),
                _dev(k_scale, "k_scale", torch.float32, blocks, k.device),
                _dev(v_scale, "v_scale", torch.float32, blocks, k.device),
                _dev(k_mean, "k_mean", torch.bfloat16, blocks + (D,), k.device)]
        struct = _Cache8Struct(*ptrs, n_pages, page_size, Hkv, D)
        self.__dict__.update(
            k=k, v=v, k_scale=k_scale, v_scale=v_scale, k_mean=k_mean, n_pages=n_pages,
            page_size=page_size, Hkv=Hkv, head_dim=D, device=k.device, index=k.get_device(),
            _struct=struct, _ref=ctypes.cast(ctypes.pointer(struct), ctypes.c_void_p),
            _ptrs=tuple(ptrs),
            _now=tuple(t.data_ptr for t in (k, v, k_scale, v_scale, k_mean)))

    def __setattr__(self, name, value):
        raise AttributeError("a Cache8 cannot be changed (%s): make another one" % name)

    def __delattr__(self, name):
        raise AttributeError("a Cache8 cannot be changed (%s): make another one" % name)


def cache8_alloc(n_pages: int, page_size: int, Hkv: int, *, head_dim: int = 128,
                 device="cuda") -> Cache8:
    """An empty 8-bit cache: n_pages pages of page_size tokens; for a dense one a page per
    sequence, page_size its capacity (a multiple of 64)."""
    torch = _t()
    kw = dict(device=device)
    blocks = (n_pages, Hkv, page_size // BLOCK8)
    return Cache8(torch.zeros((n_pages, Hkv, page_size, head_dim), dtype=torch.uint8, **kw),
                  torch.zeros((n_pages, Hkv, page_size, head_dim), dtype=torch.uint8, **kw),
                  torch.zeros(blocks, dtype=torch.float32, **kw),
                  torch.zeros(blocks, dtype=torch.float32, **kw),
                  torch.zeros(blocks + (head_dim,), dtype=torch.bfloat16, **kw))


def _new(like, stream, shape, dtype, fill=False):
    """An output (or a zeroed workspace) of a call on `stream`: from that stream's pool, so that
    neither its fill nor its reuse crosses streams."""
    make = like.new_zeros if fill else like.new_empty
    if stream is None:
        return make(shape, dtype=dtype)
    with _t().cuda.stream(stream):
        return make(shape, dtype=dtype)


def _on8(t, name, dtype, shape, index, device):
    """_dev for a tensor of a call on device `index`: the common case in one test (a small
    call's time on the host is a third of these checks), the error from _dev."""
    try:
        if (t.dtype is dtype and t.get_device() == index and t.is_contiguous()
                and (shape is None or t.shape == shape)):
            return t.data_ptr()
    except AttributeError:
        pass
    return _dev(t, name, dtype, shape, device)


def _queue(stream, index, device, name):
    """_stream of a call whose tensors are on device `index`: the library launches on the current
    one, so that has to be it."""
    torch = _t()
    try:
        now = torch._C._cuda_getDevice()
        raw = torch._C._cuda_getCurrentRawStream(now) if stream is None else stream.cuda_stream
    except AttributeError:
        now, raw = torch.cuda.current_device(), _stream(stream)
    if index != now:
        raise ValueError("%s is on %s, the current device is cuda:%d" % (name, device, now))
    return raw


def _int(x, name) -> int:
    """An int argument of the library: ctypes would drop the bits past 32."""
    x = int(x)
    if not -0x80000000 <= x <= 0x7fffffff:
        raise ValueError("%s must fit 32 bits, got %d" % (name, x))
    return x


def _query8(q, cache):
    """(B, Hq, pointer) of a query over an 8-bit cache."""
    if not isinstance(cache, Cache8):
        raise TypeError("cache must be a Cache8")
    ptr = _on8(q, "q", _t().bfloat16, None, cache.index, cache.device)
    shape = q.shape
    if len(shape) != 3 or shape[2] != cache.head_dim:
        raise ValueError("q must be [B, Hq, %d]" % cache.head_dim)
    return shape[0], shape[1], ptr


def _cache8(cache, block_table, B, stream):
    """The checks of a call of B sequences on a cache -> (jl_cache8 pointer, table pointer,
    max_pages, capacity, raw stream)."""
    raw = _queue(stream, cache.index, cache.device, "cache")
    k, v, k_scale, v_scale, k_mean = cache._now
    if (k(), v(), k_scale(), v_scale(), k_mean()) != cache._ptrs:
        raise ValueError("the cache's tensors have moved since it was made")
    if block_table is None:
        if B > cache.n_pages:
            raise ValueError("a dense cache of %d sequences cannot hold %d" % (cache.n_pages, B))
        return cache._ref, None, 0, cache.page_size, raw
    table = _on8(block_table, "block_table", _t().int32, None, cache.index, cache.device)
    shape = block_table.shape
    if len(shape) != 2 or shape[0] != B or shape[1] < 1:
        raise ValueError("block_table must be [B, max_pages]")
    max_pages = _int(shape[1], "max_pages")
    return cache._ref, table, max_pages, max_pages * cache.page_size, raw


def _ints(t, name, cache, shape):
    return _on8(t, name, _t().int32, shape, cache.index, cache.device)


def cache8_append(cache, k, v, starts, *, n_new=None, block_table=None, stream=None) -> None:
    """jl_cache8_append: rows k, v [B, n, Hkv, 128] bf16 to positions starts[b] .. of sequence
    b (starts int32 [B]); n_new int32 [B]: only the first n_new[b] of them."""
    if not isinstance(cache, Cache8):
        raise TypeError("cache must be a Cache8")
    bf16 = _t().bfloat16
    kp = _on8(k, "k", bf16, None, cache.index, cache.device)
    shape = k.shape
    if len(shape) != 4 or shape[2] != cache.Hkv or shape[3] != cache.head_dim:
        raise ValueError("k and v must be [B, n, %d, %d]" % (cache.Hkv, cache.head_dim))
    B, n = shape[0], shape[1]
    ref, table, max_pages, _, raw = _cache8(cache, block_table, B, stream)
    _check(lib().jl_cache8_append(
        ref, table, max_pages, kp, _on8(v, "v", bf16, shape, cache.index, cache.device),
        _ints(starts, "starts", cache, (B,)),
        None if n_new is None else _ints(n_new, "n_new", cache, (B,)), B, n, raw))


def cache8_read(cache, n: int, *, start: int = 0, B=None, block_table=None, k_out=None, v_out=None,
                stream=None):
    """jl_cache8_read: rows start .. start + n - 1 of every sequence as bf16 (k, v), each
    [B, n, Hkv, 128].  B: sequences of a dense cache, all of them if not given."""
    if not isinstance(cache, Cache8):
        raise TypeError("cache must be a Cache8")
    bf16 = _t().bfloat16
    if B is None:
        B = cache.n_pages if block_table is None else block_table.shape[0]
    ref, table, max_pages, cap, raw = _cache8(cache, block_table, B, stream)
    start, n, B = _int(start, "start"), _int(n, "n"), _int(B, "B")
    shape = (B, n, cache.Hkv, cache.head_dim)
    if (k_out is None or v_out is None) and 0 < n <= cap:  # the library refuses other lengths
        if k_out is None:
            k_out = _new(cache.k_mean, stream, shape, bf16)
        if v_out is None:
            v_out = _new(cache.k_mean, stream, shape, bf16)
    kp, vp = (None if t is None else _on8(t, name, bf16, shape, cache.index, cache.device)
              for t, name in ((k_out, "k_out"), (v_out, "v_out")))
    _check(lib().jl_cache8_read(ref, table, max_pages, kp, vp, B, start, n, raw))
    return k_out, v_out


def decode8_workspace_bytes(Hq: int, Hkv: int, head_dim: int = 128) -> int:
    return int(lib().jl_decode8_workspace_bytes(Hq, Hkv, head_dim))


def decode8_workspace(Hq: int, Hkv: int, *, head_dim: int = 128, device="cuda"):
    """A workspace for decode8 and decode8_blocks, zeroed as they need it before their first
    call; a decoding loop keeps one per stream."""
    torch = _t()
    return torch.zeros(decode8_workspace_bytes(Hq, Hkv, head_dim), dtype=torch.uint8,
                       device=device)


def _decode8(q, cache, kv_lens, blocks, w_pretrained, w_local, rope_theta, bifocal, block_table,
             out, workspace, stream):
    torch = _t()
    B, Hq, qp = _query8(q, cache)
    ref, table, max_pages, _, raw = _cache8(cache, block_table, B, stream)
    if out is None:
        out = _new(q, stream, q.shape, torch.bfloat16)
        op = out.data_ptr()
    else:
        op = _on8(out, "out", torch.bfloat16, q.shape, cache.index, cache.device)
    if workspace is None:
        need = decode8_workspace_bytes(Hq, cache.Hkv, cache.head_dim)
        workspace = _new(q, stream, (max(need, 16),), torch.uint8, fill=True)
    wp = _on8(workspace, "workspace", getattr(workspace, "dtype", None), None, cache.index, cache.device)
    lens = _ints(kv_lens, "kv_lens", cache, (B,))
    L = lib()
    if blocks is None:
        args = (ref, table, max_pages, qp, lens, op, B, Hq, float(rope_theta))
        call = L.jl_bifocal_decode8 if bifocal else L.jl_rope_attention_decode8
    else:
        bp = _ints(blocks, "blocks", cache, None)
        if blocks.dim() != 3 or blocks.shape[0] != B or blocks.shape[1] != cache.Hkv:
            raise ValueError("blocks must be [B, Hkv, n_select]")
        args = (ref, table, max_pages, qp, lens, bp, _int(blocks.shape[2], "n_select"), op, B, Hq,
                float(rope_theta))
        call = L.jl_bifocal_decode8_blocks if bifocal else L.jl_rope_attention_decode8_blocks
    if bifocal:
        _check(call(*args, _int(w_pretrained, "w_pretrained"), _int(w_local, "w_local"), wp,
                    workspace.nbytes, raw))
    else:
        _check(call(*args, wp, workspace.nbytes, raw))
    return out


def decode8(q, cache, kv_lens, *, w_pretrained: int = 1, w_local: int = 0,
            rope_theta: float = 1e6, bifocal: bool = True, block_table=None, out=None,
            workspace=None, stream=None):
    """jl_bifocal_decode8 / jl_rope_attention_decode8: q [B, Hq, 128] raw over an 8-bit cache,
    kv_lens int32 [B] (0: zeros).  workspace: decode8_workspace(Hq, Hkv), kept between calls;
    without one every call fills one of its own."""
    return _decode8(q, cache, kv_lens, None, w_pretrained, w_local, rope_theta, bifocal,
                    block_table, out, workspace, stream)


def decode8_blocks(q, cache, kv_lens, blocks, *, w_pretrained: int = 1, w_local: int = 0,
                   rope_theta: float = 1e6, bifocal: bool = True, block_table=None, out=None,
                   workspace=None, stream=None):
    """jl_bifocal_decode8_blocks / jl_rope_attention_decode8_blocks: decode8 over the blocks that
    blocks int32 [B, Hkv, n_select] lists (select_blocks)."""
    if blocks is None:
        raise ValueError("blocks must be [B, Hkv, n_select]")
    return _decode8(q, cache, kv_lens, blocks, w_pretrained, w_local, rope_theta, bifocal,
                    block_table, out, workspace, stream)


def block_scores8(q, cache, kv_lens, *, w_pretrained: int = 1, rope_theta: float = 1e6,
                  bifocal: bool = True, block_table=None, out=None, stream=None):
    """jl_bifocal_block_scores8 / jl_rope_block_scores8: fp32 [B, Hkv, capacity // 64], the score
    of every block's mean key, -inf past the sequence."""
    torch = _t()
    B, Hq, qp = _query8(q, cache)
    ref, table, max_pages, cap, raw = _cache8(cache, block_table, B, stream)
    shape = (B, cache.Hkv, cap // BLOCK8)
    if out is None:
        out = _new(q, stream, shape, torch.float32)
        op = out.data_ptr()
    else:
        op = _on8(out, "out", torch.float32, shape, cache.index, cache.device)
    args = (ref, table, max_pages, qp, _ints(kv_lens, "kv_lens", cache, (B,)), op, B, Hq,
            float(rope_theta))
    if bifocal:
        _check(lib().jl_bifocal_block_scores8(*args, _int(w_pretrained, "w_pretrained"),
                                              raw))
    else:
        _check(lib().jl_rope_block_scores8(*args, raw))
    return out


def select_blocks(scores, kv_lens, n_select: int, *, w_local: int, n_first: int = 1, out=None,
                  stream=None):
    """jl_select_blocks: int32 [B, Hkv, n_select] from scores fp32 [B, Hkv, n_blocks]: the first
    n_first blocks and those of the local band always, then the largest scores; ascending,
    -1 behind the last."""
    torch = _t()
    ptr = _dev(scores, "scores", torch.float32)
    if scores.dim() != 3:
        raise ValueError("scores must be [B, Hkv, n_blocks]")
    B, Hkv, n_blocks = scores.shape
    index, device = scores.get_device(), scores.device
    raw = _queue(stream, index, device, "scores")
    n_blocks, n_select = _int(n_blocks, "n_blocks"), _int(n_select, "n_select")
    w_local, n_first = _int(w_local, "w_local"), _int(n_first, "n_first")
    if out is None:
        if n_select < 1:
            raise ValueError("n_select must be >= 1")
        out = _new(scores, stream, (B, Hkv, n_select), torch.int32)
        op = out.data_ptr()
    else:
        op = _on8(out, "out", torch.int32, (B, Hkv, n_select), index, device)
    _check(lib().jl_select_blocks(
        ptr, _on8(kv_lens, "kv_lens", torch.int32, (B,), index, device), op, B, Hkv, n_blocks,
        n_select, w_local, n_first, raw))
    return out


# ------------------------------------------------------------ pages of a batch
class _PagesStruct(ctypes.Structure):  # jl_pages
    _fields_ = ([(n, ctypes.c_void_p) for n in ("table", "lens", "refs")]
                + [(n, ctypes.c_int) for n in ("B", "max_pages", "n_pages", "page_size")])


class _PoolStruct(ctypes.Structure):  # jl_page_pool
    _fields_ = [("ptr", ctypes.c_void_p), ("page_bytes", ctypes.c_size_t)]


class PageTable:
    """The tables of B sequences over a pool of pages (jl_pages): lens int32 [B], refs int32
    [n_pages], table int32 [B, max_pages], on one device.  pages_alloc makes an empty one.  The
    paged calls take table as block_table and lens as kv_lens.  The tensors are the caller's to
    read and to restore by copy_; none can be replaced.  lens may be lowered in place (rejected
    drafts): the next pages_reserve frees the pages behind."""

    def __init__(self, lens, refs, table, page_size: int):
        if table.dim() != 2:
            raise ValueError("table must be [B, max_pages]")
        (B, max_pages), device, index = table.shape, table.device, table.get_device()
        i32 = _t().int32
        page_size = _int(page_size, "page_size")
        struct = _PagesStruct(
            _dev(table, "table", i32), _on8(lens, "lens", i32, (B,), index, device),
            _on8(refs, "refs", i32, (refs.numel(),), index, device), B, max_pages, refs.numel(),
            page_size)
        self.__dict__.update(lens=lens, refs=refs, table=table, B=B, max_pages=max_pages,
                             n_pages=refs.numel(), page_size=page_size, device=device,
                             index=index, _struct=struct, _ref=ctypes.byref(struct),
                             _ptrs=(table.data_ptr(), lens.data_ptr(), refs.data_ptr()))

    def __setattr__(self, name, value):
        raise AttributeError("a PageTable cannot be changed (%s): make another one" % name)

    def __delattr__(self, name):
        raise AttributeError("a PageTable cannot be changed (%s): make another one" % name)


def pages_alloc(B: int, max_pages: int, n_pages: int, page_size: int, *, device="cuda") -> PageTable:
    """A table of B empty sequences over a pool of n_pages free pages."""
    kw = dict(dtype=_t().int32, device=device)
    return PageTable(_t().zeros(B, **kw), _t().zeros(n_pages, **kw),
                     _t().full((B, max_pages), -1, **kw), page_size)


def _pages(pages, stream):
    """The checks of a call on a table -> (jl_pages pointer, raw stream)."""
    if not isinstance(pages, PageTable):
        raise TypeError("pages must be a PageTable")
    if (pages.table.data_ptr(), pages.lens.data_ptr(), pages.refs.data_ptr()) != pages._ptrs:
        raise ValueError("the table's tensors have moved since it was made")
    return pages._ref, _queue(stream, pages.index, pages.device, "table")


def pages_fork(pages, parent, *, stream=None) -> None:
    """jl_pages_fork: row b becomes what row parent[b] was, or empty (parent int32 [B]; -1 frees),
    all rows at once."""
    ref, raw = _pages(pages, stream)
    _check(lib().jl_pages_fork(ref, _on8(parent, "parent", _t().int32, (pages.B,), pages.index,
                                         pages.device), raw))


def pages_reserve(pages, n_new, *, stream=None):
    """jl_pages_reserve: room for n_new[b] (int32 [B]) more rows of every sequence, whose lens
    grow -> (starts, granted, moves, info): starts and granted for the append calls, moves and
    info for copy_pages, which has to come before them."""
    ref, raw = _pages(pages, stream)
    B, i32 = pages.B, _t().int32
    n = _on8(n_new, "n_new", i32, (B,), pages.index, pages.device)
    out = _new(pages.lens, stream, (4 + 4 * B,), i32)
    at = out.data_ptr()
    info, moves, starts, granted = out.split((4, 2 * B, B, B))
    _check(lib().jl_pages_reserve(ref, n, at + 16 + 8 * B, at + 16 + 12 * B, at + 16, at, raw))
    return starts, granted, moves.view(B, 2), info


def pages_compact(pages, *, stream=None):
    """jl_pages_compact: the pages in use become the first ones of the pool -> (moves, info) for
    copy_pages."""
    ref, raw = _pages(pages, stream)
    n, i32 = pages.n_pages, _t().int32
    out = _new(pages.lens, stream, (4 + n // 2 * 2,), i32)
    to = _new(pages.lens, stream, (n,), i32)
    at = out.data_ptr()
    _check(lib().jl_pages_compact(ref, at + 16, to.data_ptr(), at, raw))
    return out[4:].view(n // 2, 2), out[:4]


def copy_pages(pools, moves, info, *, stream=None) -> None:
    """jl_copy_pages: pages of every pool are copied as moves int32 [m, 2] says, the first info[0]
    pairs.  pools: tensors [n_pages, ...] or Cache8s, all of as many pages and on one device."""
    torch = _t()
    tensors = []
    for p in pools if isinstance(pools, (list, tuple)) else [pools]:
        tensors.extend([p.k, p.v, p.k_scale, p.v_scale, p.k_mean] if isinstance(p, Cache8) else [p])
    if not tensors:
        raise ValueError("pools must name a tensor")
    index, device = moves.get_device(), moves.device
    mp = _dev(moves, "moves", torch.int32)
    if moves.dim() != 2 or moves.shape[1] != 2:
        raise ValueError("moves must be [m, 2]")
    ip = _on8(info, "info", torch.int32, None, index, device)
    if info.numel() < 1:
        raise ValueError("info must hold the number of moves")
    raw = _queue(stream, index, device, "moves")
    n_pages = tensors[0].shape[0] if tensors[0].dim() else 0
    array = (_PoolStruct * len(tensors))()
    for slot, t in zip(array, tensors):
        if t.dim() < 1 or t.shape[0] != n_pages or n_pages < 1:
            raise ValueError("every pool must be [n_pages, ...] of the same n_pages")
        slot.ptr = _on8(t, "pool", t.dtype, None, index, device)
        slot.page_bytes = t.nbytes // n_pages
    _check(lib().jl_copy_pages(array, len(tensors), _int(n_pages, "n_pages"), mp, ip,
                               _int(moves.shape[0], "max_moves"), raw))


def cache_append(k_cache, v_cache, k, v, starts, *, n_new=None, cu_seqlens=None, block_table=None,
                 stream=None) -> None:
    """jl_cache_append: rows k, v [B, n, Hkv, 128] bf16, or packed [T, Hkv, 128] with cu_seqlens int32
    [B + 1], to positions starts[b] .. of sequence b in caches [B, max_len, Hkv, 128] or, with
    block_table int32 [B, max_pages], pools [n_pages, page_size, Hkv, 128].  n_new int32 [B]: only
    the first n_new[b] rows of sequence b."""
    torch = _t()
    bf16, i32 = torch.bfloat16, torch.int32
    kcp = _dev(k_cache, "k_cache", bf16)
    index, device = k_cache.get_device(), k_cache.device
    if k_cache.dim() != 4:
        raise ValueError("k_cache must be [n_pages, page_size, Hkv, D]")
    n_pages, page_size, Hkv, D = k_cache.shape
    vcp = _on8(v_cache, "v_cache", bf16, k_cache.shape, index, device)
    kp = _on8(k, "k", bf16, None, index, device)
    vp = _on8(v, "v", bf16, k.shape, index, device)
    shape = k.shape
    if cu_seqlens is not None:
        if len(shape) != 3 or shape[1:] != (Hkv, D):
            raise ValueError("packed k and v must be [T, %d, %d]" % (Hkv, D))
        if cu_seqlens.dim() != 1 or cu_seqlens.numel() < 2:
            raise ValueError("cu_seqlens must be [B + 1] with B >= 1")
        B, n = cu_seqlens.numel() - 1, shape[0]
        cp = _on8(cu_seqlens, "cu_seqlens", i32, None, index, device)
    else:
        if len(shape) != 4 or shape[2:] != (Hkv, D):
            raise ValueError("k and v must be [B, n, %d, %d]" % (Hkv, D))
        B, n, cp = shape[0], shape[1], None
    tp, max_pages = None, 0
    if block_table is not None:
        tp = _on8(block_table, "block_table", i32, None, index, device)
        if block_table.dim() != 2 or block_table.shape[0] != B:
            raise ValueError("block_table must be [B, max_pages]")
        max_pages = block_table.shape[1]
    _check(lib().jl_cache_append(
        kcp, vcp, _int(n_pages, "n_pages"), _int(page_size, "page_size"), tp,
        _int(max_pages, "max_pages"), kp, vp, _on8(starts, "starts", i32, (B,), index, device),
        None if n_new is None else _on8(n_new, "n_new", i32, (B,), index, device), cp,
        _int(B, "B"), _int(n, "n"), _int(Hkv, "Hkv"), D, _queue(stream, index, device, "k_cache")))


# ------------------------------------------- decode over shared prefixes
class SharedPlan:
    """What the decode calls of one step have in common (shared_plan): made for these sizes, windows
    and lengths, for every layer."""

    __slots__ = ("buf", "B", "n_groups", "Hq", "Hkv", "page_size", "max_pages", "w_pretrained",
                 "w_local", "bifocal", "index", "device", "ptr", "nbytes")


def shared_plan_bytes(B: int, n_groups: int, Hq: int, Hkv: int) -> int:
    return int(lib().jl_shared_plan_bytes(B, n_groups, Hq, Hkv))


def shared_plan(kv_lens, group_starts, shared, *, Hq: int, Hkv: int, page_size: int,
                max_pages: int, members=None, w_pretrained: int = 1, w_local: int = 0,
                bifocal: bool = True, out=None, stream=None) -> SharedPlan:
    """jl_bifocal_shared_plan / jl_rope_shared_plan: kv_lens int32 [B]; group i is the sequences
    members[group_starts[i]] .. members[group_starts[i + 1] - 1] (group_starts int32 [n_groups + 1],
    members int32 [B], all in order if not given), which have their first shared[i] (int32
    [n_groups]) tokens' pages in common.  out: a plan of the same sizes to write again, as a
    captured step does."""
    i32 = _t().int32
    lp = _dev(kv_lens, "kv_lens", i32)
    index, device = kv_lens.get_device(), kv_lens.device
    if kv_lens.dim() != 1 or shared.dim() != 1:
        raise ValueError("kv_lens must be [B], shared [n_groups]")
    B, n = _int(kv_lens.shape[0], "B"), _int(shared.shape[0], "n_groups")
    Hq, Hkv = _int(Hq, "Hq"), _int(Hkv, "Hkv")
    page_size, max_pages = _int(page_size, "page_size"), _int(max_pages, "max_pages")
    w_pretrained, w_local = _int(w_pretrained, "w_pretrained"), _int(w_local, "w_local")
    raw = _queue(stream, index, device, "kv_lens")
    key = (B, n, Hq, Hkv, page_size, max_pages, w_pretrained, w_local, bool(bifocal), index)
    if out is None:
        p = SharedPlan()
        (p.B, p.n_groups, p.Hq, p.Hkv, p.page_size, p.max_pages, p.w_pretrained, p.w_local,
         p.bifocal, p.index) = key
        p.device = device
        p.buf = _new(kv_lens, stream, (max(shared_plan_bytes(B, n, Hq, Hkv), 16),), _t().uint8)
        p.ptr, p.nbytes = p.buf.data_ptr(), p.buf.numel()
    else:
        p = out
        if not isinstance(p, SharedPlan) or key != (
                p.B, p.n_groups, p.Hq, p.Hkv, p.page_size, p.max_pages, p.w_pretrained, p.w_local,
                p.bifocal, p.index):
            raise ValueError("out must be a plan of the same sizes and windows")
    args = (lp, None if members is None else _on8(members, "members", i32, (B,), index, device),
            _on8(group_starts, "group_starts", i32, (n + 1,), index, device),
            _on8(shared, "shared", i32, (n,), index, device), B, n, Hq, Hkv, 128, max_pages,
            page_size)
    if bifocal:
        _check(lib().jl_bifocal_shared_plan(*args, w_pretrained, w_local, p.ptr, p.nbytes, raw))
    else:
        _check(lib().jl_rope_shared_plan(*args, p.ptr, p.nbytes, raw))
    return p


def decode_shared_workspace_bytes(B: int, Hq: int, Hkv: int, head_dim: int = 128) -> int:
    return int(lib().jl_decode_shared_workspace_bytes(B, Hq, Hkv, head_dim))


def decode_shared(q, k_pages, v_pages, block_table, plan, *, rope_theta: float = 1e6, out=None,
                  workspace=None, stream=None):
    """jl_bifocal_decode_shared / jl_rope_attention_decode_shared, as the plan was made: q [B, Hq,
    128] raw over pools [n_pages, page_size, Hkv, 128] raw, block_table int32 [B, max_pages].  Rows
    of `out` for sequences that no group of the plan has stay as they were."""
    torch = _t()
    if not isinstance(plan, SharedPlan):
        raise TypeError("plan must be a SharedPlan")
    bf16, index, device = torch.bfloat16, plan.index, plan.device
    B, Hq, Hkv = plan.B, plan.Hq, plan.Hkv
    qp = _on8(q, "q", bf16, (B, Hq, 128), index, device)
    kp = _on8(k_pages, "k_pages", bf16, None, index, device)
    shape = k_pages.shape
    if len(shape) != 4 or shape[1:] != (plan.page_size, Hkv, 128):
        raise ValueError("page pools must be [n_pages, %d, %d, 128]" % (plan.page_size, Hkv))
    vp = _on8(v_pages, "v_pages", bf16, shape, index, device)
    tp = _on8(block_table, "block_table", torch.int32, (B, plan.max_pages), index, device)
    raw = _queue(stream, index, device, "plan")
    if out is None:
        out = _new(q, stream, q.shape, bf16)
        op = out.data_ptr()
    else:
        op = _on8(out, "out", bf16, (B, Hq, 128), index, device)
    if workspace is None:
        workspace = _new(q, stream, (decode_shared_workspace_bytes(B, Hq, Hkv),), torch.uint8)
    wp = _on8(workspace, "workspace", getattr(workspace, "dtype", None), None, index, device)
    args = (qp, kp, vp, tp, plan.max_pages, plan.page_size, _int(shape[0], "n_pages"), plan.ptr,
            plan.nbytes, op, B, plan.n_groups, Hq, Hkv, 128, float(rope_theta))
    if plan.bifocal:
        _check(lib().jl_bifocal_decode_shared(*args, plan.w_pretrained, plan.w_local, wp,
                                              workspace.nbytes, raw))
    else:
        _check(lib().jl_rope_attention_decode_shared(*args, wp, workspace.nbytes, raw))
    return out


def varlen_paged_workspace_bytes(B: int, T: int, Hq: int, Hkv: int, max_pages: int, page_size: int,
                                 head_dim: int = 128) -> int:
    return int(lib().jl_varlen_paged_workspace_bytes(B, T, Hq, Hkv, head_dim, max_pages, page_size))


def prefill_varlen_paged(q, k_pages, v_pages, block_table, cu_seqlens, kv_lens, *,
                         w_pretrained: int = 1, w_local: int = 0, rope_theta: float = 1e6,
                         bifocal: bool = True, out=None, lse=None, want_lse: bool = False,
                         workspace=None, stream=None):
    """jl_bifocal_prefill_varlen_paged / jl_rope_attention_varlen_paged: packed raw queries q [T, Hq,
    128], sequence b's cu_seqlens[b] .. cu_seqlens[b + 1] - 1 (int32 [B + 1]) at the last of its
    kv_lens[b] (int32 [B]) positions, over pools [n_pages, page_size, Hkv, 128] raw, block_table
    int32 [B, max_pages]; lse is [Hq, T]."""
    torch = _t()
    bf16, i32 = torch.bfloat16, torch.int32
    qp = _dev(q, "q", bf16)
    index, device = q.get_device(), q.device
    kp = _on8(k_pages, "k_pages", bf16, None, index, device)
    shape = k_pages.shape
    if q.dim() != 3 or len(shape) != 4 or shape[3] != q.shape[2]:
        raise ValueError("q must be [T, Hq, D], page pools [n_pages, page_size, Hkv, D]")
    T, Hq, D = q.shape
    vp = _on8(v_pages, "v_pages", bf16, shape, index, device)
    tp = _on8(block_table, "block_table", i32, None, index, device)
    if block_table.dim() != 2:
        raise ValueError("block_table must be [B, max_pages]")
    B, max_pages = block_table.shape
    cp = _on8(cu_seqlens, "cu_seqlens", i32, (B + 1,), index, device)
    lp = _on8(kv_lens, "kv_lens", i32, (B,), index, device)
    raw = _queue(stream, index, device, "q")
    if out is None:
        out = _new(q, stream, q.shape, bf16)
        op = out.data_ptr()
    else:
        op = _on8(out, "out", bf16, q.shape, index, device)
    want_lse = want_lse or lse is not None
    if lse is None and want_lse:
        lse = _new(q, stream, (Hq, T), torch.float32)
    args = (qp, kp, vp, tp, _int(max_pages, "max_pages"), _int(shape[1], "page_size"),
            _int(shape[0], "n_pages"), cp, lp, op,
            None if lse is None else _on8(lse, "lse", torch.float32, (Hq, T), index, device),
            _int(B, "B"), _int(T, "T"), Hq, _int(shape[2], "Hkv"), D, float(rope_theta))
    if workspace is None:
        workspace = _new(q, stream, (varlen_paged_workspace_bytes(
            B, T, Hq, shape[2], max_pages, shape[1], D),), torch.uint8)
    wp = _on8(workspace, "workspace", getattr(workspace, "dtype", None), None, index, device)
    if bifocal:
        _check(lib().jl_bifocal_prefill_varlen_paged(
            *args, _int(w_pretrained, "w_pretrained"), _int(w_local, "w_local"), wp,
            workspace.nbytes, raw))
    else:
        _check(lib().jl_rope_attention_varlen_paged(*args, wp, workspace.nbytes, raw))
    return (out, lse) if want_lse else out


def debug_schedule(lengths, positions, w_pretrained: int, stream=None):
    """jl_debug_schedule: device-computed G(L), f(x), Delta(x) (int32 CUDA tensors)."""
    torch = _t()
    nl, npos = lengths.numel(), positions.numel()
    g = torch.empty(nl, dtype=torch.int32, device=lengths.device)
    f = torch.empty((nl, npos), dtype=torch.int32, device=lengths.device)
    dlt = torch.empty((nl, npos), dtype=torch.int32, device=lengths.device)
    _check(lib().jl_debug_schedule(_dev(lengths, "lengths", torch.int32), nl,
                                   _dev(positions, "positions", torch.int32), npos,
                                   int(w_pretrained), _dev(g, "g"), _dev(f, "f"), _dev(dlt, "d"),
                                   _stream(stream)))
    return g, f, dlt


def debug_prefill_tiles(L: int, Hq: int, Hkv: int, w_local: int, device="cuda", stream=None):
    """jl_debug_prefill_tiles: (classes int8 [n_qblocks, n_ktiles], block_q, block_k)."""
    torch = _t()
    bq, bk, nq, nk = (ctypes.c_int(), ctypes.c_int(), ctypes.c_int(), ctypes.c_int())
    # first call with no buffer reports the geometry
    lib().jl_debug_prefill_tiles(L, Hq, Hkv, w_local, None, 0, ctypes.byref(bq),
                                 ctypes.byref(bk), ctypes.byref(nq), ctypes.byref(nk), None)
    if nq.value <= 0:
        _check(JL_ERR_INVALID_ARG)
    out = torch.empty((nq.value, nk.value), dtype=torch.int8, device=device)
    _check(lib().jl_debug_prefill_tiles(L, Hq, Hkv, w_local, _dev(out, "classes"), out.numel(),
                                        ctypes.byref(bq), ctypes.byref(bk), ctypes.byref(nq),
                                        ctypes.byref(nk), _stream(stream)))
    return out, bq.value, bk.value


def release_caches() -> None:
    lib().jl_release_caches()


def debug_prefill_rescale_log2(log2_bound: float) -> float:
    """jl_debug_prefill_rescale_log2: set the prefill rescale bound, return the old one."""
    return float(lib().jl_debug_prefill_rescale_log2(float(log2_bound)))


def debug_kernel_events(which: int, start=None, stop=None) -> None:
    """jl_debug_kernel_events: record torch.cuda.Event pair (start, stop) around
    the prefill attention kernel (which = 0) or the decode split kernel
    (which = 1) of every later call; no events clears the hook."""
    def ev(e):
        if e is None:
            return None
        if e.cuda_event == 0:  # torch creates the HIP event at its first record
            e.record()
        return ctypes.c_void_p(e.cuda_event)
    _check(lib().jl_debug_kernel_events(int(which), ev(start), ev(stop)))
