"""ctypes binding of libsnapstream.so: argument marshalling only.

Every function mirrors one entry point of include/snapstream.h and takes torch tensors
(used purely as device memory) or raw integers.  Nothing is computed here; if the shared
library is missing the import of this module's symbols fails loudly -- there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

# SNAP_LIBRARY names another build of the library in this directory (the checked build, libsnapstream_dbg.so)
_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)),
                         os.path.basename(os.environ.get("SNAP_LIBRARY", "libsnapstream.so")))

SNAP_F32, SNAP_BF16 = 0, 1
SNAP_POOL_AVG, SNAP_POOL_MAX = 0, 1
SNAP_DEV_BAD_SLOT, SNAP_DEV_WAIT_TIMEOUT, SNAP_DEV_BAND_OVERFLOW, SNAP_DEV_INDEX_CHECK = 1, 2, 4, 8
SNAP_DEV_BAD_PAGE = 16
SNAP_ROPE_PLAIN, SNAP_ROPE_LINEAR, SNAP_ROPE_LLAMA3, SNAP_ROPE_YARN = range(4)


class SnapConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_q_heads", "n_kv_heads", "d_qk", "d_v", "v_aliases_k", "dtype",
                                         "l_sink", "l_recent", "topk", "l_obs", "pool_kernel", "pool_mode")]
    _fields_ += [("softmax_scale", C.c_float), ("max_seqs", C.c_int32)]


class SnapLayout(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("slots", "sink_off", "ring_off", "topk_off")]
    _fields_ += [(n, C.c_int64) for n in ("k_row_bytes", "v_row_bytes", "k_head_stride_bytes",
                                          "v_head_stride_bytes", "k_seq_stride_bytes", "v_seq_stride_bytes",
                                          "k_cache_bytes", "v_cache_bytes")]


class SnapRope(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rot_dim", "rot_offset", "interleaved", "scaling")]
    _fields_ += [(n, C.c_double) for n in ("base", "factor", "original_len", "low_freq", "high_freq", "beta_fast", "beta_slow",
                                           "magnitude")]


class SnapPaged(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("page_tokens", "n_pages", "max_pages", "reserved")]
    _fields_ += [(n, C.c_int64) for n in ("k_page_stride", "k_head_stride", "k_row_stride", "v_page_stride", "v_head_stride",
                                          "v_row_stride")]


class SnapError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} ({code})")


_lib = None


def lib() -> C.CDLL:
    """Load libsnapstream.so (built by paper_2511_03092_b200.build); raises if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is missing: run `python -m paper_2511_03092_b200.build` "
                           "(there is no CPU fallback)")
    L = C.CDLL(_LIB_PATH)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    pcfg, play = C.POINTER(SnapConfig), C.POINTER(SnapLayout)
    L.snap_status_string.restype = C.c_char_p
    L.snap_status_string.argtypes = [C.c_int]
    L.snap_kernel_launch_count.restype = i64
    L.snap_kernel_launch_count.argtypes = []
    L.snap_cache_layout.restype = C.c_int
    L.snap_cache_layout.argtypes = [pcfg, play]
    L.snap_compress_workspace_bytes.restype = i64
    L.snap_compress_workspace_bytes.argtypes = [pcfg, C.POINTER(i32), i32]
    L.snap_decode_workspace_bytes.restype = i64
    L.snap_decode_workspace_bytes.argtypes = [pcfg, i32]
    L.snap_compress.restype = C.c_int
    L.snap_compress.argtypes = [pcfg, play, vp, vp, i64, i64, vp, i64, i64, C.POINTER(i32), C.POINTER(i32), i32,
                                vp, vp, vp, vp, vp, vp, sz, vp, vp]
    L.snap_compress_with_row_stats.restype = C.c_int
    L.snap_compress_with_row_stats.argtypes = [pcfg, play, vp, vp, vp, i64, i64, vp, i64, i64, C.POINTER(i32),
                                               C.POINTER(i32), i32, vp, vp, vp, vp, vp, vp, sz, vp, vp]
    L.snap_prefill_attn.restype = C.c_int
    L.snap_prefill_attn.argtypes = [pcfg, vp, vp, i64, i64, vp, i64, i64, C.POINTER(i32), i32, vp, vp, vp, vp]
    L.snap_append_kv.restype = C.c_int
    L.snap_append_kv.argtypes = [pcfg, play, vp, vp, vp, i32, vp, vp, vp, vp, vp]
    L.snap_append_kv_concat.restype = C.c_int
    L.snap_append_kv_concat.argtypes = [pcfg, play, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp]
    L.snap_decode_attn.restype = C.c_int
    L.snap_decode_attn.argtypes = [pcfg, play, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp, vp]
    L.snap_decode_multi_workspace_bytes.restype = i64
    L.snap_decode_multi_workspace_bytes.argtypes = [pcfg, i32, i32]
    L.snap_decode_attn_multi.restype = C.c_int
    L.snap_decode_attn_multi.argtypes = [pcfg, play, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp, vp]
    L.snap_decode_attn_static.restype = C.c_int
    L.snap_decode_attn_static.argtypes = [pcfg, play, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp]
    L.snap_debug_set_option.restype = C.c_int
    L.snap_debug_set_option.argtypes = [C.c_int, C.c_int]
    L.snap_block_stats_bytes.restype = i64
    L.snap_block_stats_bytes.argtypes = [pcfg, i32]
    L.snap_block_stats.restype = C.c_int
    L.snap_block_stats.argtypes = [pcfg, play, vp, i32, vp, vp, i32, vp, vp, vp]
    L.snap_block_select.restype = C.c_int
    L.snap_block_select.argtypes = [pcfg, play, vp, vp, i32, vp, vp, i32, i32, vp, vp, vp, sz, vp, vp]
    L.snap_block_select_workspace_bytes.restype = i64
    L.snap_block_select_workspace_bytes.argtypes = [pcfg, i32, i32]
    L.snap_decode_blocks_workspace_bytes.restype = i64
    L.snap_decode_blocks_workspace_bytes.argtypes = [pcfg, i32, i32, i32]
    L.snap_decode_attn_blocks.restype = C.c_int
    L.snap_decode_attn_blocks.argtypes = [pcfg, play, vp, vp, vp, vp, i32, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp, sz, vp, vp]
    prope, ppaged = C.POINTER(SnapRope), C.POINTER(SnapPaged)
    L.snap_rope_table.restype = C.c_int
    L.snap_rope_table.argtypes = [prope, C.POINTER(C.c_double), C.POINTER(C.c_double)]
    L.snap_rope.restype = C.c_int
    L.snap_rope.argtypes = [pcfg, prope, vp, vp, i32] + [vp, i64, i64] * 4 + [i32, vp]
    L.snap_paged_append.restype = C.c_int
    L.snap_paged_append.argtypes = [pcfg, ppaged, vp, vp, i32, prope, vp, vp, vp, i64, i64, vp, vp, i64, i64, vp, vp, i64, i64,
                                    vp, vp, vp, vp, vp, vp, vp]
    L.snap_paged_decode_workspace_bytes.restype = i64
    L.snap_paged_decode_workspace_bytes.argtypes = [pcfg, ppaged, i32, i32]
    L.snap_paged_decode_attn.restype = C.c_int
    L.snap_paged_decode_attn.argtypes = [pcfg, ppaged, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp]
    L.snap_paged_evict_workspace_bytes.restype = i64
    L.snap_paged_evict_workspace_bytes.argtypes = [pcfg, ppaged, i32]
    L.snap_paged_evict.restype = C.c_int
    L.snap_paged_evict.argtypes = [pcfg, ppaged, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp]
    _lib = L
    return L


EXPORTS = ("snap_cache_layout", "snap_compress_workspace_bytes", "snap_decode_workspace_bytes",
           "snap_compress", "snap_append_kv", "snap_append_kv_concat", "snap_decode_attn",
           "snap_decode_multi_workspace_bytes", "snap_decode_attn_multi", "snap_decode_attn_static", "snap_status_string",
           "snap_kernel_launch_count", "snap_prefill_attn", "snap_compress_with_row_stats", "snap_debug_set_option",
           "snap_block_stats_bytes", "snap_block_stats", "snap_block_select", "snap_block_select_workspace_bytes",
           "snap_decode_blocks_workspace_bytes",
           "snap_decode_attn_blocks", "snap_rope_table", "snap_rope", "snap_paged_append", "snap_paged_decode_workspace_bytes",
           "snap_paged_decode_attn", "snap_paged_evict_workspace_bytes", "snap_paged_evict")

# testing / tuning options of snap_debug_set_option
(SNAP_OPT_SCORE_KERNEL, SNAP_OPT_DECODE_GQA_KERNEL, SNAP_OPT_DECODE_LATENT_KERNEL, SNAP_OPT_DECODE_NSPLIT,
 SNAP_OPT_SCORE_NSPLIT, SNAP_OPT_WIDE_STAGES, SNAP_OPT_PREFILL_KERNEL, SNAP_OPT_PREFILL_SINGLE_HEADS,
 SNAP_OPT_REFINE_OFF) = range(9)


def status_string(code: int) -> str:
    return lib().snap_status_string(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != 0:
        raise SnapError(int(code), where)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _i32_array(xs: Sequence[int]):
    return (C.c_int32 * len(xs))(*[int(x) for x in xs])


def make_config(*, n_q_heads, n_kv_heads, d_qk, d_v, dtype, l_sink, l_recent, topk, l_obs, pool_kernel,
                softmax_scale, max_seqs, pool_mode=SNAP_POOL_AVG, v_aliases_k=False) -> SnapConfig:
    if isinstance(dtype, torch.dtype):
        dtype = {torch.float32: SNAP_F32, torch.bfloat16: SNAP_BF16}[dtype]
    if isinstance(pool_mode, str):
        pool_mode = {"avg": SNAP_POOL_AVG, "max": SNAP_POOL_MAX}[pool_mode]
    return SnapConfig(n_q_heads, n_kv_heads, d_qk, d_v, int(bool(v_aliases_k)), dtype, l_sink, l_recent, topk,
                      l_obs, pool_kernel, pool_mode, float(softmax_scale), max_seqs)


def snap_debug_set_option(option: int, value: int) -> int:
    """Set a process-wide testing / tuning option; returns its previous value."""
    old = lib().snap_debug_set_option(int(option), int(value))
    if old < 0:
        raise SnapError(int(old), "snap_debug_set_option")
    return int(old)


def snap_kernel_launch_count() -> int:
    return int(lib().snap_kernel_launch_count())


def snap_cache_layout(cfg: SnapConfig) -> SnapLayout:
    lay = SnapLayout()
    _check(lib().snap_cache_layout(C.byref(cfg), C.byref(lay)), "snap_cache_layout")
    return lay


def snap_compress_workspace_bytes(cfg: SnapConfig, cu_seqlens: Sequence[int]) -> int:
    cu = _i32_array(cu_seqlens)
    n = lib().snap_compress_workspace_bytes(C.byref(cfg), cu, len(cu_seqlens) - 1)
    if n < 0:
        raise SnapError(int(n), "snap_compress_workspace_bytes")
    return int(n)


def snap_decode_workspace_bytes(cfg: SnapConfig, n_active: int) -> int:
    n = lib().snap_decode_workspace_bytes(C.byref(cfg), int(n_active))
    if n < 0:
        raise SnapError(int(n), "snap_decode_workspace_bytes")
    return int(n)


def snap_compress(cfg: SnapConfig, layout: SnapLayout, q_obs, k, v, cu_seqlens: Sequence[int],
                  slot_ids: Sequence[int], k_cache, v_cache, seq_len, valid_topk, topk_idx=None,
                  workspace=None, status=None, stream=None, k_strides=None, v_strides=None) -> None:
    """k, v: [total_tokens, Hkv, d] tensors (any strides with a dense last dim), or pass
    k_strides/v_strides = (token_stride, head_stride) in elements explicitly."""
    ks = k_strides if k_strides is not None else (k.stride(0), k.stride(1))
    if v is not None:
        vs = v_strides if v_strides is not None else (v.stride(0), v.stride(1))
    else:
        vs = (0, 0)
    cu = _i32_array(cu_seqlens)
    sl = _i32_array(slot_ids)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().snap_compress(C.byref(cfg), C.byref(layout), _ptr(q_obs), _ptr(k), ks[0], ks[1], _ptr(v),
                               vs[0], vs[1], cu, sl, len(slot_ids), _ptr(k_cache), _ptr(v_cache),
                               _ptr(seq_len), _ptr(valid_topk), _ptr(topk_idx), _ptr(workspace), ws_bytes,
                               _ptr(status), _stream(stream)), "snap_compress")


def snap_compress_with_row_stats(cfg: SnapConfig, layout: SnapLayout, q_obs, row_mu, k, v, cu_seqlens: Sequence[int],
                                 slot_ids: Sequence[int], k_cache, v_cache, seq_len, valid_topk, topk_idx=None,
                                 workspace=None, status=None, stream=None) -> None:
    """snap_compress with the Eq. 4 normalisers (row_mu: [n_seq, Hq, Lo] float32, as written by
    snap_prefill_attn) supplied instead of computed."""
    vs = (v.stride(0), v.stride(1)) if v is not None else (0, 0)
    cu = _i32_array(cu_seqlens)
    sl = _i32_array(slot_ids)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().snap_compress_with_row_stats(C.byref(cfg), C.byref(layout), _ptr(q_obs), _ptr(row_mu), _ptr(k),
                                              k.stride(0), k.stride(1), _ptr(v), vs[0], vs[1], cu, sl, len(slot_ids),
                                              _ptr(k_cache), _ptr(v_cache), _ptr(seq_len), _ptr(valid_topk),
                                              _ptr(topk_idx), _ptr(workspace), ws_bytes, _ptr(status),
                                              _stream(stream)), "snap_compress_with_row_stats")


def snap_prefill_attn(cfg: SnapConfig, q, k, v, cu_seqlens: Sequence[int], out, row_mu=None, status=None,
                      stream=None) -> None:
    """Causal attention of whole prompts.  q: [T, Hq, d] dense; k, v: [T, Hkv, d] (dense last dim; v None for
    the latent layout);
    out: [T, Hq, d_v]; row_mu: None or [n_seq, Hq, Lo] float32 receiving the Eq. 4 normalisers."""
    cu = _i32_array(cu_seqlens)
    vs = (v.stride(0), v.stride(1)) if v is not None else (0, 0)
    _check(lib().snap_prefill_attn(C.byref(cfg), _ptr(q), _ptr(k), k.stride(0), k.stride(1), _ptr(v), vs[0], vs[1], cu,
                                   len(cu_seqlens) - 1, _ptr(out), _ptr(row_mu), _ptr(status), _stream(stream)),
           "snap_prefill_attn")


def snap_append_kv(cfg: SnapConfig, layout: SnapLayout, k_new, v_new, slot_ids_dev, n_active: int, k_cache,
                   v_cache, seq_len, status=None, stream=None) -> None:
    _check(lib().snap_append_kv(C.byref(cfg), C.byref(layout), _ptr(k_new), _ptr(v_new), _ptr(slot_ids_dev),
                                int(n_active), _ptr(k_cache), _ptr(v_cache), _ptr(seq_len), _ptr(status),
                                _stream(stream)), "snap_append_kv")


def snap_append_kv_concat(cfg: SnapConfig, layout: SnapLayout, k_new, v_new, slot_ids_dev, n_active: int,
                          k_cache_in, v_cache_in, k_cache_out, v_cache_out, seq_len, status=None,
                          stream=None) -> None:
    """Baseline update by slicing and concatenating into a second cache (position-ordered window)."""
    _check(lib().snap_append_kv_concat(C.byref(cfg), C.byref(layout), _ptr(k_new), _ptr(v_new),
                                       _ptr(slot_ids_dev), int(n_active), _ptr(k_cache_in), _ptr(v_cache_in),
                                       _ptr(k_cache_out), _ptr(v_cache_out), _ptr(seq_len), _ptr(status),
                                       _stream(stream)), "snap_append_kv_concat")


def snap_decode_attn(cfg: SnapConfig, layout: SnapLayout, q, k_new, v_new, slot_ids_dev, n_active: int,
                     k_cache, v_cache, seq_len, valid_topk, out, workspace, status=None, stream=None) -> None:
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().snap_decode_attn(C.byref(cfg), C.byref(layout), _ptr(q), _ptr(k_new), _ptr(v_new),
                                  _ptr(slot_ids_dev), int(n_active), _ptr(k_cache), _ptr(v_cache),
                                  _ptr(seq_len), _ptr(valid_topk), _ptr(out), _ptr(workspace), ws_bytes,
                                  _ptr(status), _stream(stream)), "snap_decode_attn")


def snap_decode_multi_workspace_bytes(cfg: SnapConfig, n_active: int, q_len: int) -> int:
    n = lib().snap_decode_multi_workspace_bytes(C.byref(cfg), int(n_active), int(q_len))
    if n < 0:
        raise SnapError(int(n), "snap_decode_multi_workspace_bytes")
    return int(n)


def snap_decode_attn_multi(cfg: SnapConfig, layout: SnapLayout, q, k_new, v_new, slot_ids_dev, n_active: int,
                           q_len: int, k_cache, v_cache, seq_len, valid_topk, out, workspace, status=None,
                           stream=None) -> None:
    """q_len new tokens per sequence in one pass over the cache (q [n][q_len][Hq][d], out alike)."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().snap_decode_attn_multi(C.byref(cfg), C.byref(layout), _ptr(q), _ptr(k_new), _ptr(v_new),
                                        _ptr(slot_ids_dev), int(n_active), int(q_len), _ptr(k_cache),
                                        _ptr(v_cache), _ptr(seq_len), _ptr(valid_topk), _ptr(out),
                                        _ptr(workspace), ws_bytes, _ptr(status), _stream(stream)),
           "snap_decode_attn_multi")


def snap_decode_attn_static(cfg: SnapConfig, layout: SnapLayout, q, k_new, v_new, slot_ids_dev, n_active: int,
                            k_cache, v_cache, seq_len, valid_topk, out, status=None, stream=None) -> None:
    """Decode step without a workspace argument: scratch is a fixed array inside the library, for
    callers that must not allocate.  Raises SnapError(-6) when the batch does not fit that array."""
    _check(lib().snap_decode_attn_static(C.byref(cfg), C.byref(layout), _ptr(q), _ptr(k_new), _ptr(v_new),
                                         _ptr(slot_ids_dev), int(n_active), _ptr(k_cache), _ptr(v_cache),
                                         _ptr(seq_len), _ptr(valid_topk), _ptr(out), _ptr(status),
                                         _stream(stream)), "snap_decode_attn_static")


@dataclass
class CacheBuffers:
    """Device buffers of one layer's compressed cache (torch is used only as the allocator)."""
    k_cache: torch.Tensor
    v_cache: Optional[torch.Tensor]
    seq_len: torch.Tensor
    valid_topk: torch.Tensor
    status: torch.Tensor


def alloc_cache(cfg: SnapConfig, layout: SnapLayout, device="cuda") -> CacheBuffers:
    dt = torch.float32 if cfg.dtype == SNAP_F32 else torch.bfloat16
    kc = torch.zeros(cfg.max_seqs, cfg.n_kv_heads, layout.slots, cfg.d_qk, dtype=dt, device=device)
    vc = None
    if not cfg.v_aliases_k:
        vc = torch.zeros(cfg.max_seqs, cfg.n_kv_heads, layout.slots, cfg.d_v, dtype=dt, device=device)
    return CacheBuffers(kc, vc, torch.zeros(cfg.max_seqs, dtype=torch.int32, device=device),
                        torch.zeros(cfg.max_seqs, dtype=torch.int32, device=device),
                        torch.zeros(1, dtype=torch.int32, device=device))


def snap_block_stats_bytes(cfg: SnapConfig, block_tokens: int) -> int:
    n = lib().snap_block_stats_bytes(C.byref(cfg), int(block_tokens))
    if n < 0:
        raise SnapError(int(n), "snap_block_stats_bytes")
    return int(n)


def snap_block_stats(cfg: SnapConfig, layout: SnapLayout, slot_ids_dev, n_seqs: int, k_cache, valid_topk,
                     block_tokens: int, stats, status=None, stream=None) -> None:
    """Per-block key minima and maxima of the third section of the given slots' caches."""
    _check(lib().snap_block_stats(C.byref(cfg), C.byref(layout), _ptr(slot_ids_dev), int(n_seqs), _ptr(k_cache),
                                  _ptr(valid_topk), int(block_tokens), _ptr(stats), _ptr(status), _stream(stream)),
           "snap_block_stats")


def snap_block_select(cfg: SnapConfig, layout: SnapLayout, q, slot_ids_dev, n_active: int, stats, valid_topk,
                      block_tokens: int, n_blocks: int, block_idx, n_selected, workspace, status=None, stream=None) -> None:
    """The n_blocks highest-scoring blocks per (sequence, KV head) for this step's queries."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().snap_block_select(C.byref(cfg), C.byref(layout), _ptr(q), _ptr(slot_ids_dev), int(n_active), _ptr(stats),
                                   _ptr(valid_topk), int(block_tokens), int(n_blocks), _ptr(block_idx), _ptr(n_selected),
                                   _ptr(workspace), ws_bytes, _ptr(status), _stream(stream)), "snap_block_select")


def snap_block_select_workspace_bytes(cfg: SnapConfig, n_active: int, block_tokens: int) -> int:
    n = lib().snap_block_select_workspace_bytes(C.byref(cfg), int(n_active), int(block_tokens))
    if n < 0:
        raise SnapError(int(n), "snap_block_select_workspace_bytes")
    return int(n)


def snap_decode_blocks_workspace_bytes(cfg: SnapConfig, n_active: int, block_tokens: int, n_blocks: int) -> int:
    n = lib().snap_decode_blocks_workspace_bytes(C.byref(cfg), int(n_active), int(block_tokens), int(n_blocks))
    if n < 0:
        raise SnapError(int(n), "snap_decode_blocks_workspace_bytes")
    return int(n)


def snap_decode_attn_blocks(cfg: SnapConfig, layout: SnapLayout, q, k_new, v_new, slot_ids_dev, n_active: int, k_cache,
                            v_cache, seq_len, valid_topk, block_tokens: int, n_blocks: int, block_idx, n_selected, out,
                            workspace, status=None, stream=None) -> None:
    """snap_decode_attn over the sinks, the window and the listed blocks of the third section."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().snap_decode_attn_blocks(C.byref(cfg), C.byref(layout), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(slot_ids_dev),
                                         int(n_active), _ptr(k_cache), _ptr(v_cache), _ptr(seq_len), _ptr(valid_topk),
                                         int(block_tokens), int(n_blocks), _ptr(block_idx), _ptr(n_selected), _ptr(out),
                                         _ptr(workspace), ws_bytes, _ptr(status), _stream(stream)), "snap_decode_attn_blocks")


# --- rotary positions and the paged cache ---
# The library sees addresses only, so the tensors of these calls are checked first (type, shape, strides, device), by the
# compiled module _marshal: a serving step makes them once per layer.  What it turns down, _refuse finds the words for.
_DTYPES = {SNAP_F32: torch.float32, SNAP_BF16: torch.bfloat16}
_I32, _F32, _F64 = torch.int32, torch.float32, torch.float64
_native = None


def _calls():
    """(the module _marshal, addresses of the entry points it calls); raises if either is absent."""
    global _native
    if _native is None:
        L = lib()
        try:
            from . import _marshal
        except ImportError as e:
            raise RuntimeError(f"the module _marshal is missing ({e}): run `python -m paper_2511_03092_b200.build`") from e
        if getattr(_marshal, "torch_version", "") != str(torch.__version__):
            raise RuntimeError(f"the module _marshal is not built for torch {torch.__version__}: run `python -m paper_2511_03092_b200.build`")
        _native = (_marshal, {name: C.cast(getattr(L, name), C.c_void_p).value
                              for name in ("snap_rope", "snap_paged_append", "snap_paged_decode_attn", "snap_paged_evict")})
    return _native


def _refuse(where: str, *named) -> None:
    """Raise for the first of (name, tensor or None, dtype, shape or None, dense) that is not what the call is told it is."""
    for name, t, dtype, shape, dense in named:
        if t is None:
            continue
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{where}: {name} is a {type(t).__name__}, not a tensor")
        if dtype is not None and t.dtype != dtype:
            raise ValueError(f"{where}: {name} is {t.dtype}, expected {dtype}")
        if shape is not None and tuple(t.shape) != tuple(shape):
            raise ValueError(f"{where}: {name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
        if dense and not t.is_contiguous():
            raise ValueError(f"{where}: {name} must be dense")
        if not dense and t.stride()[-1] != 1:
            raise ValueError(f"{where}: {name} needs a dense last dim")
    device = None
    for name, t, *_ in named:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError(f"{where}: {name} is not on a CUDA device")
        if device is None:
            device = t.get_device()
        if t.get_device() != device:
            raise ValueError(f"{where}: {name} is on device {t.get_device()}, not {device}")
    if device is not None and device != torch.cuda.current_device():
        raise ValueError(f"{where}: the tensors are on device {device}, the current device is {torch.cuda.current_device()}")
    raise ValueError(f"{where}: a tensor is missing, or the pages' strides are not those of the description")


def _count(where: str, name: str, n) -> int:
    if int(n) >= 2 ** 31:
        raise ValueError(f"{where}: {name} counts {int(n)}, at most 2^31 - 1")
    return int(n)


def _tokens(where: str, name: str, t) -> int:
    """Length of the list whose entries are the call's tokens."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{where}: {name} is a {type(t).__name__}, not a tensor")
    if t.dim() != 1:
        raise ValueError(f"{where}: {name} has shape {tuple(t.shape)}, expected one dim")
    return _count(where, name, t.shape[0])


def _answer(status: Optional[int], where: str, named) -> None:
    """Raise for a call's status; None: a tensor was turned down (only then are the arguments looked at)."""
    if status is None:
        _refuse(where, *named())
    _check(status, where)


def _handle(stream):
    return None if stream is None else _stream(stream)


def make_rope(*, rot_dim: int, rot_offset: int = 0, interleaved: bool = False, scaling="plain", base: float = 10000.0,
              factor: float = 1.0, original_len: float = 0.0, low_freq: float = 1.0, high_freq: float = 4.0,
              beta_fast: float = 32.0, beta_slow: float = 1.0, magnitude: float = 0.0) -> SnapRope:
    if isinstance(scaling, str):
        scaling = {"plain": SNAP_ROPE_PLAIN, "linear": SNAP_ROPE_LINEAR, "llama3": SNAP_ROPE_LLAMA3, "yarn": SNAP_ROPE_YARN}[scaling]
    return SnapRope(int(rot_dim), int(rot_offset), int(bool(interleaved)), int(scaling), float(base), float(factor), float(original_len),
                    float(low_freq), float(high_freq), float(beta_fast), float(beta_slow), float(magnitude))


def snap_rope_table(rope: SnapRope):
    """(frequencies [rot_dim / 2] float64 on the host, magnitude)."""
    freqs, magnitude = (C.c_double * max(rope.rot_dim // 2, 1))(), C.c_double()
    _check(lib().snap_rope_table(C.byref(rope), freqs, C.byref(magnitude)), "snap_rope_table")
    return torch.tensor(list(freqs), dtype=torch.float64), magnitude.value


def snap_rope(cfg: SnapConfig, rope: SnapRope, freqs, positions, q=None, k=None, q_out=None, k_out=None, inverse: bool = False,
              stream=None) -> None:
    """Rotate q [T, Hq, d] and / or k [T, Hkv, d] (any strides with a dense last dim) into q_out and k_out, which may be
    the inputs themselves.  freqs: float64 [rot_dim / 2], positions: int32 [T], on the device.  inverse: by minus the
    angle (the gradient's direction)."""
    native, entry = _native or _calls()
    status = native.rope(entry["snap_rope"], cfg, rope, freqs, positions, q, k, q_out, k_out, 1 if inverse else 0, _handle(stream))
    if status != 0:
        def named():
            n, dt = _tokens("snap_rope", "positions", positions), _DTYPES.get(cfg.dtype)
            sq, sk = (n, cfg.n_q_heads, cfg.d_qk), (n, cfg.n_kv_heads, cfg.d_qk)
            return (("freqs", freqs, _F64, (rope.rot_dim // 2,), True), ("positions", positions, _I32, (n,), True), ("q", q, dt, sq, False),
                    ("k", k, dt, sk, False), ("q_out", q_out, dt, sq, False), ("k_out", k_out, dt, sk, False))
        _answer(status, "snap_rope", named)


def make_paged(k_pages, v_pages, page_table) -> SnapPaged:
    """Describe a paged cache: k_pages [n_pages, Hkv, page_tokens, d_qk], v_pages [n_pages, Hkv, page_tokens, d_v] (any
    strides with a dense last dim: pages stored rows first are passed as their transposed view), page_table
    [max_seqs, max_pages]."""
    if k_pages.dim() != 4 or v_pages.dim() != 4 or k_pages.shape[:3] != v_pages.shape[:3] or page_table.dim() != 2:
        raise ValueError("make_paged: k_pages and v_pages are [pages, heads, rows, dim], page_table [seqs, pages]")
    (kp, kh, kr, _), (vp, vh, vr, _) = k_pages.stride(), v_pages.stride()
    return SnapPaged(k_pages.shape[2], k_pages.shape[0], page_table.shape[1], 0, kp, kh, kr, vp, vh, vr)


def _paged_named(cfg, paged, dt, k_pages, v_pages, page_table, seq_len, status):
    head = (paged.n_pages, cfg.n_kv_heads, paged.page_tokens)
    return (("k_pages", k_pages, dt, head + (cfg.d_qk,), False), ("v_pages", v_pages, dt, head + (cfg.d_v,), False),
            ("page_table", page_table, _I32, (cfg.max_seqs, paged.max_pages), True), ("seq_len", seq_len, _I32, (cfg.max_seqs,), True),
            ("status", status, _I32, None, True))


def _weights_shape(cfg, paged):
    return (cfg.max_seqs, cfg.n_kv_heads, paged.max_pages * paged.page_tokens)


def snap_paged_append(cfg: SnapConfig, paged: SnapPaged, slot_ids_dev, rows_dev, k, v, k_pages, v_pages, page_table, seq_len,
                      rope: Optional[SnapRope] = None, freqs=None, positions=None, q=None, q_out=None, k_out=None, weights=None,
                      status=None, stream=None) -> None:
    """Write the rows of k [T, Hkv, d_qk], v [T, Hkv, d_v] into the pages, rotated on the way when rope is given; rows_dev
    None: each token is its sequence's next row.  q -> q_out and k_out: the rotated queries and keys, dense."""
    native, entry = _native or _calls()
    status_code = native.paged_append(entry["snap_paged_append"], cfg, paged, slot_ids_dev, rows_dev, k, v, k_pages, v_pages, page_table,
                                      seq_len, rope, freqs, positions, q, q_out, k_out, weights, status, _handle(stream))
    if status_code != 0:
        def named():
            n, dt, hkv = _tokens("snap_paged_append", "slot_ids", slot_ids_dev), _DTYPES.get(cfg.dtype), cfg.n_kv_heads
            sq, sk, sv, one = (n, cfg.n_q_heads, cfg.d_qk), (n, hkv, cfg.d_qk), (n, hkv, cfg.d_v), (n,)
            return (("slot_ids", slot_ids_dev, _I32, one, True), ("rows", rows_dev, _I32, one, True),
                    ("freqs", freqs, _F64, None if rope is None else (rope.rot_dim // 2,), True), ("positions", positions, _I32, one, True),
                    ("q", q, dt, sq, False), ("q_out", q_out, dt, sq, True), ("k", k, dt, sk, False), ("k_out", k_out, dt, sk, True),
                    ("v", v, dt, sv, False), ("weights", weights, _F32, _weights_shape(cfg, paged), True),
                    *_paged_named(cfg, paged, dt, k_pages, v_pages, page_table, seq_len, status))
        _answer(status_code, "snap_paged_append", named)


def snap_paged_decode_workspace_bytes(cfg: SnapConfig, paged: SnapPaged, n_active: int, with_weights: bool = False) -> int:
    n = lib().snap_paged_decode_workspace_bytes(C.byref(cfg), C.byref(paged), int(n_active), int(bool(with_weights)))
    if n < 0:
        raise SnapError(int(n), "snap_paged_decode_workspace_bytes")
    return int(n)


def snap_paged_decode_attn(cfg: SnapConfig, paged: SnapPaged, q, slot_ids_dev, n_active: int, k_pages, v_pages, page_table,
                           seq_len, out, workspace, weights_in=None, weights_out=None, status=None, stream=None) -> None:
    """Attention of one token per sequence, q [n, Hq, d_qk] -> out [n, Hq, d_v], over the rows in its pages; weights_out
    [max_seqs, Hkv, max_pages * page_tokens] float32 receives weights_in (None = 0) plus the group's softmax weights."""
    native, entry = _native or _calls()
    status_code = native.paged_decode_attn(entry["snap_paged_decode_attn"], cfg, paged, q, slot_ids_dev, n_active, k_pages, v_pages,
                                           page_table, seq_len, out, workspace, weights_in, weights_out, status, _handle(stream))
    if status_code != 0:
        def named():
            n, dt, sw = _count("snap_paged_decode_attn", "n_active", n_active), _DTYPES.get(cfg.dtype), _weights_shape(cfg, paged)
            return (("q", q, dt, (n, cfg.n_q_heads, cfg.d_qk), True), ("out", out, dt, (n, cfg.n_q_heads, cfg.d_v), True),
                    ("slot_ids", slot_ids_dev, _I32, (n,), True), ("weights_in", weights_in, _F32, sw, True),
                    ("weights_out", weights_out, _F32, sw, True), ("workspace", workspace, None, None, True),
                    *_paged_named(cfg, paged, dt, k_pages, v_pages, page_table, seq_len, status))
        _answer(status_code, "snap_paged_decode_attn", named)


def snap_paged_evict_workspace_bytes(cfg: SnapConfig, paged: SnapPaged, n_seqs: int) -> int:
    n = lib().snap_paged_evict_workspace_bytes(C.byref(cfg), C.byref(paged), int(n_seqs))
    if n < 0:
        raise SnapError(int(n), "snap_paged_evict_workspace_bytes")
    return int(n)


def snap_paged_evict(cfg: SnapConfig, paged: SnapPaged, src_slots_dev, dst_slots_dev, n_seqs: int, k_pages, v_pages, page_table,
                     seq_len, weights_in, weights_out, workspace, kept_rows=None, status=None, stream=None) -> None:
    """Copy the rows that stay (sinks, the topk of the middle by weight, the recent ones) of each source slot to its
    destination slot's pages; kept_rows [n, Hkv, l_sink + topk + l_recent] int32 receives their source rows."""
    native, entry = _native or _calls()
    status_code = native.paged_evict(entry["snap_paged_evict"], cfg, paged, src_slots_dev, dst_slots_dev, n_seqs, k_pages, v_pages,
                                     page_table, seq_len, weights_in, weights_out, workspace, kept_rows, status, _handle(stream))
    if status_code != 0:
        def named():
            n, dt, sw = _count("snap_paged_evict", "n_seqs", n_seqs), _DTYPES.get(cfg.dtype), _weights_shape(cfg, paged)
            return (("src_slots", src_slots_dev, _I32, (n,), True), ("dst_slots", dst_slots_dev, _I32, (n,), True),
                    ("weights_in", weights_in, _F32, sw, True), ("weights_out", weights_out, _F32, sw, True),
                    ("kept_rows", kept_rows, _I32, (n, cfg.n_kv_heads, cfg.l_sink + cfg.topk + cfg.l_recent), True),
                    ("workspace", workspace, None, None, True),
                    *_paged_named(cfg, paged, dt, k_pages, v_pages, page_table, seq_len, status))
        _answer(status_code, "snap_paged_evict", named)
