"""ctypes binding of ``libpda.so`` with the C ABI's own names.

Argument marshalling only: tensors are torch CUDA tensors whose ``data_ptr``s,
shapes and strides are passed straight to the C entry points declared in
``include/pda.h``. There is no fallback: if the library is missing or a call
fails, a ``RuntimeError`` is raised.
"""
from __future__ import annotations

import contextlib
import functools
import ctypes as C
import operator
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpda.so")

PDA_BF16, PDA_FP8_E4M3 = 0, 1
PDA_FLAG_FORCE_GENERIC = 1
PDA_FLAG_MQ_MMA_SYNC = 2
PDA_FLAG_MQ_ONE_UNIT = 4
DEV_STATUS = {0: "ok", 1: "bad page id", 2: "seq_len exceeds block table", 3: "copy wait timed out",
              4: "too few free pages", 5: "too few slot map entries"}

EXPORTS = ["pda_version", "pda_status_string", "pda_max_chunks", "kv_append",
           "paged_decode_attention", "paged_decode_reduce", "paged_decode_step_host",
           "pda_debug_e4m3_decode", "paged_decode_attention_static", "pda_workspace_ints",
           "paged_decode_step", "pda_advance_seq_lens", "paged_window_decode_attention", "kv_append_tokens",
           "paged_verify_attention", "paged_prefix_decode_attention", "kv_append_fp8", "kv_append_tokens_fp8",
           "pda_set_persistent_threshold", "pda_debug_wait_timeout", "pda_debug_read_probe",
           "paged_build_tables", "latent_append", "paged_latent_attention", "pda_latent_workspace_bytes",
           "latent_prefill_attention", "rope_kv_append", "paged_prefill_attention", "pda_prefill_workspace_bytes",
           "paged_biased_decode_attention"]
STATIC_SCRATCH_BYTES = 16 * 1024 * 1024


class CacheDesc(C.Structure):
    _fields_ = [("page_stride", C.c_int64), ("head_stride", C.c_int64), ("slot_stride", C.c_int64),
                ("num_pages", C.c_int32), ("page_size", C.c_int32), ("num_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32)]


class LatentDesc(C.Structure):
    _fields_ = [("page_stride", C.c_int64), ("slot_stride", C.c_int64), ("num_pages", C.c_int32),
                ("page_size", C.c_int32), ("latent_dim", C.c_int32), ("rope_dim", C.c_int32), ("dtype", C.c_int32)]


class ScoreDesc(C.Structure):
    _fields_ = [("scale", C.c_float), ("softcap", C.c_float), ("slopes", C.c_void_p), ("window", C.c_int32)]


_lib = None


def lib():
    """Loads ``libpda.so`` on first use; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} not found: build it with `python -m paper_2605_06068_b200.build` "
                "(there is no CPU or PyTorch fallback)")
        L = C.CDLL(LIB_PATH)
        L.pda_status_string.restype = C.c_char_p
        L.pda_status_string.argtypes = [C.c_int]
        vp, i32, f32, u32 = C.c_void_p, C.c_int32, C.c_float, C.c_uint32
        dp = C.POINTER(CacheDesc)
        L.pda_max_chunks.argtypes = [i32, i32]
        L.kv_append.argtypes = [vp, vp, vp, vp, dp, vp, i32, vp, i32, vp, vp]
        L.paged_decode_attention.argtypes = [vp, vp, vp, dp, vp, vp, vp, i32, vp, i32, i32, f32,
                                             i32, vp, vp, vp, i32, u32, vp, vp]
        L.paged_decode_reduce.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, vp, vp]
        L.paged_decode_step_host.argtypes = [vp] * 5 + [vp] * 5 + [vp, vp, dp, i32, i32, i32, f32,
                                                                 i32, vp, vp, i32, vp, vp, vp, vp, vp]
        L.pda_workspace_ints.argtypes = [i32, i32]
        L.pda_set_persistent_threshold.argtypes = [i32]
        L.kv_append_fp8.argtypes = [vp, vp, vp, vp, dp, vp, vp, vp, i32, vp, i32, vp, vp]
        L.kv_append_tokens_fp8.argtypes = [vp, vp, vp, vp, dp, vp, vp, vp, i32, vp, i32, i32, vp, vp]
        L.kv_append_tokens.argtypes = [vp, vp, vp, vp, dp, vp, i32, vp, i32, i32, vp, vp]
        L.paged_verify_attention.argtypes = [vp, vp, vp, dp, vp, vp, vp, i32, vp, i32, i32, i32, f32,
                                             i32, vp, vp, vp, i32, u32, vp, vp]
        L.paged_prefix_decode_attention.argtypes = [vp, vp, vp, dp, vp, vp, vp, i32, vp, i32, i32, f32,
                                                    i32, i32, i32, vp, vp, vp, i32, u32, vp, vp]
        L.paged_window_decode_attention.argtypes = [vp, vp, vp, dp, vp, vp, vp, i32, vp, i32, i32, f32,
                                                    i32, i32, vp, vp, vp, i32, u32, vp, vp]
        L.pda_advance_seq_lens.argtypes = [vp, i32, i32, vp]
        L.paged_decode_step.argtypes = [vp, vp, vp, vp, vp, dp, vp, vp, vp, i32, vp, i32, i32, f32,
                                        i32, vp, vp, vp, i32, vp, vp, vp]
        L.pda_debug_e4m3_decode.argtypes = [vp, vp]
        L.pda_debug_wait_timeout.argtypes = [u32, vp, vp, vp]
        L.pda_debug_read_probe.argtypes = [vp, C.c_uint64, vp, vp]
        L.paged_decode_attention_static.argtypes = [vp, vp, vp, dp, vp, vp, vp, i32, vp, i32, i32,
                                                    f32, i32, i32, vp, vp, vp]
        i64, lp = C.c_int64, C.POINTER(LatentDesc)
        L.paged_build_tables.argtypes = [vp, vp, i32, i32, vp, i32, vp, vp, vp, i32, vp, vp, vp, i32, vp, vp]
        L.latent_append.argtypes = [vp, i64, vp, i64, vp, lp, vp, f32, vp, i32, vp, vp]
        L.paged_latent_attention.argtypes = [vp, i64, i64, vp, i64, i64, vp, lp, vp, i32, vp, i32, i32, i32, f32,
                                             vp, i64, i64, vp, i64, u32, vp, vp]
        L.pda_latent_workspace_bytes.restype = i64
        L.pda_latent_workspace_bytes.argtypes = [i32, i32, i32, i32]
        L.latent_prefill_attention.argtypes = [vp, i64, i64, vp, i64, i64, vp, i64, vp, i64, i64, vp, vp, i32, i32,
                                               i32, i32, i32, i32, i32, i32, f32, vp, i64, i64, u32, vp, vp]
        sp = C.POINTER(ScoreDesc)
        L.rope_kv_append.argtypes = [vp, i64, i64, vp, i64, i64, vp, i64, i64, vp, i64, i32, vp, vp, i32, i32, i32, vp, vp, f32, vp,
                                     i32, i32, vp, i64, i64, vp, vp, dp, vp, vp, vp, vp]
        L.paged_prefill_attention.argtypes = [vp, i64, i64, vp, vp, dp, vp, vp, vp, i32, vp, vp, i32, i32, i32, i32, sp, vp, vp, vp,
                                              i64, i64, vp, i64, u32, vp, vp]
        L.pda_prefill_workspace_bytes.restype = i64
        L.pda_prefill_workspace_bytes.argtypes = [i32, i32]
        L.paged_biased_decode_attention.argtypes = [vp, vp, vp, dp, vp, vp, vp, i32, vp, i32, i32, sp, vp, i32, vp, vp, vp, i32, vp,
                                                    u32, vp, vp]
        _lib = L
    return _lib


def status_string(code: int) -> str:
    return lib().pda_status_string(int(code)).decode()


def _check(rc: int, what: str):
    if rc != 0:
        raise RuntimeError(f"{what} failed with code {rc}: {status_string(rc)}")


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is not None:
        return C.c_void_p(stream.cuda_stream)
    if _raw_stream is not None:   # the current stream's handle without building a Stream object (~10x cheaper)
        return C.c_void_p(_raw_stream(torch.cuda.current_device()))
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def cache_desc(cache: torch.Tensor) -> CacheDesc:
    """Descriptor of a ``[num_pages, Hkv, P, D]`` cache tensor (bf16, or uint8 /
    float8_e4m3fn for e4m3)."""
    assert cache.dim() == 4 and cache.stride(3) == 1
    if cache.dtype == torch.bfloat16:
        dt = PDA_BF16
    elif cache.dtype in (torch.uint8, torch.float8_e4m3fn):
        dt = PDA_FP8_E4M3
    else:
        raise TypeError(f"unsupported cache dtype {cache.dtype}")
    n, Hkv, P, D = cache.shape
    return CacheDesc(cache.stride(0), cache.stride(1), cache.stride(2), n, P, Hkv, D, dt)


def max_chunks(max_seq_len: int, chunk_tokens: int) -> int:
    return int(lib().pda_max_chunks(max_seq_len, chunk_tokens))


def kv_append(k_new, v_new, k_cache, v_cache, block_table, seq_lens, status=None, stream=None):
    desc = cache_desc(k_cache)
    assert k_new.is_contiguous() and v_new.is_contiguous() and block_table.stride(1) == 1
    assert v_cache.stride() == k_cache.stride() and v_cache.shape == k_cache.shape
    rc = lib().kv_append(_ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), C.byref(desc),
                         _ptr(block_table), block_table.stride(0), _ptr(seq_lens),
                         seq_lens.shape[0], _ptr(status), _stream(stream))
    _check(rc, "kv_append")


def paged_decode_attention(q, k_cache, v_cache, block_table, seq_lens, scale, chunk_tokens=0,
                           out=None, part_o=None, part_lse=None, k_scale=None, v_scale=None,
                           flags=0, status=None, stream=None):
    """Unsplit (``chunk_tokens == 0``): fills and returns ``out`` ``[B,Hq,D]`` bf16.
    Split: fills ``part_o`` ``[B,Hq,C,D]`` / ``part_lse`` ``[B,Hq,C]`` fp32 and returns them."""
    desc = cache_desc(k_cache)
    assert q.is_contiguous() and q.dtype == torch.bfloat16 and block_table.stride(1) == 1
    assert v_cache.stride() == k_cache.stride() and v_cache.shape == k_cache.shape
    B, Hq, D = q.shape
    mc = 0
    if chunk_tokens == 0:
        if out is None:
            out = torch.empty_like(q)
    else:
        assert part_o is not None and part_lse is not None
        assert part_o.is_contiguous() and part_lse.is_contiguous()
        mc = part_o.shape[2]
        assert tuple(part_o.shape) == (B, Hq, mc, D) and tuple(part_lse.shape) == (B, Hq, mc)
    rc = lib().paged_decode_attention(
        _ptr(q), _ptr(k_cache), _ptr(v_cache), C.byref(desc), _ptr(k_scale), _ptr(v_scale),
        _ptr(block_table), block_table.stride(0), _ptr(seq_lens), B, Hq, float(scale),
        chunk_tokens, _ptr(out), _ptr(part_o), _ptr(part_lse), mc, flags, _ptr(status),
        _stream(stream))
    _check(rc, "paged_decode_attention")
    return out if chunk_tokens == 0 else (part_o, part_lse)


def paged_window_decode_attention(q, k_cache, v_cache, block_table, seq_lens, scale, window,
                                  chunk_tokens=0, out=None, part_o=None, part_lse=None,
                                  k_scale=None, v_scale=None, flags=0, status=None, stream=None):
    """``paged_decode_attention`` over each sequence's last ``window`` tokens only."""
    desc = cache_desc(k_cache)
    B, Hq, D = q.shape
    mc = 0
    if chunk_tokens == 0:
        if out is None:
            out = torch.empty_like(q)
    else:
        mc = part_o.shape[2]
        assert tuple(part_o.shape) == (B, Hq, mc, D) and tuple(part_lse.shape) == (B, Hq, mc)
    rc = lib().paged_window_decode_attention(
        _ptr(q), _ptr(k_cache), _ptr(v_cache), C.byref(desc), _ptr(k_scale), _ptr(v_scale),
        _ptr(block_table), block_table.stride(0), _ptr(seq_lens), B, Hq, float(scale), int(window),
        chunk_tokens, _ptr(out), _ptr(part_o), _ptr(part_lse), mc, flags, _ptr(status),
        _stream(stream))
    _check(rc, "paged_window_decode_attention")
    return out if chunk_tokens == 0 else (part_o, part_lse)


def paged_decode_reduce(part_o, part_lse, seq_lens, chunk_tokens, out=None, stream=None):
    B, Hq, mc, D = part_o.shape
    if out is None:
        out = torch.empty((B, Hq, D), dtype=torch.bfloat16, device=part_o.device)
    rc = lib().paged_decode_reduce(_ptr(part_o), _ptr(part_lse), _ptr(seq_lens), B, Hq, D,
                                   chunk_tokens, mc, _ptr(out), _stream(stream))
    _check(rc, "paged_decode_reduce")
    return out


def workspace_ints(batch: int, num_kv_heads: int) -> int:
    return int(lib().pda_workspace_ints(batch, num_kv_heads))


def new_workspace(batch: int, num_kv_heads: int, device="cuda") -> torch.Tensor:
    """Zeroed int32 workspace for ``paged_decode_step`` (zero it once; calls leave it zeroed)."""
    return torch.zeros(workspace_ints(batch, num_kv_heads), dtype=torch.int32, device=device)


def paged_decode_step(q, k_new, v_new, k_cache, v_cache, block_table, seq_lens, scale,
                      chunk_tokens=0, out=None, part_o=None, part_lse=None, workspace=None,
                      k_scale=None, v_scale=None, status=None, stream=None):
    """Fused append + attention (+ reduce) in one launch; fills and returns ``out``."""
    desc = cache_desc(k_cache)
    assert q.is_contiguous() and q.dtype == torch.bfloat16 and block_table.stride(1) == 1
    B, Hq, D = q.shape
    if out is None:
        out = torch.empty_like(q)
    mc = 0
    if chunk_tokens:
        mc = part_o.shape[2]
        assert tuple(part_o.shape) == (B, Hq, mc, D) and tuple(part_lse.shape) == (B, Hq, mc)
    rc = lib().paged_decode_step(
        _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), C.byref(desc),
        _ptr(k_scale), _ptr(v_scale), _ptr(block_table), block_table.stride(0), _ptr(seq_lens),
        B, Hq, float(scale), chunk_tokens, _ptr(out), _ptr(part_o), _ptr(part_lse), mc,
        _ptr(workspace), _ptr(status), _stream(stream))
    _check(rc, "paged_decode_step")
    return out


def paged_decode_step_host(q_host, k_new_host, v_new_host, block_table_host, seq_lens_host,
                           q_dev, k_new_dev, v_new_dev, block_table_dev, seq_lens_dev,
                           k_cache, v_cache, scale, chunk_tokens, part_o, part_lse,
                           out_dev, out_host, workspace=None, status=None, stream=None):
    """Fused decode step from pinned host inputs to a host output. ``q_dev``, ``k_new_dev``,
    ``v_new_dev`` and ``out_dev`` may be None: the kernel then works on the pinned host buffers in
    place (see ``include/pda.h``)."""
    desc = cache_desc(k_cache)
    B, Hq, _ = q_host.shape
    mc = 0 if part_o is None else part_o.shape[2]
    rc = lib().paged_decode_step_host(
        _ptr(q_host), _ptr(k_new_host), _ptr(v_new_host), _ptr(block_table_host),
        _ptr(seq_lens_host), _ptr(q_dev), _ptr(k_new_dev), _ptr(v_new_dev), _ptr(block_table_dev),
        _ptr(seq_lens_dev), _ptr(k_cache), _ptr(v_cache), C.byref(desc),
        block_table_host.stride(0), B, Hq, float(scale), chunk_tokens, _ptr(part_o),
        _ptr(part_lse), mc, _ptr(workspace), _ptr(out_dev), _ptr(out_host), _ptr(status),
        _stream(stream))
    _check(rc, "paged_decode_step_host")
    return out_host


def debug_e4m3_decode(stream=None):
    out = torch.empty(256, dtype=torch.float32, device="cuda")
    _check(lib().pda_debug_e4m3_decode(_ptr(out), _stream(stream)), "pda_debug_e4m3_decode")
    return out


def paged_decode_attention_static(q, k_cache, v_cache, block_table, seq_lens, scale, chunk_tokens,
                                  max_chunks, out=None, k_scale=None, v_scale=None, status=None,
                                  stream=None):
    """Split-KV attention + reduce using the library's built-in scratch array, for
    callers that cannot allocate partial buffers (see ``include/pda.h``). ``out`` should
    be passed in by such callers; it is only created here as a convenience. Raises if
    ``batch*Hq*max_chunks*(D+1)*4`` bytes exceed ``STATIC_SCRATCH_BYTES``."""
    desc = cache_desc(k_cache)
    B, Hq, _ = q.shape
    if out is None:
        out = torch.empty_like(q)
    rc = lib().paged_decode_attention_static(
        _ptr(q), _ptr(k_cache), _ptr(v_cache), C.byref(desc), _ptr(k_scale), _ptr(v_scale),
        _ptr(block_table), block_table.stride(0), _ptr(seq_lens), B, Hq, float(scale),
        chunk_tokens, max_chunks, _ptr(out), _ptr(status), _stream(stream))
    _check(rc, "paged_decode_attention_static")
    return out


def debug_wait_timeout(polls, status, result=None, stream=None):
    """Runs the kernels' two bounded waits on a barrier nobody arrives at, with ``polls`` as the limit;
    ``status`` (int32[1]) receives PDA_DEV_TIMEOUT, ``result`` (int64[3]) the two durations in ns and the
    mask of waits that wrongly reported completion."""
    _check(lib().pda_debug_wait_timeout(int(polls), _ptr(status), _ptr(result), _stream(stream)),
           "pda_debug_wait_timeout")


def debug_read_probe(buf, sink, stream=None):
    """Enqueues one read-only pass over ``buf`` (any dtype, contiguous, a multiple of 16 bytes)."""
    nbytes = buf.numel() * buf.element_size()
    _check(lib().pda_debug_read_probe(_ptr(buf), nbytes, _ptr(sink), _stream(stream)), "pda_debug_read_probe")


def advance_seq_lens(seq_lens, delta=1, stream=None):
    """``seq_lens += delta`` on the device, in stream order (graph-capturable)."""
    _check(lib().pda_advance_seq_lens(_ptr(seq_lens), seq_lens.shape[0], int(delta), _stream(stream)),
           "pda_advance_seq_lens")


def kv_append_tokens(k_new, v_new, k_cache, v_cache, block_table, seq_lens, status=None, stream=None):
    """Append ``k_new``/``v_new`` ``[B,n_new,Hkv,D]``; ``seq_lens`` is the length after the append."""
    desc = cache_desc(k_cache)
    assert k_new.is_contiguous() and v_new.is_contiguous() and k_new.dim() == 4
    rc = lib().kv_append_tokens(_ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), C.byref(desc),
                                _ptr(block_table), block_table.stride(0), _ptr(seq_lens),
                                seq_lens.shape[0], k_new.shape[1], _ptr(status), _stream(stream))
    _check(rc, "kv_append_tokens")


def paged_verify_attention(q, k_cache, v_cache, block_table, seq_lens, scale, chunk_tokens=0, out=None,
                           part_o=None, part_lse=None, k_scale=None, v_scale=None, flags=0, status=None,
                           stream=None):
    """Causal attention of a block of query tokens ``q [B,T,Hq,D]``; returns ``out [B,T,Hq,D]``."""
    desc = cache_desc(k_cache)
    assert q.is_contiguous() and q.dim() == 4
    B, T, Hq, D = q.shape
    if out is None:
        out = torch.empty_like(q)
    mc = 0
    if chunk_tokens:
        mc = part_o.shape[3]
        assert tuple(part_o.shape) == (B, T, Hq, mc, D) and tuple(part_lse.shape) == (B, T, Hq, mc)
    rc = lib().paged_verify_attention(
        _ptr(q), _ptr(k_cache), _ptr(v_cache), C.byref(desc), _ptr(k_scale), _ptr(v_scale),
        _ptr(block_table), block_table.stride(0), _ptr(seq_lens), B, Hq, T, float(scale),
        chunk_tokens, _ptr(out), _ptr(part_o), _ptr(part_lse), mc, flags, _ptr(status),
        _stream(stream))
    _check(rc, "paged_verify_attention")
    return out


def paged_prefix_decode_attention(q, k_cache, v_cache, block_table, seq_lens, scale, prefix_tokens,
                                  prefix_chunk_tokens, chunk_tokens, part_o, part_lse, out=None,
                                  k_scale=None, v_scale=None, flags=0, status=None, stream=None):
    """Decode attention of a batch sharing its first ``prefix_tokens`` tokens' pages."""
    desc = cache_desc(k_cache)
    B, Hq, D = q.shape
    if out is None:
        out = torch.empty_like(q)
    mc = part_o.shape[2]
    assert tuple(part_o.shape) == (B, Hq, mc, D) and tuple(part_lse.shape) == (B, Hq, mc)
    rc = lib().paged_prefix_decode_attention(
        _ptr(q), _ptr(k_cache), _ptr(v_cache), C.byref(desc), _ptr(k_scale), _ptr(v_scale),
        _ptr(block_table), block_table.stride(0), _ptr(seq_lens), B, Hq, float(scale),
        int(prefix_tokens), int(prefix_chunk_tokens), int(chunk_tokens), _ptr(out), _ptr(part_o),
        _ptr(part_lse), mc, flags, _ptr(status), _stream(stream))
    _check(rc, "paged_prefix_decode_attention")
    return out


def kv_append_fp8(k_new, v_new, k_cache, v_cache, k_scale, v_scale, block_table, seq_lens,
                  status=None, stream=None):
    """Quantising append of bf16 rows into e4m3 caches (scale fixed by each page's first row)."""
    desc = cache_desc(k_cache)
    assert k_new.is_contiguous() and v_new.is_contiguous() and k_scale.is_contiguous()
    rc = lib().kv_append_fp8(_ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), C.byref(desc),
                             _ptr(k_scale), _ptr(v_scale), _ptr(block_table), block_table.stride(0),
                             _ptr(seq_lens), seq_lens.shape[0], _ptr(status), _stream(stream))
    _check(rc, "kv_append_fp8")


def kv_append_tokens_fp8(k_new, v_new, k_cache, v_cache, k_scale, v_scale, block_table, seq_lens,
                         status=None, stream=None):
    """Quantising append of a block ``k_new, v_new [B,T,Hkv,D]`` bf16 into e4m3 caches."""
    desc = cache_desc(k_cache)
    assert k_new.is_contiguous() and v_new.is_contiguous() and k_scale.is_contiguous() and k_new.dim() == 4
    rc = lib().kv_append_tokens_fp8(_ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), C.byref(desc),
                                    _ptr(k_scale), _ptr(v_scale), _ptr(block_table), block_table.stride(0),
                                    _ptr(seq_lens), seq_lens.shape[0], k_new.shape[1], _ptr(status),
                                    _stream(stream))
    _check(rc, "kv_append_tokens_fp8")


def set_persistent_threshold(min_units_per_cta: int):
    """Units per resident CTA from which the unsplit fused step uses the persistent kernel (0: always)."""
    _check(lib().pda_set_persistent_threshold(int(min_units_per_cta)), "pda_set_persistent_threshold")


_same_context = contextlib.nullcontext()


def _device_call(device):
    """The device the call's tensors live on becomes current for the call (streams, launches)."""
    return _same_context if device == torch.cuda.current_device() else torch.cuda.device(device)


def _raw(stream, device):
    if stream is not None:
        return stream.cuda_stream
    return _raw_stream(device) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream


def _empty(shape, dtype, device, stream):
    """A buffer of the stream that the call runs on: allocated on another one, the allocator would give its memory
    away, or take it from work still queued there, without waiting for the call."""
    with _same_context if stream is None else torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _dp(t):
    return None if t is None else t.data_ptr()


def _same_device(*tensors):
    """Device index that all given tensors (None is skipped) live on."""
    dev = None
    for t in tensors:
        if t is not None:
            d = t.get_device()
            if d != dev:
                if d < 0:
                    raise ValueError("expected CUDA tensors")
                if dev is not None:
                    raise ValueError(f"tensors on different devices: {dev} and {d}")
                dev = d
    return dev


_I32, _BF16 = torch.int32, torch.bfloat16


def _int32(*tensors):
    for t in tensors:
        if t is not None and (t.dtype is not _I32 or not t.is_contiguous()):
            raise ValueError("expected contiguous int32 tensors")


def _bf16_rows(name, t):
    """The strides of a bf16 tensor whose last dimension is contiguous."""
    if t.dtype is not _BF16:
        raise TypeError(f"{name}: expected bfloat16, got {t.dtype}")
    strides = t.stride()
    if strides[-1] != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return strides


def _desc_of(cache, latent_dim):
    """Descriptor of a ``[num_pages, P, latent_dim + rope_dim]`` bf16 latent cache, shared by calls with equal layouts
    (not to be written to)."""
    if cache.dim() != 3:
        raise ValueError("a latent cache is [num_pages, page_size, latent_dim + rope_dim]")
    page, slot, _ = _bf16_rows("cache", cache)
    n, P, W = cache.shape
    # (a dimension of extent 1 may carry any stride: the one of the dense layout is taken)
    if P == 1:
        slot = max(slot, W)
    if n <= 1:
        page = max(page, P * slot)
    return _latent_desc(page, slot, n, P, latent_dim, W - latent_dim)


@functools.lru_cache(maxsize=64)
def _latent_desc(page_stride, slot_stride, num_pages, page_size, latent_dim, rope_dim):
    return LatentDesc(page_stride, slot_stride, num_pages, page_size, latent_dim, rope_dim, PDA_BF16)


def _check_table(block_table, batch):
    """Entries per row. The row stride is also the row's capacity: a view whose stride is longer than its row would be
    read past it, so rows must follow one another."""
    if block_table.dtype is not _I32 or block_table.dim() != 2 or block_table.shape[0] != batch:
        raise ValueError("block_table: expected int32 [batch, pages]")
    n = block_table.shape[1]
    if not block_table.is_contiguous():
        raise ValueError("block_table: rows must follow one another (pass a contiguous table)")
    return n


def paged_build_tables(seq_lens, new_lens, page_size, free_pages, free_count, block_table, cu_new, slot_map,
                       positions=None, free_count_out=None, status=None, stream=None):
    """A step's block-table rows, cumulative counts, slot map and positions from request lengths, on the device.

    ``free_count`` int32[1] (updated in place unless ``free_count_out`` is given); ``cu_new`` int32[B + 1];
    ``slot_map`` and ``positions`` int32[capacity]."""
    B = seq_lens.numel()
    _int32(seq_lens, new_lens, free_pages, free_count, cu_new, slot_map, positions, free_count_out, status)
    stride = _check_table(block_table, B)
    if new_lens.numel() != B or cu_new.numel() < B + 1 or (positions is not None and positions.numel() < slot_map.numel()):
        raise ValueError("new_lens, cu_new or positions too short")
    dev = _same_device(seq_lens, new_lens, free_pages, free_count, block_table, cu_new, slot_map, positions, free_count_out, status)
    if free_count_out is None:
        free_count_out = free_count
    with _device_call(dev):
        rc = lib().paged_build_tables(seq_lens.data_ptr(), new_lens.data_ptr(), B, int(page_size), free_pages.data_ptr(),
                                      free_pages.numel(), free_count.data_ptr(), free_count_out.data_ptr(),
                                      block_table.data_ptr(), stride, cu_new.data_ptr(), slot_map.data_ptr(),
                                      _dp(positions), slot_map.numel(), _dp(status), _raw(stream, dev))
    _check(rc, "paged_build_tables")


def latent_append(c_new, rope_new, cache, slot_map, norm_weight=None, eps=1e-6, status=None, stream=None):
    """Rows ``[c_new | rope_new]`` (``[T, R]``, ``[T, Dr]``) into the cache slots ``slot_map``; with ``norm_weight``
    ``[R]`` the latent's root-mean-square norm on the way."""
    T, R = c_new.shape
    desc = _desc_of(cache, R)
    # (a dimension of extent 1 may carry any stride)
    c_stride, rope_stride = _bf16_rows("c_new", c_new)[0] if T > 1 else 0, 0
    _int32(slot_map, status)
    rope = desc.rope_dim
    if rope > 0:
        rope_strides = _bf16_rows("rope_new", rope_new)
        if rope_new.shape != (T, rope):
            raise ValueError("rope_new: expected [T, rope_dim]")
        rope_stride = rope_strides[0] if T > 1 else 0
    else:
        rope_new = None
    if slot_map.numel() != T:
        raise ValueError("slot_map: expected one entry per token")
    if norm_weight is not None:
        _bf16_rows("norm_weight", norm_weight)
        if norm_weight.numel() != R or not norm_weight.is_contiguous():
            raise ValueError("norm_weight: expected [latent_dim], contiguous")
    dev = _same_device(c_new, rope_new, cache, slot_map, norm_weight, status)
    with _device_call(dev):
        rc = lib().latent_append(c_new.data_ptr(), c_stride, _dp(rope_new), rope_stride, cache.data_ptr(), C.byref(desc),
                                 _dp(norm_weight), float(eps), slot_map.data_ptr(), T, _dp(status), _raw(stream, dev))
    _check(rc, "latent_append")


def latent_workspace(batch, num_q_heads, n_query_tokens, latent_dim, device="cuda", stream=None):
    """Workspace of ``paged_latent_attention`` (uninitialised; one per stream of overlapping calls)."""
    n = int(lib().pda_latent_workspace_bytes(batch, num_q_heads, n_query_tokens, latent_dim))
    _check(min(n, 0), "pda_latent_workspace_bytes")
    return _empty(n, torch.uint8, device, stream)


def _token_strides(name, t, B, T, H):
    """(token stride, head stride) of ``[B, T, H, D]`` (or ``[B, H, D]``: ``T = 1``), tokens numbered ``b*T + t``."""
    strides = _bf16_rows(name, t)
    if len(strides) == 3:
        token, head, _ = strides
    else:
        batch, token, head, _ = strides
        if T == 1:
            token = batch
        elif B > 1 and batch != T * token:
            raise ValueError(f"{name}: batch and token dimensions must be evenly strided together")
    return (token if B * T > 1 else 0), (head if H > 1 else 0)


def paged_latent_attention(q_latent, q_rope, cache, block_table, seq_lens, scale, out=None, workspace=None, flags=0,
                           status=None, stream=None):
    """Absorbed attention over the paged latent cache: ``q_latent [B,T,H,R]`` (or ``[B,H,R]``), ``q_rope [B,T,H,Dr]``;
    fills and returns ``out`` like ``q_latent``. Without ``workspace`` one is allocated for the call."""
    shape = q_latent.shape
    if len(shape) == 4:
        B, T, H, R = shape
    else:
        (B, H, R), T = shape, 1
    if out is None:
        out = _empty(shape, q_latent.dtype, q_latent.device, stream)
    elif out.shape != shape:
        raise ValueError("out: expected the shape of q_latent")
    desc = _desc_of(cache, R)
    rope = desc.rope_dim
    if rope > 0:
        if q_rope.shape != ((B, T, H, rope) if len(shape) == 4 else (B, H, rope)):
            raise ValueError("q_rope: expected [batch, tokens, heads, rope_dim]")
        qr_token, qr_head = _token_strides("q_rope", q_rope, B, T, H)
    else:
        q_rope, qr_token, qr_head = None, 0, 0
    ql_token, ql_head = _token_strides("q_latent", q_latent, B, T, H)
    out_token, out_head = _token_strides("out", out, B, T, H)
    _int32(seq_lens, status)
    if seq_lens.numel() != B:
        raise ValueError("seq_lens: expected one entry per sequence")
    stride = _check_table(block_table, B)
    if workspace is None:
        workspace = latent_workspace(B, H, T, R, device=cache.device, stream=stream)
    elif not workspace.is_contiguous():
        raise ValueError("workspace: must be contiguous")
    dev = _same_device(q_latent, q_rope, out, cache, block_table, seq_lens, workspace, status)
    with _device_call(dev):
        rc = lib().paged_latent_attention(
            q_latent.data_ptr(), ql_token, ql_head, _dp(q_rope), qr_token, qr_head, cache.data_ptr(), C.byref(desc),
            block_table.data_ptr(), stride, seq_lens.data_ptr(), B, H, T, scale, out.data_ptr(), out_token, out_head,
            workspace.data_ptr(), workspace.nbytes, flags, _dp(status), _raw(stream, dev))
    if rc:
        _check(rc, "paged_latent_attention")
    return out


def latent_prefill_attention(q, k_nope, k_rope, v, cu_q, cu_k, max_q, scale, out=None, flags=0, status=None, stream=None):
    """Expanded causal attention over packed sequences: ``q [Tq,H,Dn+Dr]``, ``k_nope [Tk,H,Dn]``, ``k_rope [Tk,Dr]``,
    ``v [Tk,H,Dv]``, ``cu_q``/``cu_k`` int32[B + 1]; fills and returns ``out [Tq,H,Dv]``."""
    tq, H, D = q.shape
    tk, kh, dn = k_nope.shape
    dv, dr = v.shape[2], D - dn
    if out is None:
        out = _empty((tq, H, dv), q.dtype, q.device, stream)
    strides = _bf16_rows("q", q), _bf16_rows("k_nope", k_nope), _bf16_rows("v", v), _bf16_rows("out", out)
    if kh != H or v.shape != (tk, H, dv):
        raise ValueError("k_nope and v: expected [key tokens, heads, dim]")
    if out.shape != (tq, H, dv):
        raise ValueError("out: expected [query tokens, heads, value dim]")
    kr_token = 0
    if dr:
        rope_strides = _bf16_rows("k_rope", k_rope)
        if k_rope.shape != (tk, dr):
            raise ValueError("k_rope: expected [key tokens, rope_dim]")
        kr_token = rope_strides[0] if tk > 1 else 0
    else:
        k_rope = None
    _int32(cu_q, cu_k, status)
    n = cu_q.numel()
    if n != cu_k.numel() or n < 1:
        raise ValueError("cu_q and cu_k: expected batch + 1 entries each")
    dev = _same_device(q, k_nope, k_rope, v, out, cu_q, cu_k, status)

    # (a dimension of extent 1 may carry any stride)
    (qt, qh, _), (kt, kh, _), (vt, vh, _), (ot, oh, _) = strides
    if H == 1:
        qh = kh = vh = oh = 0
    if tq <= 1:
        qt = ot = 0
    if tk <= 1:
        kt = vt = 0
    with _device_call(dev):
        rc = lib().latent_prefill_attention(
            q.data_ptr(), qt, qh, k_nope.data_ptr(), kt, kh, _dp(k_rope), kr_token, v.data_ptr(), vt, vh,
            cu_q.data_ptr(), cu_k.data_ptr(), n - 1, H, dn, dr, dv, min(int(max_q), tq), tq, tk, scale, out.data_ptr(), ot, oh,
            flags, _dp(status), _raw(stream, dev))
    if rc:
        _check(rc, "latent_prefill_attention")
    return out


# What the calls below take from shapes and strides alone is checked and worked out once for each layout.

def _one_device(*tensors):
    """``_same_device`` in fewer steps where all is well."""
    devices = {t.get_device() for t in tensors if t is not None}
    return devices.pop() if len(devices) == 1 and min(devices) >= 0 else _same_device(*tensors)


def _on_device(dev, call, *args):
    """The call with the device of its tensors current."""
    if dev == torch.cuda.current_device():
        return call(*args)
    with torch.cuda.device(dev):
        return call(*args)


@functools.lru_cache(maxsize=64)
def _kv_layout(shape, k_stride, v_shape, v_stride, dtype, v_dtype):
    """Descriptor of two ``[num_pages, Hkv, 16, D]`` caches (not to be written to)."""
    if len(shape) != 4 or v_shape != shape or v_dtype is not dtype:
        raise ValueError("k_cache and v_cache: expected two [pages, kv heads, page size, head_dim] tensors of one type")
    n, heads, P, D = shape
    strides = []
    for page, head, slot, last in (k_stride, v_stride):
        if last != 1 and D > 1:
            raise ValueError("k_cache, v_cache: the last dimension must be contiguous")
        # (a dimension of extent 1 may carry any stride: a dense one is taken)
        if P == 1:
            slot = D
        if heads == 1:
            head = P * slot
        if n <= 1:
            page = max(heads * head, P * slot)
        strides.append((page, head, slot))
    if strides[0] != strides[1]:
        raise ValueError("k_cache and v_cache: expected the same strides")
    if dtype is not _BF16 and dtype not in (torch.uint8, torch.float8_e4m3fn):
        raise TypeError(f"unsupported cache dtype {dtype}")
    return CacheDesc(*strides[0], n, P, heads, D, PDA_BF16 if dtype is _BF16 else PDA_FP8_E4M3)


def _paged_caches(k_cache, v_cache, k_scale, v_scale, head_dim):
    """Descriptor of the two caches; e4m3 ones have a scale per page and head."""
    desc = _kv_layout(k_cache.shape, k_cache.stride(), v_cache.shape, v_cache.stride(), k_cache.dtype, v_cache.dtype)
    if desc.dtype == PDA_FP8_E4M3:
        for scale in (k_scale, v_scale):
            if scale is None or scale.dtype is not torch.float32 or scale.shape != k_cache.shape[:2] or not scale.is_contiguous():
                raise ValueError("k_scale and v_scale: expected contiguous float32 [pages, kv heads] for e4m3 caches")
    if desc.head_dim != head_dim:
        raise ValueError("q and the caches differ in head_dim")
    return desc


@functools.lru_cache(maxsize=256)
def _row_layout(name, shape, stride, tokens, heads, head_dim):
    """(token stride, head stride) of rows ``[tokens, heads, head_dim]``."""
    if shape != (tokens, heads, head_dim):
        raise ValueError(f"{name}: expected [{tokens}, {heads} heads, {head_dim}]")
    if stride[2] != 1 and head_dim > 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    # (a dimension of extent 1 may carry any stride)
    return (stride[0] if tokens > 1 else 0), (stride[1] if heads > 1 else 0)


def _rows_of(name, t, tokens, heads, head_dim):
    if t.dtype is not _BF16:
        raise TypeError(f"{name}: expected bfloat16, got {t.dtype}")
    return _row_layout(name, t.shape, t.stride(), tokens, heads, head_dim)


def rope_kv_append(q, k, v, positions, cos_sin, k_cache, v_cache, slot_map, q_norm=None, k_norm=None, eps=1e-6, interleaved=False,
                   freq_axis=None, out=None, k_scale=None, v_scale=None, status=None, stream=None):
    """A step's queries, keys and values ``[T, heads, D]`` as the projection leaves them: root-mean-square norm of each query
    and key head (``q_norm``, ``k_norm`` ``[D]``), rotation by ``positions``, queries to ``out`` (``q`` itself may be given), keys
    and values into the cache slots ``slot_map``.

    ``cos_sin`` float32 ``[positions, rot_dim]``: cosines, then sines, of each position's ``rot_dim / 2`` angles; None: no
    rotation. ``positions`` int32 ``[T]``, or ``[axes, T]`` with ``freq_axis``, the axis of each of the ``rot_dim / 2``
    frequencies (a sequence of ints on the host; bytes are taken fastest). e4m3 caches take ``k_scale``/``v_scale``
    ``[pages, Hkv]``, which are updated."""
    T, Hq, D = q.shape
    desc = _paged_caches(k_cache, v_cache, k_scale, v_scale, D)
    if out is None:
        out = _empty(q.shape, q.dtype, q.device, stream)
    Hkv = desc.num_kv_heads
    q_token, q_head = _rows_of("q", q, T, Hq, D)
    k_token, k_head = _rows_of("k", k, T, Hkv, D)
    v_token, v_head = _rows_of("v", v, T, Hkv, D)
    o_token, o_head = _rows_of("out", out, T, Hq, D)
    _int32(slot_map, status)
    if slot_map.numel() != T:
        raise ValueError("slot_map: expected one entry per token")
    for name, w in (("q_norm", q_norm), ("k_norm", k_norm)):
        if w is not None and (w.dtype is not _BF16 or w.numel() != D or not w.is_contiguous()):
            raise ValueError(f"{name}: expected contiguous bfloat16 [head_dim]")
    rot = table = pos_stride = 0
    axes, axis = 1, None
    if cos_sin is not None:
        if cos_sin.dim() != 2 or cos_sin.dtype is not torch.float32 or not cos_sin.is_contiguous():
            raise ValueError("cos_sin: expected contiguous float32 [positions, rot_dim]")
        table, rot = cos_sin.shape
        where = positions.shape
        if positions.dtype is not _I32 or len(where) > 2 or where[-1] != T or (T > 1 and positions.stride(-1) != 1):
            raise ValueError("positions: expected int32 [T] or [axes, T]")
        if len(where) == 2:
            axes = where[0]
            pos_stride = positions.stride(0) if axes > 1 else T
            if freq_axis is None and axes > 1:
                raise ValueError("freq_axis: needed for positions of several axes")
        if freq_axis is not None:
            axis = freq_axis if type(freq_axis) is bytes else bytes(tuple(freq_axis))
            if len(axis) != rot // 2 or (len(axis) and max(axis) >= axes):
                raise ValueError("freq_axis: expected an axis for each of the rot_dim / 2 frequencies")
    else:
        positions = None
    dev = _one_device(q, k, v, positions, cos_sin, k_cache, v_cache, slot_map, q_norm, k_norm, out, k_scale, v_scale, status)
    rc = _on_device(
        dev, lib().rope_kv_append, q.data_ptr(), q_token, q_head, k.data_ptr(), k_token, k_head, v.data_ptr(), v_token, v_head, _dp(positions), pos_stride,
        axes, axis, _dp(cos_sin), table, rot, interleaved, _dp(q_norm), _dp(k_norm), eps, slot_map.data_ptr(), T, Hq,
        out.data_ptr(), o_token, o_head, k_cache.data_ptr(), v_cache.data_ptr(), desc, _dp(k_scale), _dp(v_scale),
        _dp(status), _raw(stream, dev))
    if rc:
        _check(rc, "rope_kv_append")
    return out


def _score_desc(scale, softcap, slopes, window, num_q_heads):
    # (as plain numbers: a tensor of one element may hold another value at the next call)
    scale, softcap, window = float(scale), float(softcap), operator.index(window)
    if slopes is None:
        return _plain_score(scale, softcap, window)
    if slopes.dtype is not torch.float32 or slopes.numel() != num_q_heads or not slopes.is_contiguous():
        raise ValueError("slopes: expected contiguous float32 [query heads]")
    return ScoreDesc(scale, softcap, slopes.data_ptr(), window)


@functools.lru_cache(maxsize=64)
def _plain_score(scale, softcap, window):
    return ScoreDesc(scale, softcap, None, window)


def prefill_workspace(num_q_heads, head_dim, device="cuda", stream=None):
    """Workspace of ``paged_prefill_attention`` (uninitialised; one per stream of overlapping calls)."""
    n = int(lib().pda_prefill_workspace_bytes(num_q_heads, head_dim))
    _check(min(n, 0), "pda_prefill_workspace_bytes")
    return _empty(n, torch.uint8, device, stream)


def paged_prefill_attention(q, k_cache, v_cache, block_table, seq_lens, cu_q, max_q, scale, softcap=0.0, slopes=None, window=0,
                            prefix_lens=None, first_keys=None, out=None, k_scale=None, v_scale=None, workspace=None, flags=0,
                            status=None, stream=None):
    """Attention of packed ragged prompts (or chunks behind a context) ``q [Tq,Hq,D]`` over the paged cache, the query tokens
    ``cu_q`` int32[B + 1] of each sequence being the last of its ``seq_lens`` tokens; fills and returns ``out``. Scores are
    capped by ``softcap``, biased by ``slopes`` [Hq] times the distance and masked by ``window``, ``prefix_lens`` [B] and
    ``first_keys`` [Tq]. Without ``workspace`` one is allocated for the call."""
    Tq, Hq, D = q.shape
    desc = _paged_caches(k_cache, v_cache, k_scale, v_scale, D)
    if out is None:
        out = _empty(q.shape, q.dtype, q.device, stream)
    q_token, q_head = _rows_of("q", q, Tq, Hq, D)
    o_token, o_head = _rows_of("out", out, Tq, Hq, D)
    _int32(seq_lens, cu_q, prefix_lens, first_keys, status)
    B = seq_lens.numel()
    if cu_q.numel() != B + 1:
        raise ValueError("cu_q: expected batch + 1 entries")
    if prefix_lens is not None and prefix_lens.numel() != B:
        raise ValueError("prefix_lens: expected one entry per sequence")
    if first_keys is not None and first_keys.numel() != Tq:
        raise ValueError("first_keys: expected one entry per query token")
    stride = _check_table(block_table, B)
    score = _score_desc(scale, softcap, slopes, window, Hq)
    if workspace is None:
        workspace = prefill_workspace(Hq, D, device=q.device, stream=stream)
    elif not workspace.is_contiguous():
        raise ValueError("workspace: must be contiguous")
    dev = _one_device(q, k_cache, v_cache, block_table, seq_lens, cu_q, slopes, prefix_lens, first_keys, out, k_scale, v_scale,
                       workspace, status)
    rc = _on_device(
        dev, lib().paged_prefill_attention, q.data_ptr(), q_token, q_head, k_cache.data_ptr(), v_cache.data_ptr(), desc, _dp(k_scale), _dp(v_scale),
        block_table.data_ptr(), stride, seq_lens.data_ptr(), cu_q.data_ptr(), B, Hq, min(int(max_q), Tq), Tq, score,
        _dp(prefix_lens), _dp(first_keys), out.data_ptr(), o_token, o_head, workspace.data_ptr(), workspace.nbytes, flags,
        _dp(status), _raw(stream, dev))
    if rc:
        _check(rc, "paged_prefill_attention")
    return out


def paged_biased_decode_attention(q, k_cache, v_cache, block_table, seq_lens, scale, softcap=0.0, slopes=None, window=0,
                                  first_keys=None, chunk_tokens=0, out=None, part_o=None, part_lse=None, workspace=None, k_scale=None,
                                  v_scale=None, flags=0, status=None, stream=None):
    """``paged_decode_attention`` with scores that are capped by ``softcap``, biased by ``slopes`` [Hq] times the distance and
    masked by ``window`` and ``first_keys`` [B]; ``q [B,Hq,D]``. ``chunk_tokens > 0`` splits the tokens (``part_o``, ``part_lse``
    as there; ``workspace`` as in ``paged_decode_step``). Always fills and returns ``out``."""
    B, Hq, D = q.shape
    desc = _paged_caches(k_cache, v_cache, k_scale, v_scale, D)
    if out is None:
        out = _empty(q.shape, q.dtype, q.device, stream)
    for name, t in (("q", q), ("out", out)):
        if t.dtype is not _BF16 or t.shape != (B, Hq, D) or not t.is_contiguous():
            raise ValueError(f"{name}: expected contiguous bfloat16 [batch, heads, head_dim]")
    _int32(seq_lens, first_keys, status)
    if seq_lens.numel() != B or (first_keys is not None and first_keys.numel() != B):
        raise ValueError("seq_lens and first_keys: expected one entry per sequence")
    stride = _check_table(block_table, B)
    mc = 0
    if chunk_tokens:
        if part_o is None or part_lse is None:
            raise ValueError("part_o and part_lse: needed with chunk_tokens")
        mc = part_lse.shape[-1]
        if part_o.shape != (B, Hq, mc, D) or part_lse.shape != (B, Hq, mc):
            raise ValueError("part_o, part_lse: expected [batch, heads, chunks, head_dim] and [batch, heads, chunks]")
        for t in (part_o, part_lse):
            if t.dtype is not torch.float32 or not t.is_contiguous():
                raise ValueError("part_o, part_lse: expected contiguous float32")
        if workspace is not None:
            _int32(workspace)
            parts = -(-(Hq // max(desc.num_kv_heads, 1)) // 8)
            if workspace.numel() < workspace_ints(B, desc.num_kv_heads * parts):
                raise ValueError("workspace: too small")
    score = _score_desc(scale, softcap, slopes, window, Hq)
    dev = _one_device(q, k_cache, v_cache, block_table, seq_lens, slopes, first_keys, out, part_o, part_lse, workspace, k_scale,
                       v_scale, status)
    rc = _on_device(
        dev, lib().paged_biased_decode_attention, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), desc, _dp(k_scale), _dp(v_scale), block_table.data_ptr(),
        stride, seq_lens.data_ptr(), B, Hq, score, _dp(first_keys), chunk_tokens, out.data_ptr(), _dp(part_o),
        _dp(part_lse), mc, _dp(workspace), flags, _dp(status), _raw(stream, dev))
    if rc:
        _check(rc, "paged_biased_decode_attention")
    return out
