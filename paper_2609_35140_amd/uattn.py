"""Python binding for libuattn.so (argument marshalling only).

Every function here checks shapes/dtypes, takes device pointers from torch
tensors and calls the C ABI declared in ``include/uattn.h`` on the current
torch stream.  All arithmetic runs in the HIP kernels; there is no CPU or
PyTorch fallback -- if the library is missing, every call raises.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
from typing import Optional, Tuple

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("UATTN_LIB") or os.path.join(_PKG, "libuattn.so")

UATTN_OK = 0
TILE_KEYS = 64
CHUNK_KEYS = 256

_lib = None


class UattnError(RuntimeError):
    pass


def _load():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise UattnError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_35140_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    c_i32, c_i64, c_f, c_p, c_sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
    lib.uattn_abi_version.restype = c_i32
    lib.uattn_abi_version.argtypes = []
    lib.uattn_status_string.restype = ctypes.c_char_p
    lib.uattn_status_string.argtypes = [c_i32]
    lib.uattn_prefill.restype = c_i32
    lib.uattn_prefill.argtypes = [c_p, c_p, c_p, c_p, c_i32, c_i32, c_i32, c_i32, c_i32, c_i32, c_f, c_p, c_p, c_p]
    lib.uattn_decode_workspace_bytes.restype = c_sz
    lib.uattn_decode_workspace_bytes.argtypes = [c_i32, c_i32, c_i32, c_i32]
    lib.uattn_decode.restype = c_i32
    lib.uattn_decode.argtypes = [c_p, c_p, c_p, c_p, c_p, c_i32, c_i32, c_i32, c_i32, c_i32, c_i32, c_i32, c_i32, c_f,
                                 c_p, c_p, c_p, c_sz, c_p]
    lib.uattn_decode_scratch_limit.restype = c_sz
    lib.uattn_decode_scratch_limit.argtypes = []
    lib.uattn_decode_noalloc.restype = c_i32
    lib.uattn_decode_noalloc.argtypes = [c_p, c_p, c_p, c_p, c_p, c_i32, c_i32, c_i32, c_i32, c_i32, c_i32, c_i32,
                                         c_i32, c_f, c_p, c_p, c_p]
    lib.uattn_logprob.restype = c_i32
    lib.uattn_logprob.argtypes = [c_p, c_i64, c_p, c_i32, c_i32, c_f, c_p, c_p]
    lib.uattn_qk_norm_rope.restype = c_i32
    lib.uattn_qk_norm_rope.argtypes = [c_p, c_p, c_p, c_p, c_p, c_f, c_p, c_i32, c_i32, c_i32, c_i32, c_i32, c_p, c_p,
                                       c_p]
    lib.uattn_rope_cache.restype = c_i32
    lib.uattn_rope_cache.argtypes = [c_p, c_i32, c_i32, ctypes.c_double, c_p]
    lib.uattn_lm_head.restype = c_i32
    lib.uattn_lm_head.argtypes = [c_p, c_i64, c_p, c_i64, c_i32, c_i32, c_i32, c_p, c_i64, c_p]
    lib.uattn_lm_head_logprob_workspace_bytes.restype = c_sz
    lib.uattn_lm_head_logprob_workspace_bytes.argtypes = [c_i32, c_i32]
    lib.uattn_lm_head_logprob.restype = c_i32
    lib.uattn_lm_head_logprob.argtypes = [c_p, c_i64, c_p, c_i64, c_p, c_i32, c_i32, c_i32, c_f, c_p, c_p, c_i64, c_p,
                                          c_sz, c_p]
    lib.uattn_prefill_backward_workspace_bytes.restype = c_sz
    lib.uattn_prefill_backward_workspace_bytes.argtypes = [c_i32, c_i32]
    lib.uattn_prefill_backward.restype = c_i32
    lib.uattn_prefill_backward.argtypes = [c_p, c_p, c_p, c_p, c_p, c_p, c_p, c_i32, c_i32, c_i32, c_i32, c_i32,
                                           c_i32, c_f, c_p, c_p, c_p, c_p, c_sz, c_p]
    lib.uattn_kv_write.restype = c_i32
    lib.uattn_kv_write.argtypes = [c_p, c_p, c_i64, c_p, c_p, c_p, c_i32, c_i32, c_i32, c_i32, c_i32, c_i32, c_i32,
                                   c_p, c_p, c_p]
    lib.uattn_residual_norm.restype = c_i32
    lib.uattn_residual_norm.argtypes = [c_p, c_p, c_p, c_i64, c_f, c_p, c_p, c_f, c_i32, c_i32, c_p, c_p, c_p]
    lib.uattn_residual_norm_backward_workspace_bytes.restype = c_sz
    lib.uattn_residual_norm_backward_workspace_bytes.argtypes = [c_i32, c_i32]
    lib.uattn_residual_norm_backward.restype = c_i32
    lib.uattn_residual_norm_backward.argtypes = [c_p, c_p, c_p, c_p, c_p, c_p, c_p, c_i64, c_f, c_f, c_i32, c_i32, c_p,
                                                 c_p, c_p, c_p, c_p, c_p, c_sz, c_p]
    lib.uattn_embedding.restype = c_i32
    lib.uattn_embedding.argtypes = [c_p, c_p, c_i64, c_f, c_i32, c_i32, c_i32, c_p, c_i64, c_p]
    lib.uattn_embedding_backward_workspace_bytes.restype = c_sz
    lib.uattn_embedding_backward_workspace_bytes.argtypes = [c_i32, c_i32]
    lib.uattn_embedding_backward.restype = c_i32
    lib.uattn_embedding_backward.argtypes = [c_p, c_i64, c_p, c_f, c_i32, c_i32, c_i32, c_p, c_i64, c_i32, c_i32, c_p,
                                             c_sz, c_p]
    lib.uattn_logits_process.restype = c_i32
    lib.uattn_logits_process.argtypes = [c_p, c_i64, c_i32, c_i32, c_p, c_i32, c_p, c_p, c_p, c_p, c_i32, c_p, c_p,
                                         c_i64, c_i32, c_p, c_p, c_i64, c_p]
    lib.uattn_logits_process_backward.restype = c_i32
    lib.uattn_logits_process_backward.argtypes = [c_p, c_i64, c_p, c_i64, c_i32, c_i32, c_p, c_i32, c_p, c_p, c_p,
                                                  c_i64, c_i32, c_p, c_p, c_i64, c_p]
    lib.uattn_logprob_backward.restype = c_i32
    lib.uattn_logprob_backward.argtypes = [c_p, c_i64, c_p, c_p, c_i32, c_i32, c_f, c_p, c_i64, c_p]
    lib.uattn_kv_write_mx.restype = c_i32
    lib.uattn_kv_write_mx.argtypes = [c_p, c_p, c_i64, c_p, c_p, c_p] + [c_i32] * 9 + [c_p] * 5
    lib.uattn_kv_read_mx.restype = c_i32
    lib.uattn_kv_read_mx.argtypes = [c_p] * 4 + [c_i32] * 2 + [c_p] * 3 + [c_i32] * 7 + [c_p, c_p, c_i64, c_p]
    lib.uattn_kv_round_mx.restype = c_i32
    lib.uattn_kv_round_mx.argtypes = [c_p, c_p, c_i64] + [c_i32] * 5 + [c_p, c_p, c_i64, c_p]
    lib.uattn_decode_mx_workspace_bytes.restype = c_sz
    lib.uattn_decode_mx_workspace_bytes.argtypes = [c_i32] * 5
    lib.uattn_decode_mx.restype = c_i32
    lib.uattn_decode_mx.argtypes = [c_p] * 5 + [c_i32] * 2 + [c_p] * 2 + [c_i32] * 8 + [c_f, c_p, c_p, c_p, c_sz, c_p]
    _lib = lib
    return lib


def lib():
    """The loaded ctypes library (raises if it is not built)."""
    return _load()


def abi_version() -> int:
    return int(_load().uattn_abi_version())


def status_string(code: int) -> str:
    return _load().uattn_status_string(int(code)).decode()


def _check(code: int):
    if code != UATTN_OK:
        raise UattnError(status_string(code))


# What a small call costs here is Python: of 12 us for a decode-sized kv_write,
# 4 were the C call with its launch, 3 the Stream object that
# torch.cuda.current_stream() builds, the rest checks whose messages were
# formatted whether or not they failed.  So the current stream's handle is asked
# for itself, and a message is formed only by the check that fails.
def _stream(stream) -> int:
    if stream is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return raw(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _need(cond: bool, msg: str):
    if not cond:
        raise ValueError(msg)


_MOST = 2 ** 31 - 1


# ctypes drops what of a number does not fit the library's 32-bit sizes, so they are checked before.
def _fits(*sizes) -> bool:
    for n in sizes:
        if not -_MOST <= n <= _MOST:
            return False
    return True


def _sizes(*sizes):
    if not _fits(*sizes):
        raise ValueError(f"sizes are at most 2^31 - 1, got {max(sizes, key=abs)}")


def _bf16_cuda(t, name):
    import torch
    if t.is_cuda and t.dtype == torch.bfloat16 and t.is_contiguous():
        return
    _need(t.is_cuda, f"{name} must be a GPU tensor")
    _need(t.dtype == torch.bfloat16, f"{name} must be bfloat16")
    _need(False, f"{name} must be contiguous")


def _i32_cuda(t, name, msg="must be contiguous int32 on the GPU"):
    import torch
    if not (t.dtype == torch.int32 and t.is_cuda and t.is_contiguous()):
        raise ValueError(f"{name} {msg}")


def _bf16_rows(t, name):
    import torch
    if not (t.is_cuda and t.dtype == torch.bfloat16 and t.dim() == 2 and t.stride(1) == 1):
        raise ValueError(f"{name} must be a 2-D bfloat16 GPU tensor with contiguous rows")


def default_scale(head_dim: int) -> float:
    return 1.0 / math.sqrt(head_dim)


def prefill(q, k, v, cu_seqlens, max_seqlen: int, softmax_scale: Optional[float] = None, out=None,
            return_lse: bool = False, lse=None, stream=None):
    """Full-sequence causal attention (uattn_prefill).

    q [T,Hq,d], k/v [T,Hkv,d] bf16 CUDA; cu_seqlens int32 CUDA [B+1].
    Returns out [T,Hq,d] (and lse [T,Hq] fp32 if requested).
    """
    import torch
    _bf16_cuda(q, "q")
    _bf16_cuda(k, "k")
    _bf16_cuda(v, "v")
    _need(q.dim() == 3 and k.dim() == 3 and v.dim() == 3, "q/k/v must be [T, H, d]")
    T, hq, d = q.shape
    _need(k.shape == v.shape and k.shape[0] == T and k.shape[2] == d, "k/v shape mismatch")
    _need(cu_seqlens.dtype == torch.int32 and cu_seqlens.is_cuda and cu_seqlens.is_contiguous(),
          "cu_seqlens must be contiguous int32 on the GPU")
    _sizes(T, hq, k.shape[1], d, cu_seqlens.numel() - 1, int(max_seqlen))
    if softmax_scale is None:
        softmax_scale = default_scale(d)
    if out is None:
        out = torch.empty_like(q)
    else:
        _bf16_cuda(out, "out")
        _need(out.shape == q.shape, "out shape")
    if return_lse and lse is None:
        lse = torch.empty((T, hq), dtype=torch.float32, device=q.device)
    if lse is not None:
        _need(lse.dtype == torch.float32 and lse.is_contiguous() and lse.shape == (T, hq), "lse must be [T,Hq] fp32")
    _check(_load().uattn_prefill(_ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens), cu_seqlens.numel() - 1, T,
                                 int(max_seqlen), hq, k.shape[1], d, float(softmax_scale), _ptr(out), _ptr(lse),
                                 _stream(stream)))
    return (out, lse) if lse is not None else out


def prefill_backward_workspace_bytes(total_tokens: int, num_q_heads: int) -> int:
    sizes = int(total_tokens), int(num_q_heads)
    return int(_load().uattn_prefill_backward_workspace_bytes(*sizes)) if _fits(*sizes) else 0


def prefill_backward(q, k, v, out, dout, lse, cu_seqlens, max_seqlen: int, softmax_scale: Optional[float] = None,
                     dq=None, dk=None, dv=None, workspace=None, stream=None):
    """Gradients of the full-sequence attention (uattn_prefill_backward).

    q, k, v, cu_seqlens, max_seqlen, softmax_scale as for prefill; out and lse
    are prefill's outputs for them; dout [T,Hq,d] bf16 is the upstream
    gradient.  Returns (dq [T,Hq,d], dk [T,Hkv,d], dv [T,Hkv,d]) bf16.
    """
    import torch
    for name, t in (("q", q), ("k", k), ("v", v), ("out", out), ("dout", dout)):
        _bf16_cuda(t, name)
    _need(q.dim() == 3 and k.dim() == 3 and v.dim() == 3, "q/k/v must be [T, H, d]")
    T, hq, d = q.shape
    hkv = k.shape[1]
    _need(k.shape == v.shape and k.shape[0] == T and k.shape[2] == d, "k/v shape mismatch")
    _need(out.shape == q.shape and dout.shape == q.shape, "out/dout must match q")
    _need(lse.dtype == torch.float32 and lse.is_cuda and lse.is_contiguous() and tuple(lse.shape) == (T, hq),
          "lse must be [T,Hq] fp32 on the GPU")
    _need(cu_seqlens.dtype == torch.int32 and cu_seqlens.is_cuda and cu_seqlens.is_contiguous(),
          "cu_seqlens must be contiguous int32 on the GPU")
    _sizes(T, hq, hkv, d, cu_seqlens.numel() - 1, int(max_seqlen))
    if softmax_scale is None:
        softmax_scale = default_scale(d)
    outs = []
    for name, t, like in (("dq", dq, q), ("dk", dk, k), ("dv", dv, v)):
        if t is None:
            t = torch.empty_like(like)
        else:
            _bf16_cuda(t, name)
            _need(t.shape == like.shape, f"{name} shape")
        outs.append(t)
    need = prefill_backward_workspace_bytes(T, hq)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)  # no initial contents needed
    _check(_load().uattn_prefill_backward(
        _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(dout), _ptr(lse), _ptr(cu_seqlens), cu_seqlens.numel() - 1, T,
        int(max_seqlen), hq, hkv, d, float(softmax_scale), _ptr(outs[0]), _ptr(outs[1]), _ptr(outs[2]),
        _ptr(workspace), workspace.numel() * workspace.element_size() if workspace is not None else 0,
        _stream(stream)))
    return tuple(outs)


def decode_workspace_bytes(batch: int, max_seqlen: int, num_q_heads: int, head_dim: int) -> int:
    sizes = batch, max_seqlen, num_q_heads, head_dim
    return int(_load().uattn_decode_workspace_bytes(*sizes)) if _fits(*sizes) else 0


def new_workspace(nbytes: int, device="cuda"):
    """A zero-filled decode workspace (the counters it holds must start at zero).

    The returned tensor carries the extent of its known-zero prefix as an
    attribute of the tensor object itself, so the binding never re-zeroes it
    needlessly and never trusts a stale record: a different tensor (even one
    at the same device address) starts with no such record.
    """
    import torch
    t = torch.zeros(int(nbytes), dtype=torch.uint8, device=device)
    t._uattn_zero_prefix = int(nbytes)
    return t


def counter_bytes(batch: int, num_q_heads: int) -> int:
    """Size of the counter region at the start of a decode workspace."""
    return (4 * batch * num_q_heads + 255) // 256 * 256


def _partials_start(ws_bytes: int, batch: int, max_seqlen: int, num_q_heads: int, head_dim: int) -> int:
    """Byte offset where a call's fp32 partials begin (they sit at the end of
    the workspace; the counters at its start)."""
    nslot = ((max_seqlen + CHUNK_KEYS - 1) // CHUNK_KEYS + 1) // 2 * 2   # chunks rounded up to even
    acc = (4 * batch * num_q_heads * nslot * head_dim + 255) // 256 * 256
    ml = (4 * batch * num_q_heads * nslot * 2 + 255) // 256 * 256
    return (ws_bytes & ~15) - acc - ml


def _prepare_workspace(workspace, batch: int, max_seqlen: int, num_q_heads: int, head_dim: int):
    """Make the counter region of ``workspace`` zero before a call, as uattn.h
    requires, and record what the call leaves zero.

    The record lives on the tensor object (``_uattn_zero_prefix``), never in
    a table keyed by address: a workspace tensor this binding has not seen
    before (or a different view of the same memory) is zeroed on first use,
    whatever an earlier tensor at that address held.  After the call the
    counters are zero again (the kernel resets them), while the partial
    region at the end of the buffer holds data.
    """
    nbytes = workspace.numel() * workspace.element_size()
    c = min(counter_bytes(batch, num_q_heads), nbytes)
    known = getattr(workspace, "_uattn_zero_prefix", 0)
    if known < c:
        workspace.view(-1)[: c // workspace.element_size()].zero_()
        known = c
    workspace._uattn_zero_prefix = max(c, min(known, _partials_start(nbytes, batch, max_seqlen, num_q_heads,
                                                                        head_dim)))


def decode(q, k_pages, v_pages, block_table, seqlens, max_seqlen: int, softmax_scale: Optional[float] = None,
           out=None, return_lse: bool = False, lse=None, workspace=None, stream=None):
    """Token-wise paged decode (uattn_decode).

    q [B,Hq,d]; k_pages/v_pages [P,Hkv,page,d] bf16 CUDA; block_table [B,maxp]
    int32; seqlens [B] int32 (context length including the current token).
    ``workspace`` is a zero-filled uint8 CUDA tensor (``new_workspace``); a
    fresh one is allocated when not given.
    """
    import torch
    _bf16_cuda(q, "q")
    _bf16_cuda(k_pages, "k_pages")
    _bf16_cuda(v_pages, "v_pages")
    _need(q.dim() == 3 and k_pages.dim() == 4 and v_pages.shape == k_pages.shape, "shapes: q [B,Hq,d], pages [P,Hkv,page,d]")
    B, hq, d = q.shape
    _, hkv, page, d2 = k_pages.shape
    _need(d2 == d, "head_dim mismatch")
    _i32_cuda(block_table, "block_table")
    _i32_cuda(seqlens, "seqlens")
    _need(block_table.dim() == 2 and block_table.shape[0] == B and seqlens.shape == (B,), "block_table/seqlens shape")
    _sizes(B, block_table.shape[1], page, k_pages.shape[0], int(max_seqlen), hq, hkv, d)
    if softmax_scale is None:
        softmax_scale = default_scale(d)
    if out is None:
        out = torch.empty_like(q)
    else:
        _bf16_cuda(out, "out")
        _need(out.shape == q.shape, "out shape")
    if return_lse and lse is None:
        lse = torch.empty((B, hq), dtype=torch.float32, device=q.device)
    need = decode_workspace_bytes(B, int(max_seqlen), hq, d) if B > 0 else 0
    if workspace is None and need > 0:
        workspace = new_workspace(need, q.device)
    if workspace is not None and need > 0:
        _need(workspace.is_cuda and workspace.is_contiguous(), "workspace must be a contiguous GPU tensor")
        _prepare_workspace(workspace, B, int(max_seqlen), hq, d)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_load().uattn_decode(_ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(block_table), _ptr(seqlens), B,
                                block_table.shape[1], page, k_pages.shape[0], int(max_seqlen), hq, hkv, d, float(softmax_scale),
                                _ptr(out), _ptr(lse), _ptr(workspace), ws_bytes, _stream(stream)))
    return (out, lse) if lse is not None else out


def decode_scratch_limit() -> int:
    """Bytes of the library's static decode scratch array (uattn_decode_noalloc)."""
    return int(_load().uattn_decode_scratch_limit())


def decode_noalloc(q, k_pages, v_pages, block_table, seqlens, max_seqlen: int, softmax_scale: Optional[float] = None,
                   out=None, return_lse: bool = False, lse=None, stream=None):
    """uattn_decode_noalloc: the token-wise decode with the library's static
    scratch array as its workspace (the call itself allocates nothing; pass
    ``out``/``lse`` to keep this binding from allocating them).  Arguments and
    results as for :func:`decode`."""
    import torch
    _bf16_cuda(q, "q")
    _bf16_cuda(k_pages, "k_pages")
    _bf16_cuda(v_pages, "v_pages")
    _need(q.dim() == 3 and k_pages.dim() == 4 and v_pages.shape == k_pages.shape, "shapes: q [B,Hq,d], pages [P,Hkv,page,d]")
    B, hq, d = q.shape
    _, hkv, page, d2 = k_pages.shape
    _need(d2 == d, "head_dim mismatch")
    _i32_cuda(block_table, "block_table")
    _i32_cuda(seqlens, "seqlens")
    _need(block_table.dim() == 2 and block_table.shape[0] == B and seqlens.shape == (B,), "block_table/seqlens shape")
    _sizes(B, block_table.shape[1], page, k_pages.shape[0], int(max_seqlen), hq, hkv, d)
    if softmax_scale is None:
        softmax_scale = default_scale(d)
    if out is None:
        out = torch.empty_like(q)
    else:
        _bf16_cuda(out, "out")
        _need(out.shape == q.shape, "out shape")
    if return_lse and lse is None:
        lse = torch.empty((B, hq), dtype=torch.float32, device=q.device)
    if lse is not None:
        _need(lse.dtype == torch.float32 and lse.is_contiguous() and tuple(lse.shape) == (B, hq), "lse must be [B,Hq] fp32")
    _check(_load().uattn_decode_noalloc(_ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(block_table), _ptr(seqlens), B,
                                        block_table.shape[1], page, k_pages.shape[0], int(max_seqlen), hq, hkv, d,
                                        float(softmax_scale), _ptr(out), _ptr(lse), _stream(stream)))
    return (out, lse) if lse is not None else out


def logprob(logits, targets, inv_temperature: float = 1.0, out=None, stream=None):
    """Per-token log-probability (uattn_logprob). logits [T,V] bf16 (row stride may exceed V)."""
    import torch
    _need(logits.is_cuda and logits.dtype == torch.bfloat16 and logits.dim() == 2, "logits must be [T,V] bf16 on the GPU")
    _need(logits.stride(1) == 1, "logits rows must be contiguous")
    T, V = logits.shape
    _need(targets.dtype == torch.int32 and targets.is_cuda and targets.shape == (T,) and targets.is_contiguous(),
          "targets must be [T] int32 on the GPU")
    _sizes(T, V)
    if out is None:
        out = torch.empty(T, dtype=torch.float32, device=logits.device)
    _check(_load().uattn_logprob(_ptr(logits), logits.stride(0), _ptr(targets), T, V, float(inv_temperature),
                                 _ptr(out), _stream(stream)))
    return out


def kv_write(k_new, v_new, block_table, seq_idx, positions, k_pages, v_pages, stream=None):
    """Write new K/V token rows into the paged cache in place (uattn_kv_write).

      k_new, v_new   [N, Hkv, d] bf16 (token rows may be strided: stride(0) elements apart)
      block_table    [B, maxp] int32; seq_idx, positions [N] int32 (position < 0: padding)
      k_pages, v_pages  [P, Hkv, page, d] bf16, updated in place
    """
    import torch
    _bf16_cuda(k_pages, "k_pages")
    _bf16_cuda(v_pages, "v_pages")
    _need(k_new.is_cuda and k_new.dtype == torch.bfloat16, "k_new must be a bfloat16 GPU tensor")
    _need(v_new.is_cuda and v_new.dtype == torch.bfloat16, "v_new must be a bfloat16 GPU tensor")
    _need(k_new.dim() == 3 and v_new.shape == k_new.shape, "k_new/v_new must be [N,Hkv,d]")
    N, hkv, d = k_new.shape
    _need(k_new.stride(2) == 1 and k_new.stride(1) == d and v_new.stride() == k_new.stride(),
          "k_new/v_new: heads and d must be contiguous, both with the same token stride")
    P, hkv2, page, d2 = k_pages.shape
    _need(hkv2 == hkv and d2 == d and v_pages.shape == k_pages.shape, "page shapes")
    _i32_cuda(block_table, "block_table", "must be int32 on the GPU")
    _i32_cuda(seq_idx, "seq_idx", "must be int32 on the GPU")
    _i32_cuda(positions, "positions", "must be int32 on the GPU")
    _need(block_table.dim() == 2 and seq_idx.shape == (N,) and positions.shape == (N,), "index shapes")
    B, maxp = block_table.shape
    _sizes(N, B, maxp, page, P, hkv, d)
    _check(_load().uattn_kv_write(_ptr(k_new), _ptr(v_new), k_new.stride(0), _ptr(block_table), _ptr(seq_idx),
                                  _ptr(positions), N, B, maxp, page, P, hkv, d, _ptr(k_pages), _ptr(v_pages),
                                  _stream(stream)))
    return k_pages, v_pages


def rope_cache(max_position: int, head_dim: int, theta: float, out=None, stream=None):
    """The NeoX rotary table [max_position, head_dim/2, 2] fp32 (uattn_rope_cache)."""
    import torch
    _sizes(max_position, head_dim)
    if out is None:
        out = torch.empty((max_position, head_dim // 2, 2), dtype=torch.float32, device="cuda")
    _need(out.dtype == torch.float32 and out.is_cuda and out.is_contiguous()
          and tuple(out.shape) == (max_position, head_dim // 2, 2), "out must be [max_position, head_dim/2, 2] fp32")
    _check(_load().uattn_rope_cache(_ptr(out), max_position, head_dim, float(theta), _stream(stream)))
    return out


def qk_norm_rope(q, k, positions, q_weight, k_weight, cos_sin, eps: float = 1e-6, q_out=None, k_out=None,
                 stream=None):
    """RMSNorm of every q and k head row, then NeoX rotary embedding (uattn_qk_norm_rope).

      q [T, Hq, d], k [T, Hkv, d] bf16; positions [T] int32; q_weight, k_weight [d] bf16;
      cos_sin [max_position, d/2, 2] fp32.  Outputs may be q and k themselves (in place).
    """
    import torch
    _bf16_cuda(q, "q")
    _bf16_cuda(k, "k")
    _bf16_cuda(q_weight, "q_weight")
    _bf16_cuda(k_weight, "k_weight")
    _need(q.dim() == 3 and k.dim() == 3 and q.shape[0] == k.shape[0] and q.shape[2] == k.shape[2], "q/k shapes")
    T, hq, d = q.shape
    hkv = k.shape[1]
    _need(q_weight.shape == (d,) and k_weight.shape == (d,), "weights must be [d]")
    _need(positions.dtype == torch.int32 and positions.is_cuda and positions.shape == (T,) and positions.is_contiguous(),
          "positions must be [T] int32 on the GPU")
    _need(cos_sin.dtype == torch.float32 and cos_sin.is_cuda and cos_sin.is_contiguous() and cos_sin.dim() == 3
          and cos_sin.shape[1:] == (d // 2, 2), "cos_sin must be [max_position, d/2, 2] fp32")
    _sizes(cos_sin.shape[0], T, hq, hkv, d)
    if q_out is None:
        q_out = torch.empty_like(q)
    if k_out is None:
        k_out = torch.empty_like(k)
    _need(q_out.shape == q.shape and k_out.shape == k.shape, "output shapes")
    _check(_load().uattn_qk_norm_rope(_ptr(q), _ptr(k), _ptr(positions), _ptr(q_weight), _ptr(k_weight), float(eps),
                                      _ptr(cos_sin), cos_sin.shape[0], T, hq, hkv, d, _ptr(q_out), _ptr(k_out),
                                      _stream(stream)))
    return q_out, k_out


def lm_head(hidden, weight, out=None, stream=None):
    """Batch-invariant logits = bf16(hidden . weight^T) (uattn_lm_head).

      hidden [T, H] bf16, weight [V, H] bf16 (rows may be strided); out [T, V] bf16 (row stride a multiple of 8).
    """
    import torch
    _bf16_rows(hidden, "hidden")
    _bf16_rows(weight, "weight")
    T, H = hidden.shape
    V, H2 = weight.shape
    _need(H2 == H, "hidden and weight widths differ")
    _sizes(T, V, H)
    if out is None:
        stride = (V + 7) // 8 * 8
        out = torch.empty((T, stride), dtype=torch.bfloat16, device=hidden.device)[:, :V]
    _need(out.dtype == torch.bfloat16 and out.is_cuda and out.shape == (T, V) and out.stride(1) == 1, "out shape")
    _check(_load().uattn_lm_head(_ptr(hidden), hidden.stride(0), _ptr(weight), weight.stride(0), T, V, H, _ptr(out),
                                 out.stride(0), _stream(stream)))
    return out


def lm_head_logprob_workspace_bytes(num_rows: int, vocab: int) -> int:
    sizes = int(num_rows), int(vocab)
    return int(_load().uattn_lm_head_logprob_workspace_bytes(*sizes)) if _fits(*sizes) else 0


def lm_head_logprob(hidden, weight, targets, inv_temperature: float = 1.0, out=None, logits=None, workspace=None,
                    stream=None):
    """LM head fused with the token log-probability (uattn_lm_head_logprob).

      hidden [T, H], weight [V, H] bf16 (rows may be strided); targets [T] int32.
      Returns logp [T] fp32.  ``logits`` ([T, V] bf16, row stride a multiple
      of 8), when given, also receives the logits.
    """
    import torch
    _bf16_rows(hidden, "hidden")
    _bf16_rows(weight, "weight")
    T, H = hidden.shape
    V, H2 = weight.shape
    _need(H2 == H, "hidden and weight widths differ")
    _sizes(T, V, H)
    _need(targets.dtype == torch.int32 and targets.is_cuda and targets.shape == (T,) and targets.is_contiguous(),
          "targets must be [T] int32 on the GPU")
    if out is None:
        out = torch.empty(T, dtype=torch.float32, device=hidden.device)
    _need(out.dtype == torch.float32 and out.is_cuda and out.shape == (T,) and out.is_contiguous(), "out must be [T] fp32")
    if logits is not None:
        _need(logits.dtype == torch.bfloat16 and logits.is_cuda and logits.shape == (T, V) and logits.stride(1) == 1,
              "logits must be [T, V] bf16 with contiguous rows")
    need = lm_head_logprob_workspace_bytes(T, V)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=hidden.device)  # no initial contents needed
    _check(_load().uattn_lm_head_logprob(_ptr(hidden), hidden.stride(0), _ptr(weight), weight.stride(0), _ptr(targets),
                                         T, V, H, float(inv_temperature), _ptr(out), _ptr(logits),
                                         logits.stride(0) if logits is not None else 0, _ptr(workspace),
                                         workspace.numel() * workspace.element_size(), _stream(stream)))
    return out


# ---------------------------------------------------------------------------
# Row-wise operators.  Their outputs and workspaces come from the stream the call
# runs on (torch's allocator reuses memory in a stream's order), and they run on
# their tensors' device where another one is current: a call for another stream or
# device repeats itself there.  A small call costs mostly Python, so a tensor is
# checked by one expression and its message formed only where that fails.
# ---------------------------------------------------------------------------
def _elsewhere(device: int, stream):
    """None where a call on `device` and `stream` runs as things are, else the context it runs in."""
    import torch
    if stream is None:
        return None if device == torch._C._cuda_getDevice() else torch.cuda.device(device)
    if not hasattr(stream, "cuda_stream"):
        # 0 and 1 (hipStreamLegacy) are the default stream's handles; ExternalStream takes 0 for none and gives a stream of its own
        handle = int(stream)
        stream = torch.cuda.default_stream(device) if handle in (0, 1) else torch.cuda.ExternalStream(handle, device=device)
    if stream.device_index != device:
        raise ValueError(f"stream is of GPU {stream.device_index}, the tensors are on GPU {device}")
    return torch.cuda.stream(stream)


def _stream_on(device: int) -> int:
    """The handle of the device's current stream."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(device) if raw is not None else torch.cuda.current_stream(device).cuda_stream


def _gpu_of(t, name) -> int:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    return t.get_device()


def _whole(t, dtype, shape, device, name):
    """A contiguous tensor of this type and shape on this GPU."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on GPU {device}")


def _rows(t, dtype, device, name):
    """A 2-D tensor with contiguous rows, any distance apart."""
    if t.dtype is not dtype or t.dim() != 2 or t.stride(1) != 1 or t.get_device() != device:
        raise ValueError(f"{name} must be a 2-D {dtype} tensor with contiguous rows on GPU {device}")


def _row_stride(t) -> int:
    """Elements from row to row (any would do for one row: torch may report what the call refuses)."""
    return t.stride(0) if t.shape[0] > 1 else max((t.shape[1] + 7) // 8 * 8, t.stride(0) // 8 * 8)


def _out_rows(out, like, rows, width):
    """``out``, or new rows of ``like``'s type and device whose starts are 16-byte aligned."""
    if out is None:
        if width % 8 == 0:
            return like.new_empty((rows, width))
        return like.new_empty((rows, (width + 7) // 8 * 8))[:, :width]
    _rows(out, like.dtype, like.get_device(), "out")
    _need(out.shape == (rows, width), "out shape")
    return out


def _workspace(workspace, need: int, like):
    if workspace is None:
        import torch
        return like.new_empty(need if need > 16 else 16, dtype=torch.uint8)  # no initial contents needed
    _need(workspace.get_device() == like.get_device() and workspace.is_contiguous(), "workspace must be a contiguous GPU tensor")
    return workspace


def residual_norm(residual, pre_weight=None, x=None, post_weight=None, gate=None, scale: float = 1.0, eps: float = 1e-6,
                  residual_out=None, y=None, stream=None):
    """The norms behind a block and before the next with the residual sum between them (uattn_residual_norm).

      u = x * r(x) * post_weight;  s = residual + scale * gate * u;  y = s * r(s) * pre_weight

      residual, x [T, H] bf16; post_weight, pre_weight [H] bf16; gate [H] or [T, H] bf16.
      Every part but residual may be left out, not x and pre_weight both.  Returns
      (residual_out, y): residual itself where there is no x, and None where there
      is no pre_weight.  residual_out may be residual, y may be x (in place).
      y is the norm of the unrounded s: that of the stored residual_out has other bits.
    """
    import torch
    dev = _gpu_of(residual, "residual")
    there = _elsewhere(dev, stream)
    if there is not None:
        with there:
            return residual_norm(residual, pre_weight, x, post_weight, gate, scale, eps, residual_out, y)
    bf16, shape = torch.bfloat16, residual.shape
    _need(len(shape) == 2, "residual must be [T, H]")
    T, H = shape
    if T > _MOST or H > _MOST:
        _sizes(T, H)
    _whole(residual, bf16, shape, dev, "residual")
    gate_stride = 0
    if x is None:
        _need(pre_weight is not None, "x or pre_weight must be given")
        _need(post_weight is None and gate is None and residual_out is None, "post_weight, gate and residual_out belong to x")
    else:
        _whole(x, bf16, shape, dev, "x")
        if post_weight is not None:
            _whole(post_weight, bf16, (H,), dev, "post_weight")
        if gate is not None:
            gate_stride = H if gate.dim() == 2 else 0
            _whole(gate, bf16, shape if gate_stride else (H,), dev, "gate")
        if residual_out is None:
            residual_out = torch.empty_like(residual)
        else:
            _whole(residual_out, bf16, shape, dev, "residual_out")
    if pre_weight is None:
        _need(y is None, "y belongs to pre_weight")
    else:
        _whole(pre_weight, bf16, (H,), dev, "pre_weight")
        if y is None:
            y = torch.empty_like(residual)
        else:
            _whole(y, bf16, shape, dev, "y")
    _check(_load().uattn_residual_norm(_ptr(x), _ptr(post_weight), _ptr(gate), gate_stride, scale, residual.data_ptr(),
                                       _ptr(pre_weight), eps, T, H, _ptr(residual_out), _ptr(y), _stream_on(dev)))
    return (residual if x is None else residual_out), y


@functools.lru_cache(maxsize=256)
def residual_norm_backward_workspace_bytes(num_tokens: int, hidden_dim: int) -> int:
    sizes = int(num_tokens), int(hidden_dim)
    return int(_load().uattn_residual_norm_backward_workspace_bytes(*sizes)) if _fits(*sizes) else 0


def residual_norm_backward(dy, dresidual_out, residual_out, pre_weight=None, x=None, post_weight=None, gate=None,
                           scale: float = 1.0, eps: float = 1e-6, dresidual=None, dx=None, has_block: Optional[bool] = None,
                           workspace=None, stream=None):
    """Gradients of residual_norm (uattn_residual_norm_backward).

      dy [T, H] bf16, gradient of y (None without pre_weight); dresidual_out [T, H]
      bf16, gradient of residual_out (None: zeros); residual_out as the forward
      returned it; x, post_weight, gate, scale, eps as passed to it.  has_block:
      whether the forward had an x (by default, whether x is given here: where it
      had neither post_weight nor gate, x itself is not read and need not be kept).
      Returns (dresidual, dx, dpre_weight, dpost_weight, dgate): bf16 rows, fp32
      [H] weight gradients, dgate fp32 [H] or bf16 [T, H] as the gate is; None for
      what the forward did not have.
    """
    import torch
    dev = _gpu_of(residual_out, "residual_out")
    there = _elsewhere(dev, stream)
    if there is not None:
        with there:
            return residual_norm_backward(dy, dresidual_out, residual_out, pre_weight, x, post_weight, gate, scale, eps,
                                          dresidual, dx, has_block, workspace)
    bf16, shape = torch.bfloat16, residual_out.shape
    _need(len(shape) == 2, "residual_out must be [T, H]")
    T, H = shape
    if T > _MOST or H > _MOST:
        _sizes(T, H)
    _whole(residual_out, bf16, shape, dev, "residual_out")
    if has_block is None:
        has_block = x is not None
    _need(has_block or (post_weight is None and gate is None and x is None and dx is None),
          "x, post_weight, gate and dx belong to a forward with a block's output")
    _need(x is not None or (post_weight is None and gate is None), "the gradients of post_weight and gate need x")
    _need((dy is None) == (pre_weight is None), "dy and pre_weight belong together")
    _need(dy is not None or dresidual_out is not None, "dy or dresidual_out must be given")
    for name, t in (("dy", dy), ("dresidual_out", dresidual_out), ("x", x), ("dresidual", dresidual), ("dx", dx)):
        if t is not None:
            _whole(t, bf16, shape, dev, name)
    gate_stride = 0
    if gate is not None:
        gate_stride = H if gate.dim() == 2 else 0
        _whole(gate, bf16, shape if gate_stride else (H,), dev, "gate")
    sums = []
    if pre_weight is not None:
        _whole(pre_weight, bf16, (H,), dev, "pre_weight")
        sums.append(0)
    if post_weight is not None:
        _whole(post_weight, bf16, (H,), dev, "post_weight")
        sums.append(1)
    if gate is not None and not gate_stride:
        sums.append(2)
    if dresidual is None:
        dresidual = torch.empty_like(residual_out)
    if has_block and dx is None:
        dx = torch.empty_like(residual_out)
    d = [None, None, torch.empty_like(gate) if gate_stride else None]
    if len(sums) == 1:
        d[sums[0]] = residual_out.new_empty(H, dtype=torch.float32)
    elif sums:
        # one allocation; every row starts 16-byte aligned, as H is a multiple of 8 in calls that are not refused
        for i, row in zip(sums, residual_out.new_empty((len(sums), H), dtype=torch.float32).unbind(0)):
            d[i] = row
    workspace = _workspace(workspace, residual_norm_backward_workspace_bytes(T, H), residual_out)
    _check(_load().uattn_residual_norm_backward(
        _ptr(dy), _ptr(dresidual_out), residual_out.data_ptr(), _ptr(pre_weight), _ptr(x), _ptr(post_weight), _ptr(gate),
        gate_stride, scale, eps, T, H, dresidual.data_ptr(), _ptr(dx), _ptr(d[0]), _ptr(d[1]), _ptr(d[2]),
        workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_on(dev)))
    return dresidual, dx, d[0], d[1], d[2]


def embedding(ids, table, scale: float = 1.0, out=None, stream=None):
    """Rows of the embedding table, scaled (uattn_embedding).

      ids [T] int32 (negative: padding, a row of zeros); table [V, H] bf16 (rows may be strided); returns [T, H] bf16.
    """
    import torch
    dev = _gpu_of(table, "table")
    there = _elsewhere(dev, stream)
    if there is not None:
        with there:
            return embedding(ids, table, scale, out)
    _rows(table, torch.bfloat16, dev, "table")
    _need(ids.dim() == 1, "ids must be [T]")
    _whole(ids, torch.int32, ids.shape, dev, "ids")
    T, (V, H) = ids.shape[0], table.shape
    if T > _MOST or V > _MOST or H > _MOST:
        _sizes(T, V, H)
    out = _out_rows(out, table, T, H)
    _check(_load().uattn_embedding(ids.data_ptr(), table.data_ptr(), _row_stride(table), scale, T, V, H, out.data_ptr(),
                                   _row_stride(out), _stream_on(dev)))
    return out


@functools.lru_cache(maxsize=256)
def embedding_backward_workspace_bytes(num_tokens: int, hidden_dim: int) -> int:
    sizes = int(num_tokens), int(hidden_dim)
    return int(_load().uattn_embedding_backward_workspace_bytes(*sizes)) if _fits(*sizes) else 0


def embedding_backward(dout, ids, vocab: int, scale: float = 1.0, grad=None, accumulate: bool = False, dtype=None,
                       workspace=None, stream=None):
    """The embedding table's gradient (uattn_embedding_backward).

      dout [T, H] bf16 (rows may be strided); ids [T] int32.  Returns grad [V, H],
      of ``dtype`` (bfloat16, or float32 by default) where none is given.  With
      ``accumulate`` the sums are added to ``grad``, whose other rows stay as they
      are; without, those rows become zeros.
    """
    import torch
    dev = _gpu_of(dout, "dout")
    there = _elsewhere(dev, stream)
    if there is not None:
        with there:
            return embedding_backward(dout, ids, vocab, scale, grad, accumulate, dtype, workspace)
    _rows(dout, torch.bfloat16, dev, "dout")
    T, H = dout.shape
    _whole(ids, torch.int32, (T,), dev, "ids")
    vocab = int(vocab)
    if T > _MOST or vocab > _MOST or H > _MOST:
        _sizes(T, vocab, H)
    if grad is None:
        _need(not accumulate, "accumulate needs grad")
        dtype = torch.float32 if dtype is None else dtype
    else:
        _need(dtype is None or dtype == grad.dtype, "grad is of another dtype")
        dtype = grad.dtype
        _rows(grad, dtype, dev, "grad")
        _need(grad.shape == (vocab, H), "grad must be [vocab, H]")
    _need(dtype in (torch.float32, torch.bfloat16), "grad must be float32 or bfloat16")
    if grad is None:
        _need(vocab >= 0, "vocab must not be negative")
        grad = dout.new_empty((vocab, H), dtype=dtype)
    workspace = _workspace(workspace, embedding_backward_workspace_bytes(T, H), dout)
    _check(_load().uattn_embedding_backward(
        dout.data_ptr(), _row_stride(dout), ids.data_ptr(), scale, T, vocab, H, grad.data_ptr(), _row_stride(grad),
        int(dtype == torch.float32), int(bool(accumulate)), workspace.data_ptr(),
        workspace.numel() * workspace.element_size(), _stream_on(dev)))
    return grad


def _penalty_parts(rows, tokens, history, penalties, dev) -> int:
    """Checks; how many tokens there are."""
    if history is None:
        _need(tokens is None and penalties is None, "tokens, history and penalties belong together")
        return 0
    import torch
    _need(tokens is not None and penalties is not None, "tokens, history and penalties belong together")
    _need(tokens.dim() == 1, "tokens must be 1-D")
    _whole(tokens, torch.int32, tokens.shape, dev, "tokens")
    _whole(history, torch.int32, (rows, 3), dev, "history")
    _whole(penalties, torch.float32, (rows, 3), dev, "penalties")
    n = tokens.shape[0]
    if n > _MOST:
        _sizes(n)
    return n


def _mask_parts(rows, vocab, mask, mask_rows, dev) -> Tuple[int, int]:
    """Checks; (masks, words from mask to mask)"""
    if mask is None:
        _need(mask_rows is None, "mask_rows belongs to mask")
        return 0, 0
    import torch
    _rows(mask, torch.int32, dev, "mask")
    masks, words = mask.shape
    if masks > _MOST:
        _sizes(masks)
    _need(words >= (vocab + 31) // 32, "mask must have a bit for every vocabulary entry")
    if mask_rows is None:
        _need(masks >= rows, "mask needs a row for every row of logits, or mask_rows")
    else:
        _whole(mask_rows, torch.int32, (rows,), dev, "mask_rows")
    return masks, mask.stride(0) if masks > 1 else words


def logits_process(logits, tokens=None, history=None, penalties=None, bias_ids=None, bias_values=None, bias_rows=None,
                   mask=None, mask_rows=None, out=None, stream=None):
    """Penalties for repeated tokens, biases and grammar masks (uattn_logits_process).

      logits [T, V] bf16 (rows may be strided); tokens [N] int32, packed sequences;
      history [T, 3] int32 (begin, start of the response, end) and penalties [T, 3]
      fp32 (repetition, frequency, presence) of every row; bias_ids [M] int32,
      bias_values [M] fp32, bias_rows [T, 2] int32 (begin, end); mask [K, >= V/32]
      int32 words (a set bit allows), mask_rows [T] int32 (negative: no mask).
      Returns bf16 [T, V]; out may be logits (in place).
    """
    import torch
    dev = _gpu_of(logits, "logits")
    there = _elsewhere(dev, stream)
    if there is not None:
        with there:
            return logits_process(logits, tokens, history, penalties, bias_ids, bias_values, bias_rows, mask, mask_rows, out)
    _rows(logits, torch.bfloat16, dev, "logits")
    T, V = logits.shape
    if T > _MOST or V > _MOST:
        _sizes(T, V)
    num_tokens = _penalty_parts(T, tokens, history, penalties, dev)
    num_masks, mask_stride = _mask_parts(T, V, mask, mask_rows, dev)
    num_bias = 0
    if bias_rows is None:
        _need(bias_ids is None and bias_values is None, "bias_ids, bias_values and bias_rows belong together")
    else:
        _need(bias_ids is not None and bias_values is not None, "bias_ids, bias_values and bias_rows belong together")
        _need(bias_ids.dim() == 1, "bias_ids must be [M]")
        _whole(bias_ids, torch.int32, bias_ids.shape, dev, "bias_ids")
        _whole(bias_values, torch.float32, bias_ids.shape, dev, "bias_values")
        _whole(bias_rows, torch.int32, (T, 2), dev, "bias_rows")
        num_bias = bias_ids.shape[0]
        if num_bias > _MOST:
            _sizes(num_bias)
    out = _out_rows(out, logits, T, V)
    _check(_load().uattn_logits_process(
        logits.data_ptr(), _row_stride(logits), T, V, _ptr(tokens), num_tokens, _ptr(history), _ptr(penalties),
        _ptr(bias_ids), _ptr(bias_values), num_bias, _ptr(bias_rows), _ptr(mask), mask_stride, num_masks,
        _ptr(mask_rows), out.data_ptr(), _row_stride(out), _stream_on(dev)))
    return out


def logits_process_backward(dout, logits, tokens=None, history=None, penalties=None, mask=None, mask_rows=None, out=None,
                            stream=None):
    """Gradient of logits_process with respect to the logits (uattn_logits_process_backward).

      dout [T, V] bf16, gradient of the processed logits; the others as passed to
      logits_process.  Returns bf16 [T, V]; out may be dout (in place).
    """
    import torch
    dev = _gpu_of(logits, "logits")
    there = _elsewhere(dev, stream)
    if there is not None:
        with there:
            return logits_process_backward(dout, logits, tokens, history, penalties, mask, mask_rows, out)
    _rows(logits, torch.bfloat16, dev, "logits")
    _rows(dout, torch.bfloat16, dev, "dout")
    T, V = logits.shape
    if T > _MOST or V > _MOST:
        _sizes(T, V)
    _need(dout.shape == (T, V), "dout must be of the logits' shape")
    num_tokens = _penalty_parts(T, tokens, history, penalties, dev)
    num_masks, mask_stride = _mask_parts(T, V, mask, mask_rows, dev)
    out = _out_rows(out, logits, T, V)
    _check(_load().uattn_logits_process_backward(
        dout.data_ptr(), _row_stride(dout), logits.data_ptr(), _row_stride(logits), T, V, _ptr(tokens), num_tokens,
        _ptr(history), _ptr(penalties), _ptr(mask), mask_stride, num_masks, _ptr(mask_rows), out.data_ptr(),
        _row_stride(out), _stream_on(dev)))
    return out


def logprob_backward(logits, targets, dlogp, inv_temperature: float = 1.0, out=None, stream=None):
    """Gradient of logprob with respect to the logits (uattn_logprob_backward).

      logits [T, V] bf16 and targets [T] int32 as passed to logprob; dlogp [T] fp32
      (0: the row gets zeros).  Returns bf16 [T, V]; out may not be logits.
    """
    import torch
    dev = _gpu_of(logits, "logits")
    there = _elsewhere(dev, stream)
    if there is not None:
        with there:
            return logprob_backward(logits, targets, dlogp, inv_temperature, out)
    _rows(logits, torch.bfloat16, dev, "logits")
    T, V = logits.shape
    if T > _MOST or V > _MOST:
        _sizes(T, V)
    _whole(targets, torch.int32, (T,), dev, "targets")
    _whole(dlogp, torch.float32, (T,), dev, "dlogp")
    out = _out_rows(out, logits, T, V)
    _check(_load().uattn_logprob_backward(logits.data_ptr(), _row_stride(logits), targets.data_ptr(), dlogp.data_ptr(), T, V,
                                          inv_temperature, out.data_ptr(), _row_stride(out), _stream_on(dev)))
    return out


# ---------------------------------------------------------------------------
# The KV cache held in 8 or 4 bits.  Its calls run where and as the row-wise
# operators' do (above).
# ---------------------------------------------------------------------------
MX_BLOCK = 32  # elements of a row to a scale


def mx_cache(num_pages: int, num_kv_heads: int, page_size: int, head_dim: int, k_bits: int = 8, v_bits: int = 8,
             device="cuda"):
    """A new cache in k_bits and v_bits (8 or 4): (k_codes, k_scales, v_codes, v_scales), uint8, of zeros.

      codes [num_pages, num_kv_heads, page_size, head_dim * bits / 8], scales [.., head_dim / 32]
    """
    import torch
    _need(k_bits in (8, 4) and v_bits in (8, 4), "k_bits and v_bits are 8 or 4")
    _need(head_dim in (64, 128), "head_dim is 64 or 128")
    rows = (num_pages, num_kv_heads, page_size)
    return tuple(torch.zeros((*rows, width), dtype=torch.uint8, device=device)
                 for width in (head_dim * k_bits // 8, head_dim // MX_BLOCK, head_dim * v_bits // 8, head_dim // MX_BLOCK))


# A step's calls are short, so what is right is found right by one expression over all
# tensors, and which of them is not is looked up only then.
def _mx_pools(k_codes, k_scales, v_codes, v_scales, dev):
    """(P, Hkv, page, d, k_bits, v_bits) of a cache's four tensors."""
    import torch
    u8, shape, ks, vs = torch.uint8, k_scales.shape, k_codes.shape, v_codes.shape
    if len(shape) != 4 or len(ks) != 4 or len(vs) != 4:
        raise ValueError("codes must be [P,Hkv,page,d] (8 bits) or [P,Hkv,page,d/2] (4), scales [P,Hkv,page,d/32]")
    P, hkv, page, blocks = shape
    d = blocks * MX_BLOCK
    kb, vb = 8 if ks[3] == d else 4, 8 if vs[3] == d else 4
    if not (k_codes.dtype is k_scales.dtype is v_codes.dtype is v_scales.dtype is u8 and v_scales.shape == shape
            and ks == (P, hkv, page, d * kb // 8) and vs == (P, hkv, page, d * vb // 8)
            and k_codes.get_device() == k_scales.get_device() == v_codes.get_device() == v_scales.get_device() == dev
            and k_codes.is_contiguous() and k_scales.is_contiguous() and v_codes.is_contiguous() and v_scales.is_contiguous()):
        for name, t, width in (("k_scales", k_scales, blocks), ("v_scales", v_scales, blocks), ("k_codes", k_codes, d * kb // 8),
                               ("v_codes", v_codes, d * vb // 8)):
            _whole(t, u8, (P, hkv, page, width), dev, name)
    return P, hkv, page, d, kb, vb


def _kv_rows(k, v, dev, names):
    """Elements from token to token of [N,Hkv,d] keys and values whose heads and elements are contiguous."""
    import torch
    shape, stride, bf16 = k.shape, k.stride(), torch.bfloat16
    if len(shape) != 3 or v.shape != shape:
        raise ValueError(f"{names} must be [N,Hkv,d], both the same")
    n, hkv, d = shape
    if not (k.dtype is bf16 and v.dtype is bf16 and k.get_device() == dev and v.get_device() == dev):
        raise ValueError(f"{names} must be bfloat16 on GPU {dev}")
    if v.stride() == stride and stride[1] == d and stride[2] == 1:
        return stride[0] if n > 1 else hkv * d  # torch may report any stride for one token
    for t in (k, v):
        if n and (t.stride(2) != 1 or (hkv > 1 and t.stride(1) != d)):
            raise ValueError(f"{names}: heads and their elements must be contiguous")
    if n <= 1:
        return hkv * d
    if k.stride(0) != v.stride(0):
        raise ValueError(f"{names} must have the same token stride")
    return stride[0]


def _kv_outputs(k_out, v_out, shape, like, dev):
    """(k_out, v_out, elements from token to token) of outputs of this shape, made where they are not given (beside a given
    one: alike)."""
    import torch
    n, hkv, d = shape
    if k_out is None and v_out is None:
        return like.new_empty(shape, dtype=torch.bfloat16), like.new_empty(shape, dtype=torch.bfloat16), hkv * d
    given = v_out if k_out is None else k_out
    _need(given.shape == shape and (v_out is None or v_out.shape == shape), "k_out/v_out shape")
    stride = _kv_rows(given, given if v_out is None else v_out, dev, "k_out/v_out")
    if k_out is None or v_out is None:
        made = torch.empty_strided(shape, (stride, d, 1), dtype=torch.bfloat16, device=given.device)
        k_out, v_out = (made, v_out) if k_out is None else (k_out, made)
    return k_out, v_out, stride


def _kv_places(block_table, seq_idx, positions, N, dev):
    """(B, maxp) of the indices that say where N tokens live."""
    import torch
    i32, shape = torch.int32, block_table.shape
    if len(shape) != 2:
        raise ValueError("block_table must be [B,maxp]")
    if not (block_table.dtype is seq_idx.dtype is positions.dtype is i32 and seq_idx.shape == positions.shape == (N,)
            and block_table.get_device() == seq_idx.get_device() == positions.get_device() == dev
            and block_table.is_contiguous() and seq_idx.is_contiguous() and positions.is_contiguous()):
        for name, t, want in (("block_table", block_table, shape), ("seq_idx", seq_idx, (N,)), ("positions", positions, (N,))):
            _whole(t, i32, want, dev, name)
    return shape


def kv_write_mx(k_new, v_new, block_table, seq_idx, positions, k_codes, k_scales, v_codes, v_scales, stream=None):
    """Write new K/V token rows into a cache in 8 or 4 bits, in place (uattn_kv_write_mx).

      k_new, v_new   [N, Hkv, d] bf16 (token rows may be strided: stride(0) elements apart)
      block_table    [B, maxp] int32; seq_idx, positions [N] int32 (position < 0: padding)
      k_codes .. v_scales   the cache (mx_cache), whose widths say in how many bits
    """
    dev = _gpu_of(k_codes, "k_codes")
    there = _elsewhere(dev, stream)
    if there is not None:
        with there:
            return kv_write_mx(k_new, v_new, block_table, seq_idx, positions, k_codes, k_scales, v_codes, v_scales)
    P, hkv, page, d, kb, vb = _mx_pools(k_codes, k_scales, v_codes, v_scales, dev)
    stride = _kv_rows(k_new, v_new, dev, "k_new/v_new")
    N, rows, width = k_new.shape
    if rows != hkv or width != d:
        raise ValueError("the cache is of other heads")
    B, maxp = _kv_places(block_table, seq_idx, positions, N, dev)
    if max(N, B, maxp, page, P, hkv) > _MOST:
        _sizes(N, B, maxp, page, P, hkv)
    _check(_load().uattn_kv_write_mx(k_new.data_ptr(), v_new.data_ptr(), stride, block_table.data_ptr(), seq_idx.data_ptr(),
                                     positions.data_ptr(), N, B, maxp, page, P, hkv, d, kb, vb, k_codes.data_ptr(),
                                     k_scales.data_ptr(), v_codes.data_ptr(), v_scales.data_ptr(), _stream_on(dev)))
    return k_codes, k_scales, v_codes, v_scales


def kv_read_mx(k_codes, k_scales, v_codes, v_scales, block_table, seq_idx, positions, k_out=None, v_out=None, stream=None):
    """Rows of a cache in 8 or 4 bits as bf16, packed (uattn_kv_read_mx).  A prefill over them takes
    the queries of all rows; single queries attend to the cache itself (decode_mx).

      seq_idx, positions [N] int32: row n is the token at positions[n] of sequence seq_idx[n]
      (zeros for padding, position < 0, and tokens without a place)
    Returns (k, v) [N, Hkv, d] bf16 (of k_out and v_out one may be given alone).
    """
    dev = _gpu_of(k_codes, "k_codes")
    there = _elsewhere(dev, stream)
    if there is not None:
        with there:
            return kv_read_mx(k_codes, k_scales, v_codes, v_scales, block_table, seq_idx, positions, k_out, v_out)
    P, hkv, page, d, kb, vb = _mx_pools(k_codes, k_scales, v_codes, v_scales, dev)
    N = positions.shape[0] if positions.dim() == 1 else -1
    B, maxp = _kv_places(block_table, seq_idx, positions, N, dev)
    if max(N, B, maxp, page, P, hkv) > _MOST:
        _sizes(N, B, maxp, page, P, hkv)
    k_out, v_out, stride = _kv_outputs(k_out, v_out, (N, hkv, d), k_codes, dev)
    _check(_load().uattn_kv_read_mx(k_codes.data_ptr(), k_scales.data_ptr(), v_codes.data_ptr(), v_scales.data_ptr(), kb, vb,
                                    block_table.data_ptr(), seq_idx.data_ptr(), positions.data_ptr(), N, B, maxp, page, P, hkv,
                                    d, k_out.data_ptr(), v_out.data_ptr(), stride, _stream_on(dev)))
    return k_out, v_out


def kv_round_mx(k, v, k_bits: int = 8, v_bits: int = 8, k_out=None, v_out=None, stream=None):
    """The values that a cache in k_bits and v_bits would hold for packed rows (uattn_kv_round_mx).

      k, v [N, Hkv, d] bf16 (token rows may be strided).  Returns (k_out, v_out), which
      may be k and v themselves (in place), or one given alone.  The gradient of the
      rounded rows passes to the rows as it is.
    """
    dev = _gpu_of(k, "k")
    there = _elsewhere(dev, stream)
    if there is not None:
        with there:
            return kv_round_mx(k, v, k_bits, v_bits, k_out, v_out)
    _need(k_bits in (8, 4) and v_bits in (8, 4), "k_bits and v_bits are 8 or 4")
    stride = _kv_rows(k, v, dev, "k/v")
    N, hkv, d = shape = k.shape
    if N > _MOST or hkv > _MOST or d > _MOST:
        _sizes(N, hkv, d)
    k_out, v_out, out_stride = _kv_outputs(k_out, v_out, shape, k, dev)
    _check(_load().uattn_kv_round_mx(k.data_ptr(), v.data_ptr(), stride, N, hkv, d, k_bits, v_bits, k_out.data_ptr(),
                                     v_out.data_ptr(), out_stride, _stream_on(dev)))
    return k_out, v_out


def decode_mx(q, k_codes, k_scales, v_codes, v_scales, block_table, seqlens, max_seqlen: int,
              softmax_scale: Optional[float] = None, out=None, return_lse: bool = False, lse=None, workspace=None, stream=None):
    """Token-wise paged decode against a cache in 8 or 4 bits (uattn_decode_mx).

    q [B,Hq,d] bf16; the cache as mx_cache makes it; block_table, seqlens, max_seqlen,
    out and lse as for :func:`decode`.  ``workspace``: decode_mx_workspace_bytes(...) bytes,
    whatever they hold; one is allocated when not given.  A decode's own may serve: which of its
    counters this call leaves zero is recorded, and :func:`decode` clears the others.  A graph's
    replays and the runs of DecodeSteps neither record nor clear: one that they share holds
    these bytes and the decode's counters (counter_bytes) side by side.
    """
    import torch
    dev = _gpu_of(q, "q")
    there = _elsewhere(dev, stream)
    if there is not None:
        with there:
            return decode_mx(q, k_codes, k_scales, v_codes, v_scales, block_table, seqlens, max_seqlen, softmax_scale, out,
                             return_lse, lse, workspace)
    bf16, i32, shape, table = torch.bfloat16, torch.int32, q.shape, block_table.shape
    if len(shape) != 3 or len(table) != 2:
        raise ValueError("q must be [B,Hq,d], block_table [B,maxp]")
    B, hq, d = shape
    P, hkv, page, d2, kb, vb = _mx_pools(k_codes, k_scales, v_codes, v_scales, dev)
    if d2 != d:
        raise ValueError("head_dim mismatch")
    maxp, most = table[1], int(max_seqlen)
    if not (q.dtype is bf16 and block_table.dtype is seqlens.dtype is i32 and table[0] == B and seqlens.shape == (B,)
            and block_table.get_device() == seqlens.get_device() == dev
            and q.is_contiguous() and block_table.is_contiguous() and seqlens.is_contiguous()):
        _whole(q, bf16, shape, dev, "q")
        _whole(block_table, i32, (B, maxp), dev, "block_table")
        _whole(seqlens, i32, (B,), dev, "seqlens")
    if max(B, maxp, page, P, most, hq, hkv) > _MOST or most < -_MOST:
        _sizes(B, maxp, page, P, most, hq, hkv)
    if out is None:
        out = torch.empty_like(q)
    else:
        _whole(out, bf16, shape, dev, "out")
    if lse is not None:
        _whole(lse, torch.float32, (B, hq), dev, "lse")
    elif return_lse:
        lse = q.new_empty((B, hq), dtype=torch.float32)
    size = 0
    if workspace is not None:
        workspace = _workspace(workspace, 0, q)
        size = workspace.numel() * workspace.element_size()
        known = getattr(workspace, "_uattn_zero_prefix", 0)
        if known and _decode_mx_need(B, most, hq, hkv, d):
            # counters of a decode that the partials reach are no longer known to be zero
            workspace._uattn_zero_prefix = max(0, min(known, _partials_start(size, B, most, hq, d)))
    else:
        size = _decode_mx_need(B, most, hq, hkv, d)
        if size:
            workspace = q.new_empty(size, dtype=torch.uint8)  # no initial contents needed
    _check(_load().uattn_decode_mx(q.data_ptr(), k_codes.data_ptr(), k_scales.data_ptr(), v_codes.data_ptr(),
                                   v_scales.data_ptr(), kb, vb, block_table.data_ptr(), seqlens.data_ptr(), B, maxp, page, P,
                                   most, hq, hkv, d, default_scale(d) if softmax_scale is None else softmax_scale,
                                   out.data_ptr(), _ptr(lse), _ptr(workspace), size, _stream_on(dev)))
    return (out, lse) if lse is not None else out


def decode_mx_workspace_bytes(batch: int, max_seqlen: int, num_q_heads: int, num_kv_heads: int, head_dim: int) -> int:
    sizes = batch, max_seqlen, num_q_heads, num_kv_heads, head_dim
    return _decode_mx_need(*sizes) if _fits(*sizes) else 0


@functools.lru_cache(maxsize=256)
def _decode_mx_need(batch: int, max_seqlen: int, num_q_heads: int, num_kv_heads: int, head_dim: int) -> int:
    return int(_load().uattn_decode_mx_workspace_bytes(batch, max_seqlen, num_q_heads, num_kv_heads, head_dim))


def raw_call(name: str, *args) -> int:
    """Call a C entry point with raw arguments (for error-path tests)."""
    return int(getattr(_load(), name)(*args))


class DecodeSteps:
    """Argument lists for a run of uattn_decode calls over fixed buffers.

    A rollout loop calls decode once per generated token on the same cache,
    block table and workspace; only the query, length and output slices
    change.  This marshals every call's arguments once, so the loop pays one
    ctypes call per step.

      q_steps        [S, B, Hq, d] bf16   (step i uses q_steps[i])
      seqlens_steps  [S, B] int32
      out_steps      [S, B, Hq, d] bf16
    """

    def __init__(self, q_steps, k_pages, v_pages, block_table, seqlens_steps, max_seqlen: int, out_steps,
                 workspace=None, softmax_scale: Optional[float] = None, stream=None):
        import torch
        for name, t in (("q_steps", q_steps), ("k_pages", k_pages), ("v_pages", v_pages), ("out_steps", out_steps)):
            _bf16_cuda(t, name)
        _need(q_steps.dim() == 4 and out_steps.shape == q_steps.shape, "q_steps/out_steps must be [S,B,Hq,d]")
        S, B, hq, d = q_steps.shape
        _, hkv, page, d2 = k_pages.shape
        _need(d2 == d and v_pages.shape == k_pages.shape, "page shapes")
        _need(seqlens_steps.dtype == torch.int32 and seqlens_steps.shape == (S, B) and seqlens_steps.is_contiguous(),
              "seqlens_steps must be [S,B] int32")
        _need(block_table.dtype == torch.int32 and block_table.is_contiguous() and block_table.shape[0] == B,
              "block_table must be [B,maxp] int32")
        _sizes(B, block_table.shape[1], page, k_pages.shape[0], int(max_seqlen), hq, hkv, d)
        if softmax_scale is None:
            softmax_scale = default_scale(d)
        need = decode_workspace_bytes(B, int(max_seqlen), hq, d)
        if workspace is None and need > 0:
            workspace = new_workspace(need, q_steps.device)
        if workspace is not None and need > 0:
            _need(workspace.is_cuda and workspace.is_contiguous(), "workspace must be a contiguous GPU tensor")
            _prepare_workspace(workspace, B, int(max_seqlen), hq, d)
        self.workspace = workspace
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        st = _stream(stream)
        qstride = B * hq * d * 2
        lstride = B * 4
        self._fn = _load().uattn_decode
        self.args = [
            (q_steps.data_ptr() + i * qstride, _ptr(k_pages), _ptr(v_pages), _ptr(block_table),
             seqlens_steps.data_ptr() + i * lstride, B, block_table.shape[1], page, k_pages.shape[0], int(max_seqlen),
             hq, hkv, d, float(softmax_scale), out_steps.data_ptr() + i * qstride, None, _ptr(workspace), ws_bytes, st)
            for i in range(S)
        ]
        self._keep = (q_steps, k_pages, v_pages, block_table, seqlens_steps, out_steps)

    def __len__(self):
        return len(self.args)

    def run(self, i: int, stream=None):
        """Launch step i (on ``stream`` if given, else the stream fixed at construction)."""
        a = self.args[i]
        if stream is not None:
            a = a[:-1] + (_stream(stream),)
        code = self._fn(*a)
        if code != UATTN_OK:
            raise UattnError(status_string(code))
