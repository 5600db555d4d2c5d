"""Binding of the attention of include/zf_layer.h: between the projections
whose weights the selective update steps.

Argument marshalling only, as in layer.py, whose notes on `stream` hold here.
"""

from __future__ import annotations

import ctypes
from functools import lru_cache
from typing import NamedTuple, Optional, Tuple

import torch

from ._lib import (LIB, ZfAttention, ZfHeads, _check, _empty, _many_gpus, _ptr, _same_device,
                   _stream, _workspace)

BF16 = torch.bfloat16


def _heads(t: torch.Tensor, name: str, tokens: Optional[int] = None, heads: Optional[int] = None,
           dim: Optional[int] = None) -> ZfHeads:
    if t.dtype != BF16:
        raise TypeError(f"{name}: expected {BF16}, got {t.dtype}")
    shape = t.shape
    if len(shape) != 3:
        raise ValueError(f"{name}: expected [tokens, heads, dim], got shape {tuple(shape)}")
    n, h, d = shape
    if ((tokens is not None and n != tokens) or (heads is not None and h != heads)
            or (dim is not None and d != dim)):
        raise ValueError(f"{name}: expected {(tokens, heads, dim)} (None: any), got shape "
                         f"{tuple(shape)}")
    lt, lh, le = t.stride()
    at = t.data_ptr()
    if n and h and d:
        if not t.is_cuda:
            raise ValueError(f"{name}: must live on a GPU")
        if le != 1 and d > 1:
            raise ValueError(f"{name}: a head's elements must be contiguous (stride(2) == 1)")
        if at % 16 or (n > 1 and lt % 8) or (h > 1 and lh % 8):
            raise ValueError(f"{name}: vectors must be 16-byte aligned (data pointer and strides)")
    return ZfHeads(at or None, lt if n > 1 else 0, lh if h > 1 else 0)


def _ints(t: Optional[torch.Tensor], name: str, n: int) -> Optional[int]:
    if t is None:
        return None
    if t.dtype != torch.int32:
        raise TypeError(f"{name}: expected int32, got {t.dtype}")
    if t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name}: expected {n} contiguous elements, got shape {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError(f"{name}: must live on a GPU")
    return t.data_ptr()


def _shapes(q, k, seq_q, seq_k, len_k, causal, scale) -> ZfAttention:
    tokens, n_heads, dim = q.shape
    keys, kv, _ = k.shape
    if not n_heads or not kv or n_heads % kv:
        raise ValueError(f"q's {n_heads} heads are no multiple of k's {kv}")
    if dim % 8 or not 8 <= dim <= 128:
        raise ValueError(f"a head's width is a multiple of 8 up to 128, got {dim}")
    count = 1
    if seq_q is None:
        if seq_k is not None or len_k is not None:
            raise ValueError("seq_k and len_k go with seq_q")
        at_q = at_k = at_len = None
    else:
        count = seq_q.numel() - 1
        if count < 1:
            raise ValueError("seq_q: expected the sequences' starts and the end")
        at_q = at_k = _ints(seq_q, "seq_q", count + 1)
        if seq_k is not None:
            at_k = _ints(seq_k, "seq_k", count + 1)
        elif keys != tokens:
            raise ValueError("without seq_k the keys are as many as the queries")
        at_len = _ints(len_k, "len_k", count)
    return ZfAttention(tokens, keys, count, n_heads, kv, dim, 1 if causal else 0,
                       dim ** -0.5 if scale is None else float(scale), at_q, at_k, at_len)


@lru_cache(maxsize=4096)
def _workspace_bytes(backward: bool, tokens: int, keys: int, sequences: int, heads: int, kv: int,
                     dim: int) -> int:
    # (the sizes alone count: any addresses stand for the sequences' starts)
    shapes = ZfAttention(tokens, keys, sequences, heads, kv, dim, 1, 1.0, 16, 16, None)
    f = (LIB.zf_attention_backward_workspace_bytes if backward
         else LIB.zf_attention_forward_workspace_bytes)
    return f(ctypes.byref(shapes))


def _need(backward: bool, s: ZfAttention) -> int:
    return _workspace_bytes(backward, s.tokens_q, s.tokens_k, s.sequences, s.heads, s.kv_heads, s.dim)


class Attention(NamedTuple):
    """What attention returns; lse: None where not wanted."""
    out: torch.Tensor
    lse: Optional[torch.Tensor]


def _lse(t: torch.Tensor, heads: int, tokens: int) -> None:
    if t.dtype != torch.float32:
        raise TypeError(f"lse: expected float32, got {t.dtype}")
    if t.shape != (heads, tokens) or not t.is_contiguous():
        raise ValueError(f"lse: expected contiguous {(heads, tokens)}, got shape {tuple(t.shape)}")
    if t.numel() and not t.is_cuda:
        raise ValueError("lse: must live on a GPU")


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
              seq_q: Optional[torch.Tensor] = None, seq_k: Optional[torch.Tensor] = None,
              len_k: Optional[torch.Tensor] = None, causal: bool = True,
              scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
              lse: Optional[torch.Tensor] = None, want_lse: bool = False,
              workspace: Optional[torch.Tensor] = None, stream=None) -> Attention:
    """Attention (zf_attention_forward).  q [tokens, heads, dim], k and v [keys,
    kv_heads, dim], bf16, any strides that keep a head's elements contiguous
    and 16-byte aligned; heads a multiple of kv_heads; dim a multiple of 8 up to
    128.  scale: 1 / sqrt(dim) by default.

    seq_q, seq_k: int32 GPU tensors, each sequence's first token and, last, the
    end (seq_k None: seq_q's; both None: one sequence of all tokens).  len_k:
    int32, how many of a sequence's keys are used, for a cache with room.  They
    are read on the GPU: a captured call follows their contents.  With causal,
    a sequence's last query sees all of its keys, the one before one less, and
    so on: a prompt, a chunk of one behind a cache, or a single token.  (Long prompts
    among many single tokens are faster in a call of their own: how a call is divided
    follows its sequences' average length.)

    out: bf16 as q; lse (want_lse, or given): fp32 [heads, tokens], for
    attention_backward.  New ones hold nothing where tokens belong to no
    sequence."""
    tokens, heads, dim = q.shape if q.dim() == 3 else (None, None, None)
    c_q = _heads(q, "q")
    c_k = _heads(k, "k", None, None, dim)
    c_v = _heads(v, "v", k.shape[0], k.shape[1], dim)
    shapes = _shapes(q, k, seq_q, seq_k, len_k, causal, scale)
    if _many_gpus():
        _same_device(stream, q=q, k=k, v=v, seq_q=seq_q, seq_k=seq_k, len_k=len_k, out=out, lse=lse,
                     workspace=workspace)
    if out is None:
        out = _empty((tokens, heads, dim), BF16, q.device, stream)
    c_out = _heads(out, "out", tokens, heads, dim)
    if lse is not None:
        _lse(lse, heads, tokens)
    elif want_lse:
        lse = _empty((heads, tokens), torch.float32, q.device, stream)
    if workspace is None:
        need = _need(False, shapes)
        if need:
            workspace = _empty(need, torch.uint8, q.device, stream)
    ref = ctypes.byref
    _check("zf_attention_forward", LIB.zf_attention_forward(
        ref(shapes), ref(c_q), ref(c_k), ref(c_v), ref(c_out), _ptr(lse), _ptr(workspace),
        _workspace(workspace), _stream(stream)))
    return Attention(out, lse)


def attention_workspace_bytes(q: torch.Tensor, k: torch.Tensor, sequences: int = 1) -> int:
    """Workspace bytes of attention(q, k, ...) with so many sequences."""
    return _workspace_bytes(False, q.shape[0], k.shape[0], sequences, q.shape[1], k.shape[1],
                            q.shape[2])


def attention_backward_workspace_bytes(q: torch.Tensor, k: torch.Tensor, sequences: int = 1) -> int:
    """Workspace bytes of attention_backward(..., q, k, ...) with so many sequences."""
    return _workspace_bytes(True, q.shape[0], k.shape[0], sequences, q.shape[1], k.shape[1],
                            q.shape[2])


def attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                       out: torch.Tensor, lse: torch.Tensor, seq_q: Optional[torch.Tensor] = None,
                       seq_k: Optional[torch.Tensor] = None, causal: bool = True,
                       scale: Optional[float] = None, dq: Optional[torch.Tensor] = None,
                       dk: Optional[torch.Tensor] = None, dv: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None, stream=None
                       ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(dq, dk, dv) of attention, from its out and lse (zf_attention_backward), bf16
    in the shapes of q, k and v.  They may be given, as columns of one buffer
    for instance; gradients that are not hold nothing where tokens belong to no
    sequence."""
    tokens, heads, dim = q.shape if q.dim() == 3 else (None, None, None)
    c_q = _heads(q, "q")
    c_k = _heads(k, "k", None, None, dim)
    keys, kv = k.shape[:2]
    c_v = _heads(v, "v", keys, kv, dim)
    c_out, c_do = _heads(out, "out", tokens, heads, dim), _heads(dout, "dout", tokens, heads, dim)
    shapes = _shapes(q, k, seq_q, seq_k, None, causal, scale)
    _lse(lse, heads, tokens)
    if _many_gpus():
        _same_device(stream, q=q, k=k, v=v, out=out, lse=lse, dout=dout, seq_q=seq_q, seq_k=seq_k,
                     dq=dq, dk=dk, dv=dv, workspace=workspace)
    if dq is None:
        dq = _empty((tokens, heads, dim), BF16, q.device, stream)
    if dk is None:
        dk = _empty((keys, kv, dim), BF16, q.device, stream)
    if dv is None:
        dv = _empty((keys, kv, dim), BF16, q.device, stream)
    c_dq, c_dk, c_dv = (_heads(dq, "dq", tokens, heads, dim), _heads(dk, "dk", keys, kv, dim),
                        _heads(dv, "dv", keys, kv, dim))
    if workspace is None:
        need = _need(True, shapes)
        if need:
            workspace = _empty(need, torch.uint8, q.device, stream)
    ref = ctypes.byref
    _check("zf_attention_backward", LIB.zf_attention_backward(
        ref(shapes), ref(c_q), ref(c_k), ref(c_v), ref(c_out), _ptr(lse), ref(c_do), ref(c_dq),
        ref(c_dk), ref(c_dv), _ptr(workspace), _workspace(workspace), _stream(stream)))
    return dq, dk, dv
