"""``torch.autograd`` entry point of the MALA attention path (marshalling only: Algorithm 1 in the forward, Algorithm 2
in the backward, both in the library's kernels; the saved tensors are q, k, v, o and the log-normalizer, nothing else).

Note that, as the paper states in Section 2.2, the backward is Algorithm 2 on the LSE-derived support, not the exact
derivative of the forward's output; at tau = 0 it is the exact FullAttn gradient.
"""
from __future__ import annotations

import math
from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import mala


def _incoming(do: torch.Tensor) -> torch.Tensor:
    """An incoming gradient as the kernels read it: autograd also hands over one row for all rows (a stride of 0, from a sum or a mean)
    and slices of wider tensors, which are copied where a row does not begin on 16 bytes."""
    s = do.stride()
    if s[3] == 1 and do.data_ptr() % 16 == 0 and all(n == 1 or (x > 0 and x % 8 == 0) for n, x in zip(do.shape[:3], s)):
        return do
    return do.clone(memory_format=torch.contiguous_format)


class _MalaAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, tau: float, scale: float, causal: bool):
        o, lse, _ = mala.fwd_chunk(q, k, v, scale, tau, causal=causal)
        ctx.save_for_backward(q, k, v, o, lse)
        ctx.tau, ctx.scale, ctx.causal = tau, scale, causal
        return o

    @staticmethod
    def backward(ctx, do):
        q, k, v, o, lse = ctx.saved_tensors
        do = _incoming(do)
        dq, dk, dv, _ = mala.bwd_chunk(q, k, v, o, do, lse, ctx.scale, ctx.tau, causal=ctx.causal)
        return dq, dk, dv, None, None, None


class _MalaAttentionPacked(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, cu_q, cu_k, max_q: int, max_k: int, tau: float, scale: float, causal: bool):
        o, lse, _ = mala.fwd_varlen_prefix(q, k, v, cu_q, cu_k, max_q, max_k, scale, tau, causal=causal)
        ctx.save_for_backward(q, k, v, o, lse, cu_q, cu_k)
        ctx.args = (max_q, max_k, scale, tau, causal)
        return o

    @staticmethod
    def backward(ctx, do):
        q, k, v, o, lse, cu_q, cu_k = ctx.saved_tensors
        max_q, max_k, scale, tau, causal = ctx.args
        do = _incoming(do)
        dq, dk, dv, _ = mala.bwd_varlen_prefix(q, k, v, o, do, lse, cu_q, cu_k, max_q, max_k, scale, tau, causal=causal)
        return dq, dk, dv, None, None, None, None, None, None, None


class _MalaAttentionBias(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, table, max_distance: int, bidirectional: bool, tau: float, scale: float, causal: bool):
        bias = mala.RelativeBias(table, max_distance, bidirectional)
        o, lse, _ = mala.fwd_bias(q, k, v, bias, scale, tau, causal=causal)
        ctx.save_for_backward(q, k, v, table, o, lse)
        ctx.args = (max_distance, bidirectional, tau, scale, causal)
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, do):
        q, k, v, table, o, lse = ctx.saved_tensors
        max_distance, bidirectional, tau, scale, causal = ctx.args
        do = _incoming(do)
        dq, dk, dv, dtable, _ = mala.bwd_bias(q, k, v, o, do, lse, mala.RelativeBias(table, max_distance, bidirectional), scale,
                                              tau, causal=causal)
        return dq, dk, dv, dtable, None, None, None, None, None


class _MalaAttentionBiasPacked(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, table, cu_q, cu_k, max_q: int, max_k: int, max_distance: int, bidirectional: bool, tau: float,
                scale: float, causal: bool):
        bias = mala.RelativeBias(table, max_distance, bidirectional)
        o, lse, _ = mala.fwd_varlen_bias(q, k, v, cu_q, cu_k, max_q, max_k, bias, scale, tau, causal=causal)
        ctx.save_for_backward(q, k, v, table, o, lse, cu_q, cu_k)
        ctx.args = (max_q, max_k, max_distance, bidirectional, tau, scale, causal)
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, do):
        q, k, v, table, o, lse, cu_q, cu_k = ctx.saved_tensors
        max_q, max_k, max_distance, bidirectional, tau, scale, causal = ctx.args
        do = _incoming(do)
        dq, dk, dv, dtable, _ = mala.bwd_varlen_bias(q, k, v, o, do, lse, cu_q, cu_k, max_q, max_k,
                                                     mala.RelativeBias(table, max_distance, bidirectional), scale, tau, causal=causal)
        return dq, dk, dv, dtable, None, None, None, None, None, None, None, None, None


def mala_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, tau: float, scale: Optional[float] = None,
                   causal: bool = True) -> torch.Tensor:
    """MALA attention of bf16 q [B,Nq,Hq,d] against k, v [B,Nk,Hkv,d] on a B200 (tau = 0: FullAttn), differentiable
    with respect to q, k and v.  Causal: the queries are the last Nq of the Nk positions (Nq = Nk: self attention).
    ``scale`` defaults to 1 / sqrt(d)."""
    if scale is None:
        scale = 1.0 / math.sqrt(q.shape[-1])
    return _MalaAttention.apply(q, k, v, float(tau), float(scale), bool(causal))


def mala_attention_packed(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_seqlens_q: torch.Tensor,
                          cu_seqlens_k: torch.Tensor, max_seqlen_q: int, max_seqlen_k: int, tau: float,
                          scale: Optional[float] = None, causal: bool = True) -> torch.Tensor:
    """MALA attention on packed sequences: q [1,total_q,Hq,d], k, v [1,total_k,Hkv,d], sequence b in the rows
    cu_seqlens_q[b] .. cu_seqlens_q[b+1]-1 of q and cu_seqlens_k[b] .. of k, v (int32 on the device; pass the same
    tensor twice for self attention).  Differentiable with respect to q, k and v."""
    if scale is None:
        scale = 1.0 / math.sqrt(q.shape[-1])
    return _MalaAttentionPacked.apply(q, k, v, cu_seqlens_q, cu_seqlens_k, int(max_seqlen_q), int(max_seqlen_k),
                                      float(tau), float(scale), bool(causal))


def mala_attention_bias(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, tau: float,
                        max_distance: int = 128, bidirectional: bool = False, scale: Optional[float] = None,
                        causal: bool = True) -> torch.Tensor:
    """``mala_attention`` with a learned relative position bias: ``table`` bf16 [num_buckets, Hq], added to the scaled scores by
    the bucket of key position - query position (see ``mala_rel_bias`` in ``include/mala.h``; the queries are the last Nq of
    the Nk positions).  Differentiable with respect to q, k, v and the table (once).  To
    capture the backward pass in a CUDA graph, let no other autograd graph of the same leaves be alive: torch adds up their
    gradients on the stream on which that one was built, outside the capture."""
    if scale is None:
        scale = 1.0 / math.sqrt(q.shape[-1])
    return _MalaAttentionBias.apply(q, k, v, table, int(max_distance), bool(bidirectional), float(tau), float(scale), bool(causal))


def mala_attention_bias_packed(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, cu_seqlens_q: torch.Tensor,
                               cu_seqlens_k: torch.Tensor, max_seqlen_q: int, max_seqlen_k: int, tau: float,
                               max_distance: int = 128, bidirectional: bool = False, scale: Optional[float] = None,
                               causal: bool = True) -> torch.Tensor:
    """``mala_attention_packed`` with a learned relative position bias (``mala_attention_bias``): one table for all sequences."""
    if scale is None:
        scale = 1.0 / math.sqrt(q.shape[-1])
    return _MalaAttentionBiasPacked.apply(q, k, v, table, cu_seqlens_q, cu_seqlens_k, int(max_seqlen_q), int(max_seqlen_k),
                                          int(max_distance), bool(bidirectional), float(tau), float(scale), bool(causal))
