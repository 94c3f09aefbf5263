"""torch.autograd glue for the masked attention: argument marshalling and tensor bookkeeping only.

Every arithmetic step runs in the CUDA library (loma_masked_attn_fwd / loma_masked_attn_bwd through
the C ABI); this module allocates the outputs, keeps what the backward needs, and hands both calls
the same layout parameters.  There is no fallback: without the library the calls raise.
"""

from __future__ import annotations

import torch

from . import binding as L


class _MaskedAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, n_chunks, c, t, tail_read, flags, softmax_scale):
        if not (q.is_cuda and k.is_cuda and v.is_cuda):
            raise RuntimeError("loma_masked_attention needs CUDA tensors (there is no CPU path)")
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        B, H, S, D = q.shape
        o = torch.empty_like(q)
        lse = torch.empty((B, H, S), dtype=torch.float32, device=q.device)
        L.loma_masked_attn_fwd(q, k, v, o, lse, n_chunks, c, t, tail_read, flags, softmax_scale)
        ctx.save_for_backward(q, k, v, o, lse)
        ctx.layout = (n_chunks, c, t, tail_read, flags, softmax_scale)
        return o

    @staticmethod
    def backward(ctx, d_o):
        q, k, v, o, lse = ctx.saved_tensors
        n_chunks, c, t, tail_read, flags, softmax_scale = ctx.layout
        B, H, S, D = q.shape
        d_o = d_o.contiguous()
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        nbytes = L.loma_masked_attn_bwd_workspace_bytes(B, H, D, n_chunks, c, t, tail_read, flags)
        ws = torch.empty(max(256, nbytes), dtype=torch.uint8, device=q.device)
        L.loma_masked_attn_bwd(q, k, v, o, d_o, lse, dq, dk, dv, n_chunks, c, t, tail_read, flags, ws, softmax_scale)
        return dq, dk, dv, None, None, None, None, None, None


def loma_masked_attention(q, k, v, n_chunks: int, c: int, t: int, tail_read: int = 0, flags: int = 0,
                          softmax_scale: float = 0.0) -> torch.Tensor:
    """Zone-masked attention over the laid-out sequence (Eq. 1-3, Eq. 7) as a differentiable torch op.

    q, k, v: [B, H, S, D] CUDA tensors of one dtype (fp32 or bf16), S = n_chunks * chunk length + tail_read.
    Returns O [B, H, S, D]; gradients flow to q, k and v through the library's backward kernels.
    """
    return _MaskedAttention.apply(q, k, v, n_chunks, c, t, tail_read, flags, softmax_scale)


class _Rope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, n_chunks, c, t, tail_read, flags, theta_base, position_type):
        q, k = q.contiguous().clone(), k.contiguous().clone()
        L.loma_rope_apply(q, k, n_chunks, c, t, tail_read, flags, theta_base, position_type)
        ctx.layout = (n_chunks, c, t, tail_read, flags, theta_base, position_type)
        return q, k

    @staticmethod
    def backward(ctx, dq, dk):
        n_chunks, c, t, tail_read, flags, theta_base, position_type = ctx.layout
        dq, dk = dq.contiguous().clone(), dk.contiguous().clone()
        L.loma_rope_apply(dq, dk, n_chunks, c, t, tail_read, flags, theta_base, position_type | L.LOMA_ROPE_INVERSE)
        return dq, dk, None, None, None, None, None, None, None


def loma_rope(q, k, n_chunks: int, c: int, t: int, tail_read: int = 0, flags: int = 0, theta_base: float = 0.0,
              position_type: int = 0):
    """Rotary embedding of q and k at the layout's position ids as a differentiable torch op (out of place;
    the gradient is the rotation by the opposite angle, run by the same kernel)."""
    return _Rope.apply(q, k, n_chunks, c, t, tail_read, flags, theta_base, position_type)


def _dense16(x):
    """x contiguous and at a 16-byte address.  A contiguous view of a larger tensor may start anywhere: a slice of a flat
    parameter buffer, or the gradient that a concatenation hands back."""
    x = x.contiguous()
    return x if x.data_ptr() % 16 == 0 else x.clone()


class _QkNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, wq, wk, n_chunks, c, t, tail_read, flags, eps, theta_base, position_type):
        if not (q.is_cuda and k.is_cuda):
            raise RuntimeError("loma_qk_norm_rope needs CUDA tensors (there is no CPU path)")
        q, k = _dense16(q), _dense16(k)
        wq, wk = (None if w is None else _dense16(w) for w in (wq, wk))
        q_out, k_out = torch.empty_like(q), torch.empty_like(k)
        ctx.layout = (n_chunks, c, t, tail_read, flags)
        ctx.norm = (eps, theta_base, position_type)
        with torch.cuda.device(q.device):
            L.loma_qk_norm_rope_fwd(q, k, wq, wk, q_out, k_out, *ctx.layout, *ctx.norm)
        ctx.save_for_backward(q, k, wq, wk)
        return q_out, k_out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_q_out, d_k_out):
        q, k, wq, wk = ctx.saved_tensors
        n_chunks, c, t, tail_read, flags = ctx.layout
        eps, theta_base, position_type = ctx.norm
        d_q_out, d_k_out = _dense16(d_q_out), _dense16(d_k_out)
        dq, dk = torch.empty_like(q), torch.empty_like(k)
        dwq, dwk = (torch.empty_like(w) if w is not None and need else None
                    for w, need in ((wq, ctx.needs_input_grad[2]), (wk, ctx.needs_input_grad[3])))
        nbytes = L.loma_qk_norm_rope_bwd_workspace_bytes(q.shape[0], q.shape[1], k.shape[1], q.shape[3], n_chunks, c, t, tail_read, flags)
        ws = torch.empty(max(256, nbytes), dtype=torch.uint8, device=q.device)
        with torch.cuda.device(q.device):
            L.loma_qk_norm_rope_bwd(q, k, wq, wk, d_q_out, d_k_out, dq, dk, dwq, dwk, n_chunks, c, t, tail_read, flags, ws, eps,
                                    theta_base, position_type)
        return dq, dk, dwq, dwk, None, None, None, None, None, None, None, None


def loma_qk_norm_rope(q, k, wq, wk, n_chunks: int, c: int, t: int, tail_read: int = 0, flags: int = 0, eps: float = 0.0,
                      theta_base: float = 0.0, position_type: int = 0):
    """Per-head RMS norm of q [B, Hq, S, D] and k [B, Hk, S, D] with gains wq, wk ([D] or None) and the rotary embedding at the
    layout's position ids as one differentiable torch op; returns (q_out, k_out).  Gradients flow to q, k, wq and wk, once (no
    double backward).  To capture a step into a CUDA graph, first drop every eager graph of the same leaves: torch ties a leaf's
    gradient to the stream of its first use, and a capture may not wait for a stream outside it."""
    return _QkNormRope.apply(q, k, wq, wk, n_chunks, c, t, tail_read, flags, eps, theta_base, position_type)
