"""torch.autograd plumbing around the C-ABI binding: forward calls cotten_attn_fwd, backward
calls cotten_attn_bwd (which rebuilds the d x d state from K, V: nothing but the inputs is
saved).  The kernels return d loss / d log(scale) per slice; the one piece of arithmetic done
here, in torch, is its conversion to d loss / d scale (a division by the scale, [B,H] values).

The kernels' gradients have no derivatives of their own: a second derivative raises."""
from __future__ import annotations

import functools
from typing import Optional

import torch

from . import binding


class _LastDerivative(torch.autograd.Function):
    """The first `count` tensors as they are, tied to the others, which they depend on: going on from there raises.
    (torch's once_differentiable ties them to nothing, and `torch.autograd.grad` takes that for a derivative of zero.)"""
    @staticmethod
    def forward(ctx, count, *tensors):
        return tensors[:count]

    @staticmethod
    def backward(ctx, *upstream):
        raise RuntimeError("the gradients of this library's kernels are not differentiable: no second derivatives")


def _first_derivatives_only(backward):
    """For a `backward` whose arithmetic autograd does not see."""
    @functools.wraps(backward)
    def run(ctx, *upstream):
        if not torch.is_grad_enabled():
            return backward(ctx, *upstream)
        with torch.no_grad():    # (create_graph)
            grads = backward(ctx, *upstream)
        given = [t for t in grads if t is not None]
        sources = [t for t in (*upstream, *ctx.saved_tensors) if t is not None and t.requires_grad]
        if not given or not sources:
            return grads
        tied = iter(_LastDerivative.apply(len(given), *given, *sources))
        return tuple(None if t is None else next(tied) for t in grads)
    return run


def _aligned(t: torch.Tensor) -> torch.Tensor:
    """An upstream gradient as the library takes it: contiguous, from a 16-byte boundary on (a part of another gradient
    may begin anywhere)."""
    t = t.contiguous()
    return t.clone() if t.data_ptr() & 15 else t


class _CosineAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, K, V, mask, scale, eps, slice_scale, layout):
        ctx.save_for_backward(Q, K, V, mask, slice_scale)
        ctx.scale, ctx.eps, ctx.layout = scale, eps, layout
        return binding.cotten_attn_fwd(Q, K, V, mask, scale=scale, eps=eps, slice_scale=slice_scale,
                                       layout=layout)

    @staticmethod
    @_first_derivatives_only
    def backward(ctx, dO):
        Q, K, V, mask, slice_scale = ctx.saved_tensors
        dlog = None
        if slice_scale is not None and ctx.needs_input_grad[6]:
            B, H, _, _ = binding._dims(Q, ctx.layout)
            dlog = torch.empty(B, H, device=Q.device, dtype=torch.float32)
        dQ, dK, dV = binding.cotten_attn_bwd(Q, K, V, mask, _aligned(dO), scale=ctx.scale,
                                             eps=ctx.eps, slice_scale=slice_scale,
                                             dlog_scale=dlog, layout=ctx.layout)
        # d loss / d scale = (d loss / d log scale) / scale
        dscale = None if dlog is None else dlog / slice_scale
        return dQ, dK, dV, None, None, None, dscale, None


def cosine_attention(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor,
                     mask: Optional[torch.Tensor] = None, *, scale: Optional[float] = None,
                     eps: Optional[float] = None, slice_scale: Optional[torch.Tensor] = None,
                     layout: str = "bhnd") -> torch.Tensor:
    """O = scale * Qhat (Khat^T V) under the key mask, differentiable in Q, K, V and, when
    given, in the per-slice scales `slice_scale` ([B,H] float32)."""
    return _CosineAttention.apply(Q, K, V, mask, scale, eps, slice_scale, layout)


class _GatedDelta(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, K, V, g, beta, mask, scale, eps, initial_state, layout, return_state, recorded):
        ctx.dims = dims = binding._dims(Q, layout)
        B, H, _, d = dims
        state = g.new_empty((B, H, d, d)) if return_state else None
        kept = binding.cotten_delta_kept(Q, layout=layout) if recorded and any(ctx.needs_input_grad) else None
        O = binding.cotten_delta_fwd(Q, K, V, g, beta, mask, scale=scale, eps=eps, layout=layout,
                                     initial_state=initial_state, final_state=state, kept=kept)
        ctx.save_for_backward(Q, K, V, g, beta, mask, kept, initial_state)
        ctx.call = (binding._dtype_code(Q), 0.0 if scale is None else scale, -1.0 if eps is None else eps,
                    binding._LAYOUTS[layout])
        ctx.set_materialize_grads(False)
        return (O, state) if return_state else O

    @staticmethod
    @_first_derivatives_only
    def backward(ctx, dO, dstate=None):
        Q, K, V, g, beta, mask, kept, initial_state = ctx.saved_tensors
        dO = torch.zeros_like(Q) if dO is None else _aligned(dO)
        dfirst = None
        if initial_state is not None and ctx.needs_input_grad[8]:
            dfirst = torch.empty_like(initial_state)
        grads = binding._delta_backward_of(binding.CottenDeltaParams(*ctx.call), ctx.dims, Q, K, V, g, beta, mask, dO,
                                           initial_state, None if dstate is None else _aligned(dstate), dfirst, kept)
        return (*grads, None, None, None, dfirst, None, None, None)


def gated_delta_attention(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, g: torch.Tensor, beta: torch.Tensor,
                          mask: Optional[torch.Tensor] = None, *, scale: Optional[float] = None,
                          eps: Optional[float] = None, initial_state: Optional[torch.Tensor] = None,
                          return_state: bool = False, layout: str = "bhnd"):
    """The gated delta rule of `binding.cotten_delta_fwd`, differentiable in Q, K, V, g, beta and the initial state;
    with `return_state` (O, final state).  The states before every 32 tokens and a float32 row per token are kept for the
    backward (not under `torch.no_grad`, whatever the tensors ask for)."""
    return _GatedDelta.apply(Q, K, V, g, beta, mask, scale, eps, initial_state, layout, return_state, torch.is_grad_enabled())


class _ItemEmbedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, W, positions, scale, padding_idx, position_offset):
        ctx.save_for_backward(ids)
        P_shape = None if positions is None else positions.shape
        ctx.shapes = W.shape, P_shape
        ctx.call = (binding._dtype_code(W), ids.element_size(), scale, -1 if padding_idx is None else padding_idx,
                    0 if P_shape is None else P_shape[0], position_offset)
        return binding.cotten_embed_fwd(ids, W, positions, scale=scale, padding_idx=padding_idx,
                                        position_offset=position_offset)

    @staticmethod
    @_first_derivatives_only
    def backward(ctx, dE):
        ids, = ctx.saved_tensors
        W_shape, P_shape = ctx.shapes
        _, of_W, of_P = ctx.needs_input_grad[:3]
        if not (of_W or of_P):
            return None, None, None, None, None, None
        dW, dP = binding._embed_backward_of(binding.CottenEmbedParams(*ctx.call), ids, _aligned(dE), W_shape,
                                            P_shape if of_P else None, of_W)
        return None, dW, dP, None, None, None


def item_embedding(ids: torch.Tensor, W: torch.Tensor, positions: Optional[torch.Tensor] = None, *,
                   scale: float = 1.0, padding_idx: Optional[int] = None, position_offset: int = 0) -> torch.Tensor:
    """scale * W[ids] + positions[position_offset + n] (see `binding.cotten_embed_fwd`), differentiable in W and the
    positions; both gradients are dense."""
    return _ItemEmbedding.apply(ids, W, positions, scale, padding_idx, position_offset)
