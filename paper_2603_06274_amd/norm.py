"""Buffer plumbing around include/stem_norm.h: queries and keys whose heads are normalised before their rotary positions.  No
arithmetic here."""
from __future__ import annotations

from typing import Optional

import torch

from . import decode_binding as db
from . import norm_binding as nb
from .decode import Rotary


def _taken(g: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    """A gradient as the library takes it: with strides that it does not take, a copy."""
    return g if g is None or db.usable_rows(g) else g.clone(memory_format=torch.contiguous_format)


class _NormTurn(torch.autograd.Function):
    """NormRotary._run as a node of autograd's graph."""

    @staticmethod
    def forward(ctx, rotary, positions, q, k, q_weight, k_weight):
        ctx.rotary = rotary
        ctx.save_for_backward(positions, q, k, q_weight, k_weight)
        ctx.set_materialize_grads(False)
        out = rotary._run(q, k, positions, None, None, False)
        needs = ctx.needs_input_grad
        ctx.mark_non_differentiable(*(y for y, needed in zip(out, (needs[2] or needs[4], needs[3] or needs[5])) if y is not None and not needed))
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_q, grad_k):
        positions, q, k, q_weight, k_weight = ctx.saved_tensors
        grad_q, grad_k = _taken(grad_q), _taken(grad_k)
        wanted = ctx.needs_input_grad[4] and grad_q is not None, ctx.needs_input_grad[5] and grad_k is not None
        if grad_q is None and grad_k is None:
            return None, None, None, None, None, None
        norm = nb.HeadNorm(q_weight, k_weight, ctx.rotary.norm.eps, ctx.rotary.norm.weight_offset)
        dq, dk, dqw, dkw = ctx.rotary._gradients(norm, q if grad_q is not None else None, k if grad_k is not None else None, grad_q, grad_k,
                                                 positions, wanted)
        return (None, None, dq, dk, None if dqw is None else dqw.to(q_weight.dtype), None if dkw is None else dkw.to(k_weight.dtype))


class NormRotary(Rotary):
    """Rotary positions of heads that are normalised first: each head of queries and keys divided by its root mean square (with eps) and
    multiplied by weights [head_dim] (q_weight and k_weight, bf16, fp16 or fp32; None: by none) to which weight_offset is added.  Takes the
    place of a Rotary everywhere: StemPrefill, PagedCache, StemDecode; further arguments are Rotary's.  The weights are used as they are at
    each call."""

    def __init__(self, head_dim: int, q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor], eps: float = 1e-6,
                 weight_offset: float = 0.0, rotary_dim: Optional[int] = None, device="cuda", **positions):
        super().__init__(head_dim, rotary_dim, device=device, **positions)
        self.norm = nb.HeadNorm(q_weight, k_weight, eps, weight_offset)
        self.norm.need_fits(self.head_dim, self.turns.device)

    @classmethod
    def none(cls, head_dim: int, q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
             weight_offset: float = 0.0, device="cuda") -> "NormRotary":
        """Norms without positions."""
        r = cls(head_dim, q_weight, k_weight, eps, weight_offset, 2, device, layout="interleaved")    # (a pair that does not leave its chunk)
        r.turns.zero_()
        return r

    def _shape(self, q, k, q_out, k_out=None) -> db.RotaryShape:
        shape = super()._shape(q, k, q_out, k_out)
        self.norm.need_fits(self.head_dim, (q if q is not None else k).device)
        return shape

    def _turn(self, q, k, positions, q_out, k_out, backward: bool):
        leaves = q, k, self.norm.q_weight, self.norm.k_weight
        if torch.is_grad_enabled() and any(x is not None and x.requires_grad for x in leaves):
            if q_out is not None or k_out is not None:
                raise ValueError("outputs that are given carry no gradients: call under torch.no_grad, or without them")
            return _NormTurn.apply(self, positions, *leaves)
        return self._run(q, k, positions, q_out, k_out, False)

    def _run(self, q, k, positions, q_out, k_out, backward: bool):
        q_out = torch.empty_like(q) if q_out is None and q is not None else q_out
        k_out = torch.empty_like(k) if k_out is None and k is not None else k_out
        shape = self._shape(q, k, q_out, k_out)
        nb.stem_norm_rotary(shape, self.norm, q, k, positions, self.turns, self.attention_factor, q_out, k_out)
        return q_out, k_out

    def _append(self, shape, pages, q, k, v, positions, slots, q_out, k_pages, v_pages) -> None:
        nb.stem_norm_rotary_append(shape, self.norm, pages, q, k, v, positions, slots, self.turns, self.attention_factor, q_out, k_pages,
                                   v_pages)

    def backward(self, *_, **__):
        raise TypeError("the gradients of normalised heads go by their inputs: gradients()")

    def _gradients(self, norm: nb.HeadNorm, q, k, grad_q, grad_k, positions, weights_wanted):
        shape = super()._shape(q, k, grad_q, grad_k)
        like = [x if x is None else torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device) for x in (q, k)]
        first = q if q is not None else k
        sums = [torch.empty(self.head_dim, dtype=torch.float32, device=first.device) if w else None for w in weights_wanted]
        space = None
        if any(weights_wanted):
            space = torch.empty(nb.stem_norm_rotary_backward_workspace_bytes(shape), dtype=torch.uint8, device=first.device)
        nb.stem_norm_rotary_backward(shape, norm, q, k, positions, self.turns, self.attention_factor, grad_q, grad_k, *like, *sums, space)
        return (*like, *sums)

    def gradients(self, q, k, grad_q, grad_k, positions: torch.Tensor):
        """The gradients of apply's q and k from those of its outputs, in tensors of their strides, and those of the weights, in fp32 (None
        where there are none).  Either of q and k may be None, with its gradient."""
        norm = self.norm
        return self._gradients(norm, q, k, grad_q, grad_k, positions, (norm.q_weight is not None and q is not None,
                                                                        norm.k_weight is not None and k is not None))
