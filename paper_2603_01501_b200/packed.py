"""The operators on packed rollouts for ``torch`` autograd, and gradient clipping for lists of parameters.

A pack is a batch of finished rollouts of different lengths laid one behind the other: tensors
[tokens, heads, head_dim] and ``cu_seqlens`` (int32 on the device), where sequence b takes the tokens
cu_seqlens[b] .. cu_seqlens[b+1].

    q, k = packed.rotary(q, k, freqs, cu_seqlens=cu)                      # or, where heads are normed,
    q, k = packed.norm_rotary(q, k, q_weight, k_weight, freqs, cu_seqlens=cu)
    o = packed.attention(q, k, v, cu)
    ...
    loss.backward()
    clipper.clip(1.0)

All arithmetic is in the CUDA library (``binding``); this module only says what is saved for the way back.  These are
autograd functions, not registered torch operators: they have no fake kernels, batching rules or forward mode, and a
compiled policy breaks its graph at them.

A step that is captured into a CUDA graph holds its forward and its backward pass, and as with any autograd function no loss or
output of an earlier, uncaptured pass over the same leaves may still be alive then: autograd would order the captured
gradients behind the stream of that pass, which cannot be captured.
"""
from __future__ import annotations

from typing import Iterable, List, Optional

import numpy as np
import torch
from torch.autograd.function import once_differentiable

from . import binding as gb


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, freqs, positions, cu_seqlens, layout, scale, inverse, axes):
        # positions and cu_seqlens are versioned like any saved tensor; of freqs and axes the values of this call are kept
        ctx.save_for_backward(positions, cu_seqlens)
        ctx.how = (np.array(freqs, dtype=np.float64), layout, scale, inverse, None if axes is None else np.array(axes))
        return gb.gac_rotary(q, k, freqs, positions=positions, cu_seqlens=cu_seqlens, layout=layout, scale=scale, inverse=inverse, axes=axes)

    @staticmethod
    def backward(ctx, d_q, d_k):
        positions, cu_seqlens = ctx.saved_tensors
        freqs, layout, scale, inverse, axes = ctx.how
        # the transpose of a turn is the turn by the negative angle: itself a turn, so derivatives of any order go through
        d_q, d_k = _Rotary.apply(_rows(d_q), None if d_k is None else _rows(d_k), freqs, positions, cu_seqlens, layout, scale, not inverse, axes)
        return d_q, d_k, None, None, None, None, None, None, None


class _NormRotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, freqs, positions, cu_seqlens, axes, layout, scale, eps, offset):
        ctx.save_for_backward(q, k, q_weight, k_weight, positions, cu_seqlens)
        freqs = None if freqs is None else np.array(freqs, dtype=np.float64)
        ctx.freqs, ctx.how = freqs, {"axes": None if axes is None else np.array(axes), "layout": layout, "scale": scale, "eps": eps, "offset": offset}
        return gb.gac_norm_rotary(q, k, q_weight, k_weight, freqs, positions=positions, cu_seqlens=cu_seqlens, **ctx.how)

    @staticmethod
    @once_differentiable   # the library has no second derivative: asking for one raises
    def backward(ctx, d_q, d_k):
        q, k, q_weight, k_weight, positions, cu_seqlens = ctx.saved_tensors
        grads = gb.gac_norm_rotary_backward(_rows(d_q), None if k is None else _rows(d_k), q, k, q_weight, k_weight, ctx.freqs,
                                            positions=positions, cu_seqlens=cu_seqlens,
                                            weight_grads=ctx.needs_input_grad[2] or ctx.needs_input_grad[3], **ctx.how)
        return (*grads, None, None, None, None, None, None, None, None)


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, cu_seqlens, scale):
        o, lse = gb.gac_attn_forward(q, k, v, cu_seqlens, scale=scale)
        ctx.save_for_backward(q, k, v, o, lse, cu_seqlens)
        ctx.scale = scale
        ctx.mark_non_differentiable(lse)
        return o, lse

    @staticmethod
    @once_differentiable   # the library has no second derivative: asking for one raises
    def backward(ctx, d_o, _):
        q, k, v, o, lse, cu_seqlens = ctx.saved_tensors
        d_q, d_k, d_v = gb.gac_attn_backward(_rows(d_o, 8), q, k, v, o, lse, cu_seqlens, scale=ctx.scale)
        return d_q, d_k, d_v, None, None


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, ids, teacher, kind, temperature):
        ctx.save_for_backward(logits, ids, teacher)
        ctx.how = (kind, temperature)
        return gb.gac_distill(logits, ids, teacher, kind, temperature)

    @staticmethod
    @once_differentiable   # the library has no second derivative: asking for one raises
    def backward(ctx, d_loss):
        logits, ids, teacher = ctx.saved_tensors
        _, d_logits = gb.gac_distill(logits, ids, teacher, *ctx.how, weights=d_loss.contiguous(), grad=True, loss=False)
        return d_logits, None, None, None, None


def _rows(t: torch.Tensor, multiple: int = 1) -> torch.Tensor:
    """A gradient as autograd hands it over may be expanded, transposed or off any boundary: the library wants
    contiguous rows on boundaries of `multiple` elements."""
    s0, s1, s2 = t.stride()
    if s2 == 1 and s0 >= s1 >= t.shape[2] and s0 % multiple == 0 and s1 % multiple == 0 and \
            t.data_ptr() % (multiple * t.element_size()) == 0:
        return t
    return t.clone(memory_format=torch.contiguous_format)   # a copy even where t counts as contiguous: its base may be off


def rotary(q: torch.Tensor, k: Optional[torch.Tensor], freqs, positions: Optional[torch.Tensor] = None,
           cu_seqlens: Optional[torch.Tensor] = None, layout: str = "half", scale: float = 1.0, axes=None):
    """Rotary positions (binding.gac_rotary) with their derivatives of any order; returns (q', k')."""
    return _Rotary.apply(q, k, freqs, positions, cu_seqlens, layout, scale, False, axes)


def norm_rotary(q: torch.Tensor, k: Optional[torch.Tensor], q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor], freqs,
                positions: Optional[torch.Tensor] = None, cu_seqlens: Optional[torch.Tensor] = None, axes=None, layout: str = "half",
                scale: float = 1.0, eps: float = 1e-6, offset: float = 0.0):
    """Norms of the query and key heads with their rotation (binding.gac_norm_rotary) and the gradients of heads and weights
    (first order alone: a second derivative raises); returns (q', k')."""
    return _NormRotary.apply(q, k, q_weight, k_weight, freqs, positions, cu_seqlens, axes, layout, scale, eps, offset)


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_seqlens: torch.Tensor, scale: Optional[float] = None,
              return_lse: bool = False):
    """Causal attention over the pack (binding.gac_attn_forward) with its gradient (first order alone: a
    second derivative raises).  ``lse``, if asked for, has none."""
    o, lse = _Attention.apply(q, k, v, cu_seqlens, scale)
    return (o, lse) if return_lse else o


def distillation(logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, kind: str = "top", temperature: float = 1.0):
    """Divergence of the policy from a teacher's top logits for every token (binding.gac_distill), with its gradient at the
    logits (first order alone: a second derivative raises); the teacher gets none.  Nothing is kept for the way back but the arguments;
    where the weight of every token's loss is known beforehand, binding.gac_distill gives loss and gradient in one pass."""
    return _Distill.apply(logits, ids, teacher, kind, temperature)


class GradientClipper:
    """Clips the gradients of a list of parameters by their global norm, in place, without waiting for the host.

    The table of the list is made on first use and again when the list itself changes (a parameter without a gradient is
    left out, as an optimizer leaves it out): that allocates, and waits for the device.  Gradients that have only moved, as they
    do under ``zero_grad(set_to_none=True)``, are written into the table in stream order.  No references to gradients
    are kept between calls.  For lists that do not go through the alignment rule: with a
    GradientAlignmentController, ``HParams(clip_max_norm=...)`` clips in the rule's own pass, and in exchange mode
    that is the only way (the gradient may be the stored direction itself, which is refused here)."""

    def __init__(self, params: Iterable[torch.nn.Parameter]):
        self.params: List[torch.nn.Parameter] = [p for p in params if p.requires_grad]
        if not self.params:
            raise ValueError("no trainable parameters")
        self.norm = torch.zeros((), dtype=torch.float32, device=self.params[0].device)
        self._ctx: Optional[gb.ClipContext] = None
        self._shape: List[tuple] = []
        self._bound: List[int] = []

    def clip(self, max_norm: float, eps: float = 1e-6, error_if_nonfinite: bool = False) -> torch.Tensor:
        """Returns the norm before clipping as a 0-dim device tensor, overwritten by the next call.  A norm that is NaN or
        infinite leaves every gradient as it is; the tensor says so, and with ``error_if_nonfinite``, which waits for the
        device, GacError(GAC_ERR_NONFINITE) does."""
        grads = [p.grad for p in self.params if p.grad is not None]
        if not grads:
            self.norm.zero_()
            return self.norm
        if not all(g.is_contiguous() for g in grads):
            raise RuntimeError("gradients must be contiguous")
        if any(getattr(g, "_gac_direction", False) for g in grads):
            raise RuntimeError("a gradient is the stored direction of a controller in exchange mode and must not be "
                               "modified: clip with HParams(clip_max_norm=...)")
        shape, bound = [(g.numel(), g.dtype) for g in grads], [g.data_ptr() for g in grads]
        if self._ctx is None or shape != self._shape:
            self.close()
            self._ctx = gb.gac_clip_init(grads, keep=False)
            self._shape, self._bound = shape, bound
        elif bound != self._bound:
            self._bound = []   # should the call fail, the next one tries again
            gb.gac_clip_rebind(self._ctx, grads)
            self._bound = bound
        res = gb.gac_clip_grad_norm(self._ctx, max_norm, eps, norm_out=self.norm, fetch=error_if_nonfinite)
        if error_if_nonfinite and res.nonfinite:
            raise gb.GacError(gb.GAC_ERR_NONFINITE, "the norm of the gradients is NaN or infinite; none was changed")
        torch.autograd.graph.increment_version(grads + [self.norm])   # written behind autograd's back
        return self.norm

    def close(self) -> None:
        ctx, self._ctx, self._shape, self._bound = self._ctx, None, [], []
        if ctx is not None:
            gb.gac_clip_free(ctx)
