"""Plain float64 forms of rotary positions with several axes and of the heads' norms, and the bounds their kernels are
held to.  u = 2^-24 and v = 2^-8 are half a unit of a binary32 and of a bfloat16 number relative to it.

norm        The squares of a head of up to 1024 elements are added in chains of at most 64 and a tree of 5: their sum, of
            positive terms, is within 70 u; with 1/D, eps and the root (2 units, 4 u) r is within 42 u.  The two
            products with r and the weight and the weight's own sum with the offset add 3 u: x r w is within 45 u.
turned      12 u scale (|x| + |y|) on top of what went in (packed_ref): under 60 u scale (|x| + |y|).
way back    With A = scale (|dy_x| + |dy_y|) (|dy| where nothing is turned), B = A |w| and n = |x| r:
            a is within 12 u A, b = a w within 15 u B, its mean with x r within (15 + 45 + 70 + 4) u mean(B n), the product
            of that with x r within 180 u n mean(B n), and r adds 42 u to all: under 240 u r (B + n mean(B n)).
            The weights' gradients: terms within 60 u A n, then a chain of as many terms as a thread has heads to take (they
            are shared out over at least 64 groups of lanes as soon as there are so many tokens) and the CTA's up to 128
            groups, and binary64: (70 + chain) u sum(A n).
A bfloat16 result adds v of itself.
"""
import math

import torch

U, V = 2.0 ** -24, 2.0 ** -8
SHARES = 148 * 4     # heads of a kind are dealt out to at most as many CTAs on the way back


def wheel(pos, freqs, axis=None, scale=1.0):
    """Cosine and sine [tokens, 1, pairs]; pos: float64 [tokens], or [axes, tokens] with the axis of every pair."""
    at = pos[:, None] if axis is None else pos[torch.as_tensor(axis).long().to(pos.device)].t()
    turns = at * (freqs / (2 * math.pi))
    angle = 2 * math.pi * (turns - turns.round())
    return (scale * angle.cos())[:, None], (scale * angle.sin())[:, None]


def parts(r, layout):
    return (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))


def turn(x, cs, layout, back=False):
    if cs is None:
        return x
    c, s = cs[0], -cs[1] if back else cs[1]
    a, b = parts(2 * c.shape[-1], layout)
    y = x.clone()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def both(x, r, layout, scale):
    """scale (|x| + |y|) at both elements of a pair, |x| where nothing is turned."""
    y = x.abs()
    if r:
        a, b = parts(r, layout)
        y[..., a] = y[..., b] = abs(scale) * (x[..., a].abs() + x[..., b].abs())
    return y


def rounded(value, bound, dtype):
    return (value, bound * (1 + V) + V * value.abs()) if dtype == torch.bfloat16 else (value, bound)


def axes(x, cs, layout, scale, back=False):
    want = turn(x.double(), cs, layout, back)
    return rounded(want, 12 * U * both(x.double(), 2 * cs[0].shape[-1], layout, scale), x.dtype)


def norm(x, w, cs, layout, scale, eps, offset):
    """(value, bound); w: weight tensor or None."""
    v = x.double()
    n = v * torch.rsqrt(v.square().mean(-1, keepdim=True) + eps)
    if w is not None:
        n = n * (offset + w.double())
    return rounded(turn(n, cs, layout), 60 * U * both(n, 0 if cs is None else 2 * cs[0].shape[-1], layout, scale), x.dtype)


def norm_back(dy, x, w, cs, layout, scale, eps, offset):
    """((dx, bound), (dw, bound))."""
    r_dim = 0 if cs is None else 2 * cs[0].shape[-1]
    v, g = x.double(), dy.double()
    r = torch.rsqrt(v.square().mean(-1, keepdim=True) + eps)
    n, k = v * r, 1.0 if w is None else offset + w.double()
    a, A = turn(g, cs, layout, True), both(g, r_dim, layout, scale)
    b, B = a * k, A * (abs(k) if w is None else k.abs())
    dx = r * (b - n * (b * n).mean(-1, keepdim=True))
    dx_b = 240 * U * r * (B + n.abs() * (B * n.abs()).mean(-1, keepdim=True))
    dw, size = (a * n).sum((0, 1)), (A * n.abs()).sum((0, 1))
    chain = -(-x.shape[0] // 64) * x.shape[1] + 128
    return rounded(dx, dx_b, x.dtype), rounded(dw, (70 + chain) * U * size, torch.float32 if w is None else w.dtype)
