"""Plain float64 forms of the operators on packed rollouts, and the bounds their kernels are held to.

Bounds follow from the roundings the kernels make and nothing else (u = 2^-24, half a unit of a binary32
number relative to it; v = 2^-8, the same for bfloat16: 8 significant bits, spacing 2^-7 of the leading bit):

rotary      The angle's fraction of a turn is at most 1/2 and rounded once: the angle is off by at most
            2 pi (u / 2); sincospi adds at most 2 units (4 u), the product with the scale u, the two products
            and the sum of an output 2 u more.  Together under 12 u scale (|x| + |y|); a bfloat16 output
            adds v |result|.
clipping    The factor is rounded once (u), the product once (u, or u + v for bfloat16).
attention   E = 2^-19 scale sum_d |q_d k_d| bounds a score's error: a sum of at most 128 exact products in
            binary32, in any order and truncating, is within 128 2 u of the sum of their magnitudes, and
            the power of two taken of it is within 2^-22 of its own size.
            o      sum_j p_j |v_j| (1.25 v + 2 E + 2^-18) + v |o|: the probabilities are rounded to bfloat16
            lse    E + 2^-20 (1 + |lse|)
            d_v    sum_i p_ij |do_i| (1.25 v + 2 E + 2^-18) + v |d_v|
            ds     |ds| (1.25 v + 2 E + 2^-18) + p (Ed + Ep), with Ed = sum_d |do_d| (bound of o)_d
                   + 2^-16 sum |do o| (the row term is made from the rounded o) and Ep = 2^-16 sum_d |do_d v_d|
            d_q    scale sum_j (bound of ds)_ij |k_j| + v |d_q|, d_k alike
            1.25 instead of 1 leaves room for products of two of these.
"""
import math

import torch

U, V = 2.0 ** -24, 2.0 ** -8


def sequences(cu, tokens):
    """(start, end) of every sequence, as the library reads cu_seqlens."""
    cu = [min(max(int(c), 0), tokens) for c in cu]
    cu[0] = 0
    return [(cu[i], cu[i + 1]) for i in range(len(cu) - 1)]


def attention(q, k, v, cu, scale, d_o=None):
    """Results and bounds: dict name -> (value, bound), in float64 on the inputs' device."""
    q, k, v = q.double(), k.double(), v.double()
    tokens, heads, _ = q.shape
    group = heads // k.shape[1]
    z = lambda x: torch.zeros(x.shape, dtype=torch.float64, device=x.device)  # noqa: E731
    o, o_b = z(q), z(q)
    lse = torch.full((heads, tokens), -math.inf, dtype=torch.float64, device=q.device)
    lse_b = torch.zeros_like(lse)
    dq, dq_b, dk, dk_b, dv, dv_b = z(q), z(q), z(k), z(k), z(v), z(v)
    if d_o is not None:
        d_o = d_o.double()
    for a, b in sequences(cu, tokens):
        if b <= a:
            continue
        seen = torch.ones(b - a, b - a, dtype=torch.bool, device=q.device).tril()
        for h in range(heads):
            g = h // group
            Q, K, W = q[a:b, h], k[a:b, g], v[a:b, g]
            S = torch.where(seen, Q @ K.t() * scale, -math.inf)
            E = torch.where(seen, Q.abs() @ K.abs().t(), 0.0) * abs(scale) * 2.0 ** -19
            L = torch.logsumexp(S, 1)
            P = torch.exp(S - L[:, None])
            e = 2 * E.amax(1)
            o[a:b, h] = P @ W
            o_b[a:b, h] = (1.25 * V + e + 2.0 ** -18)[:, None] * (P @ W.abs()) + V * o[a:b, h].abs()
            lse[h, a:b] = L
            lse_b[h, a:b] = E.amax(1) + 2.0 ** -20 * (1 + L.abs())
            if d_o is None:
                continue
            G = d_o[a:b, h]
            r = (1.25 * V + e + 2.0 ** -18)[:, None]
            dv[a:b, g] += P.t() @ G
            dv_b[a:b, g] += (P * r).t() @ G.abs()
            D = (G * o[a:b, h]).sum(1, keepdim=True)
            Ed = (G.abs() * o_b[a:b, h]).sum(1, keepdim=True) + 2.0 ** -16 * (G * o[a:b, h]).abs().sum(1, keepdim=True)
            dS = P * (G @ W.t() - D)
            dS_b = dS.abs() * r + P * (Ed + 2.0 ** -16 * (G.abs() @ W.abs().t()))
            dq[a:b, h] = dS @ K * scale
            dq_b[a:b, h] = dS_b @ K.abs() * abs(scale) + V * dq[a:b, h].abs()
            dk[a:b, g] += dS.t() @ Q * scale
            dk_b[a:b, g] += dS_b.t() @ Q.abs() * abs(scale)
    res = {"o": (o, o_b), "lse": (lse, lse_b)}
    if d_o is not None:
        res.update(dq=(dq, dq_b), dk=(dk, dk_b + V * dk.abs()), dv=(dv, dv_b + V * dv.abs()))
    return res


def rotary(x, pos, freqs, layout, scale, inverse):
    """(value, bound of the float32 kernel) in float64; pos: float64 per token; freqs: float64 tensor."""
    x = x.double()
    r = 2 * freqs.numel()
    turns = pos[:, None] * (freqs / (2 * math.pi))
    angle = 2 * math.pi * (turns - turns.round()) * (-1 if inverse else 1)
    c, s = (scale * angle.cos())[:, None], (scale * angle.sin())[:, None]
    a = slice(0, r // 2) if layout == "half" else slice(0, r, 2)
    b = slice(r // 2, r) if layout == "half" else slice(1, r, 2)
    y, bound = x.clone(), torch.zeros_like(x)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    bound[..., a] = bound[..., b] = 12 * U * abs(scale) * (x[..., a].abs() + x[..., b].abs())
    return y, bound


def within(got, value, bound, what=""):
    got = got.double()
    same = torch.isneginf(got) & torch.isneginf(value)
    off = torch.where(same, 0.0, (got - value).abs())
    bad = ~(off <= bound + 1e-37)
    assert not bool(bad.any()), (what, int(bad.sum()), float((off / (bound + 1e-37)).nan_to_num(math.inf).max()))
