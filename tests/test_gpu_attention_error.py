"""How far attention and its gradients are from 64 bits on average: what the roundings that the kernels are meant to make explain,
and no more.

The bounds of single elements add every rounding up at its worst and are many times the errors' size.  These are of
the mean square.  A rounding to bfloat16 is off by at most 2^-8 of the leading bit's value and anything in between alike, so its
variance is at most r^2 x^2 with r = 2^-8 / sqrt(3); those of different numbers are independent.  Hence, at most,
    o     r^2 (sum_j p_ij^2 v_j^2 + o^2)                    probabilities and result rounded
    d_v   r^2 (sum_i p_ij^2 do_i^2 + d_v^2)                 the same
    d_k   r^2 (scale^2 sum_i ds_ij^2 q_i^2 + d_k^2)         score gradients and result rounded; the row term exact
    d_q   r^2 (scale^2 sum_j ds_ij^2 k_j^2 + d_q^2) + scale^2 (sum_j p_ij k_j)^2 Var(D_i)
          Var(D_i) = r^2 (sum_j p_ij^2 dp_ij^2 + sum_d do_id^2 o_id^2) for rows of more than one key tile, whose row term comes
          from the rounded o; 0 for the others.
Scores, exponentials and sums in binary32 are within 2^-18 of that and add less than a hundredth of r.  Over ten thousand
elements or more the mean square is within 5 % of its expectation, most of which is below the bound as mantissas spread.
"""
import math

import pytest
import torch

from paper_2603_01501_b200 import binding as gb

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
R2 = (2.0 ** -8) ** 2 / 3


def expected(q, k, v, d_o, lengths, scale):
    """name -> (value, variance), float64."""
    q, k, v, d_o = (x.double() for x in (q, k, v, d_o))
    group = q.shape[1] // k.shape[1]
    res = {n: (torch.zeros_like(x), torch.zeros_like(x)) for n, x in (("o", q), ("dq", q), ("dk", k), ("dv", k))}
    a = 0
    for n in lengths:
        at = slice(a, a + n)
        seen = torch.ones(n, n, dtype=torch.bool, device=q.device).tril()
        many = (torch.arange(n, device=q.device) >= 128)[:, None]       # rows that see more than one key tile
        for h in range(q.shape[1]):
            g = h // group
            Q, K, W, G = q[at, h], k[at, g], v[at, g], d_o[at, h]
            P = torch.softmax(torch.where(seen, Q @ K.t() * scale, -math.inf), 1)
            o, dP = P @ W, G @ W.t()
            dS = P * (dP - (P * dP).sum(1, keepdim=True))
            var_D = torch.where(many, (P ** 2 * dP ** 2).sum(1, keepdim=True) + (G ** 2 * o ** 2).sum(1, keepdim=True), 0.0)
            dq = dS @ K * scale
            for name, i, value, var in (("o", h, o, P ** 2 @ W ** 2 + o ** 2),
                                        ("dv", g, P.t() @ G, (P ** 2).t() @ G ** 2),
                                        ("dk", g, dS.t() @ Q * scale, (dS ** 2).t() @ Q ** 2 * scale ** 2),
                                        ("dq", h, dq, dS ** 2 @ K ** 2 * scale ** 2 + dq ** 2 + scale ** 2 * (P @ K) ** 2 * var_D)):
                res[name][0][at, i] += value
                res[name][1][at, i] += R2 * var
        a += n
    for name in ("dk", "dv"):
        res[name][1].add_(R2 * res[name][0] ** 2)
    return res


@pytest.mark.parametrize("offset", [0.0, 4.0], ids=["centred values", "values about 4"])
@pytest.mark.parametrize("lengths,heads,dim", [([700], (4, 2), 64), ([90, 128, 257, 513], (4, 2), 128), ([100] * 9, (3, 1), 80)], ids=str)
def test_mean_square_errors_are_those_of_the_roundings(lengths, heads, dim, offset):
    """Values about 4 make O large beside the score gradients: a row term left as it comes from the rounded O would make
    the error of d_k several times this bound."""
    gen = torch.Generator(device="cuda").manual_seed(sum(lengths) + dim)
    tokens = sum(lengths)
    q, k, v, d_o = (torch.randn(tokens, n, dim, generator=gen, device="cuda") for n in (heads[0], heads[1], heads[1], heads[0]))
    q, k, v, d_o = (x.to(BF) for x in (q, k, v + offset, d_o))
    cu = torch.tensor([0] + list(torch.tensor(lengths).cumsum(0)), dtype=torch.int32, device="cuda")
    o, lse = gb.gac_attn_forward(q, k, v, cu)
    got = dict(zip(("dq", "dk", "dv"), gb.gac_attn_backward(d_o, q, k, v, o, lse, cu)), o=o)
    for name, (value, var) in expected(q, k, v, d_o, lengths, dim ** -0.5).items():
        square = float((got[name].double() - value).square().mean())
        assert square <= 1.05 * float(var.mean()), (name, math.sqrt(square / float(var.mean())))
