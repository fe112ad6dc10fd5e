"""The autograd layer and the clipper at their edges, on the device."""
import math

import pytest
import torch

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import packed

from packed_ref import U

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def test_second_derivative_through_rotary():
    freqs = gb.gac_rotary_freqs(32, 1e4)
    pos = torch.arange(50, device="cuda", dtype=torch.int32) * 17
    q = torch.randn(50, 3, 32, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").requires_grad_()
    y, _ = packed.rotary(q, q[:, :1], freqs, positions=pos, scale=2.0)
    first, = torch.autograd.grad((y ** 2).sum() + (q ** 4).sum(), q, create_graph=True)
    second, = torch.autograd.grad(first.sum(), q)
    # |y|^2 = 4 |q|^2.  Each of the two turns is off by 12 units of 2^-24 of a pair's size, scaled by 2; a pair of ones
    # is turned there and back, by 4, doubled by the square: 2 * 12 U * 2 * 8 for each, and one rounding of the sum.
    want = 8 + 12 * q.double() ** 2
    assert bool(((second.double() - want).abs() <= 24 * 2 * 16 * U + 4 * U * want).all())


def test_second_derivative_through_attention_is_refused():
    cu = torch.tensor([0, 20], dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn(20, 2, 64, device="cuda").to(BF).requires_grad_() for _ in range(3))
    first, = torch.autograd.grad(packed.attention(q, k, v, cu).float().square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        (first.float() * q.float()).sum().backward()
