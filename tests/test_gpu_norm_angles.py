"""Sines of the heads' norms with rotation keep their own digits, however small the angle: where a pair's second element is zero,
its result is the sine itself times what the first one holds."""
import math

import pytest
import torch

from paper_2603_01501_b200 import binding as gb

import heads_ref as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim", [64, 30, 256])            # vectors, single elements, the longest heads of vectors
def test_small_sines(dim, layout):
    """A result s n of a sine s and a normed element n.  The norm and the product are within 60 u (heads_ref), the sine within 2 units,
    4 u, of its own size.  The angle is rounded once, u of it, which near half a turn is more than a small sine; where it is a whole number
    of 2^-64 turns times the position, it is off by 2^-65 turns per position on top."""
    pairs = dim // 2
    freqs = 10.0 ** -torch.linspace(0.0, 8.0, pairs, dtype=torch.float64).numpy()
    pos = torch.tensor([1, 2, 3, 1000, -1, -7, 40000, 0], dtype=torch.int32, device="cuda")
    first, second = ref.parts(dim, layout)
    x = torch.zeros(pos.numel(), 2, dim, device="cuda")
    x[..., first] = 1.0 + torch.rand(*x.shape[:2], pairs, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    turns = pos.double()[:, None] * torch.from_numpy(freqs / (2 * math.pi)).cuda()
    angle = (2 * math.pi * (turns - turns.round()))[:, None]
    n = x.double() * torch.rsqrt(x.double().square().mean(-1, keepdim=True) + 1e-6)
    want = n[..., first] * angle.sin()
    grain = 2 * math.pi * 2.0 ** -65 * pos.double().abs()[:, None, None]
    bound = 64 * U * want.abs() + (U * angle.abs() + grain) * n[..., first]
    for heads in (x, x.repeat(400, 1, 1)):                # few tokens and many
        got, _ = gb.gac_norm_rotary(heads, None, None, None, freqs, positions=pos.repeat(heads.shape[0] // 8), layout=layout)
        off = (got[:8].double()[..., second] - want).abs()
        assert bool((off <= bound).all()), float((off / bound.clamp(min=1e-300)).nan_to_num(0.0).max())


@pytest.mark.parametrize("dim", [64, 30])
def test_the_farthest_positions(dim):
    """Whole turns fall away where positions times steps pass 64 bits: with frequencies of whole parts of a turn the result is known exactly."""
    parts = torch.tensor([2, 4, 8, 3, 5, 7, 1 << 20, 12345], dtype=torch.int64).repeat(8)[:dim // 2]
    pos = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 31 - 12345, -2 ** 31 + 77, 1], dtype=torch.int32, device="cuda")
    freqs = (2 * math.pi / parts.double()).numpy()
    x = torch.randn(5, 3, dim, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    got, _ = gb.gac_norm_rotary(x, None, None, None, freqs, positions=pos)
    left = pos.long()[:, None] % parts.cuda()                       # of the position, behind the last whole turn
    angle = (2 * math.pi * left.double() / parts.cuda())[:, None]
    want, bound = ref.norm(x, None, (angle.cos(), angle.sin()), "half", 1.0, 1e-6, 0.0)
    # turns of at most a half: the frequency and their quotient are off by 2^-53 of it each, the step by 2^-65, all times the position
    n = x.double() * torch.rsqrt(x.double().square().mean(-1, keepdim=True) + 1e-6)
    bound = bound + 2 * math.pi * 2.0 ** 31 * (2 * 2.0 ** -54 + 2.0 ** -65) * ref.both(n, dim, "half", 1.0)
    assert bool(((got.double() - want).abs() <= bound).all())
