"""The weights' gradients of the heads' norms take every head of every token exactly once: sums of whole numbers, which one head that is
missing or counted twice moves by at least 1."""
import math

import numpy as np
import pytest
import torch

from paper_2603_01501_b200 import binding as gb

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("dims", [(30011, 3, 1, 64, BF), (20003, 1, 5, 32, F), (9001, 1, 1, 256, BF), (9001, 7, 1, 20, BF), (70001, 1, 1, 8, F),
                                  (12291, 12, 2, 128, BF), (4093, 7, 1, 96, F), (16384, 28, 4, 128, BF), (701, 5, 2, 300, BF), (1201, 3, 2, 33, F),
                                  (1, 1, 1, 64, BF), (593, 2, 1, 128, BF)], ids=str)
def test_every_head_counts_once(dims, turned):
    """Heads of ones, whose mean square rounds to 1 at these sizes, so that r = 1, and quarter turns, which exchange a pair's elements: the
    gradient is a sum of whole numbers, and all of its partial sums are below 2^24: there is nothing to round."""
    tokens, qh, kh, dim, dtype = dims
    gen = torch.Generator(device="cuda").manual_seed(dim)
    rot = dim // 4 * 2 if turned else 0
    how = {"freqs": np.full(rot // 2, math.pi / 2) if turned else None, "eps": 2.0 ** -40}
    place = torch.randint(0, 1000, (tokens,), generator=gen, device="cuda", dtype=torch.int32) if turned else None
    x, dy = [], []
    for heads in (qh, kh):
        x.append(torch.ones(tokens, heads, dim, dtype=dtype, device="cuda"))
        size = torch.randint(1, 8, x[-1].shape, generator=gen, device="cuda").double()
        dy.append(size * (2.0 * torch.randint(0, 2, x[-1].shape, generator=gen, device="cuda") - 1.0))
    ones = torch.ones(dim, device="cuda")
    unit, _ = gb.gac_norm_rotary(torch.ones(3, 2, dim, device="cuda"), None, None, None, None, eps=2.0 ** -40)
    assert bool((unit == 1).all())
    got = gb.gac_norm_rotary_backward(*(d.to(dtype) for d in dy), *x, ones, ones, positions=place, **how)
    for d, dw in zip(dy, got[2:]):
        if turned:
            c, s = (torch.tensor(t, device="cuda", dtype=torch.float64)[place.long() % 4][:, None, None] for t in ([1, 0, -1, 0], [0, 1, 0, -1]))
            a, b = d[..., :rot // 2], d[..., rot // 2:rot]
            d = torch.cat((a * c + b * s, b * c - a * s, d[..., rot:]), -1)
        assert torch.equal(dw.double(), d.sum((0, 1)))
