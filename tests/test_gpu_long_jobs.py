"""A job of the attention kernels that takes seconds: the waits for its end have limits that it must not reach."""
import pytest
import torch

from paper_2603_01501_b200 import binding as gb

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def test_a_group_of_4096_heads_over_a_long_sequence():
    """The gradients of the first key tile take one CTA 4096 x 640 turns here.  All heads are the same one."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    tokens, heads, dim = 81920, 4096, 8
    gen = torch.Generator(device="cuda").manual_seed(1)
    q1, k, v, g1 = (torch.randn(tokens, 1, dim, generator=gen, device="cuda").to(BF) for _ in range(4))
    cu = torch.tensor([0, tokens], dtype=torch.int32, device="cuda")
    o1, lse1 = gb.gac_attn_forward(q1, k, v, cu)
    want = gb.gac_attn_backward(g1, q1, k, v, o1, lse1, cu)
    q, g = q1.expand(tokens, heads, dim), g1.expand(tokens, heads, dim)
    o, lse = gb.gac_attn_forward(q, k, v, cu)
    got = gb.gac_attn_backward(g, q, k, v, o, lse, cu)
    gb.gac_attn_check()
    some = [0, 1, 2047, 4095]
    assert all(torch.equal(o[:, h], o1[:, 0]) and torch.equal(lse[h], lse1[0]) and torch.equal(got[0][:, h], want[0][:, 0]) for h in some)
    # What a wait that ran out leaves is NaN.  The last key tile is seen by one query tile of every head: 4096 x 8 additions,
    # each within 2^-23 of a partial sum that grows to the end's size (and a quarter for what is on the way inside a head); both
    # sides are rounded to bfloat16, 2^-8 each.  Earlier tiles add up more terms than binary32 tells apart.
    for x, y in zip(got[1:], want[1:]):
        assert bool(torch.isfinite(x).all())
        x, y = x[-128:].float(), y[-128:].float() * heads
        assert bool(((x - y).abs() <= 2.0 ** -7 * y.abs() + 1.25 * 2.0 ** -8 * y.abs().max()).all())
