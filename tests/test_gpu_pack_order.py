"""cu_seqlens whose entries are out of order: every token is of one sequence or of none, the same for attention, its
gradient and rotary positions."""
import pytest
import torch

from paper_2603_01501_b200 import binding as gb

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def in_order(cu, tokens):
    """The entries that mean the same in order, by the header's rule."""
    n, starts = len(cu) - 1, [0] * len(cu)

    def cut(lo, hi, a, b):
        if lo < hi:
            mid = (lo + hi + 1) // 2
            starts[mid] = min(max(cu[mid], 0, a), b)
            cut(lo, mid - 1, a, starts[mid])
            cut(mid, hi, starts[mid], b)

    cut(0, n, 0, tokens)
    assert starts == sorted(starts)
    return starts


def results(q, k, v, d_o, cu):
    cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
    o, lse = gb.gac_attn_forward(q, k, v, cu)
    grads = gb.gac_attn_backward(d_o, q, k, v, o, lse, cu)
    freqs = gb.gac_rotary_freqs(64, 1e4)
    turned = gb.gac_rotary(q, k, freqs, cu_seqlens=cu)
    gb.gac_attn_check()
    return [o, lse, *grads, *turned]


@pytest.mark.parametrize("cu", [[0, 200, 100, 300], [0, 100, 50, 150], [0, 100, 50], [0, 300, 1, 2, 3], [9, 250, 250, -4, 77, 2_000_000_000, 10],
                                [0, 299, 0, 298, 1, 297, 2, 150], [0, 40, 300, 20, 280, 60, 260, 80, 240, 100, 220]], ids=str)
@pytest.mark.parametrize("heads", [(4, 2), (6, 1)], ids=str)
def test_entries_out_of_order_are_moved_into_order(cu, heads):
    gen = torch.Generator(device="cuda").manual_seed(len(cu))
    tokens = 301
    q, k, v, d_o = (torch.randn(tokens, n, 64, generator=gen, device="cuda").to(BF) for n in (heads[0], heads[1], heads[1], heads[0]))
    want = results(q, k, v, d_o, in_order(cu, tokens))
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(results(q, k, v, d_o, cu), want))


def test_many_entries_out_of_order():
    """More sequences than are dealt out by height."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    tokens, n = 3000, 700
    cu = torch.arange(0, tokens, tokens // n)[:n]
    cu = [int(x) for x in cu[torch.randperm(n, generator=torch.Generator().manual_seed(6))]]
    q, k, v, d_o = (torch.randn(tokens, h, 64, generator=gen, device="cuda").to(BF) for h in (2, 1, 1, 2))
    want = results(q, k, v, d_o, in_order(cu, tokens))
    assert all(torch.equal(a, b) for a, b in zip(results(q, k, v, d_o, cu), want))
