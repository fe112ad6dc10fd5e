"""What the autograd layer saves, refuses and hands on, with plain torch in the place of the library's calls (no GPU)."""
import pytest
import torch

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import packed


@pytest.fixture
def plain(monkeypatch):
    """Stand-ins that, like the library, return tensors without a graph."""
    @torch.no_grad()
    def rotary(q, k, freqs, positions=None, cu_seqlens=None, layout="half", scale=1.0, inverse=False, **_):
        assert layout == "half" and cu_seqlens is None
        angle = positions.double()[:, None] * torch.as_tensor(freqs) * (-1 if inverse else 1)
        c, s = (scale * angle.cos())[:, None], (scale * angle.sin())[:, None]
        out = []
        for x in (q, k):
            if x is None:
                out.append(None)
                continue
            a, b = x.chunk(2, -1)
            out.append(torch.cat((a * c - b * s, a * s + b * c), -1))
        return tuple(out)

    @torch.no_grad()
    def forward(q, k, v, cu, scale=None, stream=None):
        return q * 2.0, q[..., 0].t().contiguous().float()

    @torch.no_grad()
    def backward(d_o, q, k, v, o, lse, cu, scale=None, stream=None):
        return d_o * 2.0, torch.zeros_like(k), torch.zeros_like(v)

    monkeypatch.setattr(gb, "gac_rotary", rotary)
    monkeypatch.setattr(gb, "gac_attn_forward", forward)
    monkeypatch.setattr(gb, "gac_attn_backward", backward)


def heads(n, seed):
    return torch.randn(5, n, 4, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).requires_grad_()


FREQS = [1.0, 0.1]


def test_second_derivative_through_rotary(plain):
    q, k, pos = heads(2, 1), heads(1, 2), torch.arange(5, dtype=torch.int32)
    y, _ = packed.rotary(q, k, FREQS, positions=pos, scale=2.0)
    first, = torch.autograd.grad((y ** 2).sum() + (q ** 4).sum(), q, create_graph=True)
    second, = torch.autograd.grad(first.sum(), q)
    # |y|^2 = 4 |q|^2
    assert torch.allclose(first, 8 * q + 4 * q ** 3) and torch.allclose(second, 8 + 12 * q ** 2)


def test_second_derivative_through_attention_is_refused(plain):
    q, k, v = heads(2, 3), heads(1, 4), heads(1, 5)
    o = packed.attention(q, k, v, torch.tensor([0, 5], dtype=torch.int32))
    first, = torch.autograd.grad((o ** 2).sum() + (q ** 4).sum(), q, create_graph=True)
    assert torch.allclose(first, 8 * q + 4 * q ** 3)
    with pytest.raises(RuntimeError):
        first.sum().backward()


def test_what_the_way_back_of_rotary_reads_cannot_change_unnoticed(plain):
    import numpy as np
    q, k = heads(2, 6), heads(1, 7)
    pos, freqs = torch.arange(5, dtype=torch.int32), np.array(FREQS)
    want, = torch.autograd.grad(packed.rotary(q, k, freqs, positions=pos)[0].sum(), q)
    y, _ = packed.rotary(q, k, freqs, positions=pos)
    freqs[:] = 3.0                                  # numpy keeps no versions: the values of the call count
    got, = torch.autograd.grad(y.sum(), q, retain_graph=True)
    assert torch.equal(got, want)
    pos.add_(7)                                     # a buffer refilled for the next micro-batch
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(y.sum(), q)


def test_a_gradient_that_is_contiguous_but_misaligned_is_copied(plain, monkeypatch):
    seen = []
    backward = gb.gac_attn_backward
    monkeypatch.setattr(gb, "gac_attn_backward", lambda d_o, *a, **kw: (seen.append(d_o), backward(d_o, *a, **kw))[1])
    q, k, v = (torch.randn(5, n, 8).to(torch.bfloat16).requires_grad_() for n in (2, 1, 1))
    cu = torch.tensor([0, 5], dtype=torch.int32)
    x = torch.zeros(3, dtype=torch.bfloat16)
    g = torch.randn(83).to(torch.bfloat16)
    torch.cat((x, packed.attention(q, k, v, cu).flatten())).backward(g)         # 6 bytes off a boundary
    assert torch.equal(seen[0].flatten(), g[3:])
    one = torch.randn(5, 8).to(torch.bfloat16).as_strided((5, 1, 8), (8, 3, 1))   # an odd stride of one head
    q1 = torch.randn(5, 1, 8).to(torch.bfloat16).requires_grad_()
    packed.attention(q1, k, v, cu).backward(one)
    for d in seen:
        assert d.data_ptr() % 16 == 0 and all(s % 8 == 0 for s in d.stride()[:2]) and d.stride(2) == 1


def test_rotary_of_queries_alone(plain):
    q, pos = heads(2, 8), torch.arange(5, dtype=torch.int32)
    y, none = packed.rotary(q, None, FREQS, positions=pos, scale=2.0)
    assert none is None
    got, = torch.autograd.grad((y * y).sum(), q)
    assert torch.allclose(got, 8 * q)
