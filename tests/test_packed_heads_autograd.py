"""What the autograd layer saves, refuses and hands on for the heads' norms, positions on axes and the divergence from a
teacher, with plain torch in the place of the library's calls (no GPU)."""
import numpy as np
import pytest
import torch

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import packed

import distill_ref
import heads_ref as ref

FREQS = [1.0, 0.1]


@pytest.fixture
def plain(monkeypatch):
    """Stand-ins that, like the library, return tensors without a graph."""
    seen = []

    def wheel(positions, freqs, axes, scale):
        pos = positions.double() if axes is None else positions.double()
        return ref.wheel(pos, torch.as_tensor(np.asarray(freqs)), axes, scale)

    @torch.no_grad()
    def rotary(q, k, freqs, positions=None, cu_seqlens=None, layout="half", scale=1.0, inverse=False, axes=None, **_):
        seen.append(("rotary", axes, inverse))
        cs = wheel(positions, freqs, axes, scale)
        return tuple(None if x is None else ref.turn(x, cs, layout, inverse) for x in (q, k))

    @torch.no_grad()
    def forward(q, k, wq, wk, freqs, positions=None, cu_seqlens=None, axes=None, layout="half", scale=1.0, eps=1e-6, offset=0.0, **_):
        cs = wheel(positions, freqs, axes, scale)
        return tuple(None if x is None else ref.norm(x, w, cs, layout, scale, eps, offset)[0] for x, w in ((q, wq), (k, wk)))

    @torch.no_grad()
    def backward(dq, dk, q, k, wq, wk, freqs, positions=None, cu_seqlens=None, axes=None, layout="half", scale=1.0, eps=1e-6, offset=0.0,
                 weight_grads=True, **_):
        seen.append(("backward", weight_grads, dq.is_contiguous()))
        cs, out = wheel(positions, freqs, axes, scale), []
        for d, x, w in ((dq, q, wq), (dk, k, wk)):
            (dx, _), (dw, _) = ((None, None), (None, None)) if x is None else ref.norm_back(d, x, w, cs, layout, scale, eps, offset)
            out.append((dx, dw if weight_grads and w is not None else None))
        return out[0][0], out[1][0], out[0][1], out[1][1]

    @torch.no_grad()
    def distill(logits, ids, teacher, kind="top", temperature=1.0, weights=None, grad=False, in_place=False, loss=True, **_):
        seen.append(("distill", grad, loss))
        assert weights is None or weights.is_contiguous()
        got = distill_ref.distill(logits, ids, teacher, kind, temperature, weights)
        return (None, got["grad"][0]) if grad else got["loss"][0]

    monkeypatch.setattr(gb, "gac_rotary", rotary)
    monkeypatch.setattr(gb, "gac_norm_rotary", forward)
    monkeypatch.setattr(gb, "gac_norm_rotary_backward", backward)
    monkeypatch.setattr(gb, "gac_distill", distill)
    return seen


def randn(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).requires_grad_()


def test_gradients_of_heads_and_weights(plain):
    q, k, wq, wk = randn((5, 2, 6), 1), randn((5, 1, 6), 2), randn((6,), 3), randn((6,), 4)
    pos = torch.arange(5, dtype=torch.int32)
    call = lambda *x: packed.norm_rotary(*x, FREQS, positions=pos, scale=1.5, eps=1e-2, offset=1.0)  # noqa: E731
    assert torch.autograd.gradcheck(call, (q, k, wq, wk))
    y, _ = call(q, k, wq, wk)
    y.sum().backward()                              # an expanded gradient, and none for the keys
    assert plain[-1] == ("backward", True, True) and bool((k.grad == 0).all()) and bool((wk.grad == 0).all())
    plain.clear()
    y, none = packed.norm_rotary(q, None, wq.detach(), None, FREQS, positions=pos)
    assert none is None
    y.sum().backward()
    assert plain[-1][:2] == ("backward", False)     # nobody wants the weights' gradients


def test_second_derivative_through_norms_is_refused(plain):
    q, w, pos = randn((5, 2, 6), 1), randn((6,), 2), torch.arange(5, dtype=torch.int32)
    y, _ = packed.norm_rotary(q, None, w, None, FREQS, positions=pos)
    first, = torch.autograd.grad((y ** 2).sum() + (q ** 4).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        first.sum().backward()


@pytest.mark.parametrize("op", ["rotary", "norm_rotary"])
def test_what_the_way_back_reads_cannot_change_unnoticed(plain, op):
    q, w = randn((5, 2, 6), 6), randn((6,), 7)
    pos, freqs, axes = torch.arange(15, dtype=torch.int32).view(3, 5), np.array(FREQS), np.array([2, 0], dtype=np.uint8)

    def run():
        how = {"positions": pos, "axes": axes}
        return (packed.rotary(q, None, freqs, **how) if op == "rotary" else packed.norm_rotary(q, None, w, None, freqs, **how))[0]

    want, = torch.autograd.grad(run().sum(), q)
    y = run()
    freqs[:] = 3.0                                  # numpy keeps no versions: the values of the call count
    axes[:] = 1
    got, = torch.autograd.grad(y.sum(), q, retain_graph=True)
    assert torch.equal(got, want)
    pos.add_(7)                                     # a buffer refilled for the next micro-batch
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(y.sum(), q)


def test_derivatives_of_any_order_through_positions_on_axes(plain):
    q, pos = randn((5, 2, 6), 8), torch.arange(10, dtype=torch.int32).view(2, 5)
    y, _ = packed.rotary(q, None, FREQS, positions=pos, axes=[1, 0], scale=2.0)
    first, = torch.autograd.grad((y[..., :4] ** 2).sum(), q, create_graph=True)
    second, = torch.autograd.grad(first.sum(), q)
    assert torch.allclose(first[..., :4], 8 * q[..., :4]) and torch.allclose(second[..., :4], torch.full_like(q[..., :4], 8.0))
    assert [s[0] for s in plain].count("rotary") >= 3


@pytest.mark.parametrize("kind", ["top", "forward", "reverse"])
def test_the_divergence_s_gradient(plain, kind):
    x = randn((4, 30), 9)
    ids = torch.tensor([[1, 5, 9], [0, 29, 3], [-1, -1, -1], [7, 8, 2]], dtype=torch.int32)
    teacher = torch.log_softmax(randn((4, 3), 10).detach(), 1) - 0.3
    assert torch.autograd.gradcheck(lambda z: packed.distillation(z, ids, teacher, kind, 1.5), (x,))
    packed.distillation(x, ids, teacher, kind).mean().backward()      # an expanded gradient
    assert plain[-1] == ("distill", True, False) and bool((x.grad[2] == 0).all())
    y = x * 1.0
    loss = packed.distillation(y, ids, teacher, kind)
    first, = torch.autograd.grad((loss ** 2).sum(), y, create_graph=True)
    with pytest.raises(RuntimeError):
        first.sum().backward()
    loss = packed.distillation(y, ids, teacher, kind).sum()
    y.detach().zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
