"""Rotary positions with several axes against the float64 form."""
import numpy as np
import pytest
import torch

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import packed

import heads_ref as ref
from packed_ref import within

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def randn(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", [BF, F], ids=["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dims", [(128, 128, [16, 24, 24]), (64, 64, [16, 16]), (96, 24, [3, 4, 5]), (30, 10, [2, 0, 3]), (6, 2, [1]),
                                  (256, 256, [32, 32, 32, 32]), (200, 128, [0, 64]), (80, 16, [8, 0, 0])], ids=str)
def test_layouts_sections_and_both_ways(dtype, layout, dims):
    head_dim, rot_dim, sections = dims
    freqs = gb.gac_rotary_freqs(rot_dim, 1e4)
    for interleaved in (False, True):
        axis = gb.gac_rotary_sections(sections, interleaved)
        for tokens, qh, kh in ((1, 3, 1), (67, 7, 2)):
            q, k = randn((tokens, qh, head_dim), dtype, tokens), randn((tokens, kh, head_dim), dtype, tokens + 1)
            pos = torch.randint(-9, 100000, (len(sections), tokens), device="cuda", dtype=torch.int32)
            cs = ref.wheel(pos.double(), torch.from_numpy(freqs).cuda(), axis, 1.25)
            for inverse in (False, True):
                yq, yk = gb.gac_rotary(q, k, freqs, positions=pos, axes=axis, layout=layout, scale=1.25, inverse=inverse)
                within(yq, *ref.axes(q, cs, layout, 1.25, inverse), "q")
                within(yk, *ref.axes(k, cs, layout, 1.25, inverse), "k")
                assert torch.equal(yq[..., rot_dim:], q[..., rot_dim:])


def test_equal_positions_on_all_axes_are_ordinary_ones():
    freqs, pos = gb.gac_rotary_freqs(64, 1e6), torch.randint(0, 40000, (100,), device="cuda", dtype=torch.int32)
    axis = gb.gac_rotary_sections([8, 12, 12])
    for dtype in (BF, F):
        q, k = randn((100, 4, 64), dtype, 1), randn((100, 2, 64), dtype, 2)
        want = gb.gac_rotary(q, k, freqs, positions=pos)
        for on in (pos.expand(3, 100), pos.repeat(3, 1), torch.nn.functional.pad(pos.repeat(3, 1), (0, 7))[:, :100]):   # strides 0, 100, 107
            got = gb.gac_rotary(q, k, freqs, positions=on, axes=axis)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        got = gb.gac_rotary(q.clone(), k.clone(), freqs, positions=pos.repeat(3, 1), axes=axis, in_place=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_an_image_with_a_spectrum_for_each_axis():
    rows, cols, dim = 13, 29, 64
    grid = torch.stack((torch.arange(rows).repeat_interleave(cols), torch.arange(cols).repeat(rows))).to(torch.int32).cuda()
    one = gb.gac_rotary_freqs(dim // 2, 1e4)
    freqs, axis = np.concatenate((one, one)), gb.gac_rotary_sections([dim // 4, dim // 4])
    q = randn((rows * cols, 3, dim), F, 1)
    y, _ = gb.gac_rotary(q, None, freqs, positions=grid, axes=axis)
    within(y, *ref.axes(q, ref.wheel(grid.double(), torch.from_numpy(freqs).cuda(), axis), "half", 1.0))
    # scores of two turned heads depend on the distance along each axis alone
    a, b = randn((1, 1, dim), F, 2), randn((1, 1, dim), F, 3)
    turned = [gb.gac_rotary(x.expand(rows * cols, 1, dim), None, freqs, positions=grid, axes=axis)[0][:, 0].double() for x in (a, b)]
    at = lambda r, c: r * cols + c  # noqa: E731
    s1 = float(turned[0][at(7, 20)] @ turned[1][at(4, 9)])
    s2 = float(turned[0][at(10, 11)] @ turned[1][at(7, 0)])
    assert abs(s1 - s2) <= 4 * 12 * ref.U * 2 * float(a.norm() * b.norm())


def test_derivatives_through_autograd():
    freqs, axis = gb.gac_rotary_freqs(32, 1e4), gb.gac_rotary_sections([4, 6, 6], True)
    pos = torch.randint(0, 500, (3, 50), device="cuda", dtype=torch.int32)
    q, k = (randn((50, n, 64), F, n).requires_grad_() for n in (3, 1))
    yq, yk = packed.rotary(q, k, freqs, positions=pos, axes=axis, scale=1.5)
    gq, gk = randn((50, 3, 64), F, 7), randn((50, 1, 64), F, 8)
    torch.autograd.backward((yq, yk), (gq, gk))
    cs = ref.wheel(pos.double(), torch.from_numpy(freqs).cuda(), axis, 1.5)
    within(q.grad, *ref.axes(gq, cs, "half", 1.5, True))
    within(k.grad, *ref.axes(gk, cs, "half", 1.5, True))
    y, _ = packed.rotary(q, None, freqs, positions=pos, axes=axis)
    pos.add_(1)                                    # refilled before the way back
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(y.sum(), q)


def test_streams_and_graphs():
    freqs, axis = gb.gac_rotary_freqs(32, 1e4), gb.gac_rotary_sections([8, 8])
    q, pos = randn((64, 4, 32), BF, 2), torch.randint(0, 99, (2, 64), device="cuda", dtype=torch.int32)
    want, _ = gb.gac_rotary(q, None, freqs, positions=pos, axes=axis)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got, _ = gb.gac_rotary(q, None, freqs, positions=pos, axes=axis, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    buf, graph = q.clone(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        gb.gac_rotary(buf, None, freqs, positions=pos, axes=axis, in_place=True)
    buf.copy_(q)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(buf, want)


def test_refusals():
    q, f = randn((4, 2, 64), BF, 1), gb.gac_rotary_freqs(64, 1e4)
    pos = torch.zeros(3, 4, dtype=torch.int32, device="cuda")
    axis = gb.gac_rotary_sections([8, 12, 12])
    for bad, kind in (({"positions": pos[:2]}, gb.GacError), ({"positions": pos.repeat(2, 1)}, gb.GacError), ({"positions": pos[:, :3]}, ValueError),
                      ({"positions": pos[0]}, ValueError), ({"positions": pos.long()}, ValueError), ({"positions": pos.t().contiguous().t()}, ValueError),
                      ({"positions": None, "cu_seqlens": pos[0]}, ValueError), ({"axes": axis[:31]}, ValueError), ({"axes": [0.5] * 32}, ValueError),
                      ({"axes": [-1] * 32}, ValueError), ({"axes": [300] * 32}, ValueError), ({"axes": [3] * 32}, gb.GacError)):
        with pytest.raises(kind):
            gb.gac_rotary(q, None, f, **{"positions": pos, "axes": axis, **bad})
    for bad in ([], [1, 2, 3, 4, 5], [4, -1]):
        with pytest.raises(ValueError):
            gb.gac_rotary_sections(bad)
