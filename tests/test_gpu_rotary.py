"""Rotary positions against the float64 form: layouts, parts of a head, types, strides, far positions."""
import math

import numpy as np
import pytest
import torch

from paper_2603_01501_b200 import binding as gb

from packed_ref import V, rotary, sequences, within

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def randn(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def check(x, y, pos, freqs, layout, scale, inverse):
    want, bound = rotary(x, pos, torch.from_numpy(freqs).cuda(), layout, scale, inverse)
    if x.dtype == BF:
        bound = bound * (1 + V) + V * want.abs()
    r = 2 * freqs.size
    within(y[..., :r], want[..., :r], bound[..., :r], "turned")
    assert torch.equal(y[..., r:], x[..., r:])          # what is not turned is copied as it is


@pytest.mark.parametrize("dtype", [BF, F], ids=["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dims", [(128, 128), (128, 64), (64, 64), (96, 24), (80, 16), (32, 32), (30, 10), (6, 2), (256, 256),
                                  (200, 128)], ids=str)
def test_layouts_and_parts_of_a_head(dtype, layout, dims):
    head_dim, rot_dim = dims
    freqs = gb.gac_rotary_freqs(rot_dim, 1e4)
    for tokens, qh, kh in ((1, 3, 1), (5, 4, 4), (131, 7, 1)):
        q, k = randn((tokens, qh, head_dim), dtype, tokens), randn((tokens, kh, head_dim), dtype, tokens + 1)
        pos = torch.randint(0, 5000, (tokens,), device="cuda", dtype=torch.int32)
        for inverse in (False, True):
            yq, yk = gb.gac_rotary(q, k, freqs, positions=pos, layout=layout, scale=1.25, inverse=inverse)
            check(q, yq, pos.double(), freqs, layout, 1.25, inverse)
            check(k, yk, pos.double(), freqs, layout, 1.25, inverse)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [BF, F], ids=["bf16", "f32"])
def test_places_follow_from_packed_sequences(layout, dtype):
    cu = torch.tensor([0, 1, 1, 18, 18, 301, 555], dtype=torch.int32, device="cuda")
    tokens = 560                                             # five tokens of padding
    qkv = randn((tokens, 6 + 2 + 2, 64), dtype, 3)
    q, k, _ = qkv.split([6, 2, 2], dim=1)                    # strided views of one projection
    pos = torch.zeros(tokens, dtype=torch.float64, device="cuda")
    for a, b in sequences(cu, tokens):
        pos[a:b] = torch.arange(b - a, device="cuda")
    freqs = gb.gac_rotary_freqs(64, 1e6, "parts", 8.0, trained=256.0)
    keep = qkv.clone()
    yq, yk = gb.gac_rotary(q, k, freqs, cu_seqlens=cu, layout=layout)
    check(q, yq, pos, freqs, layout, 1.0, False)
    check(k, yk, pos, freqs, layout, 1.0, False)
    assert torch.equal(qkv, keep)
    # in place on the views, values untouched
    got = gb.gac_rotary(q, k, freqs, cu_seqlens=cu, layout=layout, in_place=True)
    assert got[0].data_ptr() == q.data_ptr()
    assert torch.equal(q, yq) and torch.equal(k, yk) and torch.equal(qkv[:, 8:], keep[:, 8:])


def test_strides_and_alignment():
    freqs = gb.gac_rotary_freqs(16, 1e4)
    pos = torch.arange(37, device="cuda", dtype=torch.int32)
    for dtype in (BF, F):
        base = randn((37 * 5 * 41 + 8,), dtype, 4)
        odd = base[1:1 + 37 * 5 * 41].view(37, 5, 41)[..., :20]           # odd strides, base off 16 bytes
        swapped = randn((5, 37, 20), dtype, 5).transpose(0, 1)            # heads outermost
        shared = randn((37, 1, 20), dtype, 6).expand(37, 5, 20)           # one head seen five times
        for x in (odd, swapped, shared):
            y, none = gb.gac_rotary(x, None, freqs, positions=pos)
            assert none is None
            check(x, y, pos.double(), freqs, "half", 1.0, False)


def test_far_positions_are_as_exact_as_near_ones():
    freqs = gb.gac_rotary_freqs(128, 1e4)
    pos = torch.tensor([0, 1, 131_071, 1_000_003, 2 ** 31 - 1, -1, -70_001], dtype=torch.int32, device="cuda")
    q = randn((7, 2, 128), F, 7)
    y, _ = gb.gac_rotary(q, None, freqs, positions=pos)
    # a product of a 31-bit position with a binary64 frequency: 2^31 2^-53 turns on top
    want, bound = rotary(q, pos.double(), torch.from_numpy(freqs).cuda(), "half", 1.0, False)
    size = q.double().abs()
    within(y, want, bound + 2 * math.pi * 2.0 ** -21 * (size[..., :64] + size[..., 64:]).repeat(1, 1, 2))


def test_the_way_back_undoes_the_turn_and_is_its_transpose():
    freqs = gb.gac_rotary_freqs(64, 1e4)
    x, g = randn((50, 3, 96), F, 8), randn((50, 3, 96), F, 9)
    pos = torch.arange(50, device="cuda", dtype=torch.int32) * 100
    for layout in ("half", "interleaved"):
        y, _ = gb.gac_rotary(x, None, freqs, positions=pos, layout=layout, scale=0.5)
        back, _ = gb.gac_rotary(y, None, freqs, positions=pos, layout=layout, scale=2.0, inverse=True)
        assert float((back - x).abs().max()) <= 40 * 2.0 ** -24 * float(x.abs().max()) * 2
        gx, _ = gb.gac_rotary(g, None, freqs, positions=pos, layout=layout, scale=0.5, inverse=True)
        # <g, R x> = <R^T g, x>, and the difference quotient of the linear map along x
        left, right = float((g.double() * y.double()).sum()), float((gx.double() * x.double()).sum())
        size = float((g.double().abs() * x.double().abs()).sum())
        assert abs(left - right) <= 30 * 2.0 ** -24 * 2 * size


def test_streams_graphs_and_empty_packs():
    freqs = gb.gac_rotary_freqs(32, 1e4)
    q = randn((0, 4, 32), BF, 1)
    y, _ = gb.gac_rotary(q, None, freqs, positions=torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert y.shape == q.shape
    q, pos = randn((64, 4, 32), BF, 2), torch.arange(64, device="cuda", dtype=torch.int32)
    want, _ = gb.gac_rotary(q, None, freqs, positions=pos)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got, _ = gb.gac_rotary(q, None, freqs, positions=pos, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    buf, graph = q.clone(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        gb.gac_rotary(buf, None, freqs, positions=pos, in_place=True)
    buf.copy_(q)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(buf, want)


def test_refusals():
    q, k = randn((4, 2, 64), BF, 1), randn((4, 1, 64), BF, 2)
    pos = torch.arange(4, device="cuda", dtype=torch.int32)
    f = gb.gac_rotary_freqs(64, 1e4)
    with pytest.raises(gb.GacError) as e:
        gb.gac_rotary(q.half(), None, f, positions=pos)
    assert e.value.status == gb.GAC_ERR_DTYPE
    for bad in (np.zeros(33), np.zeros(0), np.full(32, np.nan)):
        with pytest.raises(gb.GacError) as e:
            gb.gac_rotary(q, k, bad, positions=pos)
        assert e.value.status == gb.GAC_ERR_INVALID_ARG
    with pytest.raises(gb.GacError):
        gb.gac_rotary(q, k, f, positions=pos, scale=math.inf)
    for kw in ({}, {"positions": pos, "cu_seqlens": pos}, {"positions": pos.long()}, {"positions": pos[:3]}):
        with pytest.raises(ValueError):
            gb.gac_rotary(q, k, f, **kw)
    with pytest.raises(ValueError):
        gb.gac_rotary(q.transpose(1, 2), None, f, positions=pos)
    with pytest.raises(ValueError):
        gb.gac_rotary(q, k.float(), f, positions=pos)
    with pytest.raises(gb.GacError):        # heads of the output would lie on one another
        gb.gac_rotary(q[:, :1].expand(4, 2, 64), None, f, positions=pos, in_place=True)
