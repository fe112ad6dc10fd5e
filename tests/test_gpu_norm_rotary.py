"""Norms of query and key heads with their rotation, and the way back, against the float64 forms."""
import math

import numpy as np
import pytest
import torch

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import packed

import heads_ref as ref
from packed_ref import sequences, within

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def randn(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def check(q, k, wq, wk, freqs, pos, axis=None, layout="half", scale=1.0, eps=1e-6, offset=0.0, back=True, **call):
    """Both directions against the reference; pos: float64 positions the call's positions or cu_seqlens stand for."""
    cs = None if freqs is None else ref.wheel(pos, torch.from_numpy(freqs).cuda(), axis, scale)
    how = dict(layout=layout, scale=scale, eps=eps, offset=offset, axes=axis, **call)
    out = gb.gac_norm_rotary(q, k, wq, wk, freqs, **how)
    for name, x, w, y in (("q", q, wq, out[0]), ("k", k, wk, out[1])):
        if x is not None:
            within(y, *ref.norm(x, w, cs, layout, scale, eps, offset), name)
    if not back:
        return out
    dq = randn(q.shape, q.dtype, 91)
    dk = None if k is None else randn(k.shape, k.dtype, 92)
    got = gb.gac_norm_rotary_backward(dq, dk, q, k, wq, wk, freqs, **how)
    for name, x, w, d, dx, dw in (("q", q, wq, dq, got[0], got[2]), ("k", k, wk, dk, got[1], got[3])):
        if x is None:
            assert dx is None
            continue
        want_x, want_w = ref.norm_back(d, x, w, cs, layout, scale, eps, offset)
        within(dx, *want_x, "d" + name)
        if w is None:
            assert dw is None
        else:
            assert dw.dtype == w.dtype
            within(dw, *want_w, "dw" + name)
    again = gb.gac_norm_rotary_backward(dq, dk, q, k, wq, wk, freqs, **how)
    for a, b in zip(got, again):
        assert (a is None and b is None) or torch.equal(a, b)
    return out


@pytest.mark.parametrize("dtype", [BF, F], ids=["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dims", [(128, 128), (128, 64), (64, 64), (96, 24), (80, 16), (32, 32), (8, 8), (12, 8), (30, 10), (6, 2), (256, 256),
                                  (256, 64), (1, 0), (128, 0), (252, 8), (512, 128), (1024, 256), (333, 2)], ids=str)
def test_layouts_and_parts_of_a_head(dtype, layout, dims):
    head_dim, rot_dim = dims
    freqs = gb.gac_rotary_freqs(rot_dim, 1e4) if rot_dim else None
    for tokens, qh, kh, w_type, offset in ((1, 3, 1, F, 0.0), (5, 4, 4, BF, 1.0), (131, 7, 1, F, 0.25)):
        q, k = randn((tokens, qh, head_dim), dtype, tokens), randn((tokens, kh, head_dim), dtype, tokens + 1)
        wq, wk = randn((head_dim,), w_type, 3), randn((head_dim,), w_type, 4)
        pos = torch.randint(0, 5000, (tokens,), device="cuda", dtype=torch.int32) if rot_dim else None
        check(q, k, wq, wk, freqs, None if pos is None else pos.double(), layout=layout, scale=1.25, offset=offset, positions=pos)


@pytest.mark.parametrize("dtype", [BF, F], ids=["bf16", "f32"])
def test_packed_sequences_and_views_of_one_projection(dtype):
    cu = torch.tensor([0, 1, 1, 18, 18, 301, 555], dtype=torch.int32, device="cuda")
    tokens = 560                                             # five tokens of padding: normed, not turned
    qkv = randn((tokens, 6 + 2 + 2, 64), dtype, 3)
    q, k, _ = qkv.split([6, 2, 2], dim=1)
    pos = torch.zeros(tokens, dtype=torch.float64, device="cuda")
    for a, b in sequences(cu, tokens):
        pos[a:b] = torch.arange(b - a, device="cuda")
    freqs = gb.gac_rotary_freqs(64, 1e6, "parts", 8.0, trained=256.0)
    w = randn((2, 64), F, 5)
    keep = qkv.clone()
    yq, yk = check(q, k, w[0], w[1], freqs, pos, cu_seqlens=cu)
    assert torch.equal(qkv, keep)
    got = gb.gac_norm_rotary(q, k, w[0], w[1], freqs, cu_seqlens=cu, in_place=True)
    assert got[0].data_ptr() == q.data_ptr()
    assert torch.equal(q, yq) and torch.equal(k, yk) and torch.equal(qkv[:, 8:], keep[:, 8:])


@pytest.mark.parametrize("dtype", [BF, F], ids=["bf16", "f32"])
def test_positions_on_axes(dtype):
    tokens = 203
    q, k, w = randn((tokens, 5, 64), dtype, 6), randn((tokens, 2, 64), dtype, 7), randn((2, 64), BF, 8)
    pos = torch.randint(-50, 70000, (3, tokens), device="cuda", dtype=torch.int32)
    for interleaved in (False, True):
        axis = gb.gac_rotary_sections([8, 12, 12], interleaved)
        check(q, k, w[0], w[1], gb.gac_rotary_freqs(64, 1e6), pos.double(), axis, positions=pos)


@pytest.mark.parametrize("dtype", [BF, F], ids=["bf16", "f32"])
def test_strides_alignment_and_missing_parts(dtype):
    freqs = gb.gac_rotary_freqs(16, 1e4)
    pos = torch.arange(37, device="cuda", dtype=torch.int32)
    base = randn((37 * 5 * 41 + 8,), dtype, 4)
    odd = base[1:1 + 37 * 5 * 41].view(37, 5, 41)[..., :20]           # odd strides, base off 16 bytes
    swapped = randn((5, 37, 20), dtype, 5).transpose(0, 1)            # heads outermost
    shared = randn((37, 1, 20), dtype, 6).expand(37, 5, 20)           # one head seen five times
    late = randn((21,), dtype, 7)[1:]                                 # a weight off every boundary
    for x in (odd, swapped, shared):
        check(x, None, late, None, freqs, pos.double(), positions=pos)
        check(x, swapped, None, late, freqs, pos.double(), positions=pos)
    check(swapped, odd, None, None, freqs, pos.double(), positions=pos)
    # the gradient of the results comes in with other strides than the heads
    dy = randn((5, 37, 20), dtype, 8).transpose(0, 1)
    a = gb.gac_norm_rotary_backward(dy, None, odd, None, late, None, freqs, positions=pos)
    b = gb.gac_norm_rotary_backward(dy.contiguous(), None, odd.contiguous(), None, late.clone(), None, freqs, positions=pos)
    want_x, want_w = ref.norm_back(dy, odd, late, ref.wheel(pos.double(), torch.from_numpy(freqs).cuda()), "half", 1.0, 1e-6, 0.0)
    for got in (a, b):
        within(got[0], *want_x)
        within(got[2], *want_w)


def test_more_tokens_than_shares_and_many_heads():
    pos = torch.arange(2999, device="cuda", dtype=torch.int32)
    freqs = gb.gac_rotary_freqs(32, 1e4)
    for dtype, dim in ((BF, 32), (F, 33)):
        q, k, w = randn((2999, 19, dim), dtype, 1), randn((2999, 2, dim), dtype, 2), randn((2, dim), F, 3)
        check(q, k, w[0], w[1], freqs, pos.double(), positions=pos)


def test_offsets_past_32_bits():
    freqs = gb.gac_rotary_freqs(64, 1e4)
    pos = torch.arange(3, device="cuda", dtype=torch.int32)
    far = torch.zeros(2 * (2 ** 31 + 8) + 128, dtype=BF, device="cuda")
    q = far.as_strided((3, 2, 64), (2 ** 31 + 8, 64, 1))
    q.copy_(randn((3, 2, 64), BF, 1))
    w = randn((64,), F, 2)
    check(q, None, w, None, freqs, pos.double(), positions=pos)
    want, _ = gb.gac_norm_rotary(q, None, w, None, freqs, positions=pos)
    gb.gac_norm_rotary(q, None, w, None, freqs, positions=pos, in_place=True)
    assert torch.equal(q, want)


@pytest.mark.parametrize("dim", [128, 66])
def test_far_positions_are_as_exact_as_near_ones(dim):
    freqs = gb.gac_rotary_freqs(dim // 4 * 2, 1e4)
    freqs[1], freqs[2] = -0.37, 1e6                            # turns back, and many whole turns
    pos = torch.tensor([0, 1, 131_071, 1_000_003, 2 ** 31 - 1, -1, -70_001, -2 ** 31], dtype=torch.int32, device="cuda")
    q, w = randn((8, 2, dim), F, 7), randn((dim,), F, 8)
    y, _ = gb.gac_norm_rotary(q, None, w, None, freqs, positions=pos)
    # the reference's own angle: a product of a 31-bit position with a frequency of so many turns, in binary64, and the frequency's
    # own rounding to turns
    turns = torch.from_numpy(freqs).cuda().abs() / (2 * math.pi)
    off = 2 * math.pi * 3 * 2.0 ** -53 * pos.double().abs()[:, None] * turns
    want, bound = ref.norm(q, w, ref.wheel(pos.double(), torch.from_numpy(freqs).cuda()), "half", 1.0, 1e-6, 0.0)
    n = (q.double() * torch.rsqrt(q.double().square().mean(-1, keepdim=True) + 1e-6) * w.double()).abs()
    r = freqs.size
    # an angle off by e moves x cos a - y sin a by at most e |x sin a + y cos a| <= e (|x| + |y|), and so the other
    both = off[:, None] * (n[..., :r] + n[..., r:2 * r])
    bound[..., :2 * r] += torch.cat((both, both), -1)
    within(y, want, bound)


@pytest.mark.parametrize("dim", [64, 30])
def test_values_at_the_edge(dim):
    pos = torch.zeros(6, dtype=torch.int32, device="cuda")
    freqs, w = gb.gac_rotary_freqs(dim // 2 // 2 * 2, 1e4), torch.ones(dim, device="cuda")
    q = randn((6, 2, dim), F, 1)
    q[1] = 0.0                      # r = 1 / sqrt(eps)
    q[2] *= 1e-18
    q[3] *= 1e15
    q[4, 0, 3] = math.nan
    q[5, 1, 0] = math.inf
    dy = randn(q.shape, F, 2)
    y, _ = gb.gac_norm_rotary(q, None, w, None, freqs, positions=pos)
    dx, _, dw, _ = gb.gac_norm_rotary_backward(dy, None, q, None, w, None, freqs, positions=pos)
    fine = [0, 1, 2, 3]
    cs = ref.wheel(pos[fine].double(), torch.from_numpy(freqs).cuda())
    want, bound = ref.norm(q[fine], w, cs, "half", 1.0, 1e-6, 0.0)
    # squares below the smallest binary32 number are lost beside eps, within 2^-24 of it
    within(y[fine], want, bound + 2.0 ** -24 * want.abs())
    within(dx[fine], *ref.norm_back(dy[fine], q[fine], w, cs, "half", 1.0, 1e-6, 0.0)[0])
    # a NaN or an infinity stays in its own head
    assert bool(y[4, 0].isnan().all()) and bool(dx[4, 0].isnan().all()) and bool(dx[5, 1].isnan().any())
    for t, h in ((4, 1), (5, 0)):
        a, b = ref.norm(q[t:t + 1, h:h + 1], w, (cs[0][:1], cs[1][:1]), "half", 1.0, 1e-6, 0.0)
        within(y[t:t + 1, h:h + 1], a, b)
        assert bool(dx[t, h].isfinite().all())
    assert bool(dw.isnan().any())


def test_the_gradient_against_differences():
    """Along random directions, by differences of the float64 form at the kernel's inputs: an error of the formula would show."""
    freqs = gb.gac_rotary_freqs(32, 1e4)
    pos = torch.arange(40, device="cuda", dtype=torch.int32) * 3
    cs = ref.wheel(pos.double(), torch.from_numpy(freqs).cuda(), None, 1.5)
    for layout in ("half", "interleaved"):
        q, w, dy = randn((40, 3, 48), F, 1), randn((48,), F, 2), randn((40, 3, 48), F, 3)
        dx, _, dw, _ = gb.gac_norm_rotary_backward(dy, None, q, None, w, None, freqs, positions=pos, layout=layout, scale=1.5, offset=1.0)

        def f(x, w):
            n = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * (1.0 + w)
            return float((ref.turn(n, cs, layout) * dy.double()).sum())

        ex, ew, h = randn(q.shape, F, 4).double(), randn(w.shape, F, 5).double(), 1e-4
        x, wd = q.double(), w.double()
        slope = (f(x + h * ex, wd + h * ew) - f(x - h * ex, wd - h * ew)) / (2 * h)
        told = float((dx.double() * ex).sum() + (dw.double() * ew).sum())
        size = float((dx.double().abs() * ex.abs()).sum() + (dw.double().abs() * ew.abs()).sum())
        # third derivatives of a normed head are below 100 / |x|^3: h^2 / 6 of that; the kernel's own bounds are smaller
        assert abs(slope - told) <= 1e-5 * size


def test_streams_graphs_and_empty_packs():
    freqs, w = gb.gac_rotary_freqs(32, 1e4), randn((32,), F, 9)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    q = randn((0, 4, 32), BF, 1)
    y, _ = gb.gac_norm_rotary(q, None, w, None, freqs, positions=none)
    assert y.shape == q.shape
    dq, _, dw, _ = gb.gac_norm_rotary_backward(q, None, q, None, w, None, freqs, positions=none)
    assert dq.shape == q.shape and bool((dw == 0).all())      # a sum over nothing
    q, dy, pos = randn((64, 4, 32), BF, 2), randn((64, 4, 32), BF, 3), torch.arange(64, device="cuda", dtype=torch.int32)
    want = gb.gac_norm_rotary(q, None, w, None, freqs, positions=pos)[0]
    want_b = gb.gac_norm_rotary_backward(dy, None, q, None, w, None, freqs, positions=pos)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = gb.gac_norm_rotary(q, None, w, None, freqs, positions=pos, stream=side)[0]
    got_b = gb.gac_norm_rotary_backward(dy, None, q, None, w, None, freqs, positions=pos, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(got_b[0], want_b[0]) and torch.equal(got_b[2], want_b[2])
    buf, graph = q.clone(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        back = gb.gac_norm_rotary_backward(dy, None, buf, None, w, None, freqs, positions=pos)
        gb.gac_norm_rotary(buf, None, w, None, freqs, positions=pos, in_place=True)
    for _ in range(2):
        buf.copy_(q)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(buf, want) and torch.equal(back[0], want_b[0]) and torch.equal(back[2], want_b[2])


def test_through_autograd():
    """Gradients reach heads and weights, through views of one projection and broadcast heads, and second ones are refused."""
    freqs = gb.gac_rotary_freqs(64, 1e4)
    cu = torch.tensor([0, 20, 50], dtype=torch.int32, device="cuda")
    x = randn((50, 5, 64), F, 1).requires_grad_()
    one = randn((50, 1, 64), F, 2).requires_grad_()
    wq, wk = (randn((64,), F, s).requires_grad_() for s in (3, 4))
    q, k = packed.norm_rotary(x[:, :3], one.expand(50, 2, 64), wq, wk, freqs, cu_seqlens=cu, scale=1.5, offset=1.0)
    gq, gk = randn((3, 50, 64), F, 5).transpose(0, 1), randn((50, 1, 64), F, 6).expand(50, 2, 64)
    torch.autograd.backward((q, k), (gq, gk))
    pos = torch.cat((torch.arange(20), torch.arange(30))).double().cuda()
    cs = ref.wheel(pos, torch.from_numpy(freqs).cuda(), None, 1.5)
    (dx, dx_b), (dw, dw_b) = ref.norm_back(gq, x.detach()[:, :3], wq.detach(), cs, "half", 1.5, 1e-6, 1.0)
    within(x.grad[:, :3], dx, dx_b)
    assert bool((x.grad[:, 3:] == 0).all())
    within(wq.grad, dw, dw_b)
    (dx, dx_b), (dw, dw_b) = ref.norm_back(gk, one.detach().expand(50, 2, 64), wk.detach(), cs, "half", 1.5, 1e-6, 1.0)
    total = dx.sum(1, keepdim=True)
    within(one.grad, total, dx_b.sum(1, keepdim=True) + 2 * ref.U * dx.abs().sum(1, keepdim=True))
    within(wk.grad, dw, dw_b)
    # heads without norm weights, queries alone, one result unused
    y, none = packed.norm_rotary(x, None, None, None, freqs, cu_seqlens=cu)
    assert none is None
    first, = torch.autograd.grad((y ** 2).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        first.sum().backward()
    q, k = packed.norm_rotary(x[:, :3], x[:, 3:], wq, wk, freqs, cu_seqlens=cu)
    d, dwk = torch.autograd.grad(q.sum(), (x, wk), allow_unused=True)
    assert bool((d[:, 3:] == 0).all()) and (dwk is None or bool((dwk == 0).all()))


def test_a_captured_way_back():
    freqs, pos = gb.gac_rotary_freqs(32, 1e4), torch.arange(33, device="cuda", dtype=torch.int32)
    x, w = randn((33, 2, 32), F, 1).requires_grad_(), randn((32,), F, 2).requires_grad_()

    def grads():
        return torch.autograd.grad(packed.norm_rotary(x, None, w, None, freqs, positions=pos)[0].square().sum(), (x, w))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = grads()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = grads()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_refusals():
    q, k, w = randn((4, 2, 64), BF, 1), randn((4, 1, 64), BF, 2), randn((64,), F, 3)
    pos = torch.arange(4, device="cuda", dtype=torch.int32)
    f = gb.gac_rotary_freqs(64, 1e4)
    for bad, kind in (((q.half(), None, w, None, f), gb.GacError), ((q, k, w.half(), None, f), gb.GacError),
                      ((q, k, w, w.to(BF), f), gb.GacError), ((q, k, w[:32], None, f), ValueError), ((q, k, w[::2], None, f[:8]), ValueError),
                      ((q, k, w.cpu(), None, f), ValueError), ((q, k.float(), w, w, f), ValueError), ((q, k, w, w, np.zeros(33)), gb.GacError)):
        with pytest.raises(kind):
            gb.gac_norm_rotary(*bad, positions=pos)
    for kw in ({"eps": 0.0}, {"eps": math.nan}, {"eps": 1e-60}, {"offset": math.inf}, {"scale": math.nan}):
        with pytest.raises(gb.GacError):
            gb.gac_norm_rotary(q, k, w, w, f, positions=pos, **kw)
    with pytest.raises(ValueError):
        gb.gac_norm_rotary(q, k, w, w, f)
    with pytest.raises(ValueError):
        gb.gac_norm_rotary(q, k, w, w, None, positions=pos, axes=[0] * 32)
    with pytest.raises(ValueError):
        gb.gac_norm_rotary_backward(q[:, :1], k, q, k, w, w, f, positions=pos)
    with pytest.raises(gb.GacError):        # heads of the output would lie on one another
        gb.gac_norm_rotary(q[:, :1].expand(4, 2, 64), None, w, None, f, positions=pos, in_place=True)
