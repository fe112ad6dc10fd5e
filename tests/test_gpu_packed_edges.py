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


def test_a_wait_that_ran_out_is_told_and_nothing_is_half_clipped():
    g = torch.randn(1 << 24, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    keep, out, told = g.clone(), torch.full_like(g, 5.0), torch.zeros(1, device="cuda")
    for ctx, seen in ((gb.gac_clip_init([g]), g), (gb.gac_clip_init([g], [out]), out)):
        before = seen.clone()
        gb.gac_clip_set_timeout(ctx, 0)                         # no CTA waits for the others
        gb.gac_clip_grad_norm(ctx, 1.0, norm_out=told)
        assert math.isnan(float(told)) and torch.equal(seen, before)
        gb.gac_clip_set_timeout(ctx, 1000)                      # not told yet: neither call goes on
        told.zero_()
        gb.gac_clip_grad_norm(ctx, 1.0, norm_out=told)
        assert math.isnan(float(told)) and torch.equal(seen, before)
        with pytest.raises(gb.GacError) as e:
            gb.gac_clip_apply(ctx, torch.ones(1, dtype=torch.float64, device="cuda"), 0.1, fetch=True)
        assert e.value.status == gb.GAC_ERR_TIMEOUT and torch.equal(seen, before)
        norm = float(keep.double().norm())
        res = gb.gac_clip_grad_norm(ctx, 0.5 * norm, norm_out=told, fetch=True)
        assert res.timed_out == 0 and abs(res.norm - norm) <= 1e-10 * norm and abs(float(told) - norm) <= 1e-6 * norm
        assert bool(((seen.double() - 0.5 * keep.double()).abs() <= 2.02 * U * keep.double().abs() + 1e-6 / norm * keep.abs()).all())
        gb.gac_clip_free(ctx)
        g.copy_(keep)


def test_sums_alone_do_not_wait_and_go_on_after_one_that_ran_out():
    g = torch.ones(1 << 22, device="cuda")
    ctx, total = gb.gac_clip_init([g]), torch.zeros(1, dtype=torch.float64, device="cuda")
    gb.gac_clip_set_timeout(ctx, 0)
    for _ in range(3):
        gb.gac_clip_grad_norm(ctx, 1.0)
        total.zero_()
        gb.gac_clip_sumsq(ctx, total)
        assert float(total) == 1 << 22
    assert bool((g == 1.0).all())


def test_the_first_call_may_be_on_a_stream_of_its_own():
    """A new context used at once on a stream that does not wait for the default one, which is busy."""
    side = torch.cuda.Stream()
    g = [torch.ones(n, device="cuda") for n in (3, 1 << 20, 70_001)]
    norm = math.sqrt(3 + (1 << 20) + 70_001)
    told = [torch.zeros(1, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    for t in told:
        torch.cuda._sleep(20_000_000)
        ctx = gb.gac_clip_init(g)
        gb.gac_clip_grad_norm(ctx, math.inf, norm_out=t, stream=side)
        side.synchronize()
        assert abs(float(t.item() if torch.cuda.current_stream().query() else t) - norm) <= 2 * U * norm
        gb.gac_clip_free(ctx)


def test_the_stored_direction_of_an_exchange_step_is_not_clipped():
    from paper_2603_01501_b200.controller import GradientAlignmentController
    params = [torch.nn.Parameter(torch.zeros(n, device="cuda")) for n in (1000, 77)]
    controller, clipper = GradientAlignmentController(params, exchange=True), packed.GradientClipper(params)
    for p in params:
        p.grad = torch.ones_like(p)
    controller.step()                       # the first step is safe: .grad is the stored direction
    with pytest.raises(RuntimeError, match="clip_max_norm"):
        clipper.clip(1.0)
    assert all(bool((s == 1.0).all()) for s in controller.snapshot)
    controller.zero_grad()
    for p in params:
        p.grad.add_(2.0)
    clipper.clip(1.0)                       # before the rule the gradients are the caller's
    assert abs(math.sqrt(sum(float(p.grad.double().square().sum()) for p in params)) - 1.0) < 1e-5
    controller.close()
    clipper.close()


def leaf_gradients(params, seed):
    for i, p in enumerate(params):
        gen = torch.Generator(device="cuda").manual_seed(100 * seed + i)
        p.grad = torch.empty_like(p).normal_(generator=gen)


def test_the_clipper_keeps_no_gradients_alive():
    params = [torch.nn.Parameter(torch.zeros(8 << 20, device="cuda")) for _ in range(4)]
    clipper, one_set = packed.GradientClipper(params), 4 * (32 << 20)
    torch.cuda.synchronize()
    start = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    for step in range(4):
        for p in params:
            p.grad = None                       # zero_grad's default
        leaf_gradients(params, step)
        clipper.clip(1.0)
    assert torch.cuda.max_memory_allocated() - start < one_set + (4 << 20)
    clipper.close()


def test_the_clipper_follows_moved_gradients_without_waiting():
    sizes = [(n, d) for n in (5, 70_001, 0, 1 << 18) for d in (torch.float32, BF)]
    params = [torch.nn.Parameter(torch.zeros(n, device="cuda", dtype=d)) for n, d in sizes]
    clipper, old = packed.GradientClipper(params), []
    leaf_gradients(params, 0)
    clipper.clip(1.0)
    for step in range(1, 4):
        old.append([p.grad for p in params])    # alive: the next ones lie elsewhere
        leaf_gradients(params, step)
        keep = [p.grad.clone() for p in params]
        torch.cuda.synchronize()
        torch.cuda._sleep(400_000_000)
        told = clipper.clip(0.5)
        assert not torch.cuda.current_stream().query()
        norm = math.sqrt(math.fsum(float(g.double().square().sum()) for g in keep))
        assert abs(float(told) - norm) <= 2 * U * norm
        for p, g in zip(params, keep):
            half = 2.0 ** -8 if g.dtype == BF else U
            want = g.double() * (0.5 / (norm + 1e-6))
            assert bool(((p.grad.double() - want).abs() <= (half + 3 * U) * want.abs()).all())
    clipper.close()


def test_many_tensors_rebound_out_of_place_and_in_a_graph():
    """More tensors than one launch takes, some empty; from in place to out of place and back."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    sizes = [(37 * i) % 41 * (500 if i % 97 == 0 else 1) for i in range(1300)]
    a, b, out = ([torch.randn(n, generator=gen, device="cuda") for n in sizes] for _ in range(3))
    keep = [x.clone() for x in b]
    norm = math.sqrt(math.fsum(float(x.double().square().sum()) for x in b))
    ctx = gb.gac_clip_init(a)
    gb.gac_clip_rebind(ctx, b, out)
    gb.gac_clip_grad_norm(ctx, 0.5 * norm)
    assert all(torch.equal(x, y) for x, y in zip(b, keep))
    want = [x * torch.tensor(0.5 * norm / (norm + 1e-6), dtype=torch.float64).float().cuda() for x in keep]
    assert all(torch.equal(x, y) for x, y in zip(out, want))
    gb.gac_clip_rebind(ctx, a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):               # addresses of b, whatever the table holds when it is replayed
        gb.gac_clip_rebind(ctx, b)
        gb.gac_clip_grad_norm(ctx, 0.5 * norm)
    gb.gac_clip_rebind(ctx, a, out)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(b, want))
    with pytest.raises(gb.GacError):
        gb.gac_clip_rebind(ctx, a[:-1])
    with pytest.raises(gb.GacError):
        gb.gac_clip_rebind(ctx, [x.to(BF) for x in a])
    with pytest.raises(gb.GacError):
        gb.gac_clip_rebind(ctx, [a[0]] * len(a))
    gb.gac_clip_free(ctx)


def test_a_gradient_that_is_contiguous_but_misaligned():
    cu = torch.tensor([0, 20], dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn(20, 2, 64, device="cuda").to(BF).requires_grad_() for _ in range(3))
    x, g = torch.zeros(3, dtype=BF, device="cuda"), torch.randn(3 + 20 * 128, device="cuda").to(BF)
    got = torch.autograd.grad(torch.cat((x, packed.attention(q, k, v, cu).flatten())), (q, k, v), g)
    want = torch.autograd.grad(packed.attention(q, k, v, cu), (q, k, v), g[3:].clone().view(20, 2, 64))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_rotary_of_queries_alone():
    freqs, pos = gb.gac_rotary_freqs(32, 1e4), torch.arange(50, device="cuda", dtype=torch.int32)
    q = torch.randn(50, 3, 32, device="cuda", requires_grad=True)
    k = torch.randn(50, 1, 32, device="cuda")
    y, none = packed.rotary(q, None, freqs, positions=pos)
    assert none is None
    g = torch.randn_like(y)
    got, = torch.autograd.grad(y, q, g)
    want, = torch.autograd.grad(packed.rotary(q, k, freqs, positions=pos)[0], q, g)
    assert torch.equal(got, want)


def test_in_place_results_raise_the_version_that_autograd_checks():
    freqs, pos = gb.gac_rotary_freqs(32, 1e4), torch.arange(50, device="cuda", dtype=torch.int32)
    w = torch.randn(50, 3, 32, device="cuda", requires_grad=True)
    q, k = torch.randn(50, 3, 32, device="cuda"), torch.randn(50, 1, 32, device="cuda")
    for hit in (q, k):
        loss = (w * hit).sum()              # hit is saved for the way back
        gb.gac_rotary(q, k, freqs, positions=pos, in_place=True)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    p = torch.nn.Parameter(torch.zeros(1000, device="cuda"))
    p.grad = torch.ones_like(p)
    loss = (torch.ones(1000, device="cuda", requires_grad=True) * p.grad).sum()
    clipper = packed.GradientClipper([p])
    clipper.clip(1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    told = clipper.norm
    loss = (torch.ones((), device="cuda", requires_grad=True) * told).sum()
    clipper.clip(1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_norm_that_is_not_finite_is_raised_when_asked_for(bad):
    p = torch.nn.Parameter(torch.zeros(1000, device="cuda"))
    p.grad = torch.ones_like(p)
    p.grad[7] = bad
    keep, clipper = p.grad.clone(), packed.GradientClipper([p])
    assert not math.isfinite(float(clipper.clip(1.0)))
    with pytest.raises(gb.GacError) as e:
        clipper.clip(1.0, error_if_nonfinite=True)
    assert e.value.status == gb.GAC_ERR_NONFINITE
    assert torch.equal(p.grad.nan_to_num(3.0), keep.nan_to_num(3.0))
    p.grad[7] = 1.0
    assert abs(float(clipper.clip(1.0, error_if_nonfinite=True)) - math.sqrt(1000.0)) < 1e-4


def test_gradients_as_views_of_one_fused_tensor():
    """d_q, d_k and d_v lie between each other's heads: their spans cross and no memory is shared."""
    import ctypes
    gen = torch.Generator(device="cuda").manual_seed(7)
    tokens, cu = 300, torch.tensor([0, 130, 290], dtype=torch.int32, device="cuda")
    q, k, v = torch.randn(tokens, 8, 64, generator=gen, device="cuda").to(BF).split([4, 2, 2], dim=1)
    d_o = torch.randn(tokens, 4, 64, generator=gen, device="cuda").to(BF)
    o, lse = gb.gac_attn_forward(q, k, v, cu)
    want = gb.gac_attn_backward(d_o, q, k, v, o, lse, cu)
    fused = torch.full((tokens, 8, 64), 7.0, dtype=BF, device="cuda")
    outs = fused.split([4, 2, 2], dim=1)
    heads = [gb.gac_attn_heads(t.data_ptr(), t.stride(0), t.stride(1)) for t in (q, k, v, o, d_o, *outs)]
    a = gb.gac_attn(*heads[:4], lse.data_ptr(), cu.data_ptr(), tokens, 2, 4, 2, 64, gb.GAC_BF16, 0.125, 0)
    L = gb.load_library()
    need = L.gac_attn_workspace(ctypes.byref(a))
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    g = gb.gac_attn_grad(*heads[4:], work.data_ptr(), need)
    gb._check(L.gac_attn_backward(ctypes.byref(a), ctypes.byref(g), 0, torch.cuda.current_stream().cuda_stream))
    assert all(torch.equal(x, y) for x, y in zip(outs, want))
