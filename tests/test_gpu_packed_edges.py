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
