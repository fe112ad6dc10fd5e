"""Global gradient norm and clipping over a list of tensors: against exact sums, over element types, sizes,
alignments and magnitudes."""
import ctypes
import math

import pytest
import torch

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import synth

from packed_ref import U, V

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def make(sizes, dtypes, seed=0, scale=1.0, offset=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        base = torch.empty(n + offset, dtype=dtypes[i % len(dtypes)], device="cuda")
        base.normal_(generator=gen).mul_(scale * 10.0 ** (-(i % 4)))
        out.append(base[offset:])
    return out


def exact_norm(ts):
    return math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in ts))


def check(ts, outs, norm, max_norm, eps=1e-6):
    f = min(1.0, max_norm / (norm + eps))
    for t, o in zip(ts, outs):
        want = t.double() * f
        rel = 0.0 if f == 1.0 else 2.02 * U + (1.01 * V if t.dtype == BF else 0.0)
        tiny = 2.0 ** -134 if t.dtype == BF else 2.0 ** -150     # half the smallest subnormal
        assert bool(((o.double() - want).abs() <= rel * want.abs() + tiny).all())


@pytest.mark.parametrize("types", [(F,), (BF,), (BF, F, F)], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", [[1], [7], [1, 2, 3, 4, 5, 63, 64, 65], [2047, 2048, 2049, 16383, 16384, 16385],
                                   [1 << 20], [5_000_003, 11, 900_001]], ids=lambda s: str(sum(s)))
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_norm_and_clipped_list(types, sizes, offset):
    ts = make(sizes, types, seed=len(sizes), offset=offset)
    norm = exact_norm(ts)
    for ratio in (0.3, 5.0):
        outs = make(sizes, types, seed=99, offset=offset)
        ctx = gb.gac_clip_init(ts, outs)
        told = torch.zeros(1, device="cuda")
        res = gb.gac_clip_grad_norm(ctx, ratio * norm, norm_out=told, fetch=True)
        assert abs(res.norm - norm) <= 1e-10 * norm and abs(res.sumsq - norm * norm) <= 1e-10 * norm * norm
        assert abs(float(told) - norm) <= 1.01 * U * norm + 1e-10 * norm
        assert res.nonfinite == 0
        assert abs(res.scale - min(1.0, ratio * norm / (norm + 1e-6))) <= 1.01 * U + 1e-9
        check(ts, outs, norm, ratio * norm)
        gb.gac_clip_free(ctx)


def test_input_and_output_of_different_alignment():
    ts = make([4099, 70001, 12], (BF, F), seed=3, offset=0)
    for off in (1, 2, 5):
        outs = make([4099, 70001, 12], (BF, F), seed=4, offset=off)
        ctx = gb.gac_clip_init(ts, outs)
        norm = exact_norm(ts)
        gb.gac_clip_grad_norm(ctx, 0.5 * norm)
        check(ts, outs, norm, 0.5 * norm)


def test_neighbours_of_a_view_are_not_written():
    flat = torch.full((100_000,), 7.0, device="cuda")
    views = [flat[3:10], flat[11:5000], flat[5001:99_990]]
    for v in views:
        v.fill_(1.0)
    ctx = gb.gac_clip_init(views)
    gb.gac_clip_grad_norm(ctx, 0.5)
    for i in (0, 1, 2, 10, 5000, 99_990, 99_999):
        assert float(flat[i]) == 7.0
    assert float(flat[4]) < 1.0


def test_in_place_and_untouched_below_the_limit():
    ts = make([300, 70_000, 5], (BF, F), seed=5)
    keep = [t.clone() for t in ts]
    norm = exact_norm(ts)
    ctx = gb.gac_clip_init(ts)
    res = gb.gac_clip_grad_norm(ctx, 2 * norm, fetch=True)
    assert res.scale == 1.0 and all(torch.equal(a, b) for a, b in zip(ts, keep))
    gb.gac_clip_grad_norm(ctx, 0.25 * norm)
    check(keep, ts, norm, 0.25 * norm)
    # infinity: the norm alone
    res = gb.gac_clip_grad_norm(ctx, math.inf, fetch=True)
    assert res.scale == 1.0 and abs(res.norm - exact_norm(ts)) <= 1e-10 * res.norm


@pytest.mark.parametrize("scale", [1e-30, 1e-22, 1e18, 1e30])
def test_magnitudes_whose_squares_leave_binary32(scale):
    ts = make([10_000, 77], (F,), seed=6, scale=scale)
    outs = [torch.empty_like(t) for t in ts]
    norm = exact_norm(ts)
    res = gb.gac_clip_grad_norm(gb.gac_clip_init(ts, outs), 0.5 * norm, eps=0.0, fetch=True)
    assert abs(res.norm - norm) <= 1e-10 * norm
    check(ts, outs, norm, 0.5 * norm, eps=0.0)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_nonfinite_gradient_writes_nothing(bad):
    ts = make([5000, 20], (F, BF), seed=7)
    ts[1][3] = bad
    outs = [torch.full_like(t, 5.0) for t in ts]
    ctx = gb.gac_clip_init(ts, outs)
    res = gb.gac_clip_grad_norm(ctx, 1.0, fetch=True)
    assert res.nonfinite == 1 and all(bool((o == 5.0).all()) for o in outs)
    ts[1][3] = 1.0                      # the context goes on working
    assert gb.gac_clip_grad_norm(ctx, 1.0, fetch=True).nonfinite == 0


def test_zero_gradient_and_empty_tensors():
    ts = [torch.zeros(100, device="cuda"), torch.zeros(0, device="cuda"), torch.zeros(33, dtype=BF, device="cuda")]
    outs = [torch.ones_like(t) for t in ts]
    res = gb.gac_clip_grad_norm(gb.gac_clip_init(ts, outs), 1.0, fetch=True)
    assert (res.norm, res.scale) == (0.0, 1.0) and all(not bool(o.any()) for o in outs)
    res = gb.gac_clip_grad_norm(gb.gac_clip_init([torch.zeros(0, device="cuda")]), 1.0, eps=0.0, fetch=True)
    assert (res.norm, res.scale, res.nonfinite) == (0.0, 1.0, 0)


def test_the_same_bits_every_time_and_in_a_graph():
    shapes = synth.decoder_tensor_list(synth.DIMS["small"])
    ts = make([n for _, n in shapes], (BF, F), seed=8)
    outs = [torch.empty_like(t) for t in ts]
    ctx = gb.gac_clip_init(ts, outs)
    norm = exact_norm(ts)
    first = gb.gac_clip_grad_norm(ctx, 0.5 * norm, fetch=True)
    keep = [o.clone() for o in outs]
    for _ in range(5):
        again = gb.gac_clip_grad_norm(ctx, 0.5 * norm, fetch=True)
        assert (again.sumsq, again.scale) == (first.sumsq, first.scale)
    told = torch.zeros(1, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        graph.capture_begin()
        gb.gac_clip_grad_norm(ctx, 0.5 * norm, norm_out=told)
        graph.capture_end()
    for o in outs:
        o.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, keep))
    assert float(told) == torch.tensor(first.norm).float().item()


def test_shards_give_what_the_whole_list_gives():
    ts = make([40_000, 3, 999, 123_457], (F, BF), seed=9)
    outs = [torch.empty_like(t) for t in ts]
    norm = exact_norm(ts)
    parts = [gb.gac_clip_init(ts[:2], outs[:2]), gb.gac_clip_init(ts[2:], outs[2:])]
    sums = torch.zeros(2, dtype=torch.float64, device="cuda")
    for i, c in enumerate(parts):
        gb.gac_clip_sumsq(c, sums[i:i + 1])
    total = sums.sum().reshape(1)
    assert abs(float(total) - norm * norm) <= 1e-10 * norm * norm
    for c in parts:
        res = gb.gac_clip_apply(c, total, 0.2 * norm, fetch=True)
        assert abs(res.norm - norm) <= 1e-10 * norm
    check(ts, outs, norm, 0.2 * norm)


def test_refusals():
    a, b = torch.ones(10, device="cuda"), torch.ones(10, device="cuda")
    flat = torch.ones(100, device="cuda")
    for call, status in (
            (lambda: gb.gac_clip_init([]), gb.GAC_ERR_INVALID_ARG),
            (lambda: gb.gac_clip_init([a.half()]), gb.GAC_ERR_DTYPE),
            (lambda: gb.gac_clip_init([flat[:10], flat[5:15]]), gb.GAC_ERR_INVALID_ARG),       # in place, overlapping
            (lambda: gb.gac_clip_init([flat[:10]], [flat[5:15]]), gb.GAC_ERR_INVALID_ARG),     # output over input
            (lambda: gb.gac_clip_init([flat[:10], flat[50:60]], [a, flat[:10]]), gb.GAC_ERR_INVALID_ARG)):
        with pytest.raises(gb.GacError) as e:
            call()
        assert e.value.status == status and len(str(e.value)) > 20
    with pytest.raises(ValueError):
        gb.gac_clip_init([a], [b[:5]])
    with pytest.raises(ValueError):
        gb.gac_clip_init([torch.ones(10)])
    ctx = gb.gac_clip_init([a])
    for args in ((0.0, 1e-6), (-1.0, 1e-6), (math.nan, 1e-6), (1.0, -1.0), (1.0, math.inf), (1.0, math.nan)):
        with pytest.raises(gb.GacError):
            gb.gac_clip_grad_norm(ctx, *args)
    L = gb.load_library()
    assert L.gac_clip_grad_norm(None, None, 1.0, 0.0, None, None) == gb.GAC_ERR_INVALID_ARG
    assert L.gac_clip_sumsq(ctx.handle, None, ctypes.c_void_p(4100)) == gb.GAC_ERR_INVALID_ARG
    assert L.gac_clip_free(None) == gb.GAC_OK
