"""Causal attention over packed sequences, forward and backward, against the float64 form."""
import math

import pytest
import torch

from paper_2603_01501_b200 import binding as gb

from packed_ref import attention, within

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def make(lengths, tail, qh, kh, dim, seed, fused=False, spread=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    tokens = sum(lengths) + tail
    cu = torch.tensor([0] + list(torch.tensor(lengths).cumsum(0)), dtype=torch.int32, device="cuda")
    if fused:
        q, k, v = torch.randn(tokens, qh + 2 * kh, dim, generator=gen, device="cuda").to(BF).split([qh, kh, kh], dim=1)
    else:
        q, k, v = (torch.randn(tokens, n, dim, generator=gen, device="cuda").to(BF) for n in (qh, kh, kh))
    if spread != 1.0:
        q = (q.float() * spread).to(BF)
    d_o = torch.randn(tokens, qh, dim, generator=gen, device="cuda").to(BF)
    return q, k, v, d_o, cu


def run(q, k, v, d_o, cu, scale=None, **kw):
    o, lse = gb.gac_attn_forward(q, k, v, cu, scale=scale, **kw)
    dq, dk, dv = gb.gac_attn_backward(d_o, q, k, v, o, lse, cu, scale=scale, **kw)
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def check(q, k, v, d_o, cu, scale=None):
    got = run(q, k, v, d_o, cu, scale)
    want = attention(q, k, v, cu, q.shape[2] ** -0.5 if scale is None else scale, d_o)
    gb.gac_attn_check()
    for name, (value, bound) in want.items():
        within(got[name], value, bound, name)
    return got


@pytest.mark.parametrize("lengths", [[1], [2], [7], [63], [64], [65], [127], [128], [129], [255], [256], [257], [385], [700]], ids=str)
@pytest.mark.parametrize("dim", [64, 128])
def test_one_sequence(lengths, dim):
    check(*make(lengths, 0, 2, 1, dim, sum(lengths)))


@pytest.mark.parametrize("heads", [(1, 1), (3, 1), (6, 2), (4, 4), (7, 1), (28, 4)], ids=str)
@pytest.mark.parametrize("dim", [8, 32, 72, 80, 96, 128])
def test_heads_and_head_sizes(heads, dim):
    check(*make([5, 130, 1, 261], 3, *heads, dim, dim, fused=True))


@pytest.mark.parametrize("lengths,tail", [([1, 1, 1, 1, 1], 0), ([0, 5, 0, 0, 300, 0], 0), ([17, 64, 130, 45], 7), ([128, 256, 128], 130),
                                          ([127, 1, 129, 255], 1), ([0, 0], 40), ([3] * 150, 0), ([513, 400], 0)], ids=str)
def test_packs(lengths, tail):
    got = check(*make(lengths, tail, 4, 2, 64, 11))
    if tail:
        for name in ("o", "dq", "dk", "dv"):
            assert not bool(got[name][-tail:].any())
        assert bool(torch.isneginf(got["lse"][:, -tail:]).all())


def test_a_longer_sequence_with_many_tiles():
    check(*make([2300, 1111], 5, 4, 2, 128, 12))


def test_many_more_jobs_than_sms():
    """Hundreds of short sequences, with one and with two query tiles to a job in turn: every CTA does many jobs."""
    lengths = [(37 * i) % 300 + 1 for i in range(90)]
    check(*make(lengths, 5, 6, 2, 64, 26))
    check(*make(lengths[:40], 0, 12, 4, 128, 27))


def test_more_sequences_than_are_ranked():
    """Beyond 192 sequences the blocks are dealt out in the pack's order."""
    lengths = [(11 * i) % 5 for i in range(2100)] + [260, 0, 129]
    check(*make(lengths, 3, 2, 1, 64, 28))


def test_scores_of_great_size_and_other_scales():
    check(*make([300, 77], 0, 4, 2, 64, 13, spread=30.0))
    check(*make([300, 77], 0, 4, 2, 64, 14), scale=0.0)
    check(*make([300, 77], 0, 4, 2, 64, 15), scale=-0.3)


def test_strides_and_shared_heads():
    q, k, v, d_o, cu = make([200, 90], 0, 4, 2, 64, 16)
    want = run(q, k, v, d_o, cu)
    turned = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v, d_o)]        # heads outermost
    wide = []
    for x in (q, k, v, d_o):                                                                 # rows and heads far apart
        w = torch.full((x.shape[0], 3 * x.shape[1], 136), float("nan"), dtype=BF, device="cuda")
        w[:, ::3, :64] = x
        wide.append(w[:, ::3, :64])
    for xs in (turned, wide):
        got = run(*xs, cu)
        assert all(torch.equal(got[n], want[n]) for n in want)
    one = v[:, :1].expand(290, 2, 64)                                                        # one head of values for both
    q2, k2 = q, k
    got, ref = run(q2, k2, one, d_o, cu), run(q2, k2, one.contiguous(), d_o, cu)
    assert all(torch.equal(got[n], ref[n]) for n in ref)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_non_finite_values_stay_in_their_sequence(bad):
    lengths = [100, 37, 200, 129]
    q, k, v, d_o, cu = make(lengths, 9, 4, 2, 128, 17)
    want = run(q, k, v, d_o, cu)
    for which in range(4):
        xs = [x.clone() for x in (q, k, v, d_o)]
        xs[which][100:137] = bad              # the second sequence whole
        xs[which][466:] = bad                 # and the padding
        got = run(*xs, cu)
        for name in want:
            a, b = (got[name].t(), want[name].t()) if name == "lse" else (got[name], want[name])
            for part in (slice(0, 100), slice(137, 466)):
                assert torch.equal(a[part], b[part]), (which, name)
            if name != "lse":
                assert not bool(a[466:].any()), (which, name)


def test_the_same_bits_every_time_on_any_stream_and_in_a_graph():
    q, k, v, d_o, cu = make([900, 33, 517], 4, 6, 2, 128, 18, fused=True)
    want = run(q, k, v, d_o, cu)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        got = run(q, k, v, d_o, cu, stream=side)
        side.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(q, k, v, d_o, cu)
    for t in got.values():
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in want)


def test_gradient_against_differences():
    """Along a random direction the gradient is the difference quotient of the float64 loss."""
    q, k, v, d_o, cu = make([70, 150], 0, 4, 2, 64, 19)
    got = run(q, k, v, d_o, cu)
    bounds = attention(q, k, v, cu, 0.125, d_o)
    gen = torch.Generator(device="cuda").manual_seed(20)
    for i, name in enumerate(("dq", "dk", "dv")):
        xs = [x.double() for x in (q, k, v)]
        u = torch.randn(xs[i].shape, generator=gen, device="cuda", dtype=torch.float64)
        loss = []
        for step in (1e-4, -1e-4):
            ys = list(xs)
            ys[i] = xs[i] + step * u
            loss.append(float((attention(*ys, cu, 0.125)["o"][0] * d_o.double()).sum()))
        quotient = (loss[0] - loss[1]) / 2e-4
        slope = float((got[name].double() * u).sum())
        # third derivatives enter as 1e-8; the kernel's error is bounded element by element
        assert abs(quotient - slope) <= float((bounds[name][1] * u.abs()).sum()) + 1e-5 * float(u.abs().sum())


def test_offsets_beyond_32_bits():
    """Token strides so wide that the last rows lie more than 2^32 elements behind the first."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    lengths = [200, 313]
    q, k, v, d_o, cu = make(lengths, 0, 2, 1, 64, 21)
    want = run(q, k, v, d_o, cu)
    row = 1 << 23                                     # 513 rows of 2^23 elements: 8.6 GB
    big = torch.empty(513 * row, dtype=BF, device="cuda").view(513, row)
    views, at = [], 0
    for x in (q, k, v, d_o):
        w = big[:, at:at + x.shape[1] * 64].view(513, x.shape[1], 64)
        w.copy_(x)
        views.append(w)
        at += x.shape[1] * 64
    got = run(*views, cu)
    assert all(torch.equal(got[n], want[n]) for n in want)


def test_cu_seqlens_out_of_range_is_kept_in_bounds():
    q, k, v, d_o, _ = make([300], 0, 2, 1, 64, 22)
    wild = torch.tensor([5, -7, 100, 2_000_000_000], dtype=torch.int32, device="cuda")
    got = run(q, k, v, d_o, wild)
    torch.cuda.synchronize()
    sane = torch.tensor([0, 0, 100, 300], dtype=torch.int32, device="cuda")
    want = run(q, k, v, d_o, sane)
    assert all(torch.equal(got[n], want[n]) for n in want)


def test_empty_packs():
    q, k, v, d_o, cu = make([0], 0, 2, 1, 64, 23)
    got = run(q, k, v, d_o, cu)
    assert got["o"].shape == (0, 2, 64) and got["lse"].shape == (2, 0)
    q, k, v, d_o, _ = make([], 10, 2, 1, 64, 24)
    got = run(q, k, v, d_o, torch.zeros(1, dtype=torch.int32, device="cuda"))        # no sequence at all
    assert not bool(got["o"].any()) and not bool(got["dk"].any())


def test_refusals():
    q, k, v, d_o, cu = make([20], 0, 4, 2, 64, 25)
    o, lse = gb.gac_attn_forward(q, k, v, cu)
    for args, status in (((q.float(), k.float(), v.float(), cu), gb.GAC_ERR_DTYPE),
                         ((q.half(), k.half(), v.half(), cu), gb.GAC_ERR_DTYPE),
                         ((q[..., :60], k[..., :60], v[..., :60], cu), gb.GAC_ERR_INVALID_ARG),
                         ((q[:, :3], k, v, cu), gb.GAC_ERR_INVALID_ARG)):
        with pytest.raises(gb.GacError) as e:
            gb.gac_attn_forward(*args)
        assert e.value.status == status and len(str(e.value)) > 20
    big = torch.zeros(20, 4, 200, dtype=BF, device="cuda")
    for bad in (big[..., :136], torch.zeros(20 * 4 * 64 + 1, dtype=BF, device="cuda")[1:].view(20, 4, 64),
                torch.zeros(20, 4, 68, dtype=BF, device="cuda")[..., :64]):
        with pytest.raises(gb.GacError) as e:
            gb.gac_attn_forward(bad, bad, bad, cu)
        assert e.value.status == gb.GAC_ERR_INVALID_ARG
    with pytest.raises(gb.GacError):
        gb.gac_attn_forward(q, k, v, cu, scale=math.nan)
    for call in (lambda: gb.gac_attn_forward(q, k[:10], v, cu), lambda: gb.gac_attn_forward(q, k, v[:, :1], cu),
                 lambda: gb.gac_attn_forward(q, k, v, cu.long()), lambda: gb.gac_attn_forward(q, k, v, cu.cpu()),
                 lambda: gb.gac_attn_backward(d_o[:, :2], q, k, v, o, lse, cu),
                 lambda: gb.gac_attn_backward(d_o, q, k, v, o, lse[:, :5], cu)):
        with pytest.raises(ValueError):
            call()
