"""The divergence where logits are masked with finite numbers of every size, in blocks and throughout, at several temperatures, and where
all logits lie far from zero."""
import math

import pytest
import torch

from paper_2603_01501_b200 import binding as gb

import distill_far_ref as ref
from packed_ref import within

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
LARGEST = torch.finfo(F).max


def check(x, ids, values, kind, temperature, w):
    want = ref.distill(x, ids, values, kind, temperature, w)
    loss, bound = want["loss"]
    over = loss.abs() > LARGEST                 # more than binary32 holds
    alone = gb.gac_distill(x, ids, values, kind, temperature)
    told, grad = gb.gac_distill(x, ids, values, kind, temperature, weights=w, grad=True)
    for got in (alone, told):
        within(got[~over], loss[~over], bound[~over], "loss")
        assert bool(torch.isposinf(got[over]).all())
    within(grad, *want["grad"], "grad")
    buf = x.clone()
    same = gb.gac_distill(buf, ids, values, kind, temperature, weights=w, grad=True, in_place=True, loss=False)
    assert same[1] is buf and torch.equal(buf, grad)
    return told, grad


def masked(vocab, top, kind, dtype, low, seed):
    """Rows with `low` in many places; the named tokens of each are sorted, as a list by id would be."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows = 13
    x = torch.randn(rows, vocab, generator=gen, device="cuda") * 1.5
    ids = torch.rand(rows, vocab, generator=gen, device="cuda").topk(top, 1).indices.sort(1).values
    likely = x.gather(1, ids) + 4.0 * torch.rand(ids.shape, generator=gen, device="cuda")
    hide = torch.zeros(rows, vocab, dtype=torch.bool, device="cuda")
    hide[0, 1::2] = True
    hide[1, vocab * 2 // 3:] = True                                   # a padded vocabulary's tail
    hide[2] = hide[3] = True                                          # all but 40 tokens, all but one
    hide[2, torch.randperm(vocab, generator=gen, device="cuda")[:40]] = False
    hide[3, [i for i in range(vocab) if i not in ids[3].tolist()][vocab // 2]] = False
    hide[4, :vocab // 2] = True
    hide[5] = True                                                    # all but the named tokens
    hide[11] = True
    x[hide] = low
    x.scatter_(1, ids, likely)
    x[6, ids[6, 2]] = low                                             # one named token
    x[7, ids[7, top // 2:]] = low                                     # the second half of them
    x[8, ids[8]] = low                                                # all of them
    x[9] = low                                                        # everything
    x[10] = torch.where(torch.rand(vocab, generator=gen, device="cuda") < 0.5, low, low / 2)
    x[11, ids[11, 1:]] = low                                          # all but one named token
    values = likely + 0.5 * torch.randn(ids.shape, generator=gen, device="cuda")
    if kind != "top":
        values = torch.log_softmax(values, 1) + math.log1p(-0.05)
    return x.to(dtype), ids.to(torch.int32), values, 0.5 + torch.rand(rows, generator=gen, device="cuda")


@pytest.mark.parametrize("temperature", [0.7, 1.0, 1.5, 2.0, 5.0])
@pytest.mark.parametrize("low", [-1e7, -1e9, -1e10, -1e12, -1e20, -1e30, float(torch.finfo(BF).min), float(torch.finfo(F).min)], ids=str)
@pytest.mark.parametrize("dtype", [BF, F], ids=["bf16", "f32"])
@pytest.mark.parametrize("kind", ["top", "forward", "reverse"])
def test_finite_masks(kind, dtype, low, temperature):
    low = max(low, torch.finfo(dtype).min)
    for vocab, top in ((1021, 64), (9001, 20)):
        x, ids, values, w = masked(vocab, top, kind, dtype, low, vocab)
        check(x, ids, values, kind, temperature, w)


@pytest.mark.parametrize("kind", ["top", "forward", "reverse"])
@pytest.mark.parametrize("size", [(1021, 400), (32000, 90), (151936, 60)], ids=str)
def test_finite_masks_in_rows_that_are_whole_or_split(size, kind):
    vocab, times = size
    for dtype, low in ((BF, float(torch.finfo(BF).min)), (F, -1e10)):
        x, ids, values, w = masked(vocab, 64, kind, dtype, low, 3)
        loss, grad = check(x, ids, values, kind, 2.0, w)
        want = ref.distill(x, ids, values, kind, 2.0, w)
        many, grads = gb.gac_distill(*(t.repeat(times, 1) for t in (x, ids, values)), kind, 2.0, weights=w.repeat(times), grad=True)
        many, grads = many.view(times, -1), grads.view(times, *x.shape)
        # rows that begin at the same place of 16 bytes, which every eighth copy does, are added up in the same order
        assert torch.equal(many[8:], many[:-8]) and torch.equal(grads[8:], grads[:-8])
        inside = want["loss"][0].abs() <= LARGEST
        for copy in range(8):
            within(many[copy][inside], *(t[inside] for t in want["loss"]))
            within(grads[copy], *want["grad"])


@pytest.mark.parametrize("kind", ["top", "forward", "reverse"])
@pytest.mark.parametrize("at", [1e6, 1e8, 1e10, 1e20, -1e10, -1e20, 3e38], ids=str)
def test_logits_that_are_all_far_from_zero(kind, at):
    for dtype, vocab in ((BF, 1021), (F, 20000)):
        gen = torch.Generator(device="cuda").manual_seed(7)
        step = abs(at) * torch.finfo(dtype).eps
        x = (at - step * torch.randint(0, 3, (5, vocab), generator=gen, device="cuda").double()).to(dtype)
        x[3:] = x[3:].max()
        ids = torch.rand(5, vocab, generator=gen, device="cuda").topk(9, 1).indices
        x[4].scatter_(0, ids[4], 1.0)
        values = torch.log_softmax(torch.randn(5, 9, generator=gen, device="cuda"), 1) - 0.2
        for temperature in (0.7, 1.0, 1000.0):
            check(x, ids.to(torch.int32), values, kind, temperature, torch.ones(5, device="cuda"))


@pytest.mark.parametrize("kind", ["forward", "reverse"])
def test_a_named_token_masked_alone_in_its_part(kind):
    """One named token at either end of a row that is split, one of them masked; and no other logit beside them."""
    for dtype in (BF, F):
        for low in (-1e10, -1e30, float(torch.finfo(dtype).min)):
            for rest in (0.0, low):
                x = torch.full((2, 40000), rest, dtype=dtype, device="cuda")
                ids = torch.tensor([[5, 39990], [39990, 5]], dtype=torch.int32, device="cuda")
                x[:, 5], x[:, 39990] = 3.0, low
                values = torch.tensor([[0.6, 0.3], [0.2, 0.7]], device="cuda").log()
                for temperature in (0.7, 1.0, 1.5, 2.0, 5.0):
                    check(x, ids, values, kind, temperature, torch.ones(2, device="cuda"))


@pytest.mark.parametrize("dtype", [BF, F], ids=["bf16", "f32"])
def test_far_rows_at_any_place_of_memory(dtype):
    """Rows on every boundary, a gradient on another boundary than the logits, and nothing written beside it."""
    for vocab, kind in ((1021, "forward"), (30011, "reverse"), (9, "top"), (1, "top")):
        x, ids, values, w = masked(max(vocab, 64), 20, kind, dtype, -1e20, 11)
        if vocab < 64:
            x, ids = x[:, :vocab].contiguous(), ids % vocab
        want = ref.distill(x, ids, values, kind, 1.5, w)
        for start, pitch in ((0, vocab), (3, vocab + 2), (1, vocab + 7)):
            flat = torch.full((13 * pitch + 16,), 7.0, dtype=dtype, device="cuda")
            v = flat[start:start + 13 * pitch].view(13, pitch)[:, :vocab]
            v.copy_(x)
            keep = flat.clone()
            loss, grad = gb.gac_distill(v, ids, values, kind, 1.5, weights=w, grad=True)
            within(loss, *want["loss"])
            within(grad, *want["grad"])
            gb.gac_distill(v, ids, values, kind, 1.5, weights=w, grad=True, in_place=True)
            keep[start:start + 13 * pitch].view(13, pitch)[:, :vocab] = grad
            assert torch.equal(flat, keep)


@pytest.mark.parametrize("kind", ["top", "forward", "reverse"])
def test_far_rows_with_repeats_and_with_non_finite_values(kind):
    for vocab in (700, 50000):
        x, ids, values, w = masked(vocab, 64, kind, BF, -1e20, 13)
        clean = gb.gac_distill(x, ids, values, kind, weights=w, grad=True)
        i2, v2 = ids.clone(), values.clone()
        i2[:, 40:] = ids[:, :24]                       # the first counts, whatever the others say
        v2[:, 40:] = 50.0
        check(x, i2, v2, kind, 1.5, w)
        y, t = x.clone(), values.clone()
        y[5, [i for i in range(vocab) if i not in ids[5].tolist()][vocab // 3]] = math.nan     # elsewhere in a far row
        y[8, ids[8, 1]] = math.nan                                                              # at a named token of one
        y[9, 0] = math.inf
        t[10, 3] = math.nan
        for _ in range(2):
            loss, grad = gb.gac_distill(y, ids, t, kind, weights=w, grad=True)
            for row in range(13):
                if row in (5, 8, 9, 10):
                    assert not math.isfinite(float(loss[row])), row
                else:
                    assert torch.equal(loss[row], clean[0][row]) and torch.equal(grad[row], clean[1][row]), row


def test_far_rows_on_two_streams_and_in_graphs():
    calls = []
    for seed, kind in ((17, "forward"), (19, "top")):
        x, ids, values, w = masked(40009, 64, kind, BF, -1e20, seed)
        calls.append(lambda a=(x, ids, values, kind), w=w: gb.gac_distill(*a, weights=w, grad=True))
    want = [c() for c in calls]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = calls[i]()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(want, got) for a, b in zip(x, y))
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for g, c in zip(graphs, calls):
        with torch.cuda.graph(g):
            outs.append(c())
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x, y in zip(want, outs) for a, b in zip(x, y))
