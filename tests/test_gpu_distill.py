"""Divergence from a teacher's top logits against the float64 form."""
import math

import pytest
import torch

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import packed

import distill_ref as ref
from packed_ref import within

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
KINDS = ["top", "forward", "reverse"]


def make(tokens, vocab, top, kind, dtype, seed, teacher=F, rest=0.05):
    """Logits with a few likely tokens, and a teacher that names some of them, in no order."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(tokens, vocab, generator=gen, device="cuda") * 1.5
    ids = torch.rand(tokens, vocab, generator=gen, device="cuda").topk(min(top, vocab), 1).indices
    x.scatter_add_(1, ids, 4.0 * torch.rand(ids.shape, generator=gen, device="cuda"))
    values = x.gather(1, ids) + 0.5 * torch.randn(ids.shape, generator=gen, device="cuda")
    if kind != "top":
        values = torch.log_softmax(values, 1) + math.log1p(-rest)
    w = 0.5 + torch.rand(tokens, generator=gen, device="cuda")
    return x.to(dtype), ids.to(torch.int32), values.to(teacher), w


def check(x, ids, values, kind, temperature=1.0, weights=None):
    want = ref.distill(x, ids, values, kind, temperature, weights)
    keep = x.clone()
    loss = gb.gac_distill(x, ids, values, kind, temperature)
    within(loss, *want["loss"], "loss")
    loss2, grad = gb.gac_distill(x, ids, values, kind, temperature, weights=weights, grad=True)
    within(loss2, *want["loss"], "loss beside the gradient")     # another order of the same sum
    assert torch.equal(x.nan_to_num(7.0), keep.nan_to_num(7.0)) and grad.dtype is x.dtype
    within(grad, *want["grad"], "grad")
    none, again = gb.gac_distill(x, ids, values, kind, temperature, weights=weights, grad=True, loss=False)
    assert none is None and torch.equal(grad, again)
    return loss, grad


@pytest.mark.parametrize("dtype", [BF, F], ids=["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [(1, 1, 1), (3, 2, 1), (5, 7, 7), (4, 8, 3), (9, 1021, 16), (2, 4099, 64), (3, 9001, 5), (3, 16385, 300),
                                  (2, 70001, 1000), (1, 151936, 64)], ids=str)
def test_sizes_and_kinds(dtype, kind, size):
    for temperature, teacher in ((1.0, F), (0.7, BF)):
        x, ids, values, w = make(*size, kind, dtype, sum(size), teacher)
        check(x, ids, values, kind, temperature, w)


@pytest.mark.parametrize("kind", KINDS)
def test_many_rows_are_not_split(kind):
    x, ids, values, w = make(700, 9000, 8, kind, BF, 5)
    few = gb.gac_distill(x[:20], ids[:20], values[:20], kind, weights=w[:20], grad=True)
    want = ref.distill(x[:20], ids[:20], values[:20], kind, 1.0, w[:20])
    many = gb.gac_distill(x, ids, values, kind, weights=w, grad=True)
    for loss, grad in (few, (many[0][:20], many[1][:20])):
        within(loss, *want["loss"])
        within(grad, *want["grad"])
    want = ref.distill(x[-20:], ids[-20:], values[-20:], kind, 1.0, w[-20:])
    within(many[0][-20:], *want["loss"])
    within(many[1][-20:], *want["grad"])


@pytest.mark.parametrize("dtype", [BF, F], ids=["bf16", "f32"])
def test_strides_alignment_and_in_place(dtype):
    x, ids, values, w = make(6, 5003, 9, "forward", dtype, 7)
    want = ref.distill(x, ids, values, "forward", 1.0, w)
    for pitch, start in ((5003, 1), (5010, 3), (5008, 0), (5001 + 8, 5)):      # rows on every boundary; a base off 16 bytes
        flat = torch.zeros(6 * pitch + 16, dtype=dtype, device="cuda")
        v = flat[start:start + 6 * pitch].view(6, pitch)[:, :5003]
        v.copy_(x)
        # ids and values with strides of their own
        i2, t2 = torch.nn.functional.pad(ids, (2, 3))[:, 2:-3], torch.nn.functional.pad(values, (1, 0))[:, 1:]
        loss, grad = gb.gac_distill(v, i2, t2, "forward", weights=w, grad=True)
        within(loss, *want["loss"])
        within(grad, *want["grad"])
        keep = flat.clone()
        loss2, same = gb.gac_distill(v, i2, t2, "forward", weights=w, grad=True, in_place=True)
        assert same is v and torch.equal(loss2, loss) and torch.equal(v, grad)
        keep[start:start + 6 * pitch].view(6, pitch)[:, :5003] = grad          # nothing else was written
        assert torch.equal(flat, keep)
    one = x[:1].expand(6, 5003)                                                # the same logits under six teachers
    want = ref.distill(one, ids, values, "forward", 1.0, w)
    loss, grad = gb.gac_distill(one, ids, values, "forward", weights=w, grad=True)
    within(loss, *want["loss"])
    within(grad, *want["grad"])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("vocab", [900, 20000])
def test_absent_and_repeated_entries(kind, vocab):
    x, ids, values, w = make(8, vocab, 40, kind, F, 11)
    ids[1] = -1                                    # a prompt's row: no teacher
    ids[2, 5:] = vocab                             # out of range on either side
    ids[2, 20:] = -2 ** 31
    values[3, 7:] = -math.inf
    ids[4, 10:30] = ids[4, 3].item()               # one token again and again
    ids[5] = ids[5, 0].item()
    ids[6, 1::2] = ids[6, 0::2]                    # pairs
    ids[7, 0] = -1
    values[7, 1] = -math.inf
    ids[7, 3] = ids[7, 1].item()                   # the first of the two is absent, so the second counts
    x[1, 5] = math.nan                             # not read
    loss, grad = check(x, ids, values, kind, 1.0, w)
    assert float(loss[1]) == 0.0 and bool((grad[1] == 0).all())
    x[1] = 0.0
    # the values of repeated entries do not matter
    v2 = values.clone()
    v2[4, 10:30] -= 3.0
    l2, g2 = gb.gac_distill(x, ids, v2, kind, weights=w, grad=True)
    if kind != "top":
        assert torch.equal(l2[4], loss[4]) and torch.equal(g2[4], grad[4])
    within(l2[4:5], *[r[4:5] for r in ref.distill(x, ids, v2, kind, 1.0, w)["loss"]])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [BF, F], ids=["bf16", "f32"])
def test_masked_logits(kind, dtype):
    lowest = torch.finfo(dtype).min
    x, ids, values, w = make(8, 3000, 20, kind, dtype, 13)
    for row, low in ((0, -math.inf), (1, lowest), (2, -1e4)):
        x[row, 1::2] = low                          # half of the vocabulary, some named tokens among it
    x[:3].scatter_(1, ids[:3].long(), torch.randn(3, 20, device="cuda").to(dtype))
    for row, low in ((3, -math.inf), (4, lowest)):  # all but the named tokens
        keep = x[row, ids[row].long()].clone()
        x[row] = low
        x[row, ids[row].long()] = keep
    x[5] += 60.0                                    # all far from zero
    x[6] *= 20.0                                    # one token has nearly everything
    loss, grad = check(x, ids, values, kind, 1.0, w)
    assert bool(loss.isfinite().all()) and bool(grad.isfinite().all())
    # a named token that is masked
    x[7, ids[7, 2].long()] = -math.inf
    loss, grad = gb.gac_distill(x, ids, values, kind, weights=w, grad=True)
    if kind == "reverse":
        want = ref.distill(x[7:], ids[7:], values[7:], kind, 1.0, w[7:])
        within(loss[7:], *want["loss"])
        within(grad[7:], *want["grad"])
    else:
        assert math.isinf(float(loss[7])) and bool(grad[7].isfinite().all()) and float(grad[7, ids[7, 2].long()]) < 0


@pytest.mark.parametrize("kind", KINDS)
def test_non_finite_values_stay_in_their_row(kind):
    x, ids, values, w = make(7, 9000, 12, kind, F, 17)
    clean = gb.gac_distill(x, ids, values, kind, weights=w, grad=True)
    other = [i for i in range(9000) if i not in ids[0].tolist()][0]
    x[0, other] = math.nan
    x[1, ids[1, 3].long()] = math.nan
    x[2, ids[2, 3].long()] = math.inf
    values[3, 4] = math.nan
    x[4] = -math.inf
    x[5, 8999 if 8999 not in ids[5].tolist() else 8998] = math.inf
    loss, grad = gb.gac_distill(x, ids, values, kind, weights=w, grad=True)
    for row in range(6):
        assert not math.isfinite(float(loss[row])), row
    assert torch.equal(loss[6], clean[0][6]) and torch.equal(grad[6], clean[1][6])


@pytest.mark.parametrize("kind", ["forward", "reverse"])
def test_a_teacher_that_leaves_little_or_nothing_to_the_rest(kind):
    x, ids, values, w = make(6, 2000, 30, kind, F, 19)
    p = values.double().softmax(1)
    for row, rest in enumerate((1e-2, 1e-5, 1e-7, 0.0, -1e-4)):     # the last two: none, and sums above one
        values[row] = (p[row] * (1 - rest)).log().float()
    values[5, 3] = torch.finfo(F).min                               # a token that the teacher rules out
    if kind == "reverse":
        x[5, ids[5, 3].long()] = -200.0                             # exp(-200) of the policy on it: e^-200 3e38 is nothing
    check(x, ids, values, kind, 1.0, w)


@pytest.mark.parametrize("kind", KINDS)
def test_the_gradient_against_differences(kind):
    """Differences of the float64 loss at the kernel's inputs, along random directions."""
    x, ids, values, w = make(5, 300, 12, kind, F, 23)
    _, grad = gb.gac_distill(x, ids, values, kind, 1.3, weights=w, grad=True)
    e = torch.randn(5, 300, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=torch.float64)
    h = 1e-4
    up, down = (float((ref.distill(x.double() + d * h * e, ids, values, kind, 1.3)["loss"][0] * w.double()).sum()) for d in (1, -1))
    told = float((grad.double() * e).sum())
    size = float((grad.double().abs() * e.abs()).sum())
    # h^2 / 6 times a third derivative of a few units, and what the kernel's gradient is off by
    assert abs((up - down) / (2 * h) - told) <= 1e-5 * size + 1e-7


def test_streams_graphs_and_empty_calls():
    x, ids, values, w = make(40, 12000, 20, "reverse", BF, 29)
    want = gb.gac_distill(x, ids, values, "reverse", weights=w, grad=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = gb.gac_distill(x, ids, values, "reverse", weights=w, grad=True, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    buf, graph = x.clone(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        loss, _ = gb.gac_distill(buf, ids, values, "reverse", weights=w, grad=True, in_place=True)
    for _ in range(2):
        buf.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(buf, want[1])
    loss, grad = gb.gac_distill(x[:0], ids[:0], values[:0], grad=True)
    assert loss.shape == (0,) and grad.shape == (0, 12000)


def test_through_autograd():
    for kind in KINDS:
        x, ids, values, w = make(9, 1021, 16, kind, F, 31)
        leaf = x.clone().requires_grad_()
        (packed.distillation(leaf, ids, values, kind, 1.5) * w).sum().backward()
        want = ref.distill(x, ids, values, kind, 1.5, w)
        within(leaf.grad, *want["grad"])
        leaf.grad = None
        packed.distillation(leaf, ids, values, kind, 1.5).mean().backward()         # an expanded gradient comes in
        want = ref.distill(x, ids, values, kind, 1.5, torch.full((9,), 1 / 9))
        value, bound = want["grad"]
        within(leaf.grad, value, bound + ref.U * 2 * value.abs())
    loss = packed.distillation(leaf, ids, values, kind)
    first, = torch.autograd.grad((loss ** 2).sum(), leaf, create_graph=True)
    with pytest.raises(RuntimeError):
        first.sum().backward()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y = leaf * 1.0
        loss = packed.distillation(y, ids, values, kind)
        gb.gac_distill(y.detach(), ids, values, kind, grad=True, in_place=True)
        loss.sum().backward()


def test_offsets_past_32_bits():
    x, ids, values, w = make(2, 2000, 10, "top", BF, 37)
    far = torch.zeros(2 ** 32 + 4096, dtype=BF, device="cuda")
    v = far.as_strided((2, 2000), (2 ** 32 + 17, 1))
    v.copy_(x)
    want = gb.gac_distill(x, ids, values, weights=w, grad=True)
    ref_want = ref.distill(x, ids, values, "top", 1.0, w)
    loss, grad = gb.gac_distill(v, ids, values, weights=w, grad=True)
    for a, b in ((loss, grad), want):
        within(a, *ref_want["loss"])
        within(b, *ref_want["grad"])
    gb.gac_distill(v, ids, values, weights=w, grad=True, in_place=True)
    assert torch.equal(v, grad)


def test_refusals():
    x, ids, values, w = make(4, 100, 5, "top", F, 41)
    for bad, kind in (((x.double(), ids, values), gb.GacError), ((x, ids, values.half()), gb.GacError), ((x, ids.long(), values), ValueError),
                      ((x, ids[:3], values[:3]), ValueError), ((x, ids, values[:, :4]), ValueError), ((x.t(), ids, values), ValueError),
                      ((x[0], ids, values), ValueError), ((x, ids.cpu(), values), ValueError), ((x, ids[:, :0], values[:, :0]), gb.GacError),
                      ((x, ids, values[:, ::2]), ValueError), ((x[:, :0], ids, values), gb.GacError)):
        with pytest.raises(kind):
            gb.gac_distill(*bad)
    for kw, kind in (({"temperature": 0.0}, gb.GacError), ({"temperature": math.nan}, gb.GacError), ({"temperature": 1e9}, gb.GacError),
                     ({"kind": "sideways"}, KeyError), ({"weights": w[:3]}, ValueError), ({"weights": w.double()}, ValueError),
                     ({"in_place": True}, ValueError)):
        with pytest.raises(kind):
            gb.gac_distill(x, ids, values, **kw)
    with pytest.raises(gb.GacError):        # rows of the gradient would lie on one another
        gb.gac_distill(x[:1].expand(4, 100), ids, values, grad=True, in_place=True)
