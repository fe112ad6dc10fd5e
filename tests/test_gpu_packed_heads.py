"""The heads' norms with positions on axes, packed attention and the divergence from a teacher, run together as a policy update
runs them: every operator is held to the float64 form of what reached it, forward and backward, and a pack to its sequences."""
import math

import pytest
import torch

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import packed

import distill_ref
import heads_ref
from packed_ref import attention, within

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
LENGTHS, TAIL, Q_HEADS, KV_HEADS, DIM, VOCAB, TOP = [1, 130, 257, 64], 3, 6, 2, 64, 1021, 12
AXES = gb.gac_rotary_sections([8, 12, 12], interleaved=True)
FREQS = gb.gac_rotary_freqs(DIM, 1e6)


def inputs(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    tokens = sum(LENGTHS) + TAIL
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    qkv = r(tokens, Q_HEADS + 2 * KV_HEADS, DIM).to(BF).requires_grad_()
    wq, wk = ((1 + 0.2 * r(DIM)).requires_grad_() for _ in range(2))
    head = (r(VOCAB, Q_HEADS * DIM) * (Q_HEADS * DIM) ** -0.5).to(BF).requires_grad_()
    ids = torch.rand(tokens, VOCAB, generator=gen, device="cuda").topk(TOP, 1).indices.to(torch.int32)
    teacher = torch.log_softmax(r(tokens, TOP), 1) + math.log(0.9)
    places = torch.randint(0, 9000, (3, tokens), generator=gen, device="cuda", dtype=torch.int32)
    cu = torch.tensor([0] + list(torch.tensor(LENGTHS).cumsum(0)), dtype=torch.int32, device="cuda")
    ids[cu[-1]:] = -1                                   # rows behind the last sequence have no teacher
    return qkv, wq, wk, head, ids, teacher, places, cu


def run(qkv, wq, wk, head, ids, teacher, places, cu, kind):
    q, k, v = qkv.split([Q_HEADS, KV_HEADS, KV_HEADS], dim=1)
    qn, kn = packed.norm_rotary(q, k, wq, wk, FREQS, positions=places, axes=AXES)
    o = packed.attention(qn, kn, v, cu)
    logits = o.flatten(1) @ head.t()
    return (q, k, v), (qn, kn, o, logits), packed.distillation(logits, ids, teacher, kind)


@pytest.mark.parametrize("kind", ["top", "forward", "reverse"])
def test_every_operator_beside_the_others(kind):
    qkv, wq, wk, head, ids, teacher, places, cu = inputs(1)
    (q, k, v), (qn, kn, o, logits), loss = run(qkv, wq, wk, head, ids, teacher, places, cu, kind)
    for t in (q, k, v, qn, kn, o, logits):
        t.retain_grad()
    weights = torch.rand(loss.numel(), device="cuda") / loss.numel()
    (loss * weights).sum().backward()
    cs = heads_ref.wheel(places.double(), torch.from_numpy(FREQS).cuda(), AXES)
    want = distill_ref.distill(logits.detach(), ids, teacher, kind, 1.0, weights)
    within(loss.detach(), *want["loss"])
    within(logits.grad, *want["grad"])
    want = attention(qn.detach(), kn.detach(), v.detach(), cu, DIM ** -0.5, o.grad)
    within(o.detach(), *want["o"])
    for name, t in (("dq", qn), ("dk", kn), ("dv", v)):
        within(t.grad, *want[name], name)
    for x, y, w in ((q, qn, wq), (k, kn, wk)):
        within(y.detach(), *heads_ref.norm(x.detach(), w.detach(), cs, "half", 1.0, 1e-6, 0.0))
        dx, dw = heads_ref.norm_back(y.grad, x.detach(), w.detach(), cs, "half", 1.0, 1e-6, 0.0)
        within(x.grad, *dx)
        within(w.grad, *dw)
    assert bool((qkv.grad[cu[-1]:] == 0).all()) and bool((o[cu[-1]:] == 0).all()) and bool((loss[cu[-1]:] == 0).all())


def test_a_pack_gives_what_its_sequences_give_alone():
    qkv, wq, wk, head, ids, teacher, places, cu = inputs(2)
    _, _, loss = run(qkv, wq, wk, head, ids, teacher, places, cu, "reverse")
    whole, = torch.autograd.grad(loss.sum(), qkv)
    for a, b in zip(cu.tolist()[:-1], cu.tolist()[1:]):
        x = qkv.detach()[a:b].clone().requires_grad_()
        (q, k, v), (qn, kn, o, _), _ = run(x, wq, wk, head, ids[a:b], teacher[a:b], places[:, a:b], cu[:1].new_tensor([0, b - a]), "reverse")
        both = packed.norm_rotary(*qkv.detach().split([Q_HEADS, KV_HEADS, KV_HEADS], dim=1)[:2], wq, wk, FREQS, positions=places, axes=AXES)
        assert torch.equal(both[0][a:b], qn) and torch.equal(both[1][a:b], kn)
    assert bool(whole.isfinite().all()) and bool((whole[cu[-1]:] == 0).all())


def test_two_streams_at_once():
    calls = []
    for seed in (3, 4):
        qkv, wq, wk, head, ids, teacher, places, cu = inputs(seed)
        calls.append(lambda a=(qkv, wq, wk, head, ids, teacher, places, cu): torch.autograd.grad(run(*a, "forward")[2].sum(), a[:4]))
    want = [c() for c in calls]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = calls[i]()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            for x, y in zip(a, b):
                assert torch.equal(x, y)
