"""The autograd layer over the operators on packed rollouts, and the example that runs them together."""
import importlib.util
import math
import os

import pytest
import torch

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import packed

from packed_ref import attention, within

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF = torch.bfloat16


def tensors(tokens, qh, kh, dim, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(tokens, n, dim, generator=gen, device="cuda").to(BF).requires_grad_() for n in (qh, kh, kh)]


def test_attention_gradients_through_autograd():
    cu = torch.tensor([0, 70, 71, 300], dtype=torch.int32, device="cuda")
    q, k, v = tensors(300, 4, 2, 64, 1)
    d_o = torch.randn(300, 4, 64, device="cuda").to(BF)
    packed.attention(q, k, v, cu).backward(d_o)
    want = attention(q.detach(), k.detach(), v.detach(), cu, 0.125, d_o)
    for name, t in (("dq", q), ("dk", k), ("dv", v)):
        within(t.grad, *want[name], name)
    # a gradient that autograd hands over expanded (stride 0)
    for t in (q, k, v):
        t.grad = None
    packed.attention(q, k, v, cu).sum().backward()
    want = attention(q.detach(), k.detach(), v.detach(), cu, 0.125, torch.ones(300, 4, 64, device="cuda"))
    for name, t in (("dq", q), ("dk", k), ("dv", v)):
        within(t.grad, *want[name], name)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_gradient_is_the_transpose(layout):
    freqs = gb.gac_rotary_freqs(32, 1e4)
    cu = torch.tensor([0, 20, 50], dtype=torch.int32, device="cuda")
    q, k = (torch.randn(50, n, 64, device="cuda", requires_grad=True) for n in (3, 1))
    yq, yk = packed.rotary(q, k, freqs, cu_seqlens=cu, layout=layout, scale=1.5)
    gq, gk = torch.randn_like(yq), torch.randn_like(yk)
    torch.autograd.backward((yq, yk), (gq, gk))
    for x, y, g in ((q, yq, gq), (k, yk, gk)):
        left, right = (g.double() * y.detach().double()).sum(), (x.grad.double() * x.detach().double()).sum()
        # both sides are sums of products whose factors carry at most 12 units of 2^-24 each way
        size = float(g.norm() * y.detach().norm())
        assert abs(float(left - right)) <= 30 * 2.0 ** -24 * 1.5 * size


def test_a_pack_gives_what_its_sequences_give_alone():
    lengths = [1, 130, 257, 64, 700]
    cu = torch.tensor([0] + list(torch.tensor(lengths).cumsum(0)), dtype=torch.int32, device="cuda")
    freqs = gb.gac_rotary_freqs(128, 1e6)
    q, k, v = tensors(sum(lengths), 3, 3, 128, 2)
    d_o = torch.randn(sum(lengths), 3, 128, device="cuda").to(BF)

    def run(a, b, cu):
        xs = [t.detach()[a:b].clone().requires_grad_() for t in (q, k, v)]
        qr, kr = packed.rotary(xs[0], xs[1], freqs, cu_seqlens=cu)
        o = packed.attention(qr, kr, xs[2], cu)
        o.backward(d_o[a:b])
        return [o.detach()] + [x.grad for x in xs]

    whole = run(0, sum(lengths), cu)
    for a, b in zip(cu.tolist()[:-1], cu.tolist()[1:]):
        alone = run(a, b, torch.tensor([0, b - a], dtype=torch.int32, device="cuda"))
        for x, y in zip(whole, alone):
            assert torch.equal(x[a:b], y)


def test_clipper_follows_moving_gradients():
    params = [torch.nn.Parameter(torch.zeros(n, device="cuda", dtype=d)) for n, d in ((1000, torch.float32), (77, BF), (5, BF))]
    clipper = packed.GradientClipper(params)
    assert float(clipper.clip(1.0)) == 0.0                 # no gradients yet
    for step in range(3):
        for i, p in enumerate(params):
            p.grad = None if (step == 1 and i == 2) else torch.randn_like(p)
        before = [None if p.grad is None else p.grad.clone() for p in params]
        norm = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in before if g is not None))
        told = float(clipper.clip(0.5 * norm))
        assert abs(told - norm) <= 2.0 ** -23 * norm
        for p, g in zip(params, before):
            if g is not None:
                half = 2.0 ** -8 if g.dtype == BF else 2.0 ** -24
                want = g.double() * min(1.0, 0.5 * norm / (norm + 1e-6))
                assert bool(((p.grad.double() - want).abs() <= (half + 3 * 2.0 ** -24) * want.abs()).all())
    clipper.close()
    with pytest.raises(ValueError):
        packed.GradientClipper([])


def test_the_example_runs(capsys):
    spec = importlib.util.spec_from_file_location("packed_policy_update", os.path.join(ROOT, "examples", "packed_policy_update.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    told = example.main(steps=3)
    assert len(told) == 3 and all(math.isfinite(x) for row in told for x in row)
    assert told[0][2] == 0.0 and all(norm > 0 for _, norm, _ in told)
    assert "step 2" in capsys.readouterr().out
