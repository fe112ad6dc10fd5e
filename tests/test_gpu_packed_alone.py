"""What a pack gives is what each of its sequences gives alone: attention and its gradients, and the divergence of every token, in the pack
and of the sequence by itself, are both held to the float64 form of the sequence by itself."""
import pytest
import torch

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import packed

import distill_ref
import heads_ref
from packed_ref import attention, within
from test_gpu_packed_heads import AXES, DIM, FREQS, KV_HEADS, Q_HEADS, inputs, run

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("kind", ["top", "forward", "reverse"])
def test_sequences_do_not_see_each_other(kind):
    qkv, wq, wk, head, ids, teacher, places, cu = inputs(5)
    gen = torch.Generator(device="cuda").manual_seed(9)
    with torch.no_grad():                       # sequences of very different size: what leaks from one into another is seen
        qkv[cu[1]:cu[2], Q_HEADS + KV_HEADS:] *= 50.0
    weights = torch.rand(ids.shape[0], generator=gen, device="cuda")

    def step(qkv, ids, teacher, places, cu, weights):
        """Everything that the library computes in one step, as leaves see it; the logits' gradient weighs every token by itself."""
        (q, k, v), (qn, kn, o, logits), loss = run(qkv, wq, wk, head, ids, teacher, places, cu, kind)
        return (qn, kn, v, o, logits, loss) + torch.autograd.grad((loss * weights).sum(), (q, k, v, qn, kn, o, logits))

    whole = step(qkv, ids, teacher, places, cu, weights)
    for a, b in zip(cu.tolist()[:-1], cu.tolist()[1:]):
        one = cu.new_tensor([0, b - a])
        alone = step(qkv.detach()[a:b].clone().requires_grad_(), ids[a:b], teacher[a:b], places[:, a:b], one, weights[a:b])
        assert torch.equal(alone[0], whole[0][a:b]) and torch.equal(alone[1], whole[1][a:b])
        cs = heads_ref.wheel(places[:, a:b].double(), torch.from_numpy(FREQS).cuda(), AXES)
        for name, got in (("alone", alone), ("packed", [t[a:b] for t in whole])):
            qn, kn, v, o, logits, loss, dq, dk, dv, dqn, dkn, d_o, d_logits = (t.detach() for t in got)
            want = attention(qn, kn, v, one, DIM ** -0.5, d_o)
            for key, t in (("o", o), ("dq", dqn), ("dk", dkn), ("dv", dv)):
                within(t, *want[key], f"{name} {key}")
            want = distill_ref.distill(logits, ids[a:b], teacher[a:b], kind, 1.0, weights[a:b])
            within(loss, *want["loss"], f"{name} loss")
            within(d_logits, *want["grad"], f"{name} gradient of the logits")
            for x, w, d, t in ((qkv.detach()[a:b, :Q_HEADS], wq, dqn, dq), (qkv.detach()[a:b, Q_HEADS:Q_HEADS + KV_HEADS], wk, dkn, dk)):
                within(t, *heads_ref.norm_back(d, x, w.detach(), cs, "half", 1.0, 1e-6, 0.0)[0], f"{name} heads")
        # rows of one call of the divergence know nothing of each other either
        loss, grad = gb.gac_distill(whole[4].detach()[a:b], ids[a:b], teacher[a:b], kind, weights=weights[a:b], grad=True)
        want = distill_ref.distill(whole[4].detach()[a:b], ids[a:b], teacher[a:b], kind, 1.0, weights[a:b])
        within(loss, *want["loss"])
        within(grad, *want["grad"])
    assert all(bool((t[cu[-1]:] == 0).all()) for t in whole[6:9])
    other = qkv.detach().clone()                # another first token of the last sequence moves nothing in front of it, whatever it is
    last = int(cu[-2])
    other[last:] = torch.randn(other[last:].shape, generator=gen, device="cuda").to(BF) * 9.0
    changed = step(other.requires_grad_(), ids, teacher, places, cu, weights)
    for i in (3, 6, 7, 8):
        assert torch.equal(changed[i][:last], whole[i][:last])
    assert not torch.equal(changed[3][last:], whole[3][last:])
