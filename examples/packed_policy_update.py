"""Policy updates on packed rollouts, end to end: a small decoder with grouped-query attention and normed heads, a clipped
policy-gradient loss with a divergence from the reference policy's top logits, the gradient alignment rule with clipping in
its own pass, a value head whose gradients have no stored direction and are clipped by themselves, and AdamW.

    python examples/packed_policy_update.py [steps]

Rollouts of different lengths are laid one behind the other and trained on without padding: the heads' norms with rotary
positions and causal attention run over the pack (``packed.norm_rotary``, ``packed.attention``), the divergence over its logits
(``packed.distillation``), the rest of the decoder is ordinary torch.  Some rollouts have an image in front, whose patches
stand in height and width as well as in time.  The rollouts are random tokens with random advantages: this shows the calls, it learns nothing.
"""
import copy
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import packed
from paper_2603_01501_b200.controller import GradientAlignmentController

HIDDEN, LAYERS, Q_HEADS, KV_HEADS, HEAD_DIM, INTERMEDIATE, VOCAB = 384, 2, 6, 2, 64, 1030, 1021
AXES = gb.gac_rotary_sections([16, 8, 8], interleaved=True)   # pairs of a head that time, height and width turn
TOP = 16                                                      # logits kept of the reference policy, per token


class Block(torch.nn.Module):
    def __init__(self):
        super().__init__()
        self.qkv = torch.nn.Linear(HIDDEN, (Q_HEADS + 2 * KV_HEADS) * HEAD_DIM)
        self.q_norm, self.k_norm = (torch.nn.Parameter(torch.ones(HEAD_DIM)) for _ in range(2))
        self.out = torch.nn.Linear(Q_HEADS * HEAD_DIM, HIDDEN, bias=False)
        self.norm1, self.norm2 = torch.nn.RMSNorm(HIDDEN), torch.nn.RMSNorm(HIDDEN)
        self.gate = torch.nn.Linear(HIDDEN, INTERMEDIATE, bias=False)
        self.up = torch.nn.Linear(HIDDEN, INTERMEDIATE, bias=False)
        self.down = torch.nn.Linear(INTERMEDIATE, HIDDEN, bias=False)

    def forward(self, x, cu, places, freqs):
        qkv = self.qkv(self.norm1(x)).to(torch.bfloat16).view(-1, Q_HEADS + 2 * KV_HEADS, HEAD_DIM)
        q, k, v = qkv.split([Q_HEADS, KV_HEADS, KV_HEADS], dim=1)
        q, k = packed.norm_rotary(q, k, self.q_norm, self.k_norm, freqs, positions=places, axes=AXES)
        o = packed.attention(q, k, v, cu)
        x = x + self.out(o.flatten(1).float())
        h = self.norm2(x)
        return x + self.down(F.silu(self.gate(h)) * self.up(h))


class Policy(torch.nn.Module):
    def __init__(self):
        super().__init__()
        self.embed = torch.nn.Embedding(VOCAB, HIDDEN)
        self.blocks = torch.nn.ModuleList(Block() for _ in range(LAYERS))
        self.norm = torch.nn.RMSNorm(HIDDEN)
        # positions stretched to four times the trained context
        self.freqs = gb.gac_rotary_freqs(HEAD_DIM, 1e4, "parts", 4.0, trained=512.0)

    def forward(self, tokens, cu, places):
        """Log-probability of every token's successor in the pack, the logits it comes from, and the last hidden states."""
        x = self.embed(tokens)
        for block in self.blocks:
            x = block(x, cu, places, self.freqs)
        x = self.norm(x)
        logits = (x @ self.embed.weight.t())[:-1]
        return F.log_softmax(logits, -1).gather(1, tokens[1:, None])[:, 0], logits, x


def places_of(lengths):
    """Time, height and width of every token: all the same for text; every other rollout begins with an image of 4 x 6 patches."""
    out = []
    for i, n in enumerate(lengths.tolist()):
        at = torch.arange(n).repeat(3, 1)
        if i % 2 and n > 24:
            patch = torch.arange(24)
            at[:, :24] = torch.stack((torch.zeros_like(patch), patch // 6, patch % 6))
            at[:, 24:] -= 24 - 6   # the text goes on behind the image's longer side
        out.append(at)
    return torch.cat(out, 1).to(torch.int32)


def rollouts(step, device="cuda"):
    """Random finished rollouts: tokens, cu_seqlens, places, advantage per token, and which tokens have a successor of their own."""
    gen = torch.Generator().manual_seed(step)
    lengths = torch.randint(1, 700, (8,), generator=gen)
    cu = torch.cat((torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)))
    tokens = torch.randint(0, VOCAB, (int(cu[-1]),), generator=gen)
    advantage = torch.randn(8, generator=gen).repeat_interleave(lengths)
    inner = torch.ones(int(cu[-1]), dtype=torch.bool)
    inner[cu[1:] - 1] = False
    return tokens.to(device), cu.to(torch.int32).to(device), places_of(lengths).to(device), advantage[:-1].to(device), inner[:-1].to(device)


def main(steps=5, max_norm=1.0):
    torch.manual_seed(0)
    policy, value = Policy().cuda(), torch.nn.Linear(HIDDEN, 1).cuda()
    reference = copy.deepcopy(policy).requires_grad_(False)
    optimizer = torch.optim.AdamW([*policy.parameters(), *value.parameters()], lr=1e-4)
    # the policy's gradients: the rule, clipped in the pass that applies it
    controller = GradientAlignmentController(policy.parameters(), gb.HParams(clip_max_norm=max_norm))
    # the value head's: no stored direction, norm and clipping alone
    clipper = packed.GradientClipper(value.parameters())
    told = []
    for step in range(steps):
        tokens, cu, places, advantage, inner = rollouts(step)
        with torch.no_grad():
            old, _, _ = policy(tokens, cu, places)
            known, ids = F.log_softmax(reference(tokens, cu, places)[1], -1).topk(TOP, -1)   # what is stored with the rollouts
            ids = ids.to(torch.int32).masked_fill_(~inner[:, None], -1)                       # no teacher for what is not trained on
        new, logits, states = policy(tokens, cu, places)
        ratio = (new - old).exp()
        gain = torch.minimum(ratio * advantage, ratio.clamp(0.8, 1.2) * advantage)
        error = value(states[:-1].detach())[:, 0] - advantage
        apart = packed.distillation(logits, ids, known, "reverse").sum() / inner.sum()
        loss = -gain[inner].mean() + 0.1 * apart + error[inner].square().mean()
        optimizer.zero_grad()
        loss.backward()
        go_on = controller.step()                 # the alignment rule, in place on the policy's gradients
        norm = clipper.clip(max_norm)
        if not go_on:                             # a violation: the policy stays as it is
            policy.zero_grad()
        optimizer.step()
        told.append((float(loss.detach()), float(norm), controller.last.cos))
        print("step %d  loss %+.5f  value norm %.4f  alignment %+.4f  %s" % (step, *told[-1], gb.REGIME_NAMES[controller.last.regime]))
    gb.gac_attn_check()
    controller.close()
    clipper.close()
    return told


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 5)
