"""Policy updates on packed rollouts, end to end: a small decoder with grouped-query attention, a clipped
policy-gradient loss, the gradient alignment rule with clipping in its own pass, a value head whose gradients have no
stored direction and are clipped by themselves, and AdamW.

    python examples/packed_policy_update.py [steps]

Rollouts of different lengths are laid one behind the other and trained on without padding: rotary positions and
causal attention run over the pack (``packed.rotary``, ``packed.attention``), the rest of the decoder is ordinary
torch.  The rollouts are random tokens with random advantages: this shows the calls, it learns nothing.
"""
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import packed
from paper_2603_01501_b200.controller import GradientAlignmentController

HIDDEN, LAYERS, Q_HEADS, KV_HEADS, HEAD_DIM, INTERMEDIATE, VOCAB = 384, 2, 6, 2, 64, 1030, 1021


class Block(torch.nn.Module):
    def __init__(self):
        super().__init__()
        self.qkv = torch.nn.Linear(HIDDEN, (Q_HEADS + 2 * KV_HEADS) * HEAD_DIM)
        self.out = torch.nn.Linear(Q_HEADS * HEAD_DIM, HIDDEN, bias=False)
        self.norm1, self.norm2 = torch.nn.RMSNorm(HIDDEN), torch.nn.RMSNorm(HIDDEN)
        self.gate = torch.nn.Linear(HIDDEN, INTERMEDIATE, bias=False)
        self.up = torch.nn.Linear(HIDDEN, INTERMEDIATE, bias=False)
        self.down = torch.nn.Linear(INTERMEDIATE, HIDDEN, bias=False)

    def forward(self, x, cu, freqs):
        qkv = self.qkv(self.norm1(x)).to(torch.bfloat16).view(-1, Q_HEADS + 2 * KV_HEADS, HEAD_DIM)
        q, k, v = qkv.split([Q_HEADS, KV_HEADS, KV_HEADS], dim=1)
        q, k = packed.rotary(q, k, freqs, cu_seqlens=cu)
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

    def forward(self, tokens, cu):
        """Log-probability of every token's successor in the pack, and the last hidden states."""
        x = self.embed(tokens)
        for block in self.blocks:
            x = block(x, cu, self.freqs)
        x = self.norm(x)
        return F.log_softmax((x @ self.embed.weight.t())[:-1], -1).gather(1, tokens[1:, None])[:, 0], x


def rollouts(step, device="cuda"):
    """Random finished rollouts: tokens, cu_seqlens, advantage per token, and which tokens have a successor of their own."""
    gen = torch.Generator().manual_seed(step)
    lengths = torch.randint(1, 700, (8,), generator=gen)
    cu = torch.cat((torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)))
    tokens = torch.randint(0, VOCAB, (int(cu[-1]),), generator=gen)
    advantage = torch.randn(8, generator=gen).repeat_interleave(lengths)
    inner = torch.ones(int(cu[-1]), dtype=torch.bool)
    inner[cu[1:] - 1] = False
    return tokens.to(device), cu.to(torch.int32).to(device), advantage[:-1].to(device), inner[:-1].to(device)


def main(steps=5, max_norm=1.0):
    torch.manual_seed(0)
    policy, value = Policy().cuda(), torch.nn.Linear(HIDDEN, 1).cuda()
    optimizer = torch.optim.AdamW([*policy.parameters(), *value.parameters()], lr=1e-4)
    # the policy's gradients: the rule, clipped in the pass that applies it
    controller = GradientAlignmentController(policy.parameters(), gb.HParams(clip_max_norm=max_norm))
    # the value head's: no stored direction, norm and clipping alone
    clipper = packed.GradientClipper(value.parameters())
    told = []
    for step in range(steps):
        tokens, cu, advantage, inner = rollouts(step)
        with torch.no_grad():
            old, _ = policy(tokens, cu)
        new, states = policy(tokens, cu)
        ratio = (new - old).exp()
        gain = torch.minimum(ratio * advantage, ratio.clamp(0.8, 1.2) * advantage)
        error = value(states[:-1].detach())[:, 0] - advantage
        loss = -gain[inner].mean() + error[inner].square().mean()
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
