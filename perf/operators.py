"""What a policy update on packed rollouts needs around the gradient rule, as measured cases.

Three operators that follow one another in that update: rotary positions on the queries and keys of a pack of
sequences, causal attention over the pack with grouped heads (forward, and its gradient), and the global norm
of the resulting gradient list with clipping.  ``run`` computes them in plain torch operations, or, where
``own`` is true, through this package's entry points.

Head layouts (q heads / kv heads x head size) and tensor lists are those of this repository's synthetic
decoders: 3/1 x 32, 6/2 x 64, 8/2 x 128, 12/2 x 128, 28/4 x 128, 40/8 x 128.
"""
import math
import random

import numpy as np
import torch

own = False

# hidden, layers, q heads, kv heads, head size, intermediate, vocabulary, tied embeddings
DECODERS = {
    "mini": (96, 3, 3, 1, 32, 250, 1021, True),
    "small": (384, 6, 6, 2, 64, 1030, 15013, False),
    "0.25b": (1024, 12, 8, 2, 128, 4096, 32000, False),
    "1.5b": (1536, 28, 12, 2, 128, 8960, 151936, True),
}


def listed():
    return [
        # ---- global gradient norm and clipping over a list of tensors
        # a debugging-size policy with float32 norms and biases beside bfloat16 matrices, packed without padding: latency
        {"name": "clip_mini_mixed", "op": "clip", "decoder": "mini", "layers": 3, "types": "mixed", "pad": 1, "ratio": 0.25},
        # one flat float32 vector of 2^20 elements: an adapter-size gradient
        {"name": "clip_flat_1m_f32", "op": "clip", "decoder": "flat", "layers": 0, "types": "f32", "pad": 64, "ratio": 0.5},
        # 0.25 B parameters, bfloat16 gradients
        {"name": "clip_0.25b_bf16", "op": "clip", "decoder": "0.25b", "layers": 12, "types": "bf16", "pad": 64, "ratio": 0.1},
        # 1.5 B parameters, float32 gradients
        {"name": "clip_1.5b_f32", "op": "clip", "decoder": "1.5b", "layers": 28, "types": "f32", "pad": 64, "ratio": 0.7},
        # ---- rotary positions
        # one new token for each of 16 rollouts at far positions of a stretched context: latency
        {"name": "rotary_tokens_16", "op": "rotary", "tokens": 16, "lengths": "", "q_heads": 12, "kv_heads": 2, "head_dim": 128,
         "rot_dim": 128, "layout": "half", "scaling": "parts", "type": "bf16", "inverse": False, "fused": True},
        # a training micro-batch of packed rollouts
        {"name": "rotary_pack_16k", "op": "rotary", "tokens": 16384, "lengths": "4091,2713,3300,1500,4096,660", "q_heads": 28,
         "kv_heads": 4, "head_dim": 128, "rot_dim": 128, "layout": "half", "scaling": "none", "type": "bf16", "inverse": False,
         "fused": True},
        # the gradient's way back through positions on half of the head, pairs interleaved, float32
        {"name": "rotary_back_f32", "op": "rotary", "tokens": 8189, "lengths": "2047,1,3001,3140", "q_heads": 12, "kv_heads": 2,
         "head_dim": 128, "rot_dim": 64, "layout": "interleaved", "scaling": "linear", "type": "f32", "inverse": True,
         "fused": False},
        # ---- causal attention over packed sequences
        # a few short answers of a small policy, one of a single token: latency, forward and backward
        {"name": "attn_short_train", "op": "attention", "lengths": "1,17,64,130,45", "tail": 7, "q_heads": 6, "kv_heads": 2,
         "head_dim": 64, "backward": True, "fused": True},
        # log-probabilities of finished rollouts under the current policy: forward alone
        {"name": "attn_logprob_8k", "op": "attention", "lengths": "1333,512,2048,705,1800,901,256,637", "tail": 0, "q_heads": 12,
         "kv_heads": 2, "head_dim": 128, "backward": False, "fused": True},
        # the same policy's training micro-batch
        {"name": "attn_train_8k", "op": "attention", "lengths": "2011,1024,1777,930,1490,897", "tail": 63, "q_heads": 12,
         "kv_heads": 2, "head_dim": 128, "backward": True, "fused": True},
        # 28 query heads over 4 key heads, rollouts of up to 4096 tokens
        {"name": "attn_train_7b_heads", "op": "attention", "lengths": "4096,2500,3801,1987", "tail": 0, "q_heads": 28, "kv_heads": 4,
         "head_dim": 128, "backward": True, "fused": True},
        # one long chain of thought
        {"name": "attn_train_16k", "op": "attention", "lengths": "16384", "tail": 0, "q_heads": 12, "kv_heads": 2, "head_dim": 128,
         "backward": True, "fused": False},
    ]


def _log(rng, low, high):
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return n + 1 if n == 3072 else n


def _lengths(rng, total, longest):
    """Lengths that add up to about `total`, none above `longest`."""
    got, left = [], total
    while left > 0 and len(got) < 64:
        n = min(left, longest, _log(rng, max(1, total // 64), max(2, longest)))
        got.append(n + 1 if n == 3072 else n)
        left -= n
    return got


def draw(rng):
    kind = rng.choice(["clip", "rotary", "attention", "attention"])
    if kind == "clip":
        decoder = rng.choice(["mini", "small", "0.25b", "1.5b"])
        most = {"mini": 3, "small": 6, "0.25b": 12, "1.5b": 20}[decoder]
        return {"op": "clip", "decoder": decoder, "layers": rng.randint(1, most), "types": rng.choice(["f32", "bf16", "mixed"]),
                "pad": rng.choice([1, 2, 8, 64]), "ratio": round(math.exp(rng.uniform(math.log(0.02), math.log(3.0))), 4)}
    heads = rng.choice([(3, 1, 32), (6, 2, 64), (8, 2, 128), (12, 2, 128), (28, 4, 128), (40, 8, 128), (5, 5, 80), (7, 1, 96)])
    if kind == "rotary":
        tokens = _log(rng, 1, 16384)
        packed = rng.random() < 0.6
        part = rng.choice([1.0, 1.0, 0.5, 0.25])
        return {"op": "rotary", "tokens": tokens, "lengths": ",".join(map(str, _lengths(rng, tokens, 4096))) if packed else "",
                "q_heads": min(heads[0], 28), "kv_heads": heads[1] if heads[0] <= 28 else 4, "head_dim": heads[2],
                "rot_dim": max(8, int(heads[2] * part) // 8 * 8), "layout": rng.choice(["half", "interleaved"]),
                "scaling": rng.choice(["none", "linear", "base", "parts"]), "type": rng.choice(["bf16", "bf16", "f32"]),
                "inverse": rng.random() < 0.5, "fused": rng.random() < 0.5}
    total = _log(rng, 16, 10000)
    lengths = _lengths(rng, total, min(total, 4096))
    if heads[0] == 40:  # within the largest listed case's cost
        lengths = lengths[:3]
    return {"op": "attention", "lengths": ",".join(map(str, lengths)), "tail": rng.choice([0, 0, 1, 37]), "q_heads": heads[0],
            "kv_heads": heads[1], "head_dim": heads[2], "backward": rng.random() < 0.75, "fused": rng.random() < 0.5}


# ------------------------------------------------------------------------------------------------------ inputs


def _list_sizes(case):
    """(number of elements, whether a vector) of every tensor of the list."""
    if case["decoder"] == "flat":
        return [(1 << 20, False)]
    h, _, qh, kvh, hd, inter, vocab, tied = DECODERS[case["decoder"]]
    q, kv = qh * hd, kvh * hd
    layer = [(h, True), (q * h, False), (q, True), (kv * h, False), (kv, True), (kv * h, False), (kv, True), (h * q, False),
             (h, True), (inter * h, False), (inter * h, False), (h * inter, False)]
    return [(vocab * h, False)] + layer * case["layers"] + [(h, True)] + ([] if tied else [(vocab * h, False)])


def _ints(text):
    return [int(x) for x in text.split(",")] if text else []


def _rotary_freqs(case):
    """Radians per position of each pair, stretched for contexts longer than the policy was trained on."""
    r, base, factor, trained = case["rot_dim"], 1e6, 4.0, 4096.0
    if case["scaling"] == "base":
        base *= factor ** (r / (r - 2.0))
    f = base ** (-np.arange(0, r, 2, dtype=np.float64) / r)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "parts":  # short wavelengths stay, those beyond the trained context are divided, a ramp between
        turns = trained * f / (2 * math.pi)
        keep = np.clip((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        f = f * (keep + (1 - keep) / factor)
    return f


def _heads(gen, tokens, counts, head_dim, dtype, fused):
    """Tensors [tokens, heads, head_dim]: separate ones, or views of one fused projection's output."""
    if fused:
        x = torch.randn(tokens, sum(counts), head_dim, generator=gen, device="cuda").to(dtype)
        return list(x.split(counts, dim=1))
    return [torch.randn(tokens, n, head_dim, generator=gen, device="cuda").to(dtype) for n in counts]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    if case["op"] == "clip":
        rng, pad = random.Random(seed * 31 + 7), case["pad"]
        spans, ends, square = [], {torch.float32: 0, torch.bfloat16: 0}, 0.0
        for n, vector in _list_sizes(case):
            dtype = torch.float32 if case["types"] == "f32" or (case["types"] == "mixed" and vector) else torch.bfloat16
            sigma = 10.0 ** rng.uniform(-4.0, -1.0)
            spans.append((dtype, ends[dtype], n, sigma))
            ends[dtype] += -(-n // pad) * pad
            square += sigma * sigma * n
        flats = {d: torch.zeros(n, dtype=d, device="cuda") for d, n in ends.items() if n}
        outs = {d: torch.zeros_like(f) for d, f in flats.items()}
        s["grads"] = [flats[d][o:o + n] for d, o, n, _ in spans]
        s["clipped"] = [outs[d][o:o + n] for d, o, n, _ in spans]
        for g, (_, _, _, sigma) in zip(s["grads"], spans):
            g.normal_(generator=gen).mul_(sigma)
        s["flats"], s["outs"] = list(flats.values()), list(outs.values())
        s["max_norm"] = case["ratio"] * math.sqrt(square)
        s["norm"] = torch.zeros((), device="cuda")
        if own:  # the table of the list's tensors, which a training loop builds once
            from paper_2603_01501_b200 import binding as gb
            s["list"] = gb.gac_clip_init(s["grads"], s["clipped"])
        return s
    if case["op"] == "rotary":
        dtype = torch.bfloat16 if case["type"] == "bf16" else torch.float32
        s["q"], s["k"], _ = _heads(gen, case["tokens"], [case["q_heads"], case["kv_heads"], case["kv_heads"]], case["head_dim"],
                                   dtype, case["fused"])
        s["freqs"] = _rotary_freqs(case)
        s["freqs_dev"] = torch.from_numpy(s["freqs"]).cuda()
        s["scale"] = 1.0 + 0.1 * math.log(4.0) if case["scaling"] == "parts" else 1.0
        s["cu"] = s["positions"] = None
        if case["lengths"]:
            s["cu"] = torch.tensor([0] + list(np.cumsum(_ints(case["lengths"]))), dtype=torch.int32, device="cuda")
        else:
            s["positions"] = torch.randint(0, 32768, (case["tokens"],), generator=gen, device="cuda", dtype=torch.int32)
        return s
    lengths = _ints(case["lengths"])
    tokens = sum(lengths) + case["tail"]
    s["q"], s["k"], s["v"] = _heads(gen, tokens, [case["q_heads"], case["kv_heads"], case["kv_heads"]], case["head_dim"],
                                    torch.bfloat16, case["fused"])
    s["do"] = (torch.randn(s["q"].shape, generator=gen, device="cuda") * 0.02).to(torch.bfloat16)
    s["cu"] = torch.tensor([0] + list(np.cumsum(lengths)), dtype=torch.int32, device="cuda")
    s["longest"] = max(lengths)
    s["scale"] = case["head_dim"] ** -0.5
    return s


# ------------------------------------------------------------------------------------------------------- plain


def _token_places(cu, tokens):
    """Sequence, position in it, and whether there is one, of every token of the pack."""
    t = torch.arange(tokens, device=cu.device, dtype=torch.int32)
    seq = (torch.searchsorted(cu, t, right=True) - 1).clamp(0, cu.numel() - 2)
    return seq, t - cu[seq], t < cu[-1]


def _plain_clip(s):
    norm = sum(f.float().square().sum() for f in s["flats"]).sqrt()
    factor = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
    return {"norm": norm, "clipped": [(f.float() * factor).to(f.dtype) for f in s["flats"]]}


def _plain_rotary(s):
    case, r = s["case"], s["case"]["rot_dim"]
    if s["cu"] is not None:
        _, pos, inside = _token_places(s["cu"], case["tokens"])
        pos = pos * inside  # a token after the last sequence stays where it is
    else:
        pos = s["positions"]
    # whole turns leave the angle before it is rounded to 32 bits: at far positions a 32-bit product has lost them
    turns = pos.double()[:, None] * (s["freqs_dev"] / (2 * math.pi))
    angle = (2 * math.pi * (turns - turns.round())).float()
    cos, sin = (angle.cos() * s["scale"])[:, None], (angle.sin() * s["scale"])[:, None]
    if case["inverse"]:
        sin = -sin

    def turn(x):
        x = x.float()
        a, b = (x[..., :r // 2], x[..., r // 2:r]) if case["layout"] == "half" else (x[..., 0:r:2], x[..., 1:r:2])
        a, b = a * cos - b * sin, a * sin + b * cos
        both = torch.cat((a, b), -1) if case["layout"] == "half" else torch.stack((a, b), -1).flatten(-2)
        return torch.cat((both, x[..., r:]), -1)

    return {"q": turn(s["q"]).to(s["q"].dtype), "k": turn(s["k"]).to(s["k"].dtype)}


def _plain_attention(s):
    """Every sequence padded to the longest; a query sees the keys up to its own position, so padding keys are never seen."""
    q, k, v, cu, scale, longest = s["q"], s["k"], s["v"], s["cu"], s["scale"], s["longest"]
    tokens, heads, dim = q.shape
    kv, n = k.shape[1], cu.numel() - 1
    place = torch.arange(longest, device=q.device)
    index = (cu[:-1, None] + place).clamp(max=tokens - 1)
    seq, pos, inside = _token_places(cu, tokens)
    pos = pos.clamp(max=longest - 1)

    def padded(x):  # [n * kv, heads of the group * longest, dim]
        return x.float()[index].view(n, longest, kv, -1, dim).permute(0, 2, 3, 1, 4).reshape(n * kv, -1, dim)

    def tokens_of(x, h):  # back to [tokens, h, ...]
        x = x.view(n, h, longest, *x.shape[2:])[seq, :, pos]
        return torch.where(inside.view(-1, *[1] * (x.dim() - 1)), x, 0.0)

    qp, kp, vp = padded(q), padded(k), padded(v)
    hidden = place[None, :] > place[:, None]
    p = torch.bmm(qp, kp.transpose(1, 2)).mul_(scale).view(n * kv, -1, longest, longest)
    p.masked_fill_(hidden, -math.inf)
    top = p.amax(-1, keepdim=True)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(total).view(n * kv, -1, longest)
    op = torch.bmm(p, vp)
    lse = (top + total.log()).view(n, heads, longest)[seq, :, pos]
    lse = torch.where(inside[:, None], lse, -math.inf).t().contiguous()
    out = {"o": tokens_of(op.view(n * heads, longest, dim), heads).to(q.dtype), "lse": lse}
    if not s["case"]["backward"]:
        return out
    valid = (place < (cu[1:] - cu[:-1])[:, None])[:, None, None, :, None]
    dop = (padded(s["do"]).view(n, kv, -1, longest, dim) * valid).view(n * kv, -1, dim)
    dv = torch.bmm(p.transpose(1, 2), dop)
    ds = torch.bmm(dop, vp.transpose(1, 2)).sub_((dop * op).sum(-1, keepdim=True)).mul_(p)
    dq = torch.bmm(ds, kp).mul_(scale)
    dk = torch.bmm(ds.transpose(1, 2), qp).mul_(scale)
    out["dq"] = tokens_of(dq.view(n * heads, longest, dim), heads).to(q.dtype)
    out["dk"] = tokens_of(dk.view(n * kv, longest, dim), kv).to(k.dtype)
    out["dv"] = tokens_of(dv.view(n * kv, longest, dim), kv).to(v.dtype)
    return out


def run(s):
    if not own:
        return {"clip": _plain_clip, "rotary": _plain_rotary, "attention": _plain_attention}[s["case"]["op"]](s)
    from paper_2603_01501_b200 import binding as gb
    case = s["case"]
    if case["op"] == "clip":
        gb.gac_clip_grad_norm(s["list"], s["max_norm"], norm_out=s["norm"])
        return {"norm": s["norm"], "clipped": s["outs"]}
    if case["op"] == "rotary":
        q, k = gb.gac_rotary(s["q"], s["k"], s["freqs"], positions=s["positions"], cu_seqlens=s["cu"], layout=case["layout"],
                             scale=s["scale"], inverse=case["inverse"])
        return {"q": q, "k": k}
    o, lse = gb.gac_attn_forward(s["q"], s["k"], s["v"], s["cu"], scale=s["scale"])
    out = {"o": o, "lse": lse}
    if case["backward"]:
        out["dq"], out["dk"], out["dv"] = gb.gac_attn_backward(s["do"], s["q"], s["k"], s["v"], o, lse, s["cu"], scale=s["scale"])
    return out


# -------------------------------------------------------------------------------------------------- accounting


def work(case):
    if case["op"] == "clip":
        size = {"f32": lambda vector: 4, "bf16": lambda vector: 2, "mixed": lambda vector: 4 if vector else 2}[case["types"]]
        sizes = _list_sizes(case)
        return {"bytes": sum(2 * n * size(vector) for n, vector in sizes), "flops": sum(3 * n for n, _ in sizes)}
    if case["op"] == "rotary":
        n = case["tokens"] * (case["q_heads"] + case["kv_heads"])
        size = 2 if case["type"] == "bf16" else 4
        index = 4 * (case["tokens"] if not case["lengths"] else len(_ints(case["lengths"])) + 1)
        return {"bytes": 2 * n * case["head_dim"] * size + index, "flops": 3 * n * case["rot_dim"]}
    lengths = _ints(case["lengths"])
    tokens, pairs = sum(lengths) + case["tail"], sum(n * (n + 1) // 2 for n in lengths)
    row = case["head_dim"] * 2
    q, kv = tokens * case["q_heads"] * row, tokens * case["kv_heads"] * row
    moved = 2 * q + 2 * kv + tokens * case["q_heads"] * 4 + (2 * q + 2 * kv if case["backward"] else 0)
    return {"bytes": moved, "flops": (14 if case["backward"] else 4) * case["head_dim"] * case["q_heads"] * pairs}


# ------------------------------------------------------------------------------------------------------- exact


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "clip":
        total = 0.0
        for g in s["grads"]:
            for part in g.split(1 << 26):
                x = part.double()
                total += float(torch.dot(x, x))
        norm = math.sqrt(total)
        factor = min(1.0, s["max_norm"] / (norm + 1e-6))
        return {"norm": norm, "clipped": [f.double() * factor for f in s["flats"]]}
    if case["op"] == "rotary":
        r = case["rot_dim"]
        if s["cu"] is None:
            where = s["positions"].cpu().numpy().astype(np.float64)
        else:
            where = np.concatenate([np.arange(n, dtype=np.float64) for n in _ints(case["lengths"])])
            where = np.concatenate([where, np.zeros(case["tokens"])])[:case["tokens"]]
        wheel = torch.from_numpy(s["scale"] * np.exp((-1j if case["inverse"] else 1j) * where[:, None] * s["freqs"])).cuda()[:, None]
        result = {}
        for name in ("q", "k"):
            y = s[name].double()
            first, second = (slice(0, r // 2), slice(r // 2, r)) if case["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
            z = torch.complex(y[..., first], y[..., second]) * wheel
            y[..., first], y[..., second] = z.real, z.imag
            result[name] = y
        return result
    tokens, heads, _ = s["q"].shape
    group = heads // case["kv_heads"]
    o, dq = (torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
    dk, dv = (torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
    lse = torch.full((heads, tokens), -math.inf, dtype=torch.float64, device="cuda")
    start = 0
    for n in _ints(case["lengths"]):
        at = slice(start, start + n)
        seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        for h in range(heads):
            q, k, v = (x[at, i].double().requires_grad_(case["backward"]) for x, i in
                       ((s["q"], h), (s["k"], h // group), (s["v"], h // group)))
            scores = torch.where(seen, (q @ k.t()) * s["scale"], -math.inf)
            rows = torch.logsumexp(scores, -1)
            y = torch.exp(scores - rows[:, None]) @ v
            o[at, h], lse[h, at] = y.detach(), rows.detach()
            if case["backward"]:
                a, b, c = torch.autograd.grad(y, (q, k, v), s["do"][at, h].double())
                dq[at, h] = a
                dk[at, h // group] += b
                dv[at, h // group] += c
        start += n
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv} if case["backward"] else {"o": o, "lse": lse}
