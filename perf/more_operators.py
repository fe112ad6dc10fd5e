"""What newer decoders add to a policy update on packed rollouts, as measured cases.

Three operators that such an update runs in this order: rotary positions with several axes (time, height and width of
images and video), the norm of every query and key head in the same pass as its rotation, with its gradient, and the
divergence between the policy and a teacher (or a reference policy) whose top logits were kept with the rollouts, with
its gradient.  ``run`` computes them in plain torch operations, or, where ``own`` is true, through this package's
entry points.

Head layouts (q heads / kv heads x head size) and vocabularies are those of this repository's synthetic decoders:
3/1 x 32, 6/2 x 64, 8/2 x 128, 12/2 x 128, 28/4 x 128; 1021, 15013, 32000, 151936 and 152064 tokens.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # ---- norms of query and key heads with their rotation
        # one new token for each of 16 rollouts, far into a stretched context: latency
        {"name": "norm_rotary_tokens_16", "op": "norm_rotary", "tokens": 16, "lengths": "", "axes": 1, "order": "chunks", "q_heads": 12,
         "kv_heads": 2, "head_dim": 128, "rot_dim": 128, "layout": "half", "scale": 1.1386, "offset": 0.0, "type": "bf16",
         "weights": "bf16", "train": False, "fused": True},
        # log-probabilities of finished rollouts: forward alone over a large micro-batch
        {"name": "norm_rotary_pack_16k", "op": "norm_rotary", "tokens": 16384, "lengths": "4091,2713,3300,1500,4096,660", "axes": 1,
         "order": "chunks", "q_heads": 28, "kv_heads": 4, "head_dim": 128, "rot_dim": 128, "layout": "half", "scale": 1.0,
         "offset": 0.0, "type": "bf16", "weights": "bf16", "train": False, "fused": True},
        # a training micro-batch, forward and backward with the gradients of both weights; weights kept in float32
        {"name": "norm_rotary_train_12k", "op": "norm_rotary", "tokens": 12291, "lengths": "4096,2500,3703,1987", "axes": 1,
         "order": "chunks", "q_heads": 12, "kv_heads": 2, "head_dim": 128, "rot_dim": 128, "layout": "half", "scale": 1.0,
         "offset": 0.0, "type": "bf16", "weights": "f32", "train": True, "fused": True},
        # float32 training of a small policy: odd counts, a part of the head turned, weights stored as their distance from 1
        {"name": "norm_rotary_train_f32", "op": "norm_rotary", "tokens": 4093, "lengths": "2047,1,1301,740", "axes": 1, "order": "chunks",
         "q_heads": 7, "kv_heads": 1, "head_dim": 96, "rot_dim": 48, "layout": "interleaved", "scale": 1.0, "offset": 1.0, "type": "f32",
         "weights": "f32", "train": True, "fused": False},
        # ---- rotary positions with several axes
        # one new token for each of 8 rollouts about images and video: latency
        {"name": "axes_tokens_8", "op": "axes", "tokens": 8, "axes": 3, "order": "chunks", "q_heads": 8, "kv_heads": 2, "head_dim": 128,
         "rot_dim": 128, "layout": "half", "scale": 1.0, "inverse": False, "type": "bf16", "fused": True},
        # a micro-batch of text and images: time, height and width
        {"name": "axes_images_16k", "op": "axes", "tokens": 16384, "axes": 3, "order": "interleaved", "q_heads": 28, "kv_heads": 4,
         "head_dim": 128, "rot_dim": 128, "layout": "half", "scale": 1.0, "inverse": False, "type": "bf16", "fused": True},
        # the gradient's way back through the height and width of an image's patches, float32
        {"name": "axes_patches_back_f32", "op": "axes", "tokens": 4097, "axes": 2, "order": "own", "q_heads": 6, "kv_heads": 6,
         "head_dim": 64, "rot_dim": 64, "layout": "half", "scale": 1.0, "inverse": True, "type": "f32", "fused": False},
        # ---- divergence from a teacher's top logits
        # a debugging-size policy, eight tokens, with the gradient: latency
        {"name": "distill_tokens_8", "op": "distill", "tokens": 8, "vocab": 1021, "top": 16, "kind": "top", "temperature": 2.0,
         "type": "f32", "teacher": "f32", "prompt": 0.0, "grad": True},
        # how far a policy is from its reference on finished rollouts: values alone
        {"name": "distill_values_2k", "op": "distill", "tokens": 2048, "vocab": 151936, "top": 64, "kind": "reverse", "temperature": 1.0,
         "type": "bf16", "teacher": "f32", "prompt": 0.0, "grad": False},
        # a training micro-batch, values and gradient
        {"name": "distill_train_4k", "op": "distill", "tokens": 4096, "vocab": 151936, "top": 64, "kind": "forward", "temperature": 1.0,
         "type": "bf16", "teacher": "f32", "prompt": 0.0, "grad": True},
        # the same on a smaller vocabulary in float32, a quarter of the tokens a prompt that has no teacher
        {"name": "distill_train_prompts_f32", "op": "distill", "tokens": 8191, "vocab": 32000, "top": 20, "kind": "top", "temperature": 1.5,
         "type": "f32", "teacher": "bf16", "prompt": 0.25, "grad": True},
        # a handful of tokens over the largest vocabulary: few rows, each long
        {"name": "distill_rows_5", "op": "distill", "tokens": 5, "vocab": 152064, "top": 128, "kind": "reverse", "temperature": 1.0,
         "type": "bf16", "teacher": "f32", "prompt": 0.0, "grad": True},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _lengths(rng, total):
    got, left = [], total
    while left > 0 and len(got) < 64:
        n = min(left, _log(rng, max(1, total // 64), min(max(2, total), 4096)))
        got.append(n)
        left -= n
    return got


def draw(rng):
    op = rng.choice(["norm_rotary", "norm_rotary", "axes", "distill", "distill"])
    if op == "distill":
        vocab = rng.choice([1021, 15013, 32000, 151936, 152064, _log(rng, 600, 160000)])
        size = rng.choice(["bf16", "bf16", "f32"])
        tokens = _log(rng, 1, min(8192, (4096 if size == "bf16" else 2048) * 151936 // vocab))
        return {"op": op, "tokens": tokens, "vocab": vocab, "top": rng.choice([1, 5, 16, 20, 64, 100, 128, 333]),
                "kind": rng.choice(["top", "forward", "reverse"]), "temperature": rng.choice([1.0, 1.0, 0.7, 2.0]), "type": size,
                "teacher": rng.choice(["f32", "f32", "bf16"]), "prompt": rng.choice([0.0, 0.0, 0.3]) if tokens >= 64 else 0.0,
                "grad": rng.random() < 0.7}
    q_heads, kv_heads, head_dim = rng.choice([(3, 1, 32), (6, 2, 64), (8, 2, 128), (12, 2, 128), (28, 4, 128), (5, 5, 80), (7, 1, 96),
                                              (4, 1, 256)])
    tokens = _log(rng, 1, 16384)
    case = {"op": op, "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "rot_dim": max(8, int(head_dim * rng.choice([1.0, 1.0, 0.5, 0.25])) // 8 * 8), "layout": rng.choice(["half", "interleaved"]),
            "scale": rng.choice([1.0, 1.0, 1.1386]), "type": rng.choice(["bf16", "bf16", "f32"]), "fused": rng.random() < 0.5}
    if op == "axes":
        case.update(axes=rng.choice([2, 3, 3, 4]), order=rng.choice(["chunks", "interleaved", "own"]), inverse=rng.random() < 0.5)
        return case
    axes = rng.choice([1, 1, 3])
    case.update(lengths=",".join(map(str, _lengths(rng, tokens))) if axes == 1 and rng.random() < 0.6 else "", axes=axes,
                order=rng.choice(["chunks", "interleaved"]), offset=rng.choice([0.0, 0.0, 1.0]),
                weights=rng.choice(["bf16", "f32"]), train=rng.random() < 0.7 and tokens * (q_heads + kv_heads) <= 16384 * 16)
    return case


# ------------------------------------------------------------------------------------------------------ inputs


def _ints(text):
    return [int(x) for x in text.split(",")] if text else []


def _axis_of_pairs(case):
    """Which axis turns each pair of a head: a quarter of the pairs time, the rest shared by the others; in a row one
    axis after the other ("chunks"), or dealt out in turn ("interleaved").  "own": equal shares, one after the other."""
    pairs, n = case["rot_dim"] // 2, case["axes"]
    if case["order"] == "own":
        left = [pairs // n + (i < pairs % n) for i in range(n)]
    else:
        first = max(1, pairs // 4) if n > 2 else (pairs + 1) // 2
        left = [first] + [(pairs - first) // (n - 1) + (i < (pairs - first) % (n - 1)) for i in range(n - 1)] if n > 1 else [pairs]
    if case["order"] != "interleaved":
        return np.repeat(np.arange(n), left).astype(np.uint8)
    got, at = [], 0
    while len(got) < pairs:
        if left[at]:
            left[at] -= 1
            got.append(at)
        at = (at + 1) % n
    return np.array(got, dtype=np.uint8)


def _freqs(case, axis):
    """Radians per position of each pair: one spectrum over all pairs, or ("own") one over the pairs of each axis."""
    r, base = case["rot_dim"], 1e6
    if case.get("order") != "own":
        return base ** (-np.arange(0, r, 2, dtype=np.float64) / r)
    f = np.zeros(r // 2)
    for a in range(case["axes"]):
        n = int((axis == a).sum())
        f[axis == a] = 1e4 ** (-np.arange(n) / max(n, 1))
    return f


def _places(case, rng):
    """Positions [axes, tokens]: text, where all axes agree, and grids of patches, where the last two count rows and columns."""
    n, tokens = case["axes"], case["tokens"]
    out, have, at = [], 0, rng.randrange(0, 20000)
    while have < tokens:
        if rng.random() < 0.5:
            k = rng.randint(1, 400)
            out.append(np.tile(np.arange(at, at + k), (n, 1)))
            at += k
        else:
            h, w = rng.randint(1, 40), rng.randint(1, 40)
            k = h * w
            grid = np.full((n, k), at)
            grid[n - 2] += np.repeat(np.arange(h), w)
            grid[n - 1] += np.tile(np.arange(w), h)
            out.append(grid)
            at += max(h, w)
        have += k
    return np.concatenate(out, 1)[:, :tokens].astype(np.int32)


def _heads(gen, tokens, counts, head_dim, dtype, fused):
    """Tensors [tokens, heads, head_dim]: separate ones, or views of one fused projection's output."""
    if fused:
        x = torch.randn(tokens, sum(counts), head_dim, generator=gen, device="cuda").to(dtype)
        return list(x.split(counts, dim=1))
    return [torch.randn(tokens, n, head_dim, generator=gen, device="cuda").to(dtype) for n in counts]


def _prepare_heads(case, seed, gen):
    s, tokens, dtype = {"case": case}, case["tokens"], DTYPES[case["type"]]
    s["q"], s["k"], _ = _heads(gen, tokens, [case["q_heads"], case["kv_heads"], case["kv_heads"]], case["head_dim"], dtype, case["fused"])
    rng = random.Random(seed * 31 + 7)
    s["cu"] = s["positions"] = s["axis"] = None
    axis = _axis_of_pairs(case)
    if case["axes"] > 1:
        s["axis"] = axis
        s["positions"] = torch.from_numpy(_places(case, rng)).cuda()
    elif case["lengths"]:
        s["cu"] = torch.tensor([0] + list(np.cumsum(_ints(case["lengths"]))), dtype=torch.int32, device="cuda")
    else:
        s["positions"] = torch.randint(0, 32768, (tokens,), generator=gen, device="cuda", dtype=torch.int32)
    s["freqs"] = _freqs(case, axis)
    s["freqs_dev"], s["axis_dev"] = torch.from_numpy(s["freqs"]).cuda(), torch.from_numpy(axis.astype(np.int64)).cuda()
    if case["op"] == "norm_rotary":
        for name in ("q", "k"):
            s[name] *= 0.5 + 2.0 * torch.rand(s[name].shape[1], 1, generator=gen, device="cuda").to(dtype)   # heads of different sizes
            w = 1.0 - case["offset"] + 0.2 * torch.randn(case["head_dim"], generator=gen, device="cuda")
            s["w" + name] = w.to(DTYPES[case["weights"]])
            if case["train"]:
                s["d" + name] = (torch.randn(s[name].shape, generator=gen, device="cuda") * 0.02).to(dtype)
    return s


def _prepare_distill(case, seed, gen):
    """Logits with a few likely tokens per row, as a policy's are, and a teacher that agrees with them in the main.  The
    tokens it names are distinct; a prompt's rows name none (-1)."""
    s, n, v, top = {"case": case}, case["tokens"], case["vocab"], case["top"]
    x = torch.empty(n, v, dtype=DTYPES[case["type"]], device="cuda").normal_(0.0, 1.5, generator=gen)
    first = torch.randint(0, v, (n, 1), generator=gen, device="cuda")
    step = torch.randint(1, max(2, v // top), (n, 1), generator=gen, device="cuda")
    ids = (first + step * torch.arange(top, device="cuda")) % v
    rank = 10.0 - 1.6 * torch.log1p(torch.arange(top, device="cuda", dtype=torch.float32))
    x.scatter_(1, ids, (rank + torch.randn(n, top, generator=gen, device="cuda")).to(x.dtype))
    teacher = rank + 0.7 * torch.randn(n, top, generator=gen, device="cuda")
    if case["kind"] != "top":   # log-probabilities: the tokens that are not named hold 0.1 to 10 % of the teacher's mass
        rest = 10.0 ** (-3.0 + 2.0 * torch.rand(n, 1, generator=gen, device="cuda"))
        teacher = torch.log_softmax(teacher, -1) + torch.log1p(-rest)
    if case["prompt"]:
        place = torch.arange(n, device="cuda") % max(1, n // 8)
        ids[place < case["prompt"] * max(1, n // 8)] = -1
    s["logits"], s["ids"], s["teacher"] = x, ids.to(torch.int32), teacher.to(DTYPES[case["teacher"]])
    if case["grad"]:   # what a token's divergence weighs in the loss
        s["weights"] = (0.5 + torch.rand(n, generator=gen, device="cuda")) / n
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return _prepare_distill(case, seed, gen) if case["op"] == "distill" else _prepare_heads(case, seed, gen)


# ------------------------------------------------------------------------------------------------------- plain


def _wheel(s):
    """Cosine and sine [tokens, 1, pairs] in 32 bits, the scale in them; the angle in 64, whole turns taken out."""
    case = s["case"]
    if s["cu"] is not None:
        t = torch.arange(case["tokens"], device="cuda", dtype=torch.int32)
        seq = (torch.searchsorted(s["cu"], t, right=True) - 1).clamp(0, s["cu"].numel() - 2)
        pos = ((t - s["cu"][seq]) * (t < s["cu"][-1]))[:, None]   # a token after the last sequence stays where it is
    elif s["axis"] is None:
        pos = s["positions"][:, None]
    else:
        pos = s["positions"].t()[:, s["axis_dev"]]
    turns = pos.double() * (s["freqs_dev"] / (2 * math.pi))
    angle = (2 * math.pi * (turns - turns.round())).float()
    return (angle.cos() * case["scale"])[:, None], (angle.sin() * case["scale"])[:, None]


def _turn(case, x, cos, sin):
    r = case["rot_dim"]
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if case["layout"] == "half" else (x[..., 0:r:2], x[..., 1:r:2])
    a, b = a * cos - b * sin, a * sin + b * cos
    both = torch.cat((a, b), -1) if case["layout"] == "half" else torch.stack((a, b), -1).flatten(-2)
    return torch.cat((both, x[..., r:]), -1)


def _plain_axes(s):
    cos, sin = _wheel(s)
    if s["case"]["inverse"]:
        sin = -sin
    return {n: _turn(s["case"], s[n].float(), cos, sin).to(s[n].dtype) for n in ("q", "k")}


EPS = 1e-6


def _plain_norm_rotary(s):
    case, (cos, sin), out = s["case"], _wheel(s), {}
    for n in ("q", "k"):
        x, w = s[n].float(), s["w" + n].float() + case["offset"]
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        unit = x * r
        out[n] = _turn(case, unit * w, cos, sin).to(s[n].dtype)
        if case["train"]:
            back = _turn(case, s["d" + n].float(), cos, -sin)    # the transpose of a turn turns back
            out["dw" + n] = (back * unit).sum((0, 1)).to(s["w" + n].dtype)
            back = back * w
            out["d" + n] = (r * (back - unit * (back * unit).mean(-1, keepdim=True))).to(s[n].dtype)
    return out


def _plain_distill(s):
    case, kind = s["case"], s["case"]["kind"]
    ids, named = s["ids"].long().clamp(min=0), s["ids"] >= 0
    some = named.any(-1, keepdim=True)
    z = s["logits"].float() / case["temperature"]
    top = z.amax(-1, keepdim=True)
    e = (z - top).exp_()
    total = e.sum(-1, keepdim=True)
    log_q = z.gather(1, ids) - top - total.log()
    q = e.gather(1, ids) / total
    if kind == "top":
        log_p = s["teacher"].float() / case["temperature"]
        log_p = log_p.masked_fill(~named, -math.inf)
        log_p = torch.where(some, log_p - torch.logsumexp(log_p, -1, keepdim=True), 0.0).masked_fill(~named, -math.inf)
    else:   # the tokens that are not named, as one; their share of the policy summed over them alone
        log_p = s["teacher"].float().masked_fill(~named, -math.inf)
        rest = (1.0 - log_p.double().exp().sum(-1, keepdim=True)).clamp(min=2.0 ** -24).float()
        other = torch.ones_like(e).scatter_(1, ids, torch.where(named, 0.0, 1.0))
        q_rest = (e * other).sum(-1, keepdim=True) / total
    p = log_p.exp()
    if kind == "reverse":
        away = torch.where(named, log_q - log_p, 0.0)
        away_rest = (q_rest / rest).log()
        loss = (q * away * named).sum(-1, keepdim=True) + q_rest * away_rest
    else:
        loss = torch.where(named, p * (log_p - log_q), 0.0).sum(-1, keepdim=True)
        if kind == "forward":
            loss += rest * (rest / q_rest).log()
    out = {"loss": torch.where(some, loss, 0.0)[:, 0]}
    if not case["grad"]:
        return out
    f = torch.where(some, s["weights"][:, None], 0.0) / case["temperature"]
    if kind == "reverse":
        grad, at = e.mul_((away_rest - loss) * f / total), q * (away - loss) * f
    else:
        mass = p.sum(-1, keepdim=True) + (rest if kind == "forward" else 0.0)
        others = mass - rest / q_rest if kind == "forward" else mass
        grad, at = e.mul_(others * f / total), (q * mass - p) * f
    grad = grad.scatter_(1, ids, torch.where(named, at, 0.0))
    out["grad"] = grad.to(s["logits"].dtype)
    return out


def run(s):
    case = s["case"]
    if not own:
        return {"axes": _plain_axes, "norm_rotary": _plain_norm_rotary, "distill": _plain_distill}[case["op"]](s)
    from paper_2603_01501_b200 import binding as gb
    if case["op"] == "distill":
        how = {"kind": case["kind"], "temperature": case["temperature"]}
        if not case["grad"]:
            return {"loss": gb.gac_distill(s["logits"], s["ids"], s["teacher"], **how)}
        loss, grad = gb.gac_distill(s["logits"], s["ids"], s["teacher"], weights=s["weights"], grad=True, **how)
        return {"loss": loss, "grad": grad}
    how = {"positions": s["positions"], "cu_seqlens": s["cu"], "axes": s["axis"], "layout": case["layout"], "scale": case["scale"]}
    if case["op"] == "axes":
        q, k = gb.gac_rotary(s["q"], s["k"], s["freqs"], inverse=case["inverse"], **how)
        return {"q": q, "k": k}
    how.update(eps=EPS, offset=case["offset"])
    q, k = gb.gac_norm_rotary(s["q"], s["k"], s["wq"], s["wk"], s["freqs"], **how)
    out = {"q": q, "k": k}
    if case["train"]:
        out["dq"], out["dk"], out["dwq"], out["dwk"] = gb.gac_norm_rotary_backward(s["dq"], s["dk"], s["q"], s["k"], s["wq"], s["wk"],
                                                                                   s["freqs"], **how)
    return out


# -------------------------------------------------------------------------------------------------- accounting


def work(case):
    size = 2 if case["type"] == "bf16" else 4
    if case["op"] == "distill":
        rows = case["tokens"]
        if case["prompt"]:   # rows without a teacher need not be read
            span = max(1, rows // 8)
            rows = sum(1 for t in range(rows) if t % span >= case["prompt"] * span)
        table = case["tokens"] * case["top"] * (4 + (2 if case["teacher"] == "bf16" else 4))
        moved = rows * case["vocab"] * size + table + 4 * case["tokens"]
        if case["grad"]:
            moved += case["tokens"] * (case["vocab"] * size + 4)
        return {"bytes": moved, "flops": rows * case["vocab"] * (7 if case["grad"] else 4)}
    heads = case["q_heads"] + case["kv_heads"]
    n = case["tokens"] * heads * case["head_dim"]
    index = 4 * (len(_ints(case["lengths"])) + 1 if case.get("lengths") else case["tokens"] * case["axes"])
    turned = 3 * case["tokens"] * heads * case["rot_dim"]
    if case["op"] == "axes":
        return {"bytes": 2 * n * size + index, "flops": turned}
    weights = 2 * case["head_dim"] * (2 if case["weights"] == "bf16" else 4)
    if not case["train"]:
        return {"bytes": 2 * n * size + index + weights, "flops": 4 * n + turned}
    return {"bytes": 4 * n * size + index + 2 * weights, "flops": 14 * n + 2 * turned}


# ------------------------------------------------------------------------------------------------------- exact


def _exact_turns(s):
    """The complex factor of every token and pair, in 64 bits."""
    case = s["case"]
    if s["axis"] is not None:
        pos = s["positions"].cpu().numpy().astype(np.float64)
        where = np.stack([pos[a] for a in s["axis"]], 1)
    else:
        if s["cu"] is None:
            line = s["positions"].cpu().numpy().astype(np.float64)
        else:
            line = np.concatenate([np.arange(n, dtype=np.float64) for n in _ints(case["lengths"])] + [np.zeros(case["tokens"])])
            line = line[:case["tokens"]]
        where = line[:, None]
    sign = -1j if case.get("inverse") else 1j
    return torch.from_numpy(case["scale"] * np.exp(sign * where * s["freqs"])).cuda()[:, None]


def _exact_turned(case, y, wheel):
    r = case["rot_dim"]
    first, second = (slice(0, r // 2), slice(r // 2, r)) if case["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * wheel
    out = y.clone()
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _exact_distill(s):
    case, kind = s["case"], s["case"]["kind"]
    losses, grads = [], []
    table = [row[row >= 0] for row in s["ids"].cpu().numpy()]
    for t in range(case["tokens"]):
        if len(table[t]) == 0:
            losses.append(torch.zeros((), dtype=torch.float64, device="cuda"))
            grads.append(torch.zeros(case["vocab"], dtype=s["logits"].dtype, device="cuda"))
            continue
        at = torch.from_numpy(table[t].astype(np.int64)).cuda()
        z = (s["logits"][t].double() / case["temperature"]).requires_grad_(case["grad"])
        lq = torch.log_softmax(z, 0)
        if kind == "top":
            lp = torch.log_softmax(s["teacher"][t].double() / case["temperature"], 0)
            loss = (lp.exp() * (lp - lq[at])).sum()
        else:
            lp = s["teacher"][t].double()
            rest = (1.0 - lp.exp().sum()).clamp(min=2.0 ** -24).log().reshape(1)
            lp = torch.cat((lp, rest))
            outside = torch.ones(case["vocab"], dtype=torch.bool, device="cuda")
            outside[at] = False
            lq = torch.cat((lq[at], torch.logsumexp(lq[outside], 0, keepdim=True)))
            loss = (lp.exp() * (lp - lq)).sum() if kind == "forward" else (lq.exp() * (lq - lp)).sum()
        losses.append(loss.detach())
        if case["grad"]:
            g, = torch.autograd.grad(loss, z)
            grads.append(g * (s["weights"][t].double() / case["temperature"]))
    out = {"loss": torch.stack(losses)}
    if case["grad"]:
        out["grad"] = torch.stack([g.double() for g in grads])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "distill":
        return _exact_distill(s)
    wheel = _exact_turns(s)
    if case["op"] == "axes":
        return {n: _exact_turned(case, s[n].double(), wheel) for n in ("q", "k")}
    out = {}
    for n in ("q", "k"):
        x = s[n].double().requires_grad_(case["train"])
        w = s["w" + n].double().requires_grad_(case["train"])
        size = (torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / case["head_dim"] + EPS).sqrt()
        y = _exact_turned(case, x / size * (case["offset"] + w), wheel)
        out[n] = y.detach()
        if case["train"]:
            out["d" + n], out["dw" + n] = torch.autograd.grad(y, (x, w), s["d" + n].double())
    return out
