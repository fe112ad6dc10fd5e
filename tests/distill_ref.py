"""Plain float64 form of the divergence from a teacher's top logits, row by row, and the bounds its kernel is held to.

u = 2^-24, v = 2^-8: half a unit of a binary32 and of a bfloat16 number relative to it.  Named tokens and the row's own
numbers are binary64 in the kernel, so what is off comes from the sum over the rest, in binary32:
  a term     exp2 of x = (logit - largest) c: the difference, c and the product are rounded (3 u |x|, times ln 2), the
             power itself is within 4 u: (2.1 |x| + 4) u of the term
  their sum  of positive terms in a chain of at most vocab / (256 * 4) * 2 + 48 steps: as many u
Together es of the rest's sum, relative.  It moves the loss by es G with G = the sum of the loss's gradient over the rest
(q_r, W q_r - p_r, q_r (d_r - L)), doubled for what is of second order.  1 - sum p is a difference of binary64 numbers: off by dp = 2^-50
(2 + K), which moves log p_r by dp / p_r.
Gradients are off by the same, with q, their own exponentials and the rounding at the end.  A named token's q and p are each
an exponential in binary64 (2^-52 of it) over a sum of such: with the quotient and the products under 8 2^-52, so their difference
is off by 2^-49 (q W + p) on top, which shows where the two agree to the last digit of binary32."""
import math

import torch

U, V = 2.0 ** -24, 2.0 ** -8


def named(ids, values, vocab):
    """(place, id) of the entries of a row that count."""
    seen, got = set(), []
    for i, (t, x) in enumerate(zip(ids, values)):
        if 0 <= t < vocab and x != -math.inf and t not in seen:
            seen.add(t)
            got.append((i, t))
    return got


def distill(logits, ids, teacher, kind, temperature, weights=None):
    """dict name -> (value, bound): loss [tokens] and grad [tokens, vocab], float64 on the logits' device."""
    tokens, vocab = logits.shape
    dev = logits.device
    loss, loss_b = (torch.zeros(tokens, dtype=torch.float64, device=dev) for _ in range(2))
    grad, grad_b = (torch.zeros(tokens, vocab, dtype=torch.float64, device=dev) for _ in range(2))
    id_rows, value_rows = ids.tolist(), teacher.double().tolist()
    for t in range(tokens):
        entries = named(id_rows[t], value_rows[t], vocab)
        if not entries:
            continue
        at = torch.tensor([e[1] for e in entries], device=dev)
        z = logits[t].double() / temperature
        lq = torch.log_softmax(z, 0)
        out = torch.ones(vocab, dtype=torch.bool, device=dev)
        out[at] = False
        others = out & (logits[t].double() > -1e38)
        lp = teacher[t].double()[torch.tensor([e[0] for e in entries], device=dev)]
        q, rest = lq[at].exp(), bool(others.any())
        x = torch.zeros_like(z)
        if rest:
            x = torch.where(others, (z[others].max() - z).abs() / math.log(2), 0.0)
            lr = torch.logsumexp(lq[others], 0)
            share = torch.where(others, (lq - lr).exp(), 0.0)
            es = float(((2.1 * x + 4) * share).sum()) * U + (vocab / 512 + 48) * U
        else:
            lr, share, es = torch.tensor(-math.inf, device=dev, dtype=torch.float64), torch.zeros_like(z), 0.0
        qr = float(lr.exp())
        lq_at = lq[at]
        term = lambda a, b: torch.where(a > 0, a * b, 0.0 * a)  # noqa: E731    0 log 0 = 0
        dp = 0.0
        if kind == "top":
            lp = torch.log_softmax(lp / temperature, 0)
            p = lp.exp()
            value, w, G = float(term(p, lp - lq_at).sum()), 1.0, qr
            g_at, dG = q - p, qr * es
            g_at_b = q * qr * es + 2.0 ** -49 * (q + p)
        else:
            p = lp.exp()
            pr = max(1.0 - float(p.sum()), 2.0 ** -24)
            dp = 2.0 ** -50 * (2 + len(entries)) / pr if rest else 0.0
            if kind == "forward":
                w = float(p.sum()) + (pr if rest else 0.0)
                value = float(term(p, lp - lq_at).sum()) + (pr * (math.log(pr) - float(lr)) if rest else 0.0)
                G = w * qr - pr if rest else 0.0
                g_at, dG = q * w - p, w * qr * es + dp * pr
                g_at_b = q * w * qr * es + q * dp * pr + 2.0 ** -49 * (q * w + p)
                dp *= pr * (1 + abs(math.log(pr) - float(lr))) if rest else 0.0
            else:
                d, dr = lq_at - lp, (float(lr) - math.log(pr)) if rest else 0.0
                value = float(term(q, d).sum()) + (qr * dr if rest else 0.0)
                G = qr * (dr - value) if rest else 0.0
                g_at = term(q, d - value)
                move = 2 * es * (abs(G) + es) + dp * qr
                dG = qr * (es * (abs(dr - value) + 2) + dp + move)
                g_at_b = q * (qr * es * ((d - value).abs().nan_to_num(0.0) + 1) + move)
                g_at_b += 2.0 ** -49 * term(q, lq_at.abs() + lp.abs() + abs(value) + 1)
                dp *= qr
        loss[t] = value
        loss_b[t] = 2 * es * (abs(G) + es) + dp + 2 * U * abs(value)
        f = (1.0 if weights is None else float(weights[t])) / temperature
        row = share * G * f
        # the exponential of a token that is not masked but lies below the others keeps its own error
        row_b = share * abs(f) * (abs(G) * ((2.1 * x + 8) * U + es) + dG)
        row[at], row_b[at] = g_at * f, g_at_b * abs(f)
        grad[t], grad_b[t] = row, row_b + (V if logits.dtype == torch.bfloat16 else 2 * U) * row.abs() + 2.0 ** -120
    return {"loss": (loss, loss_b + 1e-13), "grad": (grad, grad_b)}
