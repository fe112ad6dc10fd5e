"""The float64 form of the divergence from a teacher's top logits for logits of any finite size, and its bounds.

Same definitions and roundings as distill_ref, but logits are taken relative to the largest that counts, so that float64 loses
nothing where masks or common offsets are large, and the rest's shares come from its own largest logit.  The bounds are those
that distill_ref derives: a power of the rest is of (logit - largest) / temperature, whose difference, factor and product are rounded
(3 u |x|), however large the logits are."""
import math

import torch

from distill_ref import U, V, named

MASKED = -1e38      # logits that are not above it have no share


def distill(logits, ids, teacher, kind, temperature, weights=None):
    """dict name -> (value, bound): loss [tokens] and grad [tokens, vocab], float64 on the logits' device."""
    tokens, vocab = logits.shape
    dev = logits.device
    loss, loss_b = (torch.zeros(tokens, dtype=torch.float64, device=dev) for _ in range(2))
    grad, grad_b = (torch.zeros(tokens, vocab, dtype=torch.float64, device=dev) for _ in range(2))
    term = lambda a, b: torch.where(a > 0, a * b, 0.0 * a)  # noqa: E731    0 log 0 = 0
    id_rows, value_rows = ids.tolist(), teacher.double().tolist()
    for t in range(tokens):
        entries = named(id_rows[t], value_rows[t], vocab)
        if not entries:
            continue
        at = torch.tensor([e[1] for e in entries], device=dev)
        x = logits[t].double()
        others = x > MASKED
        others[at] = False
        rest = bool(others.any())
        far = x[others].max() if rest else x.new_tensor(-math.inf)
        base = torch.maximum(x[at].max(), far)
        z = (x[at] - base) / temperature
        below = torch.where(others, (x - far) / temperature, -math.inf)
        total = z.exp().sum()
        if rest:
            rest_log = (far - base) / temperature + torch.logsumexp(below, 0)
            total = total + rest_log.exp()
            lr, share = float(rest_log - total.log()), torch.softmax(below, 0)
            away = torch.where(others, below.abs() / math.log(2), 0.0)
            es = float((torch.where(share > 0, 2.1 * away + 4, 0.0) * share).sum()) * U + (vocab / 512 + 48) * U
        else:
            lr, share, away, es = -math.inf, torch.zeros_like(x), torch.zeros_like(x), 0.0
        lq, lp = z - total.log(), teacher[t].double()[torch.tensor([e[0] for e in entries], device=dev)]
        q, qr, dp = lq.exp(), math.exp(lr), 0.0
        if kind == "top":
            lp = torch.log_softmax(lp / temperature, 0)
            p = lp.exp()
            value, G, g, dG = float(term(p, lp - lq).sum()), qr, q - p, qr * es
            g_b = q * qr * es + 2.0 ** -49 * (q + p)
        else:
            p = lp.exp()
            pr = max(1.0 - float(p.sum()), 2.0 ** -24)
            dp = 2.0 ** -50 * (2 + len(entries)) / pr if rest else 0.0
            if kind == "forward":
                w = float(p.sum()) + (pr if rest else 0.0)
                value = float(term(p, lp - lq).sum()) + (pr * (math.log(pr) - lr) if rest else 0.0)
                G, g, dG = (w * qr - pr if rest else 0.0), q * w - p, w * qr * es + dp * pr
                g_b = q * w * qr * es + q * dp * pr + 2.0 ** -49 * (q * w + p)
                dp *= pr * (1 + abs(math.log(pr) - lr)) if rest else 0.0
            else:
                d, dr = lq - lp, lr - math.log(pr) if rest else 0.0
                value = float(term(q, d).sum()) + (qr * dr if qr > 0 else 0.0)
                G, g = (qr * (dr - value) if qr > 0 else 0.0), term(q, d - value)
                move = 2 * es * (abs(G) + es) + dp * qr
                dG = qr * (es * (abs(dr - value) + 2) + dp + move) if qr > 0 else 0.0
                g_b = term(q, qr * es * ((d - value).abs() + 1) + move) + 2.0 ** -49 * term(q, lq.abs() + lp.abs() + abs(value) + 1)
                dp *= qr
        loss[t], loss_b[t] = value, 2 * es * (abs(G) + es) + dp + 2 * U * abs(value)
        f = (1.0 if weights is None else float(weights[t])) / temperature
        row = share * G * f
        row_b = torch.where(share > 0, share * abs(f) * (abs(G) * ((2.1 * away + 8) * U + es) + dG), 0.0)
        row[at], row_b[at] = g * f, g_b * abs(f)
        grad[t], grad_b[t] = row, row_b + (V if logits.dtype == torch.bfloat16 else 2 * U) * row.abs() + 2.0 ** -120
    return {"loss": (loss, loss_b + 1e-13), "grad": (grad, grad_b)}
