"""Plain 64-bit CPU forms of the token log-probabilities and losses, element by
element from their definitions (numpy).  Test infrastructure, like the rest of
this package; shares no code with the HIP path."""
import numpy as np


def token_logprobs(logits, tokens, mask=None, temperature=1.0):
    """(logp, lse, entropy) of [..., V] logits; 0 where the mask is off."""
    z = np.asarray(logits, np.float64) / temperature
    logp, lse, ent = (np.zeros(z.shape[:-1]) for _ in range(3))
    for at in np.ndindex(*z.shape[:-1]):
        if mask is not None and not mask[at]:
            continue
        row = z[at]
        top = row.max()
        if top == -np.inf:
            logp[at] = lse[at] = -np.inf
            continue
        # the maximum goes first: at 1e38 even 64 bits hold nothing beside it
        log_sum = np.log(np.exp(row - top).sum())
        lse[at] = top + log_sum
        logp[at] = (row[tokens[at]] - top) - log_sum
        live = row > -np.inf
        logq = (row[live] - top) - log_sum
        ent[at] = -(np.exp(logq) * logq).sum()
    return logp, lse, ent


def logits_gradient(logits, tokens, g, h=None, mask=None, temperature=1.0):
    """Gradient of sum(g logp + h entropy) with respect to the logits."""
    z = np.asarray(logits, np.float64) / temperature
    _, lse, ent = token_logprobs(logits, tokens, mask, temperature)
    d = np.zeros(z.shape)
    for at in np.ndindex(*z.shape[:-1]):
        if (mask is not None and not mask[at]) or lse[at] == -np.inf:
            continue
        logq = z[at] - lse[at]
        p = np.exp(logq)
        d[at] = -g[at] * p
        d[at][tokens[at]] += g[at]
        if h is not None:
            live = p > 0
            d[at][live] -= h[at] * p[live] * (logq[live] + ent[at])
    return d / temperature


def policy_loss(logp, adv, old=None, ref=None, entropy=None, mask=None, clip_low=0.2, clip_high=0.2, dual_clip=0.0,
                kl_coef=0.0, entropy_coef=0.0, scale=1.0, reduction="token_mean", valid=None):
    """(stats[8], dlogp, dentropy); `valid` off: in the counts, in no sum."""
    B, T = logp.shape
    on = np.ones((B, T), bool) if mask is None else np.asarray(mask) != 0
    n = int(on.sum())
    rows = int(on.any(1).sum())
    stats, g, h = np.zeros(8), np.zeros((B, T)), np.zeros((B, T))
    stats[7] = n
    if n == 0:
        return stats, g, h
    held_n = log_sum = ratio_sum = 0.0
    for b, t in np.argwhere(on):
        w = {"token_mean": 1 / n, "sequence_mean": 1 / (rows * max(1, on[b].sum())), "sum": 1.0}[reduction]
        if valid is not None and not valid[b, t]:
            continue
        lp, a = float(logp[b, t]), float(adv[b, t])
        lr = lp - float(old[b, t]) if old is not None else 0.0
        r = np.exp(lr)
        plain = -a * r if a else 0.0
        bound = -a * min(max(r, 1 - clip_low), 1 + clip_high)
        term, held = (bound, True) if bound > plain else (plain, False)
        if dual_clip and a < 0 and term > -a * dual_clip:
            term, held = -a * dual_clip, True
        slope = 0.0 if held else plain
        kl = 0.0
        if ref is not None:
            x = float(ref[b, t]) - lp
            kl = np.expm1(x) - x if x < np.inf else x
            slope -= kl_coef * np.expm1(x) if kl_coef else 0.0  # (no term: not 0 times infinity)
        e = float(entropy[b, t]) if entropy is not None else 0.0
        stats[1] += w * term
        stats[2] += w * kl
        stats[3] += w * e
        held_n += held
        log_sum += lr
        ratio_sum += r
        g[b, t] = scale * w * slope
        h[b, t] = -scale * w * entropy_coef
    terms = [c * v for c, v in ((1.0, stats[1]), (kl_coef, stats[2]), (-entropy_coef, stats[3])) if c]
    stats[0] = scale * sum(terms)
    stats[4], stats[5], stats[6] = held_n / n, -log_sum / n, ratio_sum / n
    return stats, g, h


def preference_loss(logp, ref=None, mask=None, beta=0.1, loss="sigmoid", label_smoothing=0.0, length_norm=False,
                    scale=1.0):
    """(loss[P], chosen[P], rejected[P], stats[4], dlogp)."""
    P = logp.shape[0] // 2
    on = np.ones(logp.shape, bool) if mask is None else np.asarray(mask) != 0
    d, n = np.zeros(2 * P), np.ones(2 * P)
    for b in range(2 * P):
        x = np.asarray(logp[b], np.float64)[on[b]]
        if ref is not None:
            x = x - np.asarray(ref[b], np.float64)[on[b]]
        d[b] = x.sum()
        if length_norm:
            n[b] = max(1, on[b].sum())
            d[b] /= n[b]
    out, q = np.zeros(P), np.zeros(P)
    u = beta * (d[:P] - d[P:])
    for i in range(P):
        if loss == "sigmoid":
            e = label_smoothing
            out[i] = (1 - e) * np.logaddexp(0, -u[i]) + (e * np.logaddexp(0, u[i]) if e else 0.0)
            q[i] = beta * (e / (1 + np.exp(-u[i])) - (1 - e) / (1 + np.exp(u[i])))
        else:
            out[i] = (u[i] / beta - 0.5 / beta) ** 2
            q[i] = 2 * (u[i] / beta - 0.5 / beta)
    g = np.zeros(logp.shape)
    for b in range(2 * P):
        g[b][on[b]] = scale * (q[b] if b < P else -q[b - P]) / P / n[b]
    return out, beta * d[:P], beta * d[P:], np.array([scale * out.mean(), (u > 0).mean(), u.mean(), on.sum()]), g
