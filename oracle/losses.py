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


def _lists(ids, V, values=None):
    """[(place, number)] of a token's entries that are choices (and, with values, not at -inf)."""
    return [(k, int(j)) for k, j in enumerate(ids) if 0 <= j < V and (values is None or values[k] != -np.inf)]


def alternatives(logits, K, mask=None, temperature=1.0):
    """(numbers, log-probabilities) of the K largest logits of every row, the lowest number first among equal ones."""
    x = np.asarray(logits, np.float64)
    ids, logps = np.zeros(x.shape[:-1] + (K,), np.int64), np.zeros(x.shape[:-1] + (K,))
    for at in np.ndindex(*x.shape[:-1]):
        if mask is not None and not mask[at]:
            continue
        row = x[at]
        if np.isnan(row).any() or np.isposinf(row).any():
            ids[at], logps[at] = -1, np.nan
            continue
        best = np.argsort(-row, kind="stable")[:K]
        ids[at], logps[at] = -1, -np.inf
        ids[at][:len(best)] = best
        if row.max() > -np.inf:
            z = (row - row.max()) / temperature
            logps[at][:len(best)] = z[best] - np.log(np.exp(z).sum())
    return ids, logps


def _row_of(row, listed, temperature):
    """(log-probability of every choice, log-probability of those not in `listed`, log-normaliser) of a row."""
    top = row.max()
    if top == -np.inf:
        return np.full(row.shape, -np.inf), -np.inf, -np.inf
    z = (row - top) / temperature
    log_sum = np.log(np.exp(z).sum())
    rest = np.delete(z, sorted(set(listed)))
    near = rest.max() if rest.size else -np.inf
    logrest = near + np.log(np.exp(rest - near).sum()) - log_sum if near > -np.inf else -np.inf
    return z - log_sum, logrest, top / temperature + log_sum


def _shares(row, listed, temperature):
    """Every choice's share of the probability of those not in `listed`, 0 for these: by the others' own largest score (a
    difference of log-probabilities of 1e30 holds nothing of it)."""
    out, others = np.zeros(row.shape), np.ones(row.shape, bool)
    others[sorted(set(listed))] = False
    if others.any() and row[others].max() > -np.inf:
        out[others] = np.exp((row[others] - row[others].max()) / temperature)
        out /= out.sum()
    return out


def listed_logprobs(logits, ids, mask=None, temperature=1.0):
    """(log-probabilities of ids, log-probability of all others, log-normaliser)."""
    x = np.asarray(logits, np.float64)
    logps, rest, lse = np.zeros(ids.shape), np.zeros(x.shape[:-1]), np.zeros(x.shape[:-1])
    for at in np.ndindex(*x.shape[:-1]):
        if mask is not None and not mask[at]:
            continue
        entries = _lists(ids[at], x.shape[-1])
        logp, rest[at], lse[at] = _row_of(x[at], [j for _, j in entries], temperature)
        logps[at] = -np.inf
        for k, j in entries:
            logps[at][k] = logp[j]
    return logps, rest, lse


def listed_gradient(logits, ids, g, h=None, mask=None, temperature=1.0):
    """Gradient of sum(g logps + h rest) with respect to the logits."""
    x = np.asarray(logits, np.float64)
    d = np.zeros(x.shape)
    for at in np.ndindex(*x.shape[:-1]):
        entries = _lists(ids[at], x.shape[-1])
        logp, rest, lse = _row_of(x[at], [j for _, j in entries], temperature)
        if (mask is not None and not mask[at]) or lse == -np.inf:
            continue
        p = np.exp(logp)
        for k, j in entries:
            d[at] -= g[at][k] * p
            d[at][j] += g[at][k]
        if h is not None and rest > -np.inf:
            d[at] += h[at] * (_shares(x[at], [j for _, j in entries], temperature) - p)
    return d / temperature


def distill_loss(logits, ids, teacher, loss="forward", rest=False, teacher_temperature=1.0, scale=1.0,
                 reduction="token_mean", weight=None, mask=None, temperature=1.0, sizes=None):
    """(loss per token, stats[3], gradient).  sizes: a list that receives, for every token, what its rounding errors go
    by: the largest |log(q / p)| that counts, and exp(log(q / p)) of the rest."""
    x = np.asarray(logits, np.float64)
    B, T, V = x.shape
    on = np.ones((B, T), bool) if mask is None else np.asarray(mask) != 0
    n, rows = int(on.sum()), int(on.any(1).sum())
    out, d, total = np.zeros((B, T)), np.zeros(x.shape), 0.0
    for b, t in np.argwhere(on):
        w = {"token_mean": 1 / n, "sequence_mean": 1 / (rows * max(1, on[b].sum())), "sum": 1.0}[reduction]
        w *= 1.0 if weight is None else float(weight[b, t])
        at = (b, t)
        y, first = np.asarray(teacher[at], np.float64), {}
        for k, j in _lists(ids[at], V, y):
            first.setdefault(j, y[k])
        js = np.array(sorted(first), int)
        y = np.array([first[j] for j in js])
        logp, logrest, lse = _row_of(x[at], js, temperature)
        if not rest and not len(js):
            continue
        if lse == -np.inf:
            out[at] = np.inf
            total += w * np.inf if w else 0.0
            continue
        p = np.exp(logp)
        if not rest:
            y = y / teacher_temperature
            y = y - y.max()
            logq = y - np.log(np.exp(y).sum())
            q, q_rest = np.exp(logq), 0.0
            some = False
        else:
            logq, q = y, np.exp(y)
            some = logrest > -np.inf
            q_rest = max(1 - q.sum(), 2.0 ** -23) if some else 0.0
        away = np.log(q_rest) - logrest if some else 0.0
        others = np.ones(V, bool)
        others[js] = False
        g = np.zeros(V)
        if loss == "forward":
            terms = np.where(q > 0, q * (logq - logp[js]), 0.0)
            out[at] = terms.sum() + q_rest * away
            g = p * (q.sum() + q_rest)
            g[js] -= q
            if some:
                g -= _shares(x[at], js, temperature) * q_rest
            used = q > 0
        else:
            used = p[js] > 0
            terms = p[js][used] * (logp[js][used] - logq[used])
            out[at] = terms.sum() - (np.exp(logrest) * away if some else 0.0)
            by = np.zeros(V)  # log(p / q) of every choice, of the rest as one
            by[js[used]] = logp[js][used] - logq[used]
            by[others] = -away
            g = p * (by - out[at])
        if w:
            d[at] = scale * w * g / temperature
            total += w * out[at]
        if sizes is not None:
            u = (logq - logp[js])[used & np.isfinite(logp[js])]
            sizes.append((at, w, p, js, q, max(np.abs(u).max() if u.size else 0.0, abs(away)), np.exp(min(away, 80.0)) if some else 0.0))
    stats = np.array([scale * total, out[on].sum() / n if n else 0.0, n])
    return out, stats, d
