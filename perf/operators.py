"""The language-model operators whose speed this framework is judged by, as a training program calls them.

A learner that was handed a batch of token sequences (tokens, mask, behaviour log-probabilities, advantages) scores
it and takes the loss with its gradient.  Every per-token array is [B, T]; a mask of uint8 says which tokens count.

  logprobs    log-probabilities of the taken tokens, log-normalisers and entropies from logits [B, T, V]
              (`conduit_token_logprobs`)
  backward    the gradient of those logits (`conduit_token_logprobs_backward`)
  policy      the clipped policy loss with a KL term and an entropy bonus, and its gradient, from log-probabilities
              (`conduit_policy_loss`)
  fused       the same from logits, to the logits' gradient, in one call (`conduit_policy_loss_logits`)
  preference  the preference loss over pairs of sequences, and its gradient (`conduit_preference_loss`)
  head        log-probabilities from the last hidden states and the output projection, no logits kept
              (`conduit_head_logprobs`)
  headgrad    the gradients of those hidden states and of the projection (`conduit_head_logprobs_backward`)

With `own` false a pass is computed with elementary torch operations in 32 bits and rounded once at the end.
Inputs are seeded and synthetic; `exact` works the outputs out in 64 bits.
"""
import math

import torch

own = False

VOCAB = 128000
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # one PPO minibatch of a discrete-action agent: 16,384 samples, 18 actions, an entropy bonus, some actions
        # not allowed (their logits are -inf)
        _fused("ppo-actions", B=1, T=16384, V=18, dtype="f32", mask=False, forbid=True, kl=0.0, ent=0.01),
        # one microbatch of a language model's policy update: 8 sequences of up to 1,024 tokens, bf16 logits
        _fused("tokens-update", B=8, T=1024, V=VOCAB, dtype="bf16", kl=0.05, ent=0.0),
        # a small vocabulary of odd size in fp32, logits and tokens taken one position apart out of the full sequences
        _logprobs("score-shifted", B=16, T=511, V=32001, dtype="f32", shifted=True),
        # one new token for each of 64 sequences while they are generated
        _logprobs("score-step", B=64, T=1, V=VOCAB, dtype="bf16", mask=False),
        # the gradient that goes back into a model that returned fp32 logits, entropies among the loss's terms
        _backward("logits-gradient", B=4, T=512, V=50001, dtype="f32", ent=True),
        # the smallest policy loss: a few short answers
        _policy("policy-short", B=8, T=333, kl=0.05, ent=0.0, reduction="token_mean"),
        # the delivered token batch: 256 sequences of up to 4,096 tokens, each sequence of the same weight
        _policy("policy-batch", B=256, T=4096, kl=0.05, ent=0.01, reduction="sequence_mean"),
        # 128 pairs of answers
        _preference("preference-pairs", P=128, T=2048, loss="sigmoid", smoothing=0.1, length_norm=False),
        # two pairs of very long ones
        _preference("preference-long", P=2, T=65537, loss="squared", smoothing=0.0, length_norm=True),
        # behaviour or reference log-probabilities of a batch of rollouts
        _head("head-score", B=8, T=1024, H=4096, V=VOCAB),
        # one new token for each of 16 sequences
        _head("head-step", B=16, T=1, H=2048, V=VOCAB, mask=False),
        # the training step's gradients through the projection
        _headgrad("head-gradient", B=4, T=1024, H=2048, V=VOCAB),
    ]


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    kind = rng.choice(["fused", "fused", "logprobs", "backward", "policy", "preference", "head", "headgrad"])
    dtype = rng.choice(["f32", "bf16"])
    shifted = rng.random() < 0.3
    mask = rng.random() < 0.75
    if kind in ("fused", "logprobs", "backward"):
        # actions of an agent, bytes, or tokens of a vocabulary
        V = rng.choice([_log(rng, 2, 1024), _log(rng, 1000, 200_000), _log(rng, 20_000, 160_000)])
        rows = _log(rng, 1, max(2, min(262_144, 500_000_000 // V)))
        B, T = _split(rng, rows)
        if kind == "fused":
            return _fused(None, B=B, T=T, V=V, dtype=dtype, mask=mask, shifted=shifted, forbid=rng.random() < 0.3,
                          kl=rng.choice([0.0, 0.05]), ent=rng.choice([0.0, 0.01]),
                          reduction=rng.choice(["token_mean", "sequence_mean"]))
        if kind == "logprobs":
            return _logprobs(None, B=B, T=T, V=V, dtype=dtype, mask=mask, shifted=shifted)
        return _backward(None, B=B, T=T, V=V, dtype=dtype, mask=mask, shifted=shifted, ent=rng.random() < 0.5)
    if kind == "policy":
        B, T = _split(rng, _log(rng, 64, 1_000_000))
        return _policy(None, B=B, T=T, mask=mask, shifted=shifted, kl=rng.choice([0.0, 0.05]),
                       ent=rng.choice([0.0, 0.01]), reduction=rng.choice(["token_mean", "sequence_mean"]))
    if kind == "preference":
        P, T = _split(rng, _log(rng, 64, 400_000))
        return _preference(None, P=P, T=T, mask=mask, shifted=shifted, loss=rng.choice(["sigmoid", "squared"]),
                           smoothing=rng.choice([0.0, 0.1]), length_norm=rng.random() < 0.5)
    H = rng.choice([64 * _log(rng, 2, 64), 64 * _log(rng, 2, 64), _log(rng, 64, 2500)])
    V = _log(rng, 1000, 130_000)
    flops = 8e12 if kind == "head" else 2e12
    rows = _log(rng, 1, max(2, min(8192, int(flops / (2 * H * V)))))
    B, T = _split(rng, rows)
    return (_head if kind == "head" else _headgrad)(None, B=B, T=T, H=H, V=V, mask=mask, shifted=shifted)


def _log(rng, lo, hi):
    """A whole number in [lo, hi], uniform in its logarithm."""
    return max(lo, min(hi, int(round(lo * (max(lo, hi) / lo) ** rng.random()))))


def _split(rng, n):
    """About n tokens as B sequences of T."""
    B = _log(rng, 1, max(1, min(n, 512)))
    return B, max(1, n // B)


def _case(kind, name, **c):
    c["kind"] = kind
    if name is not None:
        c["name"] = name
    return c


def _fused(name, B, T, V, dtype, kl, ent, mask=True, shifted=False, forbid=False, reduction="token_mean"):
    return _case("fused", name, B=B, T=T, V=V, dtype=dtype, mask=mask, shifted=shifted, forbid=forbid, kl=kl, ent=ent,
                 reduction=reduction)


def _logprobs(name, B, T, V, dtype, mask=True, shifted=False):
    return _case("logprobs", name, B=B, T=T, V=V, dtype=dtype, mask=mask, shifted=shifted, forbid=False)


def _backward(name, B, T, V, dtype, ent, mask=True, shifted=False):
    return _case("backward", name, B=B, T=T, V=V, dtype=dtype, mask=mask, shifted=shifted, forbid=False, ent=ent)


def _policy(name, B, T, kl, ent, reduction, mask=True, shifted=False):
    return _case("policy", name, B=B, T=T, mask=mask, shifted=shifted, kl=kl, ent=ent, reduction=reduction)


def _preference(name, P, T, loss, smoothing, length_norm, mask=True, shifted=False):
    return _case("preference", name, P=P, T=T, mask=mask, shifted=shifted, loss=loss, smoothing=smoothing,
                 length_norm=length_norm)


def _head(name, B, T, H, V, mask=True, shifted=False):
    return _case("head", name, B=B, T=T, H=H, V=V, mask=mask, shifted=shifted)


def _headgrad(name, B, T, H, V, mask=True, shifted=False):
    return _case("headgrad", name, B=B, T=T, H=H, V=V, mask=mask, shifted=shifted)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
TAU = 0.9  # sampling temperature
CLIP_LOW, CLIP_HIGH, DUAL = 0.2, 0.28, 3.0
BETA = 0.1


def _spans(B, T, mask):
    """(first, last + 1) counted token of each row: lengths spread evenly over [T / 8, T], a prompt of a quarter of
    the length, and from 8 rows on one row with nothing in it.  No mask: every token counts."""
    if not mask:
        return [(0, T)] * B
    spans = []
    for b in range(B):
        n = T if B == 1 else max(1, T // 8 + (T - T // 8) * b // (B - 1))
        spans.append((n // 4, n))
    if B >= 8:
        spans[B // 2] = (0, 0)
    return spans


def _count(B, T, mask):
    return sum(b - a for a, b in _spans(B, T, mask))


class _Inputs:
    """Seeded device inputs of a [B, T] token batch; `shifted` ones are views, one position in, of arrays with T + 1
    columns (the predictions of position t and the tokens of position t + 1)."""

    def __init__(self, c, seed, rows=None):
        self.c, self.B, self.T = c, (rows or c["B"]), c["T"]
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda")

    def rand(self, *shape):
        return torch.rand(shape, generator=self.g, device="cuda")

    def empty(self, dtype=torch.float32):
        """An uninitialised per-token array in the case's layout."""
        if self.c["shifted"]:
            return torch.empty((self.B, self.T + 1), dtype=dtype, device="cuda")[:, 1:]
        return torch.empty((self.B, self.T), dtype=dtype, device="cuda")

    def token(self, x):
        out = self.empty(x.dtype)
        out.copy_(x)
        return out

    def wide(self, width, dtype, zero=False):
        """An array of one row of `width` elements a token, in the case's layout."""
        make = torch.zeros if zero else torch.empty
        if self.c["shifted"]:
            return make((self.B, self.T + 1, width), dtype=dtype, device="cuda")[:, :-1]
        return make((self.B, self.T, width), dtype=dtype, device="cuda")

    def mask(self):
        if not self.c["mask"]:
            return None
        spans = torch.tensor(_spans(self.B, self.T, True), device="cuda")
        spans = spans[torch.randperm(self.B, generator=self.g, device="cuda")]
        t = torch.arange(self.T, device="cuda")
        return self.token(((t >= spans[:, :1]) & (t < spans[:, 1:])).to(torch.uint8))

    def tokens(self, V):
        return torch.randint(0, V, (self.B, self.T), generator=self.g, device="cuda", dtype=torch.int32)

    def logits(self, tokens):
        """A row's logits spread like a trained model's: unit noise of scale 2, the taken token ahead by up to 12."""
        c = self.c
        x = self.wide(c["V"], TYPES[c["dtype"]])
        lead = 12 * self.rand(self.B, self.T)
        for b in range(self.B):
            for a in range(0, self.T, 4096):
                z = min(self.T, a + 4096)
                rows = 2 * self.randn(z - a, c["V"])
                rows.scatter_add_(1, tokens[b, a:z, None].long(), lead[b, a:z, None])
                if c["forbid"]:  # a fifth of the choices are not allowed, never the taken one
                    taken = rows.gather(1, tokens[b, a:z, None].long())
                    rows.masked_fill_(self.rand(z - a, c["V"]) < 0.2, -math.inf)
                    rows.scatter_(1, tokens[b, a:z, None].long(), taken)
                x[b, a:z] = rows.to(x.dtype)
        return x

    def old(self, logp):
        """Log-probabilities of the policy that acted, a few updates ago.  No ratio lies within half a percent of a
        kink of the clipped loss, where the gradient jumps."""
        d = 0.2 * self.randn(self.B, self.T)
        d = torch.where(self.rand(self.B, self.T) < 0.01, d + 1.5, d)
        for kink in (math.log(1 - CLIP_LOW), math.log(1 + CLIP_HIGH), math.log(DUAL)):
            d = torch.where((d - kink).abs() < 0.005, d + 0.01, d)
        return logp - d


def prepare(case, seed):
    c = case
    k = c["kind"]
    s = {"case": c}
    if k == "preference":
        x = _Inputs(c, seed, rows=2 * c["P"])
        logp = -torch.empty((x.B, x.T), device="cuda").exponential_(1.0, generator=x.g)
        s["logp"], s["mask"] = x.token(logp), x.mask()
        s["ref"] = x.token(logp + 0.05 * x.randn(x.B, x.T))
        s["dlogp"] = x.empty()
        for name in ("loss", "chosen", "rejected"):
            s[name] = torch.empty(c["P"], device="cuda")
        s["stats"] = torch.empty(4, device="cuda")
    elif k == "policy":
        x = _Inputs(c, seed)
        logp = -torch.empty((x.B, x.T), device="cuda").exponential_(1.0, generator=x.g)
        s["logp"], s["mask"], s["adv"] = x.token(logp), x.mask(), x.token(x.randn(x.B, x.T))
        s["old"], s["ref"] = x.token(x.old(logp)), x.token(logp + 0.1 * x.randn(x.B, x.T))
        s["entropy"] = x.token(3 * x.rand(x.B, x.T))
        s["dlogp"], s["dentropy"] = x.empty(), x.empty()
        s["stats"] = torch.empty(8, device="cuda")
    else:
        x = _Inputs(c, seed)
        s["mask"] = x.mask()
        tokens = x.tokens(c["V"])
        s["tokens"] = x.token(tokens)
        if k in ("head", "headgrad"):
            s["hidden"] = x.wide(c["H"], torch.bfloat16)
            s["hidden"].copy_(x.randn(x.B, x.T, c["H"]))
            s["weight"] = (x.randn(c["V"], c["H"]) * (2 / math.sqrt(c["H"]))).to(torch.bfloat16)
        else:
            s["logits"] = x.logits(tokens)
        if k in ("fused", "backward", "headgrad"):
            logp, lse, entropy = _forward(s, chunk=512)
        if k == "fused":
            s["adv"], s["old"] = x.token(x.randn(x.B, x.T)), x.token(x.old(logp))
            s["ref"] = x.token(logp + 0.1 * x.randn(x.B, x.T))
            s["stats"] = torch.empty(8, device="cuda")
        if k in ("backward", "headgrad"):
            s["lse"], s["entropy"] = x.token(lse), x.token(entropy)
            s["dlogp"] = x.token(x.randn(x.B, x.T) / max(1, _count(c["B"], c["T"], c["mask"])))
            s["dentropy"] = x.token(0.1 * x.randn(x.B, x.T) / max(1, _count(c["B"], c["T"], c["mask"]))) \
                if c.get("ent") else None
        if k in ("fused", "backward"):  # what a pass does not write (the last position of a shifted one) stays 0
            s["dlogits"] = x.wide(c["V"], TYPES[c["dtype"]], zero=True)
        if k == "headgrad":
            s["dhidden"] = x.wide(c["H"], torch.bfloat16, zero=True)
            s["dweight"] = torch.empty_like(s["weight"])
        else:
            s["out"] = [x.empty() for _ in range(3)]
    if own:
        from paper_2609_24456_amd import conduit as cd
        n = 0
        if k in ("fused", "policy"):
            s["opts"] = cd.policy_opts(clip_low=CLIP_LOW, clip_high=CLIP_HIGH, dual_clip=DUAL, kl_coef=c["kl"],
                                       entropy_coef=c["ent"], reduction=c["reduction"])
            n = cd.policy_loss_logits_workspace(s["logits"]) if k == "fused" else cd.policy_loss_workspace(c["B"], c["T"])
        elif k == "logprobs":
            n = cd.token_logprobs_workspace(s["logits"])
        elif k == "preference":
            s["opts"] = cd.preference_opts(beta=BETA, loss=c["loss"], label_smoothing=c["smoothing"],
                                           length_norm=c["length_norm"])
            n = cd.preference_loss_workspace(c["P"], c["T"])
        elif k == "head":
            n = cd.head_logprobs_workspace(s["hidden"], s["weight"])
        elif k == "headgrad":
            n = cd.head_logprobs_backward_workspace(s["hidden"], s["weight"])
        s["workspace"] = cd.workspace(n)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2609_24456_amd import conduit as cd
    c = s["case"]
    k = c["kind"]
    ws = s["workspace"]
    if k == "logprobs":
        logp, lse, entropy = s["out"]
        cd.conduit_token_logprobs(s["logits"], s["tokens"], logp, lse=lse, entropy=entropy, mask=s["mask"],
                                  temperature=TAU, workspace=ws)
        return {"logp": logp, "lse": lse, "entropy": entropy}
    if k == "backward":
        cd.conduit_token_logprobs_backward(s["logits"], s["tokens"], s["lse"], s["dlogp"], s["dlogits"],
                                           entropy=s["entropy"] if c["ent"] else None, dentropy=s["dentropy"],
                                           mask=s["mask"], temperature=TAU)
        return {"dlogits": s["dlogits"]}
    if k == "policy":
        cd.conduit_policy_loss(s["opts"], s["logp"], s["adv"], s["stats"], s["dlogp"], old_logp=s["old"],
                               ref_logp=s["ref"], entropy=s["entropy"], dentropy=s["dentropy"], mask=s["mask"],
                               workspace=ws)
        return {"stats": s["stats"], "dlogp": s["dlogp"], "dentropy": s["dentropy"]}
    if k == "fused":
        logp, _, entropy = s["out"]
        cd.conduit_policy_loss_logits(s["opts"], s["logits"], s["tokens"], s["adv"], s["stats"], s["dlogits"],
                                      old_logp=s["old"], ref_logp=s["ref"], logp=logp, entropy=entropy, mask=s["mask"],
                                      temperature=TAU, workspace=ws)
        return {"stats": s["stats"], "logp": logp, "entropy": entropy, "dlogits": s["dlogits"]}
    if k == "preference":
        cd.conduit_preference_loss(s["opts"], s["logp"], s["loss"], s["stats"], s["dlogp"], ref_logp=s["ref"],
                                   mask=s["mask"], chosen=s["chosen"], rejected=s["rejected"], workspace=ws)
        return {x: s[x] for x in ("loss", "chosen", "rejected", "stats", "dlogp")}
    if k == "head":
        logp, lse, entropy = s["out"]
        cd.conduit_head_logprobs(s["hidden"], s["weight"], s["tokens"], logp, lse=lse, entropy=entropy, mask=s["mask"],
                                 temperature=TAU, workspace=ws)
        return {"logp": logp, "lse": lse, "entropy": entropy}
    cd.conduit_head_logprobs_backward(s["hidden"], s["weight"], s["tokens"], s["lse"], s["dlogp"], s["dhidden"],
                                      s["dweight"], mask=s["mask"], temperature=TAU, workspace=ws)
    return {"dhidden": s["dhidden"], "dweight": s["dweight"]}


def _on(s):
    """The mask as truth values."""
    if s["mask"] is not None:
        return s["mask"] != 0
    return torch.ones(s["tokens" if "tokens" in s else "logp"].shape, dtype=torch.bool, device="cuda")


def _scores(s, b=slice(None), t=slice(None)):
    """Tempered logits of some positions in 32 bits."""
    if "logits" in s:
        return s["logits"][b, t].float() / TAU
    h = s["hidden"][b, t].float()
    return (h.reshape(-1, h.shape[-1]) @ s["weight"].float().t()).reshape(*h.shape[:-1], -1) / TAU


def _statistics(z, tokens):
    """(log-probability of the token, log-normaliser, entropy) of scores z."""
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(-1, keepdim=True)
    lse = (top + torch.log(total))[..., 0]
    mean = torch.where(e > 0, e * z, 0.0).sum(-1) / total[..., 0]  # nothing of a choice whose score is -inf
    taken = z.gather(-1, tokens.long()[..., None])[..., 0]
    return taken - lse, lse, lse - mean


def _forward(s, chunk=None):
    """The statistics of every position, 0 where the mask is off."""
    T = s["tokens"].shape[1]
    step = chunk or T
    parts = [_statistics(_scores(s, b, slice(a, a + step)), s["tokens"][b, a:a + step])
             for b in ([slice(None)] if chunk is None else [slice(i, i + 1) for i in range(s["tokens"].shape[0])])
             for a in range(0, T, step)]
    if chunk is None:
        out = parts[0]
    else:
        per = -(-T // step)
        out = [torch.cat([torch.cat([p[i] for p in parts[r:r + per]], 1) for r in range(0, len(parts), per)])
               for i in range(3)]
    on = _on(s)
    return [torch.where(on, x, 0.0) for x in out]


def _score_gradient(z, tokens, lse, entropy, g, h):
    """The gradient of the untempered logits for gradients g of the log-probability and h of the entropy."""
    logq = z - lse[..., None]
    p = torch.exp(logq)
    d = -g[..., None] * p
    if h is not None:
        d = d - torch.where(p > 0, h[..., None] * p * (logq + entropy[..., None]), 0.0)
    # at the taken token g (1 - p), without the cancellation of a probability near 1
    at = tokens.long()[..., None]
    lead = -g[..., None] * torch.expm1(logq.gather(-1, at)) + g[..., None] * p.gather(-1, at)
    return d.scatter_add(-1, at, lead) / TAU


def _policy_terms(c, on, logp, old, ref, adv, entropy):
    """(stats, gradient of logp, gradient of the entropy) of the policy loss."""
    on_f = on.float()
    tokens = on_f.sum()
    per_row = on_f.sum(1, keepdim=True)
    if c["reduction"] == "token_mean":
        w = on_f / tokens.clamp(min=1)
    else:
        w = on_f / (per_row.clamp(min=1) * (per_row > 0).sum().clamp(min=1))
    zero = torch.zeros_like(logp)
    lr, lk = torch.where(on, logp - old, zero), torch.where(on, ref - logp, zero)
    adv, entropy = torch.where(on, adv, zero), torch.where(on, entropy, zero)
    ratio = torch.exp(lr)
    plain, bound = -adv * ratio, -adv * ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH)
    clipped = bound > plain
    term = torch.maximum(plain, bound)
    dual = (adv < 0) & (term > -adv * DUAL)
    term = torch.where(dual, -adv * DUAL, term)
    kl = torch.expm1(lk) - lk
    # the mean KL term is a statistic whether it is part of the loss or not
    s_pol, s_kl, s_ent = (w * term).sum(), (w * kl).sum(), (w * entropy).sum()
    n = tokens.clamp(min=1)
    stats = torch.stack([s_pol + c["kl"] * s_kl - c["ent"] * s_ent, s_pol, s_kl, s_ent,
                         (on & (clipped | dual)).sum() / n, torch.where(on, -lr, zero).sum() / n,
                         torch.where(on, ratio, zero).sum() / n, tokens])
    g = w * (torch.where(clipped | dual, zero, plain) - c["kl"] * torch.expm1(lk))
    return stats, g, -c["ent"] * w


def _run_plain(s):
    c = s["case"]
    k = c["kind"]
    on = _on(s)
    if k in ("logprobs", "head"):
        logp, lse, entropy = _forward(s)
        return {"logp": logp, "lse": lse, "entropy": entropy}
    if k == "backward":
        d = _score_gradient(_scores(s), s["tokens"], s["lse"], s["entropy"], s["dlogp"], s["dentropy"])
        return {"dlogits": torch.where(on[..., None], d, 0.0).to(s["logits"].dtype)}
    if k == "policy":
        stats, g, h = _policy_terms(c, on, s["logp"], s["old"], s["ref"], s["adv"], s["entropy"])
        return {"stats": stats, "dlogp": g, "dentropy": h}
    if k == "fused":
        z = _scores(s)
        logp, lse, entropy = [torch.where(on, x, 0.0) for x in _statistics(z, s["tokens"])]
        stats, g, h = _policy_terms(c, on, logp, s["old"], s["ref"], s["adv"], entropy)
        d = _score_gradient(z, s["tokens"], lse, entropy, g, h if c["ent"] else None)
        return {"stats": stats, "logp": logp, "entropy": entropy,
                "dlogits": torch.where(on[..., None], d, 0.0).to(s["logits"].dtype)}
    if k == "preference":
        P = c["P"]
        n = on.sum(1).clamp(min=1).float() if c["length_norm"] else torch.ones(2 * P, device="cuda")
        d = torch.where(on, s["logp"] - s["ref"], 0.0).sum(1) / n
        margin = d[:P] - d[P:]
        u = BETA * margin
        if c["loss"] == "sigmoid":
            e = c["smoothing"]
            soft = lambda x: torch.clamp(-x, min=0) + torch.log1p(torch.exp(-x.abs()))  # noqa: E731  -log sigmoid
            loss = (1 - e) * soft(u) + e * soft(-u)
            q = BETA * (e / (1 + torch.exp(-u)) - (1 - e) / (1 + torch.exp(u)))
        else:
            loss = (margin - 1 / (2 * BETA)) ** 2
            q = 2 * (margin - 1 / (2 * BETA))
        stats = torch.stack([loss.mean(), (margin > 0).float().mean(), u.mean(), on.sum().float()])
        q = torch.cat([q, -q]) / (P * n)
        return {"loss": loss, "chosen": BETA * d[:P], "rejected": BETA * d[P:], "stats": stats,
                "dlogp": torch.where(on, q[:, None], 0.0)}
    # headgrad
    d = _score_gradient(_scores(s), s["tokens"], s["lse"], s["entropy"], s["dlogp"], s["dentropy"])
    d = torch.where(on[..., None], d, 0.0).reshape(-1, c["V"])
    h = s["hidden"].float()
    return {"dhidden": (d @ s["weight"].float()).reshape(h.shape).to(torch.bfloat16),
            "dweight": (d.t() @ h.reshape(-1, c["H"])).to(torch.bfloat16)}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(c):
    """Bytes: each input that counts read once, each output written once; rows that the mask leaves out are read
    nowhere but written (as zeros) in a gradient.  Flops: the matrix products' multiplications and additions, and a
    handful an element elsewhere."""
    k = c["kind"]
    if k == "preference":
        n, on = 2 * c["P"] * c["T"], _count(2 * c["P"], c["T"], c["mask"])
        return {"bytes": on * 8 + n * (4 + (1 if c["mask"] else 0)) + 12 * c["P"], "flops": 4 * on}
    n, on = c["B"] * c["T"], _count(c["B"], c["T"], c["mask"])
    flag = n if c["mask"] else 0
    if k == "policy":
        return {"bytes": on * 20 + n * 8 + flag, "flops": 40 * on}
    if k in ("fused", "logprobs", "backward"):
        size = 4 if c["dtype"] == "f32" else 2
        row = c["V"] * size
        if k == "logprobs":
            return {"bytes": on * (row + 4) + n * 12 + flag, "flops": 5 * on * c["V"]}
        if k == "backward":
            return {"bytes": on * (row + 12 + (8 if c["ent"] else 0)) + n * row + flag, "flops": 6 * on * c["V"]}
        return {"bytes": on * (row + 16) + n * (row + 8) + flag, "flops": 9 * on * c["V"]}
    wide = c["V"] * c["H"] * 2
    if k == "head":
        return {"bytes": wide + on * (c["H"] * 2 + 4) + n * 12 + flag, "flops": 2 * on * c["V"] * c["H"]}
    return {"bytes": 2 * wide + on * (c["H"] * 2 + 12) + n * c["H"] * 2 + flag, "flops": 6 * on * c["V"] * c["H"]}


# ---------------------------------------------------------------------------
# the outputs in 64 bits
# ---------------------------------------------------------------------------
def _exact_token(c, on, n_tokens, row_tokens, n_rows, lp, old, ref, adv, ent):
    """Weight, loss terms and derivatives of every token of the policy loss, case by case from its definition."""
    w = on / n_tokens if c["reduction"] == "token_mean" else on / (row_tokens * n_rows)
    r = (lp - old).exp()
    inside = (r >= 1 - CLIP_LOW) & (r <= 1 + CLIP_HIGH)
    # the pessimistic choice: for a gain only the upper bound holds back, for a loss only the lower one
    held = torch.where(adv >= 0, r > 1 + CLIP_HIGH, r < 1 - CLIP_LOW) & ~inside & (adv != 0)
    limit = torch.where(adv >= 0, torch.full_like(r, 1 + CLIP_HIGH), torch.full_like(r, 1 - CLIP_LOW))
    steep = (adv < 0) & (r > DUAL)
    used = torch.where(steep, torch.full_like(r, DUAL), torch.where(held, limit, r))
    term = -adv * used
    x = ref - lp
    kl = x.exp() - 1 - x
    slope = torch.where(held | steep, torch.zeros_like(r), -adv * r) + c["kl"] * (1 - x.exp())
    return w, r, held | steep, term, kl, w * slope


def _exact_policy(c, mask, lp, old, ref, adv, ent):
    on = mask.double()
    n = on.sum().clamp(min=1)
    rows = on.sum(1, keepdim=True)
    z = torch.zeros_like(on)
    lp, old, ref, adv, ent = [torch.where(mask, x.double(), z) for x in (lp, old, ref, adv, ent)]
    w, r, held, term, kl, g = _exact_token(c, on, n, rows.clamp(min=1), (rows > 0).sum().clamp(min=1), lp, old, ref,
                                           adv, ent)
    a, b, h = (w * term).sum(), (w * kl).sum(), (w * ent).sum()
    stats = torch.stack([a + c["kl"] * b - c["ent"] * h, a, b, h, (held.double() * on).sum() / n,
                         ((old - lp) * on).sum() / n, (r * on).sum() / n, on.sum()])
    return stats, g, -c["ent"] * w


def exact(case, seed):
    c = case
    k = c["kind"]
    s = prepare(c, seed)
    if k == "preference":
        on = _on(s)
        P = c["P"]
        d = (s["logp"].double() - s["ref"].double()).masked_fill(~on, 0)
        length = on.double().sum(1)
        sums = d.sum(1) / (length.clamp(min=1) if c["length_norm"] else 1)
        better, worse = sums[:P], sums[P:]
        u = BETA * (better - worse)
        e = c["smoothing"]
        if c["loss"] == "sigmoid":
            logsig = torch.nn.functional.logsigmoid
            loss = -(1 - e) * logsig(u) - e * logsig(-u)
            slope = BETA * (torch.sigmoid(u) - (1 - e))
        else:
            loss = (u / BETA - 0.5 / BETA).square()
            slope = 2 * (u / BETA - 0.5 / BETA)
        each = torch.stack([slope, -slope]).reshape(-1, 1) / P
        if c["length_norm"]:
            each = each / length.clamp(min=1)[:, None]
        return {"loss": loss, "chosen": BETA * better, "rejected": BETA * worse,
                "stats": torch.stack([loss.mean(), (u > 0).double().mean(), u.mean(), length.sum()]),
                "dlogp": each * on}
    if k == "policy":
        stats, g, h = _exact_policy(c, _on(s), s["logp"], s["old"], s["ref"], s["adv"], s["entropy"])
        return {"stats": stats, "dlogp": g, "dentropy": h}
    # the others: some rows at a time, so that 64-bit logits stay small
    B, T, V = c["B"], c["T"], c["V"]
    on, tok = _on(s).reshape(-1), s["tokens"].reshape(-1).long()
    rows = (s["logits"] if "logits" in s else s["hidden"]).reshape(B * T, -1)
    weight = s["weight"].double() if "weight" in s else None
    step = max(1, 200_000_000 // V)
    scores = lambda a: (rows[a:a + step].double() if weight is None  # noqa: E731
                        else rows[a:a + step].double() @ weight.t()) / TAU
    flat = torch.zeros((3, B * T), dtype=torch.float64, device="cuda")
    if k in ("logprobs", "head", "fused"):
        for a in range(0, B * T, step):
            logq = torch.log_softmax(scores(a), -1)
            at = tok[a:a + step, None]
            flat[0, a:a + step] = logq.gather(1, at)[:, 0]
            flat[1, a:a + step] = torch.logsumexp(scores(a), -1)
            flat[2, a:a + step] = -(logq.exp() * logq.masked_fill(logq == -math.inf, 0)).sum(-1)
            del logq
        flat *= on
    logp, lse, entropy = flat.reshape(3, B, T)
    if k in ("logprobs", "head"):
        return {"logp": logp, "lse": lse, "entropy": entropy}
    if k == "fused":
        stats, g, h = _exact_policy(c, _on(s), logp, s["old"], s["ref"], s["adv"], entropy)
        if not c["ent"]:
            h = None
    else:
        lse, entropy, g = s["lse"].double(), s["entropy"].double(), s["dlogp"].double()
        h = s["dentropy"].double() if s["dentropy"] is not None else None
    lse, entropy, g = lse.reshape(-1), entropy.reshape(-1), g.reshape(-1)
    h = h.reshape(-1) if h is not None else None
    out = None
    if k == "headgrad":
        dh = torch.empty((B * T, c["H"]), dtype=torch.float64, device="cuda")
        dw = torch.zeros((V, c["H"]), dtype=torch.float64, device="cuda")
    else:
        out = torch.empty((B * T, V), dtype=torch.float64, device="cuda")
    for a in range(0, B * T, step):
        logq = scores(a) - lse[a:a + step, None]
        p = logq.exp()
        d = -p * g[a:a + step, None]
        d[torch.arange(d.shape[0], device="cuda"), tok[a:a + step]] += g[a:a + step]
        if h is not None:
            d -= h[a:a + step, None] * (p * (logq.masked_fill(logq == -math.inf, 0) + entropy[a:a + step, None]))
        d = (d / TAU).masked_fill(~on[a:a + step, None], 0)
        if k == "headgrad":
            dh[a:a + step] = d @ weight
            dw += d.t() @ rows[a:a + step].double()
        else:
            out[a:a + step] = d
        del logq, p, d
    if k == "headgrad":
        return {"dhidden": dh.reshape(B, T, -1), "dweight": dw}
    if k == "fused":
        return {"stats": stats, "logp": logp, "entropy": entropy, "dlogits": out.reshape(B, T, V)}
    return {"dlogits": out.reshape(B, T, V)}
