"""The operators on listed choices whose speed this framework is judged by, as a training or serving program calls them.

A teacher's answer is kept as a few choices for each position (their numbers and log-probabilities) instead of a whole
row of logits; a student is scored at those choices and drawn towards them.  Per-token arrays are [B, T], listed ones
[B, T, K]; a mask of uint8 says which tokens count.

  alternatives  the K most probable choices of every position with their log-probabilities, beside the taken token's
                log-probability, the log-normaliser and the entropy (`conduit_token_alternatives`)
  listed        log-probabilities of K given choices and of all others together (`conduit_listed_logprobs`)
  listedgrad    the gradient of those (`conduit_listed_logprobs_backward`)
  distill       the divergence from a teacher's K listed choices and its gradient, logits to their gradient in one call
                (`conduit_distill_loss`)

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
        # one new token for each of 64 sequences while they are generated, with its 20 best alternatives
        _alternatives("step-alternatives", B=64, T=1, V=VOCAB, K=20, dtype="bf16", mask=False),
        # a teacher's scoring of a batch of delivered sequences, kept as 64 choices a position
        _alternatives("teacher-alternatives", B=8, T=512, V=VOCAB, K=64, dtype="bf16"),
        # a small vocabulary of odd size in fp32, logits and tokens taken one position apart out of the full sequences
        _alternatives("shifted-alternatives", B=16, T=511, V=32001, K=50, dtype="f32", shifted=True),
        # a discrete-action agent: 16,384 samples, 18 actions, some of them not allowed (their logits are -inf)
        _alternatives("action-alternatives", B=1, T=16384, V=18, K=5, dtype="f32", mask=False, forbid=True),
        # five answers to choose from at the last position of 64 sequences
        _listed("answer-options", B=64, T=1, V=VOCAB, K=5, dtype="bf16", mask=False),
        # a student scored at a teacher's choices, one position apart
        _listed("listed-shifted", B=8, T=511, V=50001, K=32, dtype="f32", shifted=True),
        # the gradient that goes back into a model that returned fp32 logits
        _listedgrad("listed-gradient", B=4, T=512, V=50001, K=32, dtype="f32", rest=True),
        # the smallest distillation step: a few short sequences over bytes
        _distill("distill-bytes", B=4, T=61, V=257, K=8, dtype="f32", loss="forward", rest=False,
                 reduction="token_mean"),
        # the training step of a distilled student
        _distill("distill-batch", B=8, T=1024, V=VOCAB, K=64, dtype="bf16", loss="forward", rest=False,
                 reduction="token_mean"),
        # the same over an odd vocabulary in fp32, the choices that the teacher did not list as one
        _distill("distill-rest", B=8, T=511, V=32001, K=100, dtype="f32", loss="forward", rest=True,
                 reduction="sequence_mean", shifted=True),
        # a student drawn towards the teacher on its own answers, tokens weighted
        _distill("distill-reverse", B=4, T=512, V=50001, K=20, dtype="bf16", loss="reverse", rest=True,
                 reduction="token_mean", weight=True),
        # a few positions of a vocabulary: fewer rows than the GPU has compute units
        _distill("distill-few", B=4, T=9, V=VOCAB, K=32, dtype="bf16", loss="forward", rest=True,
                 reduction="token_mean", mask=False),
    ]


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    kind = rng.choice(["alternatives", "alternatives", "listed", "listedgrad", "distill", "distill"])
    # actions of an agent, bytes, or tokens of a vocabulary
    V = rng.choice([_log(rng, 2, 1024), _log(rng, 1000, 200_000), _log(rng, 20_000, 160_000)])
    rows = _log(rng, 1, max(2, min(65_536, 400_000_000 // V)))
    B, T = _split(rng, rows)
    c = dict(B=B, T=T, V=V, K=min(V, _log(rng, 1, 128)), dtype=rng.choice(["f32", "bf16"]),
             mask=rng.random() < 0.75, shifted=rng.random() < 0.3)
    if kind == "alternatives":
        return _alternatives(None, forbid=rng.random() < 0.3, **c)
    if kind == "listed":
        return _listed(None, **c)
    if kind == "listedgrad":
        return _listedgrad(None, rest=rng.random() < 0.5, **c)
    loss, rest = rng.choice([("forward", False), ("forward", True), ("reverse", True)])
    return _distill(None, loss=loss, rest=rest, reduction=rng.choice(["token_mean", "sequence_mean"]),
                    weight=rng.random() < 0.3, **c)


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


def _alternatives(name, B, T, V, K, dtype, mask=True, shifted=False, forbid=False):
    return _case("alternatives", name, B=B, T=T, V=V, K=K, dtype=dtype, mask=mask, shifted=shifted, forbid=forbid)


def _listed(name, B, T, V, K, dtype, mask=True, shifted=False):
    return _case("listed", name, B=B, T=T, V=V, K=K, dtype=dtype, mask=mask, shifted=shifted, forbid=False)


def _listedgrad(name, B, T, V, K, dtype, rest, mask=True, shifted=False):
    return _case("listedgrad", name, B=B, T=T, V=V, K=K, dtype=dtype, mask=mask, shifted=shifted, forbid=False,
                 rest=rest)


def _distill(name, B, T, V, K, dtype, loss, rest, reduction, mask=True, shifted=False, weight=False):
    return _case("distill", name, B=B, T=T, V=V, K=K, dtype=dtype, mask=mask, shifted=shifted, forbid=False, loss=loss,
                 rest=rest, reduction=reduction, weight=weight)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
TAU = 0.9  # sampling temperature of the logits
TEACHER_TAU = 2.0  # further softening of a teacher's choices where the others are left out
LEAST = 2.0 ** -23  # least probability that a teacher leaves to the choices it did not list
NONE = -math.inf


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


def _count(c):
    return sum(b - a for a, b in _spans(c["B"], c["T"], c["mask"]))


class _Inputs:
    """Seeded device inputs of a [B, T] token batch; `shifted` ones are views, one position in, of arrays with T + 1
    columns (the predictions of position t and the tokens of position t + 1)."""

    def __init__(self, c, seed):
        self.c, self.B, self.T = c, c["B"], c["T"]
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

    def tokens(self):
        return torch.randint(0, self.c["V"], (self.B, self.T), generator=self.g, device="cuda", dtype=torch.int32)

    def rows(self):
        """(first, last + 1, sequence) of the pieces that whole rows are made in."""
        step = max(1, 4096 * 32000 // self.c["V"])
        return [(a, min(self.T, a + step), b) for b in range(self.B) for a in range(0, self.T, step)]

    def model(self, tokens, a, z, b):
        """Rows of logits spread like a trained model's: unit noise of scale 2, eight choices ahead by up to 12 (by less
        among few choices, which stay uncertain), the taken token among them."""
        V = self.c["V"]
        x = 2 * self.randn(z - a, V)
        ahead = torch.randint(0, V, (z - a, 8), generator=self.g, device="cuda")
        ahead[:, 0] = tokens[b, a:z]
        return x.scatter_add_(1, ahead, min(12.0, 1.15 * math.log(V)) * self.rand(z - a, 8))

    def logits(self, tokens):
        c = self.c
        out = self.wide(c["V"], TYPES[c["dtype"]])
        for a, z, b in self.rows():
            x = self.model(tokens, a, z, b)
            if c["forbid"]:  # a fifth of the choices are not allowed, never the taken one
                taken = x.gather(1, tokens[b, a:z, None].long())
                x.masked_fill_(self.rand(z - a, c["V"]) < 0.2, NONE)
                x.scatter_(1, tokens[b, a:z, None].long(), taken)
            out[b, a:z] = x.to(out.dtype)
        return out

    def teacher_and_student(self, tokens):
        """(logits of a student, numbers and log-probabilities of its teacher's K best choices): the student's scores
        are the teacher's with noise."""
        c = self.c
        out = self.wide(c["V"], TYPES[c["dtype"]])
        ids, values = self.wide(c["K"], torch.int32), self.wide(c["K"], torch.float32)
        for a, z, b in self.rows():
            x = self.model(tokens, a, z, b)
            best, at = torch.topk(x, c["K"], dim=-1)
            values[b, a:z] = best - torch.logsumexp(x, -1, keepdim=True)
            ids[b, a:z] = at.int()
            out[b, a:z] = x.add_(self.randn(z - a, c["V"]), alpha=0.7).to(out.dtype)
        return out, ids, values


def prepare(case, seed):
    c = case
    k = c["kind"]
    x = _Inputs(c, seed)
    s = {"case": c, "mask": x.mask()}
    tokens = x.tokens()
    if k == "alternatives":
        s["tokens"], s["logits"] = x.token(tokens), x.logits(tokens)
        s["ids"], s["logps"] = x.wide(c["K"], torch.int32, zero=True), x.wide(c["K"], torch.float32, zero=True)
        s["out"] = [x.empty() for _ in range(3)]
    else:
        s["logits"], s["ids"], s["teacher"] = x.teacher_and_student(tokens)
    if k == "listed":
        s["logps"], s["out"] = x.wide(c["K"], torch.float32, zero=True), [x.empty() for _ in range(2)]
    if k == "listedgrad":
        n = max(1, _count(c))
        lse, rest = torch.zeros((2, x.B, x.T), device="cuda")
        for a, z, b in x.rows():
            scores = s["logits"][b, a:z].float() / TAU
            lse[b, a:z] = torch.logsumexp(scores, -1)
            scores.scatter_(1, s["ids"][b, a:z].long(), NONE)
            rest[b, a:z] = torch.logsumexp(scores, -1) - lse[b, a:z]
        s["lse"], s["rest"] = x.token(lse), x.token(rest)
        s["dlogps"] = x.wide(c["K"], torch.float32)
        s["dlogps"].copy_(x.randn(x.B, x.T, c["K"]) / n)
        s["drest"] = x.token(x.randn(x.B, x.T) / n) if c["rest"] and c["K"] < c["V"] else None
    if k == "distill":
        s["weight"] = x.token(2 * x.rand(x.B, x.T)) if c["weight"] else None
        s["out"], s["stats"] = [x.empty()], torch.empty(3, device="cuda")
    if k in ("listedgrad", "distill"):  # what a pass does not write (the last position of a shifted one) stays 0
        s["dlogits"] = x.wide(c["V"], TYPES[c["dtype"]], zero=True)
    if own:
        from paper_2609_24456_amd import conduit as cd
        n = 0
        if k == "alternatives":
            n = cd.token_alternatives_workspace(s["logits"], c["K"])
        elif k == "listed":
            n = cd.listed_logprobs_workspace(s["logits"], c["K"])
        elif k == "distill":
            s["opts"] = cd.distill_opts(loss=c["loss"], rest=c["rest"], reduction=c["reduction"],
                                        teacher_temperature=1.0 if c["rest"] else TEACHER_TAU)
            n = cd.distill_loss_workspace(s["logits"], c["K"])
        s["workspace"] = cd.workspace(n)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2609_24456_amd import conduit as cd
    k = s["case"]["kind"]
    if k == "alternatives":
        logp, lse, entropy = s["out"]
        cd.conduit_token_alternatives(s["logits"], s["ids"], s["logps"], tokens=s["tokens"], logp=logp, lse=lse,
                                      entropy=entropy, mask=s["mask"], temperature=TAU, workspace=s["workspace"])
        return {"ids": s["ids"], "logps": s["logps"], "logp": logp, "lse": lse, "entropy": entropy}
    if k == "listed":
        rest, lse = s["out"]
        cd.conduit_listed_logprobs(s["logits"], s["ids"], s["logps"], rest=rest, lse=lse, mask=s["mask"],
                                   temperature=TAU, workspace=s["workspace"])
        return {"logps": s["logps"], "rest": rest, "lse": lse}
    if k == "listedgrad":
        cd.conduit_listed_logprobs_backward(s["logits"], s["ids"], s["lse"], s["dlogps"], s["dlogits"],
                                            rest=s["rest"] if s["drest"] is not None else None, drest=s["drest"],
                                            mask=s["mask"], temperature=TAU)
        return {"dlogits": s["dlogits"]}
    loss, = s["out"]
    cd.conduit_distill_loss(s["opts"], s["logits"], s["ids"], s["teacher"], loss, s["stats"], dlogits=s["dlogits"],
                            weight=s["weight"], mask=s["mask"], temperature=TAU, workspace=s["workspace"])
    return {"stats": s["stats"], "loss": loss, "dlogits": s["dlogits"]}


def _on(s):
    """The mask as truth values."""
    if s["mask"] is not None:
        return s["mask"] != 0
    return torch.ones(s["ids"].shape[:2], dtype=torch.bool, device="cuda")


def _ranking(x, K):
    """The K largest of each row in order, the lowest number first among equal ones: of whole numbers that hold an
    element's rank in their upper 32 bits and its place, counted from the end, in the lower ones."""
    bits = torch.where(x == 0, 0.0, x).view(torch.int32).long()
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
    last = x.shape[-1] - 1
    keys = (order << 32) + (last - torch.arange(last + 1, device=x.device))
    best = torch.topk(keys, K, dim=-1).values
    return (last - (best & 0xFFFFFFFF)).int()


def _log_sum(z):
    """(largest score, log of the sum of exponentials), by the largest score; -inf of nothing."""
    top = z.amax(-1, keepdim=True)
    base = torch.where(top > NONE, top, 0.0)
    return top[..., 0], (base + torch.log(torch.exp(z - base).sum(-1, keepdim=True)))[..., 0]


def _plain_alternatives(s):
    on, x = _on(s), s["logits"].float()
    z = x / TAU
    top, lse = _log_sum(z)
    # by the largest score: the entropy of a row with one probable choice is far below its scores
    far = z - top[..., None]
    e = torch.exp(far)
    total = e.sum(-1)
    entropy = torch.log(total) - torch.where(e > 0, e * far, 0.0).sum(-1) / total
    at = _ranking(x, s["case"]["K"])
    logps = z.gather(-1, at.long()) - lse[..., None]
    logp = z.gather(-1, s["tokens"].long()[..., None])[..., 0] - lse
    return {"ids": torch.where(on[..., None], at, 0), "logps": torch.where(on[..., None], logps, 0.0),
            "logp": torch.where(on, logp, 0.0), "lse": torch.where(on, lse, 0.0),
            "entropy": torch.where(on, entropy, 0.0)}


def _parts(s, z):
    """(log-normaliser, log-probabilities of the listed choices, log-probability of all others) of scores z, by the
    largest score: a probability near 1 has a logarithm far below the scores."""
    at = s["ids"].long()
    top, lse = _log_sum(z)
    base = torch.where(top > NONE, top, 0.0)[..., None]
    far = z - base
    log_total = torch.log(torch.exp(far).sum(-1, keepdim=True))
    _, others = _log_sum(far.scatter(-1, at, NONE))
    return lse, far.gather(-1, at) - log_total, others - log_total[..., 0]


def _curve(x):
    """exp(x) - 1 - x, in 64 bits: next to 0 little is left of the difference."""
    return (torch.expm1(x.double()) - x.double()).float()


def _token_weights(c, on):
    """Every token's part of the loss, by the reduction."""
    f = on.float()
    if c["reduction"] == "token_mean":
        return f / f.sum().clamp(min=1)
    per_row = f.sum(1, keepdim=True)
    return f / (per_row.clamp(min=1) * (per_row > 0).sum().clamp(min=1))


def _run_plain(s):
    c = s["case"]
    k = c["kind"]
    if k == "alternatives":
        return _plain_alternatives(s)
    on, at = _on(s), s["ids"].long()
    z = s["logits"].float() / TAU
    if k == "listedgrad":
        p = torch.exp(z - s["lse"][..., None])
        g, total = s["dlogps"], s["dlogps"].sum(-1, keepdim=True)
        lead = g - (total + (s["drest"][..., None] if s["drest"] is not None else 0.0)) * p.gather(-1, at)
        others = -total
        if s["drest"] is not None:  # exp(-rest) - 1: without the cancellation of a rest near 1
            others = others + s["drest"][..., None] * torch.expm1(-s["rest"])[..., None]
        d = (others * p).scatter(-1, at, lead) / TAU
        return {"dlogits": torch.where(on[..., None], d, 0.0).to(s["logits"].dtype)}
    lse, logps, rest = _parts(s, z)
    if k == "listed":
        return {"logps": torch.where(on[..., None], logps, 0.0), "rest": torch.where(on, rest, 0.0),
                "lse": torch.where(on, lse, 0.0)}
    # sum q log(q / p) as sum q (exp(-u) - 1 + u) + sum q - sum p with u = log(q / p): no terms of both signs
    y = s["teacher"]
    if not c["rest"]:
        logq = y / TEACHER_TAU
        logq = logq - logq.amax(-1, keepdim=True)
        logq = logq - torch.log(torch.exp(logq).sum(-1, keepdim=True))
        q, u = torch.exp(logq), logq - logps
        loss = (q * _curve(-u)).sum(-1) + torch.exp(rest)
        lead, others = q * torch.expm1(-u), torch.ones_like(loss)
    else:
        # 64 bits: the difference of 1 and a sum next to it
        left = 1 - torch.exp(y.double()).sum(-1)
        some = rest > NONE  # where nothing is left to the others, they add nothing
        kept = torch.where(some, left.clamp(min=LEAST), 0.0)
        over = (kept - left).float()  # what the teacher's probabilities are above 1
        logq_rest = torch.where(some, torch.log(kept), 0.0).float()
        q, p, u = torch.exp(y), torch.exp(logps), y - logps
        away = torch.where(some, logq_rest - rest, 0.0)
        if c["loss"] == "forward":
            loss = (q * _curve(-u)).sum(-1) + kept.float() * _curve(-away) + over
            lead, others = q * torch.expm1(-u) + p * over[..., None], over - torch.expm1(away)
        else:
            loss = (p * _curve(u)).sum(-1) + torch.exp(rest) * _curve(away) - over
            lead, others = -p * (u + loss[..., None]), -away - loss
    w = _token_weights(c, on)
    if s["weight"] is not None:
        w = w * s["weight"]
    loss = torch.where(on, loss, 0.0)
    stats = torch.stack([(w * loss).sum(), loss.sum() / on.sum().clamp(min=1), on.sum().float()])
    w = torch.where(on, w, 0.0)[..., None]
    d = torch.exp(z.sub_(lse[..., None])).mul_(w * others[..., None]).scatter_(-1, at, w * lead).div_(TAU)
    return {"stats": stats, "loss": loss, "dlogits": torch.where(on[..., None], d, 0.0).to(s["logits"].dtype)}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(c):
    """Bytes: each input that counts read once, each output written once; rows that the mask leaves out are read
    nowhere but written (as zeros) in a gradient.  Flops: a handful an element."""
    k = c["kind"]
    n, on = c["B"] * c["T"], _count(c)
    flag = n if c["mask"] else 0
    row, K = c["V"] * (4 if c["dtype"] == "f32" else 2), c["K"]
    if k == "alternatives":
        return {"bytes": on * (row + 4) + n * (12 + 8 * K) + flag, "flops": 6 * on * c["V"]}
    if k == "listed":
        return {"bytes": on * (row + 4 * K) + n * (8 + 4 * K) + flag, "flops": 4 * on * c["V"]}
    if k == "listedgrad":
        return {"bytes": on * (row + 4 + 8 * K + (8 if c["rest"] else 0)) + n * row + flag, "flops": 5 * on * c["V"]}
    return {"bytes": on * (row + 8 * K + (4 if c["weight"] else 0)) + n * (row + 4) + flag, "flops": 7 * on * c["V"]}


# ---------------------------------------------------------------------------
# the outputs in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    c = case
    k = c["kind"]
    s = prepare(c, seed)
    B, T, V, K = c["B"], c["T"], c["V"], c["K"]
    N = B * T
    on = _on(s).reshape(-1)
    x = s["logits"].reshape(N, V)
    ids = s["ids"].reshape(N, K).long()
    step = max(1, 100_000_000 // V)
    pieces = [slice(a, min(N, a + step)) for a in range(0, N, step)]
    f64 = dict(dtype=torch.float64, device="cuda")
    if k == "alternatives":
        tok = s["tokens"].reshape(-1).long()
        out_ids = torch.zeros((N, K), dtype=torch.int32, device="cuda")
        logps, logp, lse, entropy = torch.zeros((N, K), **f64), *torch.zeros((3, N), **f64)
        for r in pieces:
            logq = torch.log_softmax(x[r].double() / TAU, -1)
            order = torch.sort(x[r].double(), dim=-1, descending=True, stable=True).indices[:, :K]
            out_ids[r], logps[r] = order.int(), logq.gather(1, order)
            logp[r] = logq.gather(1, tok[r, None])[:, 0]
            lse[r] = torch.logsumexp(x[r].double() / TAU, -1)
            entropy[r] = -(logq.exp() * logq.masked_fill(logq == NONE, 0)).sum(-1)
        out_ids[~on], logps[~on], logp[~on], lse[~on], entropy[~on] = 0, 0, 0, 0, 0
        return {"ids": out_ids.reshape(B, T, K), "logps": logps.reshape(B, T, K), "logp": logp.reshape(B, T),
                "lse": lse.reshape(B, T), "entropy": entropy.reshape(B, T)}
    if k == "listed":
        logps, rest, lse = torch.zeros((N, K), **f64), *torch.zeros((2, N), **f64)
        for r in pieces:
            z = x[r].double() / TAU
            lse[r] = torch.logsumexp(z, -1)
            logps[r] = z.gather(1, ids[r]) - lse[r, None]
            rest[r] = torch.logsumexp(z.scatter(1, ids[r], NONE), -1) - lse[r]
        logps[~on], rest[~on], lse[~on] = 0, 0, 0
        return {"logps": logps.reshape(B, T, K), "rest": rest.reshape(B, T), "lse": lse.reshape(B, T)}
    grad = torch.zeros((N, V), **f64)
    if k == "listedgrad":
        lse, g = s["lse"].reshape(-1).double(), s["dlogps"].reshape(N, K).double()
        for r in pieces:
            p = (x[r].double() / TAU - lse[r, None]).exp()
            d = -p * g[r].sum(-1, keepdim=True)
            d.scatter_add_(1, ids[r], g[r])
            if s["drest"] is not None:
                h, rest = s["drest"].reshape(-1)[r, None].double(), s["rest"].reshape(-1)[r, None].double()
                d += h * (p.scatter(1, ids[r], 0.0) * (-rest).exp() - p)
            grad[r] = d / TAU
        grad[~on] = 0
        return {"dlogits": grad.reshape(B, T, V)}
    y = s["teacher"].reshape(N, K).double()
    live = on.double()
    if c["reduction"] == "token_mean":
        w = live / live.sum().clamp(min=1)
    else:
        rows = live.reshape(B, T).sum(1)
        w = live / (rows.clamp(min=1) * (rows > 0).sum().clamp(min=1)).repeat_interleave(T)
    if s["weight"] is not None:
        w = w * s["weight"].reshape(-1).double()
    loss = torch.zeros(N, **f64)
    for r in pieces:
        logq = torch.log_softmax(x[r].double() / TAU, -1)  # the student's
        p = logq.exp()
        mine = logq.gather(1, ids[r])
        inside = torch.zeros_like(p).scatter_(1, ids[r], 1.0) > 0
        # the derivative by the log-probability of each listed choice, and of the others together
        if not c["rest"]:
            t = torch.softmax(y[r] / TEACHER_TAU, -1)
            loss[r] = (t * (t.log() - mine)).sum(-1)
            by_listed, by_rest, outside = -t, torch.zeros_like(loss[r]), False
        else:
            t = y[r].exp()
            t_rest = (1 - t.sum(-1)).clamp(min=LEAST)
            rest = torch.logsumexp(logq.masked_fill(inside, NONE), -1)
            outside = (rest > NONE).double()
            gap = torch.where(outside > 0, rest - t_rest.log(), 0.0)  # log of student over teacher
            if c["loss"] == "forward":
                loss[r] = (t * (y[r] - mine)).sum(-1) - outside * t_rest * gap
                by_listed, by_rest = -t, -outside * t_rest
            else:
                loss[r] = (mine.exp() * (mine - y[r])).sum(-1) + outside * rest.exp() * gap
                by_listed, by_rest = mine.exp() * (mine - y[r] + 1), outside * rest.exp() * (gap + 1)
        d = -p * (by_listed.sum(-1) + by_rest)[:, None]
        d.scatter_add_(1, ids[r], by_listed)
        if outside is not False:
            share = torch.where(inside, 0.0, (logq - torch.where(outside > 0, rest, 0.0)[:, None]).exp())
            d += by_rest[:, None] * share
        grad[r] = d * (w[r, None] / TAU)
        del logq, p, inside, d
    loss[~on], grad[~on] = 0, 0
    n = live.sum()
    stats = torch.stack([(w * loss).sum(), loss.sum() / n.clamp(min=1), n])
    return {"stats": stats, "loss": loss.reshape(B, T), "dlogits": grad.reshape(B, T, V)}
