"""One post-training iteration of a language model's policy on delivered token batches, end to end on the library.

The "model" is the part that the library's operators meet: the last hidden states of every position (here a free
parameter of each sequence) and the output projection.  An iteration

  1. delivers a prioritised batch of recorded sequences, right-padded, with its mask, the behaviour policy's
     log-probabilities and the advantages, in one launch (ReplayBuffer.sample_pack_gae);
  2. scores it under the current policy without its logits ever being in memory (conduit_head_logprobs);
  3. takes the clipped policy loss with a KL term to a reference policy and its gradient (conduit_policy_loss);
  4. takes the gradients of the hidden states and the projection (conduit_head_logprobs_backward) and steps both;
  5. hands the sequences' new priorities back (ReplayBuffer.update).

With --logits the same through logits that a model returned (conduit_policy_loss_logits), and with --preference a
step of the preference loss over pairs of the batch's sequences.  With --distill the start's scores are kept as a few
choices a position (conduit_token_alternatives), and the gradient back towards them is taken (conduit_distill_loss).

Position t predicts token t + 1, so what is scored are the columns [:, 1:] of the delivered arrays against the hidden
states [:, :-1]: views, nothing is copied.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_24456_amd import conduit as cd  # noqa: E402


def record(capacity, max_len, vocab, seed):
    """A replay of recorded sequences: tokens, behaviour log-probabilities, an outcome reward each."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    lengths = torch.randint(max_len // 8, max_len + 1, (capacity,), generator=g, device="cuda")
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), lengths.cumsum(0)])
    total = int(offsets[-1])
    buf = cd.ReplayBuffer(capacity, (max_len,), torch.int32, ragged=True, aux_elem_bytes=4, action_bytes=0)
    buf.ingest(torch.randint(0, vocab, (total,), generator=g, device="cuda", dtype=torch.int32), offsets=offsets,
               aux=torch.full((total,), -float(torch.log(torch.tensor(float(vocab)))), device="cuda"),
               reward=torch.randn(capacity, generator=g, device="cuda"))
    return buf


class Batch:
    """A delivered batch's tensors, and the views that the losses take."""

    def __init__(self, n, max_len):
        f = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
        self.tokens = torch.empty((n, max_len), dtype=torch.int32, device="cuda")
        self.mask = torch.empty((n, max_len), dtype=torch.uint8, device="cuda")
        self.old, self.adv, self.ret = f(n, max_len), f(n, max_len), f(n, max_len)
        self.reward, self.length = f(n), torch.empty(n, dtype=torch.int32, device="cuda")

    def deliver(self, buf, uniforms):
        xf = cd.transform(cd.XF_TOKENS_PAD, pad_id=0)
        idx, w = buf.sample_pack_gae(uniforms, xf, 1.0, 0.95, self.adv, self.ret, obs=self.tokens, mask=self.mask,
                                     aux=self.old, reward=self.reward, length=self.length)
        return idx, w


def per_token(batch):
    """A new per-token tensor in the layout of the views."""
    return torch.zeros(batch.tokens.shape, device="cuda")[:, 1:]


def policy_step(batch, hidden, weight, ref_logp, opts, lr, workspaces):
    """Steps 2 to 4: the loss's statistics; hidden and weight are moved against their gradients."""
    tokens, mask = batch.tokens[:, 1:], batch.mask[:, 1:]
    logp, lse, entropy = per_token(batch), per_token(batch), per_token(batch)
    cd.conduit_head_logprobs(hidden[:, :-1], weight, tokens, logp, lse=lse, entropy=entropy, mask=mask,
                             workspace=workspaces[0])
    stats = torch.empty(8, device="cuda")
    dlogp, dentropy = per_token(batch), per_token(batch)
    cd.conduit_policy_loss(opts, logp, batch.adv[:, 1:], stats, dlogp, old_logp=batch.old[:, 1:], ref_logp=ref_logp,
                           entropy=entropy, dentropy=dentropy, mask=mask, workspace=workspaces[1])
    dhidden, dweight = torch.zeros_like(hidden), torch.empty_like(weight)
    cd.conduit_head_logprobs_backward(hidden[:, :-1], weight, tokens, lse, dlogp, dhidden[:, :-1], dweight, entropy=entropy,
                                      dentropy=dentropy, mask=mask, workspace=workspaces[0])
    for x, dx in ((hidden, dhidden), (weight, dweight)):  # a step of `lr` of the parameter's own norm
        x.sub_(dx * (lr * x.norm() / dx.norm().clamp_min(1e-20)))
    return stats


def logits_step(batch, logits, opts):
    """The same loss from logits, their gradient in their place."""
    stats, logp, entropy = torch.empty(8, device="cuda"), per_token(batch), per_token(batch)
    view = logits[:, :-1]
    cd.conduit_policy_loss_logits(opts, view, batch.tokens[:, 1:], batch.adv[:, 1:], stats, view, logp, entropy,
                                  old_logp=batch.old[:, 1:], mask=batch.mask[:, 1:])
    return stats, logits


def preference_step(batch, logits, ref_logp):
    """The preference loss over the batch's first half of sequences against its second, back to the logits."""
    tokens, mask, view = batch.tokens[:, 1:], batch.mask[:, 1:], logits[:, :-1]
    logp, lse, dlogp = per_token(batch), per_token(batch), per_token(batch)
    cd.conduit_token_logprobs(view, tokens, logp, lse=lse, mask=mask)
    loss, stats = torch.empty(len(tokens) // 2, device="cuda"), torch.empty(4, device="cuda")
    cd.conduit_preference_loss(cd.preference_opts(beta=0.1), logp, loss, stats, dlogp, ref_logp=ref_logp, mask=mask)
    grad = torch.zeros_like(logits)
    cd.conduit_token_logprobs_backward(view, tokens, lse, dlogp, grad[:, :-1], mask=mask)
    return stats, grad


def teacher_choices(batch, logits, choices):
    """What is kept of a teacher: its best choices of every position and their log-probabilities."""
    shape = tuple(batch.tokens[:, 1:].shape) + (choices,)
    ids, logps = torch.empty(shape, dtype=torch.int32, device="cuda"), torch.empty(shape, device="cuda")
    cd.conduit_token_alternatives(logits[:, :-1], ids, logps, mask=batch.mask[:, 1:])
    return ids, logps


def distill_step(batch, logits, ids, logps, opts):
    """The divergence from a teacher's choices, and its gradient in the logits' place; how likely the student finds the
    teacher's choices, and all others together."""
    view, mask = logits[:, :-1], batch.mask[:, 1:]
    scores, rest, loss, stats = torch.empty_like(logps), per_token(batch), per_token(batch), torch.empty(3, device="cuda")
    cd.conduit_listed_logprobs(view, ids, scores, rest=rest, mask=mask)
    cd.conduit_distill_loss(opts, view, ids, logps, loss, stats, dlogits=view, mask=mask)
    return stats, scores, rest, logits


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--sequences", type=int, default=16)
    p.add_argument("--max-len", type=int, default=256)
    p.add_argument("--vocab", type=int, default=32000)
    p.add_argument("--hidden", type=int, default=512)
    p.add_argument("--steps", type=int, default=5)
    p.add_argument("--lr", type=float, default=0.003, help="step, relative to each parameter's norm")
    p.add_argument("--logits", action="store_true", help="also the loss from logits")
    p.add_argument("--preference", action="store_true", help="also the preference loss")
    p.add_argument("--distill", action="store_true", help="also the divergence from the start's best choices")
    p.add_argument("--choices", type=int, default=16, help="choices a position that --distill keeps")
    a = p.parse_args(argv)
    n, T, V, H = a.sequences, a.max_len, a.vocab, a.hidden
    buf = record(4 * n, T, V, seed=0)
    batch = Batch(n, T)
    g = torch.Generator(device="cuda").manual_seed(1)
    hidden = torch.randn((n, T, H), generator=g, device="cuda").to(torch.bfloat16)
    weight = (torch.randn((V, H), generator=g, device="cuda") * H ** -0.5).to(torch.bfloat16)
    opts = cd.policy_opts(clip_low=0.2, clip_high=0.2, dual_clip=3.0, kl_coef=0.02, entropy_coef=0.001,
                          reduction="sequence_mean")
    workspaces = (cd.workspace(max(cd.head_logprobs_workspace(hidden[:, :-1], weight),
                                   cd.head_logprobs_backward_workspace(hidden[:, :-1], weight))),
                  cd.workspace(cd.policy_loss_workspace(n, T - 1)))
    uniforms = torch.randint(-2 ** 63, 2 ** 63 - 1, (n,), generator=g, dtype=torch.int64, device="cuda")
    idx, _ = batch.deliver(buf, uniforms)
    # the reference policy, and here also the one that acted: the start
    ref = per_token(batch)
    cd.conduit_head_logprobs(hidden[:, :-1], weight, batch.tokens[:, 1:], ref, mask=batch.mask[:, 1:],
                             workspace=workspaces[0])
    batch.old[:, 1:].copy_(ref)
    scores = lambda: (hidden.float().reshape(-1, H) @ weight.float().t()).reshape(n, T, V).to(torch.bfloat16)  # noqa: E731
    if a.distill:
        kept = teacher_choices(batch, scores(), a.choices)
    losses = []
    for step in range(a.steps):
        stats = policy_step(batch, hidden, weight, ref, opts, a.lr, workspaces)
        named = dict(zip(cd.POLICY_STATS, stats.tolist()))
        losses.append(named["loss"])
        print(f"step {step}: " + "  ".join(f"{k} {v:.4g}" for k, v in named.items()), flush=True)
    buf.update(idx, (batch.adv.abs().sum(1) * 1000).to(torch.int32) + 1)
    out = {"losses": losses}
    if a.distill:
        stats = distill_step(batch, scores(), *kept, cd.distill_opts(rest=True))[0]
        out["distill"] = stats.tolist()
        print("distill: " + "  ".join(f"{k} {v:.4g}" for k, v in zip(cd.DISTILL_STATS, out["distill"])), flush=True)
    if a.logits or a.preference:
        logits = scores()
    if a.preference:
        stats, grad = preference_step(batch, logits, ref)
        out["preference"] = stats.tolist()
        print("preference: " + "  ".join(f"{k} {v:.4g}" for k, v in zip(cd.PREFERENCE_STATS, out["preference"])), flush=True)
    if a.logits:
        stats, grad = logits_step(batch, logits, opts)
        out["logits"] = stats.tolist()
        print("from logits: " + "  ".join(f"{k} {v:.4g}" for k, v in zip(cd.POLICY_STATS, out["logits"])), flush=True)
    if cd.conduit_sync_check() != cd.OK:
        raise cd.ConduitError(cd.ESTATE, cd.last_error())
    buf.close()
    return out


if __name__ == "__main__":
    main()
