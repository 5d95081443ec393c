"""Logits far from 0 and near-certain tokens: log-normalisers and gradients against 64 bits on the same inputs, in every
kernel.

Tolerances, with u = 2^-24.  Scores are at most R powers of two below a row's maximum; a kernel's own probabilities carry
a relative error of u (8 R + 128), as in test_gpu_losses.py, whatever the maximum is.  A log-normaliser is rounded once
where it is formed (u |lse|) beside the error of its logarithm, u (8 R + 128); a gradient taken from it forms log p with
one more rounding of that size.  bf16 gradients add half a unit of their last place."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2609_24456_amd import conduit as cd  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
TAU = 0.9

# short rows, a wavefront a row, a workgroup of 256 and of 1,024 lanes, split rows
SHAPES = [(300, 18), (300, 700), (300, 9001), (260, 40002), (3, 9001), (2, 40002), (1, 128000)]


def _batch(T, V, dtype, offset, lead=0.0):
    g = torch.Generator(device="cuda").manual_seed(T + V)
    x = torch.randn((1, T, V), generator=g, device="cuda").mul_(2)
    tok = torch.randint(0, V, (1, T), generator=g, device="cuda", dtype=torch.int32)
    if lead:
        x.clamp_(-4, 4)
        x.scatter_(-1, tok.long()[..., None], lead)
    x += offset * (1 + torch.rand((1, T, 1), generator=g, device="cuda") / 8)
    return x.to(dtype), tok


def _exact(x, tok):
    z = x.double() / TAU
    lse = torch.logsumexp(z, -1)
    logq = z - lse[..., None]
    p = logq.exp()
    at = tok.long()[..., None]
    R = 1.4427 * float((z.amax(-1, keepdim=True) - z).max())
    rest = p.clone().scatter_(-1, at, 0.0).sum(-1)  # 1 - p of the taken token, without a difference
    return lse, logq, p, rest, (p * -logq).sum(-1), R


def _check(dx, want, p, size, tol, dtype, what):
    """|dx - want| within tol of size times the choice's probability (and, bf16, half a unit of the last place)"""
    bound = tol * size * p + (2.0 ** -8 * want.abs() if dtype == BF16 else 0.0) + 1e-30
    bad = ~((dx.double() - want).abs() <= bound)
    assert not bool(bad.any()), (what, float(((dx.double() - want).abs() / bound).max()), int(bad.sum()))


@pytest.mark.parametrize("offset", [0.0, 1000.0, -30000.0, 30000.0])
@pytest.mark.parametrize("T,V", SHAPES)
def test_log_normalisers_and_gradients_of_offset_logits(T, V, offset):
    x, tok = _batch(T, V, F32, offset)
    lse, logq, p, rest, ent, R = _exact(x, tok)
    f = lambda: torch.empty((1, T), device="cuda")  # noqa: E731
    lp, ls, en = f(), f(), f()
    cd.conduit_token_logprobs(x, tok, lp, lse=ls, entropy=en, temperature=TAU)
    own = U * (8 * R + 128)
    top = float(lse.abs().max())
    err = (ls.double() - lse).abs()
    assert bool((err <= U * lse.abs() + own).all()), float((err / (U * lse.abs() + own)).max())
    # the gradient that the library takes from its own log-normaliser
    one, dx = torch.ones((1, T), device="cuda"), torch.empty_like(x)
    cd.conduit_token_logprobs_backward(x, tok, ls, one, dx, temperature=TAU)
    at = tok.long()[..., None]
    tol = 2 * U * top + own
    others = dx.clone().scatter_(-1, at, 0.0)
    _check(others, (-p / TAU).scatter_(-1, at, 0.0), p, 1.0 / TAU, 2 * tol, F32, "others")
    taken = dx.gather(-1, at)[..., 0].double()
    assert bool(((taken - rest / TAU).abs() <= 2 * tol / TAU).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("ec", [0.0, 0.5])
@pytest.mark.parametrize("offset", [1000.0, 30000.0])
@pytest.mark.parametrize("T,V", SHAPES)
def test_the_fused_loss_of_offset_logits(T, V, offset, ec, dtype):
    """The loss's own gradient does not pass through a rounded log-normaliser: no part of its error grows with the logits."""
    x, tok = _batch(T, V, dtype, offset)
    lse, logq, p, rest, ent, R = _exact(x, tok)
    f = lambda v=0.0: torch.full((1, T), v, device="cuda")  # noqa: E731
    stats, dx = torch.empty(8, device="cuda"), torch.empty_like(x)
    cd.conduit_policy_loss_logits(cd.policy_opts(reduction="sum", entropy_coef=ec), x, tok, f(-1.0), stats, dx, f(), f(), temperature=TAU)
    # the loss is the sum of ratios of 1 minus ec times the entropy: g = 1, h = -ec
    at = tok.long()[..., None]
    want = (-p + ec * p * (logq + ent[..., None])) / TAU
    want.scatter_add_(-1, at, torch.full_like(lse, 1.0 / TAU)[..., None])
    own = U * (8 * R + 128)
    size = (1 + ec * (R + 2)) / TAU
    others = dx.clone().scatter_(-1, at, 0.0)
    _check(others, want.clone().scatter_(-1, at, 0.0), p, size, 2 * own, dtype, "others")
    taken, w = dx.gather(-1, at)[..., 0].double(), want.gather(-1, at)[..., 0]
    assert bool(((taken - w).abs() <= 2 * own * size + (2.0 ** -8 * w.abs() if dtype == BF16 else 0.0)).all())


@pytest.mark.parametrize("T,V", SHAPES)
def test_the_fused_loss_of_a_near_certain_token(T, V):
    """A taken token so far ahead that every other term is lost beside 1 in 32 bits (their sum is below u / 2): 1 - p comes
    out as 0, and nothing larger than what is lost."""
    x, tok = _batch(T, V, F32, 0.0, lead=34.0)
    lse, logq, p, rest, ent, R = _exact(x, tok)
    assert float(rest.max()) < U / 2
    f = lambda v=0.0: torch.full((1, T), v, device="cuda")  # noqa: E731
    stats, dx = torch.empty(8, device="cuda"), torch.empty_like(x)
    cd.conduit_policy_loss_logits(cd.policy_opts(reduction="sum"), x, tok, f(-1.0), stats, dx, f(), f(), temperature=TAU)
    taken = dx.gather(-1, tok.long()[..., None])[..., 0].double()
    assert bool(((taken - rest / TAU).abs() <= U / 2 / TAU).all()), float((taken - rest / TAU).abs().max())
