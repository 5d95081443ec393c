"""Scores x / temperature past the largest float: log-normalisers are the infinity of their sign, and gradients of choices
at -infinity or at the type's lowest value are those of a probability of 0.

Temperatures of which 1 / temperature rounds up and down (what its rounding left has either sign).  Where the largest
score is 0 the log-normaliser is the logarithm of how many choices share it, and a gradient is a sum of at most 5 products,
each of at most 8 roundings of 2^-24 of its parts."""
import numpy as np
import pytest
import torch

from gpu_util import host
from oracle import losses as ref

pytestmark = pytest.mark.gpu

from paper_2609_24456_amd import conduit as cd  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
WIDTHS = [40, 300, 2100, 5000, 40000]


def _left(tau):
    """What rounding 1 / tau to 32 bits left of it."""
    return np.float64(1.0) / tau - np.float64(np.float32(1.0 / tau))


def _taus(k):
    """Small temperatures, k of either sign of _left."""
    t = 10.0 ** -np.linspace(9.03, 20.3, 40)
    return [float(v) for s in (1, -1) for v in [v for v in t if s * _left(v) > 1][:: max(1, 18 // k)][:k]]


def test_temperatures_of_both_signs():
    signs = [np.sign(_left(t)) for t in _taus(3)]
    assert signs.count(1.0) == 3 and signs.count(-1.0) == 3


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", WIDTHS)
def test_log_normalisers_past_the_largest_float(V, dtype):
    rng = np.random.default_rng(V)
    low, high = float(torch.finfo(dtype).min), float(torch.finfo(dtype).max)
    a = np.stack([np.full(V, low), np.full(V, high), -1e38 * (1 + rng.random(V)), 1e38 * (1 + rng.random(V)), np.where(np.arange(V) == 2, high, low)])
    x = torch.from_numpy(a.astype(np.float32)).to(dtype).cuda()
    n = len(a)
    tok = torch.full((n,), 2, dtype=torch.int32, device="cuda")
    ids = torch.tensor([[0, 2, V - 1]] * n, dtype=torch.int32, device="cuda")
    want = np.array([-np.inf, np.inf, -np.inf, np.inf, np.inf])
    for tau in _taus(3):
        out = torch.full((3, n), float("nan"), device="cuda")
        i, lps = torch.empty((n, 3), dtype=torch.int32, device="cuda"), torch.empty((n, 3), device="cuda")
        cd.conduit_token_logprobs(x, tok, torch.empty(n, device="cuda"), lse=out[0], temperature=tau)
        cd.conduit_token_alternatives(x, i, lps, tokens=tok, lse=out[1], temperature=tau)
        cd.conduit_listed_logprobs(x, ids, lps, lse=out[2], temperature=tau)
        for o in host(out):
            assert (o == want).all(), (tau, o)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", WIDTHS)
def test_gradients_of_choices_without_weight_at_small_temperatures(V, dtype):
    rng = np.random.default_rng(V + 1)
    a = -1.0 - rng.random((6, V))
    a[np.arange(6), rng.integers(0, V, 6)] = 0.0
    a[1, 3] = a[1, 9] = 0.0
    a[2, ::3], a[3, 1::3] = -np.inf, float(torch.finfo(dtype).min)
    a[4, V - 1], a[5, 0] = -np.inf, float(torch.finfo(dtype).min)
    a[np.arange(6), 20] = 0.0
    x = torch.from_numpy(a.astype(np.float32)).to(dtype)
    z = x.double().numpy()
    x = x.cuda()
    ids = np.tile(np.array([20, 3, 1, V - 1], np.int32), (6, 1))
    g, h = rng.standard_normal((6, 4)).astype(np.float32), rng.standard_normal(6).astype(np.float32)
    tok = rng.integers(0, V, 6).astype(np.int32)
    dev = lambda t: torch.from_numpy(np.ascontiguousarray(t, np.float32)).cuda()  # noqa: E731
    for tau in _taus(3):
        step = 2.0 ** -24 * 40 * (np.abs(g).sum(-1) + np.abs(h))[:, None] / tau
        _, rest, lse = ref.listed_logprobs(z, ids, temperature=tau)
        want = ref.listed_gradient(z, ids, g, temperature=tau)
        dx = torch.full_like(x, float("nan"))
        cd.conduit_listed_logprobs_backward(x, torch.from_numpy(ids).cuda(), dev(lse), dev(g), dx, temperature=tau)
        got = host(dx.float()).astype(np.float64)
        half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
        assert (np.abs(got - want) <= step + half * np.abs(want)).all(), (tau, np.argwhere(~(np.abs(got - want) <= step + half * np.abs(want)))[:5])
        want = ref.logits_gradient(z, tok, h, temperature=tau)
        dx.fill_(float("nan"))
        cd.conduit_token_logprobs_backward(x, torch.from_numpy(tok).cuda(), dev(lse), dev(h), dx, temperature=tau)
        got = host(dx.float()).astype(np.float64)
        assert (np.abs(got - want) <= step + half * np.abs(want)).all(), (tau, np.argwhere(~(np.abs(got - want) <= step + half * np.abs(want)))[:5])
