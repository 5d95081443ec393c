"""Scores x / temperature past the largest float: log-normalisers are the infinity of their sign.  At temperatures of which
1 / temperature rounds up and down (what its rounding left has either sign)."""
import numpy as np
import pytest
import torch

from gpu_util import host

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
