"""Policy loss at the edges of its types and of its launches, against the 64-bit forms of oracle/losses.py."""
import numpy as np
import pytest
import torch

from gpu_util import host
from oracle import losses as ref

pytestmark = pytest.mark.gpu

from paper_2609_24456_amd import conduit as cd  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("n", [5, 20000])  # one workgroup, many
@pytest.mark.parametrize("kl", [0.0, 0.1])
def test_a_divergence_from_nothing_is_infinite(n, kl):
    """logp = -inf under a finite reference: k = exp(x) - 1 - x at x = infinity is infinity, not a difference of two; a
    loss without the KL term does not see it, and with it the gradient is -infinity there alone."""
    lp = np.full((1, n), -1.0, np.float32)
    lp[0, 3] = -np.inf
    old, rf, adv = np.full((1, n), -1.0, np.float32), np.full((1, n), -1.5, np.float32), np.ones((1, n), np.float32)
    stats, g = torch.empty(8, device="cuda"), torch.empty((1, n), device="cuda")
    t = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    cd.conduit_policy_loss(cd.policy_opts(kl_coef=kl, reduction="sum"), t(lp), t(adv), stats, g, old_logp=t(old), ref_logp=t(rf))
    want, wg, _ = ref.policy_loss(lp, adv, old, rf, kl_coef=kl, reduction="sum")
    s = host(stats)
    assert s[2] == want[2] == np.inf and s[5] == want[5] == np.inf
    assert (s[0] == np.inf) == (kl > 0) and not np.isnan(s).any()
    d = host(g)
    assert d[0, 3] == wg[0, 3] == (-np.inf if kl else 0.0) and np.isfinite(np.delete(d[0], 3)).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,V", [(6, 18), (6, 700), (300, 700), (600, 5000), (6, 40000), (300, 40000)])
def test_a_taken_choice_without_weight_has_an_infinite_divergence(T, V, dtype):
    """The same from logits: the taken choice's logit is -inf now.  Short rows, wavefronts, workgroups, split rows."""
    g = torch.Generator(device="cuda").manual_seed(V + T)
    x = torch.randn((1, T, V), generator=g, device="cuda").to(dtype)
    tok = torch.randint(0, V, (1, T), generator=g, device="cuda", dtype=torch.int32)
    x[0, 2, int(tok[0, 2])] = float("-inf")
    old = torch.full((1, T), -5.0, device="cuda")
    adv = torch.ones((1, T), device="cuda")
    stats, lp, en, dx = torch.empty(8, device="cuda"), torch.empty((1, T), device="cuda"), torch.empty((1, T), device="cuda"), \
        torch.empty_like(x)
    cd.conduit_policy_loss_logits(cd.policy_opts(entropy_coef=0.01), x, tok, adv, stats, dx, lp, en, old_logp=old, ref_logp=old)
    s = host(stats)
    assert host(lp)[0, 2] == -np.inf and s[2] == np.inf and np.isfinite(s[[0, 1, 3, 4, 6, 7]]).all()
    assert torch.isfinite(dx.float()).all()
