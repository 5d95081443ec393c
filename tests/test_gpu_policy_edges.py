"""Policy loss at the edges of its types and of its launches, against the 64-bit forms of oracle/losses.py."""
import numpy as np
import pytest
import torch

from gpu_util import host
from oracle import losses as ref
from test_gpu_losses import _mask, _policy_check, _policy_inputs

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


def _sums(adv, reduction, mask=None):
    """The statistics of a loss whose terms are -adv themselves (ratio 1), and its gradient."""
    stats, g, lp = torch.empty(8, device="cuda"), torch.empty_like(adv), torch.zeros_like(adv)
    cd.conduit_policy_loss(cd.policy_opts(reduction=reduction), lp, adv, stats, g, mask=mask)
    assert torch.equal(g, (-adv).masked_fill(mask == 0, 0.0) if mask is not None else -adv) or reduction != "sum"
    return host(stats).astype(np.float64)


@pytest.mark.parametrize("n", [600, 20000, 300001])  # one workgroup, one chunk a lane, several
def test_sums_of_terms_of_both_signs_are_in_64_bits(n):
    """Terms up to 2^30 in steps of 2^-5 that nearly cancel: every partial sum fits 64 bits, whatever the order, so the total
    is exact but for its last rounding, where sums in 32 bits would be off by 2^5 and more."""
    g = torch.Generator(device="cuda").manual_seed(n)
    a = torch.randint(-(1 << 23), 1 << 23, (n,), generator=g, device="cuda").double()
    big = a * torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, 128.0, 2.0 ** -5)
    half = big[: n // 2]
    x = torch.cat([half, -half, torch.full((n - 2 * (n // 2),), 3.0, device="cuda", dtype=torch.float64)])
    x = x[torch.randperm(n, generator=g, device="cuda")]
    x[0] += 2.0 ** -5
    adv = x.float()[None]
    want = -float(adv.double().sum())
    assert abs(want) <= 200.0
    s = _sums(adv, "sum")
    assert s[1] == s[0] == np.float32(want), (s[1], want)


@pytest.mark.parametrize("n", [600, 20000])
def test_partial_sums_beyond_the_largest_float(n):
    """Partial sums may pass the largest float: the total is what counts."""
    adv = torch.full((1, n), 3e38, device="cuda")
    adv[0, n // 2:] = -3e38
    s = _sums(adv, "sum")
    assert s[0] == 0.0 and s[1] == 0.0


@pytest.mark.parametrize("B,T", [(3, 200), (7, 3001), (1, 300001)])
@pytest.mark.parametrize("reduction", ["token_mean", "sequence_mean"])
@pytest.mark.parametrize("masked", [False, True])
def test_means_are_rounded_once(B, T, reduction, masked):
    """Positive terms that are whole numbers, so the 64-bit sum is exact: a mean is right to one rounding to 32 bits (and a
    few of 64), the weights' included."""
    g = torch.Generator(device="cuda").manual_seed(B + T)
    adv = -torch.randint(1, 1 << 20, (B, T), generator=g, device="cuda").float()
    mask = (torch.rand((B, T), generator=g, device="cuda") < 0.7).to(torch.uint8) if masked else None
    on = mask.double() if masked else torch.ones((B, T), device="cuda", dtype=torch.float64)
    x = -adv.double() * on
    want = float(x.sum() / on.sum()) if reduction == "token_mean" else float((x.sum(1) / on.sum(1)).mean())
    s = _sums(adv, reduction, mask)
    assert abs(s[1] - want) <= 2.0 ** -24 * (1 + 1e-5) * want, (s[1] / want - 1) * 2 ** 24


# up to 2,048 chunks of 4 tokens of a row, and up to 2,048 rows with weights of their own, one workgroup takes by itself:
# both sides of each edge
@pytest.mark.parametrize("B,T", [(1, 8192), (1, 8193), (2048, 1), (2049, 1), (2048, 4), (2047, 5), (1024, 8), (1025, 8)])
@pytest.mark.parametrize("reduction", ["token_mean", "sequence_mean", "sum"])
@pytest.mark.parametrize("columns", [False, True])
def test_both_sides_of_the_largest_batch_of_one_workgroup(B, T, reduction, columns):
    """`columns`: columns [1, T + 1) of wider arrays, whose rows are never taken as one."""
    rng = np.random.default_rng(B + T)
    x, mask = _policy_inputs(rng, B, T), _mask(rng, B, T)

    def dev(a):
        if not columns:
            return torch.from_numpy(a).cuda()
        w = torch.zeros((B, T + 1), dtype=torch.from_numpy(a).dtype, device="cuda")
        w[:, 1:] = torch.from_numpy(a).cuda()
        return w[:, 1:]

    kw = dict(clip_low=0.2, clip_high=0.2, dual_clip=3.0, kl_coef=0.05, entropy_coef=0.01, reduction=reduction)
    for m in (None, mask):
        nine = np.full((B, T), 9.0, np.float32)
        stats, g, h = torch.full((8,), 9.0, device="cuda"), dev(nine), dev(nine)
        cd.conduit_policy_loss(cd.policy_opts(**kw), dev(x["logp"]), dev(x["adv"]), stats, g, old_logp=dev(x["old"]),
                               ref_logp=dev(x["ref"]), entropy=dev(x["entropy"]), dentropy=h, mask=None if m is None else dev(m))
        _policy_check(x, m, kw, (host(stats), host(g.contiguous()), host(h.contiguous())))
