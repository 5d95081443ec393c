"""Distillation of batches whose tokens of weight 0 have rows that are not finite: they add nothing to the loss's sum and
have gradient 0, and every other row is what it would be beside finite ones, bit for bit."""
import numpy as np
import pytest
import torch

from gpu_util import host

pytestmark = pytest.mark.gpu

from paper_2609_24456_amd import conduit as cd  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
FORMS = [dict(loss="forward", teacher_temperature=2.0), dict(loss="forward", rest=True, reduction="sequence_mean", scale=1.5),
         dict(loss="reverse", rest=True, reduction="sum", scale=0.01)]
K = 5
# rows that share a wavefront, of a wavefront (by elements and in vectors), of 4 and 16 wavefronts, in parts, in parts that a
# launch of its own joins
SHAPES = [(18, 1, 9), (18, 3, 200), (300, 2, 9), (2100, 2, 9), (9000, 2, 150), (40000, 1, 300), (40000, 1, 9), (140001, 1, 9),
          (140001, 1, 515)]


def _batch(V, B, T, dtype):
    g = torch.Generator(device="cuda").manual_seed(V + T)
    x = torch.randn((B, T, V), generator=g, device="cuda").mul_(3).to(dtype)
    ids = torch.stack([torch.randperm(V, generator=g, device="cuda")[:K] for _ in range(B * T)]).reshape(B, T, K).int()
    y = torch.log_softmax(torch.randn((B, T, K), generator=g, device="cuda"), -1) - 0.1
    weight = torch.rand((B, T), generator=g, device="cuda") + 0.1
    return x, ids, y, weight


def _spoil(x, ids):
    """(a copy with rows 1 to 5 of each sequence not finite, those rows)"""
    bad, x = torch.zeros(x.shape[:2], dtype=torch.bool, device="cuda"), x.clone()
    bad[:, 1:6] = True
    for b in range(x.shape[0]):
        free = next(j for j in range(x.shape[-1]) if j not in set(ids[b, 2].tolist()))
        x[b, 1, int(ids[b, 1, 2])], x[b, 2, free], x[b, 3, int(ids[b, 3, 0])] = float("nan"), float("nan"), float("inf")
        x[b, 4], x[b, 5, x.shape[-1] - 1] = float("nan"), float("inf")
    return x, bad


def _distill(opts, x, ids, y, weight, gradient=True):
    loss, stats = torch.empty(ids.shape[:-1], device="cuda"), torch.empty(3, device="cuda")
    dx = torch.full_like(x, float("nan")) if gradient else None
    cd.conduit_distill_loss(cd.distill_opts(**opts), x, ids, y, loss, stats, dlogits=dx, weight=weight)
    return loss, host(stats), dx


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,B,T", SHAPES)
def test_rows_of_weight_zero_that_are_not_finite(V, B, T, dtype):
    x, ids, y, weight = _batch(V, B, T, dtype)
    spoilt, bad = _spoil(x, ids)
    weight[bad] = 0.0
    for opts in FORMS:
        for gradient in (True, False):
            want, got = (_distill(opts, t, ids, y, weight, gradient) for t in (x, spoilt))
            assert torch.equal(torch.isnan(got[0]), bad) and torch.equal(got[0][~bad], want[0][~bad])
            assert np.isfinite(got[1][0]) and got[1][0] == want[1][0] and got[1][2] == B * T
            if gradient:
                assert not got[2][bad].float().abs().sum() > 0 and not torch.isnan(got[2]).any(), opts
                assert torch.equal(got[2], want[2])


@pytest.mark.parametrize("V,B,T", SHAPES)
def test_no_gradient_of_a_loss_scaled_to_nothing(V, B, T):
    x, ids, y, weight = _batch(V, B, T, F32)
    spoilt, _ = _spoil(x, ids)
    for opts in FORMS:
        dx = _distill(dict(opts, scale=0.0), spoilt, ids, y, weight)[2]
        assert bool((dx == 0).all()), opts
