"""Choices forbidden by large finite logits, the type's lowest value among them, in the calls on listed choices, against
the 64-bit forms of oracle/losses.py: the list holds every allowed choice, so that all others together have next to no
weight, and some forbidden ones.

Tolerances.  With R0 the spread in powers of two of the allowed scores, 2^-24 (8 R0 + 128) =: e bounds their
log-probabilities (the others add nothing to the sums); those of forbidden ones are off by at most 8 roundings of their own
size besides.  The divergence and its gradient inherit that as in test_gpu_listed.py, with U0 the largest |log(q / p)| of
the allowed choices: 4 e (1 + U0) and 8 e (1 + U0) (p + q) w / temperature, q that of the rest shared by the others that
hold it, whose exponents at equal scores are exact; terms of q times a forbidden one's distance are off by 16 roundings of
themselves.  bf16 adds half a step, 2^-8 of the value."""
import numpy as np
import pytest
import torch

from gpu_util import host
from oracle import losses as ref

pytestmark = pytest.mark.gpu

from paper_2609_24456_amd import conduit as cd  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
FORMS = [dict(loss="forward", teacher_temperature=2.0), dict(loss="forward", rest=True, reduction="sequence_mean", scale=1.5),
         dict(loss="reverse", rest=True, reduction="sum", scale=0.01)]
# rows that share a wavefront, a wavefront each (by elements and in vectors), a workgroup each, in parts
SHAPES = [(18, 3, 200), (300, 2, 9), (2100, 2, 9), (9000, 1, 260), (40000, 1, 9)]
K, ALLOWED = 12, 9


def _batch(V, B, T, dtype, low):
    """(device logits, the same in 64 bits, numbers of the 9 allowed choices of every row and 3 of -1)"""
    rng = np.random.default_rng(V)
    a, ids = np.full((B, T, V), low), np.full((B, T, K), -1, np.int32)
    for at in np.ndindex(B, T):
        ids[at][:ALLOWED] = rng.permutation(V)[:ALLOWED]
        a[at][ids[at][:ALLOWED]] = 3 * rng.standard_normal(ALLOWED)
    x = torch.from_numpy(a.astype(np.float32)).to(dtype)
    return x.cuda(), x.double().numpy(), ids


def _lows(dtype):
    return [-1e4, -1e9, -1e12, -1e30, float(torch.finfo(dtype).min)]


def _e(z, tau):
    fin = np.where(z > -9e3, z, 0.0) / tau * 1.4427
    return 2.0 ** -24 * (8 * (fin.max() - fin.min() + np.abs(fin).max()) + 128)


def _close(got, want, tol):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        same = (got == want) | (got == want.astype(np.float32))  # (past the largest float: infinity)
        bad = ~same & ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5].tolist(), got[bad][:5], want[bad][:5])


def _gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,B,T", SHAPES)
def test_log_probabilities_of_forbidden_choices(V, B, T, dtype):
    for low in _lows(dtype):
        x, z, ids = _batch(V, B, T, dtype, low)
        ids[:, :, ALLOWED] = (ids[:, :, 0] + 1) % V  # (often a forbidden one)
        for tau in (0.9, 1.0, 1.2, 3.0):
            e = _e(z, tau)
            tol = lambda w: e + 8 * 2.0 ** -24 * np.abs(np.where(np.isfinite(w), w, 0.0))  # noqa: E731
            want = ref.listed_logprobs(z, ids, temperature=tau)
            out = [torch.full(s, float("nan"), device="cuda") for s in ((B, T, K), (B, T), (B, T))]
            cd.conduit_listed_logprobs(x, _gpu(ids), out[0], rest=out[1], lse=out[2], temperature=tau)
            for g, w in zip(out, want):
                _close(host(g), w, tol(w))
            want = ref.alternatives(z, K, temperature=tau)
            tok = ids[:, :, ALLOWED].astype(np.int32)
            i, lps, lp = torch.empty((B, T, K), dtype=torch.int32, device="cuda"), torch.empty((B, T, K), device="cuda"), torch.empty((B, T), device="cuda")
            cd.conduit_token_alternatives(x, i, lps, tokens=_gpu(tok), logp=lp, temperature=tau)
            assert (host(i) == want[0]).all()
            _close(host(lps), want[1], tol(want[1]))
            w = ref.token_logprobs(z, tok, temperature=tau)[0]
            _close(host(lp), w, tol(w))
            cd.conduit_token_logprobs(x, _gpu(tok), lp, temperature=tau)
            _close(host(lp), w, tol(w))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,B,T", SHAPES)
def test_distillation_where_all_others_are_forbidden(V, B, T, dtype):
    rng = np.random.default_rng(V + 1)
    for low in _lows(dtype):
        x, z, ids = _batch(V, B, T, dtype, low)
        q = rng.random((B, T, ALLOWED)) + 0.05
        y = np.full((B, T, K), -np.inf, np.float32)
        y[..., :ALLOWED] = np.log(q / q.sum(-1, keepdims=True) * rng.choice([0.7, 0.99, 1.0], (B, T, 1)))
        for tau in (0.9, 1.0, 1.3):
            for opts in FORMS:
                e = _e(z, tau)
                want = ref.distill_loss(z, ids, y, temperature=tau, **opts)
                dx = torch.full_like(x, float("nan"))
                loss, stats = torch.empty((B, T), device="cuda"), torch.empty(3, device="cuda")
                cd.conduit_distill_loss(cd.distill_opts(**opts), x, _gpu(ids), _gpu(y), loss, stats, dlogits=dx, temperature=tau)
                logp, rest, _ = ref.listed_logprobs(z, ids, temperature=tau)
                t = y[..., :ALLOWED].astype(np.float64) / (opts.get("teacher_temperature", 1.0))
                if not opts.get("rest"):
                    t = t - np.log(np.exp(t).sum(-1, keepdims=True))
                U = 1 + np.abs(t - logp[..., :ALLOWED]).max(-1)
                far = 16 * 2.0 ** -24 * np.abs(want[0]) if opts["loss"] == "forward" else 0.0
                _close(host(loss), want[0], 4 * e * U + far)
                total = abs(opts.get("scale", 1.0)) * (B * T if opts.get("reduction") == "sum" else 1)
                _close(host(stats)[0], want[1][0], total * (4 * e * U.max() + 2.0 ** -22 * np.abs(want[0]).max()))
                size = np.zeros(z.shape)
                np.put_along_axis(size, ids[..., :ALLOWED].astype(np.int64), np.exp(t) + np.exp(logp[..., :ALLOWED]), -1)
                if opts.get("rest") and V > ALLOWED:
                    others = np.ones(z.shape, bool)
                    np.put_along_axis(others, ids[..., :ALLOWED].astype(np.int64), False, -1)
                    size[others] = 1.0 / (V - ALLOWED)
                w = abs(opts.get("scale", 1.0)) / (1 if opts.get("reduction") == "sum" else B * T)
                _close(host(dx.float()), want[2],
                       8 * e * U[..., None] * size * w / tau + 1e-44 + (2.0 ** -8 * np.abs(want[2]) if dtype == BF16 else 0.0))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,B,T", SHAPES)
def test_distillation_towards_a_forbidden_choice(V, B, T, dtype):
    """The teacher gives weight to a choice that the student's logits forbid; at -infinity the divergence is infinite."""
    rng = np.random.default_rng(V + 3)
    for low in _lows(dtype)[1:] + [-np.inf]:
        x, z, ids = _batch(V, B, T, dtype, low)
        free = np.ones(z.shape, bool)
        np.put_along_axis(free, ids[..., :ALLOWED].astype(np.int64), False, -1)
        ids[..., ALLOWED] = free.argmax(-1)  # the first forbidden one
        q = rng.random((B, T, ALLOWED + 1)) + 0.05
        y = np.full((B, T, K), -np.inf, np.float32)
        y[..., :ALLOWED + 1] = np.log(q / q.sum(-1, keepdims=True))
        for tau in (0.9, 1.0, 1.3):
            for opts in FORMS[:2]:
                want = ref.distill_loss(z, ids, y, temperature=tau, **opts)
                dx = torch.full_like(x, float("nan"))
                loss, stats = torch.empty((B, T), device="cuda"), torch.empty(3, device="cuda")
                cd.conduit_distill_loss(cd.distill_opts(**opts), x, _gpu(ids), _gpu(y), loss, stats, dlogits=dx, temperature=tau)
                # (sums of up to 11 terms of one sign, each of 4 roundings and the exponential's)
                _close(host(loss), want[0], 32 * 2.0 ** -24 * np.abs(np.where(np.isfinite(want[0]), want[0], 0)) + _e(z, tau) * 100)
                e = _e(z, tau)
                logp = ref.listed_logprobs(z, ids, temperature=tau)[0][..., :ALLOWED + 1]
                t = y[..., :ALLOWED + 1].astype(np.float64) / opts.get("teacher_temperature", 1.0)
                if not opts.get("rest"):
                    t = t - np.log(np.exp(t).sum(-1, keepdims=True))
                U = 1 + np.abs(t - logp)[..., :ALLOWED].max(-1)
                size = np.full(z.shape, 1.0 / V)
                np.put_along_axis(size, ids[..., :ALLOWED + 1].astype(np.int64), np.exp(t) + np.exp(logp), -1)
                w = abs(opts.get("scale", 1.0)) / (B * T)
                _close(host(dx.float()), want[2],
                       8 * e * U[..., None] * size * w / tau + 1e-44 + (2.0 ** -8 * np.abs(want[2]) if dtype == BF16 else 0.0))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,B,T", SHAPES)
def test_gradient_of_a_rest_without_weight(V, B, T, dtype):
    """By lse and rest as they are given, whose roundings are as large as |rest| 2^-24: an other's share of the rest is
    within them, and never above 1."""
    rng = np.random.default_rng(V + 2)
    for low in _lows(dtype):
        x, z, ids = _batch(V, B, T, dtype, low)
        g, h = rng.standard_normal((B, T, K)).astype(np.float32), rng.standard_normal((B, T)).astype(np.float32)
        gz = np.where(ids < 0, 0, g)
        for tau in (0.9, 1.0, 1.2, 3.0):
            out = [torch.empty(s, device="cuda") for s in ((B, T, K), (B, T), (B, T))]
            cd.conduit_listed_logprobs(x, _gpu(ids), out[0], rest=out[1], lse=out[2], temperature=tau)
            dx = torch.full_like(x, float("nan"))
            cd.conduit_listed_logprobs_backward(x, _gpu(ids), out[2], _gpu(g), dx, rest=out[1], drest=_gpu(h), temperature=tau)
            got, rest = host(dx.float()).astype(np.float64), host(out[1])
            # (a rest past the largest float is -infinity as given, and has no gradient)
            want = ref.listed_gradient(z, ids, gz, np.where(rest > -np.inf, h, 0), temperature=tau)
            half = 1 + (2.0 ** -8 if dtype == BF16 else 2.0 ** -24)
            others = np.ones(z.shape, bool)
            np.put_along_axis(others, ids[..., :ALLOWED].astype(np.int64), False, -1)
            most = np.broadcast_to(np.where(rest > -np.inf, np.abs(h), 0)[..., None] / tau * half * (1 + 2.0 ** -20), z.shape)
            assert np.isfinite(got).all() and (np.abs(got)[others] <= most[others]).all(), (low, tau)
            size = (np.abs(gz).sum(-1) + np.abs(h))[..., None] / tau
            _close(got[~others], want[~others], np.broadcast_to(4 * _e(z, tau) * size, z.shape)[~others] + 2.0 ** -8 * (dtype == BF16) * np.abs(want[~others]))
            if low == -1e4:  # 4 roundings of |rest| and |lse|
                tol = np.expm1(8 * 2.0 ** -24 * 1.2e4 / tau) + _e(z, tau)
                _close(got[others], want[others], (tol + half - 1) * np.abs(want[others]))
