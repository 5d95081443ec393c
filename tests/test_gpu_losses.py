"""Token log-probabilities and losses through the Python binding against the
64-bit forms of oracle/losses.py: every kernel a row's width and the batch's
size select, masks that leave rows empty, values that nothing may read, strides,
in-place gradients, workspaces handed from call to call, graphs and streams.

Tolerances.  With R the spread of a row's scores in powers of two, every score's
distance to the maximum carries two roundings of 2^-24 R, the sum over n scores a
lane at most n + 6 more of 2^-24 (n <= 64 for the widths here), the logarithm and
the last products a few: 2^-24 (8 R + 128) bounds a log-probability.  A gradient
inherits that as a relative error of its probability, times g or h (R + 2);
bf16 (8 significant bits) adds half a unit of the last place, at most 2^-8 of the value."""
import numpy as np
import pytest
import torch

from gpu_util import host
from oracle import losses as ref

pytestmark = pytest.mark.gpu

from paper_2609_24456_amd import conduit as cd  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16


def _gpu(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def _logits(rng, B, T, V, dtype, spread=3.0):
    """(device tensor, the same values in 64 bits)"""
    x = torch.from_numpy((spread * rng.standard_normal((B, T, V))).astype(np.float32)).to(dtype)
    return x.cuda(), x.double().numpy()


def _mask(rng, B, T):
    m = (rng.random((B, T)) < 0.7).astype(np.uint8) * rng.integers(1, 256, (B, T)).astype(np.uint8)
    if B > 1:
        m[B // 2] = 0
    return m


def _bound(z, temperature):
    """2^-24 (8 R + 128), R the widest spread of finite scores in powers of two (and the largest score itself)."""
    fin = np.where(np.isfinite(z), z, 0.0) / temperature * 1.4427
    return 2.0 ** -24 * (8 * (fin.max() - fin.min() + np.abs(fin).max()) + 128)


def _close(got, want, tol):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        bad = ~same & ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


def _forward(x, tok, mask=None, temperature=1.0, **kw):
    out = [torch.full(tok.shape, float("nan"), device="cuda") for _ in range(3)]
    cd.conduit_token_logprobs(x, tok, out[0], lse=out[1], entropy=out[2], mask=mask, temperature=temperature, **kw)
    return [host(o) for o in out]


# V: one choice, groups of 4 to 64 lanes and their edges, a wavefront a row (up to 8 vectors a lane), a workgroup of
# 256, one of 1,024 (whole and with a remainder read twice), each with and without elements after the last vector
WIDTHS = [1, 2, 3, 18, 32, 33, 64, 65, 128, 129, 255, 256, 257, 511, 512, 513, 1000, 2047, 4096, 4097, 5001, 16385, 33001]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", WIDTHS)
def test_logprobs_and_gradient(V, dtype):
    rng = np.random.default_rng(V)
    B, T = (3, 7) if V > 6000 else (4, 81)  # fewer rows than compute units (split where wide), or more
    tau = 0.7
    x, z = _logits(rng, B, T, V, dtype)
    tok = rng.integers(0, V, (B, T)).astype(np.int32)
    mask = _mask(rng, B, T)
    tol = _bound(z, tau)
    want = ref.token_logprobs(z, tok, mask, tau)
    got = _forward(x, _gpu(tok), _gpu(mask), tau)
    for g, w, k in zip(got, want, (1, 1, 2)):
        _close(g, w, k * tol)
    g, h = rng.standard_normal((B, T)), rng.standard_normal((B, T))
    lse, ent = _gpu(want[1].astype(np.float32)), _gpu(want[2].astype(np.float32))
    R = tol * 2.0 ** 24 / 8
    for hh in (None, h):
        dx = torch.full_like(x, float("nan"))
        cd.conduit_token_logprobs_backward(x, _gpu(tok), lse, _gpu(g.astype(np.float32)), dx,
                                           entropy=None if hh is None else ent,
                                           dentropy=None if hh is None else _gpu(hh.astype(np.float32)),
                                           mask=_gpu(mask), temperature=tau)
        w = ref.logits_gradient(z, tok, g.astype(np.float32), None if hh is None else hh.astype(np.float32), mask, tau)
        size = (np.abs(g) + (0 if hh is None else np.abs(hh) * (R + 2)))[..., None] / tau
        _close(host(dx.float()), w, 2 * tol * size + (2.0 ** -8 * np.abs(w) if dtype == BF16 else 0))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,V", [(2, 150, 6001), (1, 270, 17001), (1, 260, 66001), (1, 1, 128001), (5, 1, 70002)])
def test_logprobs_of_wide_rows(B, T, V, dtype):
    """Whole rows a workgroup of 256 or 1,024 lanes (one wider than its registers hold), and split rows."""
    rng = np.random.default_rng(V)
    x = torch.randn((B, T, V), generator=torch.Generator(device="cuda").manual_seed(V), device="cuda").mul_(2).to(dtype)
    tok = rng.integers(0, V, (B, T)).astype(np.int32)
    tok[0, 0] = V - 1
    z = x.double()
    lse = torch.logsumexp(z, -1)
    logp = z.gather(-1, _gpu(tok).long()[..., None])[..., 0] - lse
    p = torch.exp(z - lse[..., None])
    ent = -(p * (z - lse[..., None])).sum(-1)
    tol = 2.0 ** -24 * (8 * 2 * 1.4427 * float(z.abs().max()) + 128)
    for g, w, k in zip(_forward(x, _gpu(tok)), (logp, lse, ent), (1, 1, 2)):
        _close(g, host(w), k * tol)


def test_rows_without_weight_and_extreme_values():
    """-inf choices, rows of nothing else, rows at the type's lowest value, large logits, a taken choice at -inf,
    a NaN, in every kernel."""
    for dtype in (F32, BF16):
        for V in (7, 300, 700, 5000, 40000):
            T = 12
            rng = np.random.default_rng(V)
            x, z = _logits(rng, 1, T, V, dtype)
            low = torch.finfo(dtype).min
            tok = rng.integers(1, V, (1, T)).astype(np.int32)
            z = x.clone()
            z[0, 0] = -np.inf
            z[0, 1, :V // 2] = -np.inf
            tok[0, 1] = V - 1
            z[0, 2] = low
            z[0, 3, 0] = -np.inf
            tok[0, 3] = 0
            z[0, 4] += 30000.0
            z[0, 5] = low
            z[0, 5, V // 2] = 1.0
            tok[0, 5] = V // 2
            z[0, 6] = -np.inf
            z[0, 6, V - 1] = -5.0
            tok[0, 6] = V - 1
            z[0, 7, V // 3] = float("nan")
            z64 = z.double().cpu().numpy()
            rows = [0, 1, 2, 3, 4, 5, 6] + list(range(8, T))
            logp, lse, ent = _forward(z, _gpu(tok))
            assert all(np.isnan(v[0, 7]) for v in (logp, lse, ent)), V
            want = ref.token_logprobs(z64[:, rows], tok[:, rows])
            for r, (k, t) in enumerate(zip(rows, tok[0, rows])):
                # (the lowest value is far beyond what the other terms of an error could see: its own size counts)
                tol = 2.0 ** -24 * (8 * 1.45 * 40 + 128) + (0 if k not in (2, 4) else 2.0 ** -23 * abs(want[1][0, r]))
                for name, g, w in (("logp", logp, want[0]), ("lse", lse, want[1]), ("entropy", ent, want[2])):
                    slack = tol if name == "lse" else 2.0 ** -24 * (8 * 1.45 * 40 + 128)
                    a, b = float(g[0, k]), float(w[0, r])
                    assert a == b or abs(a - b) <= 2 * slack, (V, dtype, k, name, a, b)
            # gradients: nothing at a row without weight, finite everywhere but the NaN's row
            dx = torch.full_like(z, 7.0)
            gg = torch.ones((1, T), device="cuda")
            cd.conduit_token_logprobs_backward(z, _gpu(tok), _gpu(lse), gg, dx, entropy=_gpu(ent), dentropy=gg)
            d = host(dx.float())
            assert (d[0, 0] == 0).all()
            assert np.isfinite(d[0, [1, 3, 5, 6]]).all(), (V, dtype)
            assert np.abs(d[0, 6]).max() <= 1e-5 and abs(d[0, 5]).max() <= 1e-5


def test_masked_places_are_not_read():
    for V in (18, 700, 6000, 40000):
        for T in (6, 300):
            rng = np.random.default_rng(T + V)
            x, z = _logits(rng, 1, T, V, BF16)
            tok = rng.integers(0, V, (1, T)).astype(np.int32)
            mask = np.ones((1, T), np.uint8)
            mask[0, 1::2] = 0
            clean = _forward(x, _gpu(tok), _gpu(mask))
            x[0, 1::4] = float("nan")
            x[0, 3::4] = float("inf")
            tok[0, 1::2] = -100  # what a padded label holds
            dirty = _forward(x, _gpu(tok), _gpu(mask))
            for a, b in zip(clean, dirty):
                assert np.array_equal(a, b) and (a[0, 1::2] == 0).all()
            nan = torch.full((1, T), float("nan"), device="cuda")
            m = _gpu(mask) != 0
            zero = torch.zeros((1, T), device="cuda")
            at = lambda v: torch.where(m, v, nan)  # noqa: E731
            dx = torch.full_like(x, 5.0)
            cd.conduit_token_logprobs_backward(x, _gpu(tok), at(_gpu(clean[1])), at(zero + 1), dx, entropy=at(_gpu(clean[2])),
                                               dentropy=at(zero + 1), mask=_gpu(mask))
            assert torch.isfinite(dx.float()).all() and (dx[0, 1::2] == 0).all()
            stats = torch.empty(8, device="cuda")
            dx = torch.full_like(x, 5.0)
            cd.conduit_policy_loss_logits(cd.policy_opts(kl_coef=0.1, entropy_coef=0.1, reduction="sequence_mean"), x,
                                          _gpu(tok), at(zero + 1), stats, dx, zero.clone(), zero.clone(),
                                          old_logp=at(_gpu(clean[0])), ref_logp=at(_gpu(clean[0])), mask=_gpu(mask))
            assert torch.isfinite(stats).all() and torch.isfinite(dx.float()).all() and (dx[0, 1::2] == 0).all()
    assert cd.conduit_sync_check() == cd.OK, cd.last_error()


def test_tokens_outside_the_vocabulary_are_flagged():
    for V in (18, 700, 40000):
        for T in (4, 300):
            for call in ("forward", "gradient", "loss"):
                rng = np.random.default_rng(V)
                x, z = _logits(rng, 1, T, V, F32)
                tok = rng.integers(0, V, (1, T)).astype(np.int32)
                tok[0, 1], tok[0, 2] = V, -1
                f = lambda v=0.0: torch.full((1, T), v, device="cuda")  # noqa: E731
                dx = torch.full_like(x, 5.0)
                if call == "forward":
                    out = _forward(x, _gpu(tok))
                    assert all((o[0, 1:3] == 0).all() for o in out)
                elif call == "gradient":
                    cd.conduit_token_logprobs_backward(x, _gpu(tok), f(3.0), f(1.0), dx)
                    assert (dx[0, 1:3] == 0).all() and (dx[0, 3] != 0).any()
                else:
                    stats = torch.empty(8, device="cuda")
                    cd.conduit_policy_loss_logits(cd.policy_opts(), x, _gpu(tok), f(1.0), stats, dx, f(), f())
                    assert (dx[0, 1:3] == 0).all()
                    # two of the T add nothing, and the count is the mask's
                    s = host(stats)
                    assert s[7] == T and abs(s[1] + (T - 2) / T) <= 1e-6
                assert cd.conduit_sync_check() == cd.ESTATE and "token outside" in cd.last_error()
                cd.conduit_clear_error()
    assert cd.conduit_sync_check() == cd.OK, cd.last_error()


def test_strides_and_in_place_gradients():
    for dtype in (F32, BF16):
        for V in (19, 513, 5003, 9001):
            rng = np.random.default_rng(V)
            B, T = 3, 9
            full, z = _logits(rng, B, T + 1, V, dtype)
            tok = rng.integers(0, V, (B, T + 1)).astype(np.int32)
            mask = _mask(rng, B, T + 1)
            g = rng.standard_normal((B, T + 1)).astype(np.float32)
            tol = _bound(z, 1.0)
            x, t, m = full[:, :-1], _gpu(tok)[:, 1:], _gpu(mask)[:, 1:]
            out = [torch.full((B, T + 1), -3.0, device="cuda") for _ in range(3)]
            cd.conduit_token_logprobs(x, t, out[0][:, 1:], lse=out[1][:, 1:], entropy=out[2][:, 1:], mask=m)
            want = ref.token_logprobs(z[:, :-1], tok[:, 1:], mask[:, 1:])
            for o, w, k in zip(out, want, (1, 1, 2)):
                _close(host(o)[:, 1:], w, k * tol)
                assert (o[:, 0] == -3.0).all()  # nothing outside the view is written
            wg = ref.logits_gradient(z[:, :-1], tok[:, 1:], g[:, 1:], None, mask[:, 1:])
            last = full[:, -1].clone()
            cd.conduit_token_logprobs_backward(x, t, out[1][:, 1:], _gpu(g)[:, 1:], x, mask=m)
            _close(host(full.float())[:, :-1], wg,
                   2 * tol * np.abs(g[:, 1:, None]) + (2.0 ** -8 * np.abs(wg) if dtype == BF16 else 0))
            assert torch.equal(full[:, -1], last)
            # one row of logits for every token (broadcast), [T, V] and [T] forms, transposed sequences
            row, zr = _logits(rng, 1, 1, V, dtype)
            tt = rng.integers(0, V, 5).astype(np.int32)
            w = ref.token_logprobs(np.broadcast_to(zr[0], (5, V)), tt)
            for a, b, k in zip(_forward(row[0].expand(5, V), _gpu(tt)), w, (1, 1, 2)):
                _close(a, b, k * tol)
            time_major = torch.from_numpy(z[:, :-1]).to(dtype).transpose(0, 1).contiguous().cuda().transpose(0, 1)
            for a, b, k in zip(_forward(time_major, t.contiguous(), m.contiguous()), want, (1, 1, 2)):
                _close(a, b, k * tol)


# ---------------------------------------------------------------------------
# policy loss
# ---------------------------------------------------------------------------
def _policy_inputs(rng, B, T):
    logp = -rng.exponential(1.0, (B, T))
    d = 0.4 * rng.standard_normal((B, T))
    for kink in (np.log(0.8), np.log(1.2), np.log(3.0)):
        d = np.where(np.abs(d - kink) < 1e-3, d + 3e-3, d)
    d.flat[::17] += 1.4
    adv = rng.standard_normal((B, T))
    adv.flat[::13] = 0.0
    f = lambda a: a.astype(np.float32)  # noqa: E731
    logp = f(logp)
    return dict(logp=logp, old=f(logp - d), ref=f(logp + 0.1 * rng.standard_normal((B, T))), adv=f(adv),
                entropy=f(3 * rng.random((B, T))))


def _policy_check(x, mask, kw, got, valid=None, tol=2.0 ** -20):
    """fp32 terms: a few roundings of exponentials (2^-22 each), sums in 64 bits, one rounding at the end."""
    stats, g, h = ref.policy_loss(x["logp"], x["adv"], x.get("old"), x.get("ref"), x.get("entropy"), mask, valid=valid, **kw)
    on = np.ones(x["logp"].shape, bool) if mask is None else mask != 0
    n = max(1, on.sum())
    w = {"token_mean": 1.0 / n, "sequence_mean": 1.0, "sum": 1.0}[kw.get("reduction", "token_mean")]
    size = (np.abs(x["adv"]) * np.exp(x["logp"] - x.get("old", x["logp"])) + 1) * kw.get("scale", 1.0)
    _close(got[1], g, tol * size * w + 2.0 ** -22 * np.abs(g))
    if got[2] is not None:
        _close(got[2], h, 2.0 ** -22 * np.abs(h) + 1e-12)
    total = n if kw.get("reduction") == "sum" else 1
    top = float(np.where(on, size, 0).max(initial=1.0))
    _close(got[0][:4], stats[:4], tol * top * total * 4)
    _close(got[0][4:], stats[4:], 1e-6 * np.maximum(1, np.abs(stats[4:])))


# one workgroup (up to 4,096 chunks of 4), many; rows of one token, rows longer than one count's reach
@pytest.mark.parametrize("B,T", [(1, 1), (7, 1), (1, 5), (3, 7), (8, 333), (1, 16384), (1, 16385), (5000, 1), (4097, 3),
                                 (300, 71), (3, 20001), (2, 70001)])
@pytest.mark.parametrize("reduction", ["token_mean", "sequence_mean", "sum"])
def test_policy_loss(B, T, reduction):
    rng = np.random.default_rng(B * 7 + T)
    x = _policy_inputs(rng, B, T)
    dev = {k: _gpu(v) for k, v in x.items()}
    ws = cd.workspace(cd.policy_loss_workspace(B, T))
    for masked in (False, True):
        mask = _mask(rng, B, T) if masked else None
        kw = dict(clip_low=0.2, clip_high=0.2, dual_clip=3.0, kl_coef=0.05, entropy_coef=0.01, scale=0.5, reduction=reduction)
        stats, g, h = torch.full((8,), 9.0, device="cuda"), torch.full((B, T), 9.0, device="cuda"), torch.full((B, T), 9.0, device="cuda")
        cd.conduit_policy_loss(cd.policy_opts(**kw), dev["logp"], dev["adv"], stats, g, old_logp=dev["old"], ref_logp=dev["ref"],
                               entropy=dev["entropy"], dentropy=h, mask=None if mask is None else _gpu(mask), workspace=ws)
        _policy_check(x, mask, kw, (host(stats), host(g), host(h)))
    if B * T < 3000:  # the absent inputs, and gradients in place
        for drop in ({"old"}, {"ref"}, {"entropy"}, {"old", "ref", "entropy"}):
            y = {k: v for k, v in x.items() if k not in drop}
            kw = dict(kl_coef=0.2, entropy_coef=0.3, reduction=reduction)
            stats, lp = torch.empty(8, device="cuda"), dev["logp"].clone()
            cd.conduit_policy_loss(cd.policy_opts(**kw), lp, dev["adv"], stats, lp, old_logp=_gpu(x["old"]) if "old" in y else None,
                                   ref_logp=_gpu(x["ref"]) if "ref" in y else None,
                                   entropy=_gpu(x["entropy"]) if "entropy" in y else None)
            _policy_check(y, None, kw, (host(stats), host(lp), None))


def test_policy_loss_of_nothing():
    for B, T, mask in [(0, 5, None), (3, 0, None), (4, 6, np.zeros((4, 6), np.uint8)), (300, 200, np.zeros((300, 200), np.uint8))]:
        for reduction in ("token_mean", "sequence_mean"):
            f = torch.full((B, T), float("nan"), device="cuda")
            stats, g = torch.full((8,), 9.0, device="cuda"), torch.full((B, T), 9.0, device="cuda")
            cd.conduit_policy_loss(cd.policy_opts(kl_coef=0.1, reduction=reduction), f, f, stats, g, old_logp=f, ref_logp=f,
                                   mask=None if mask is None else _gpu(mask))
            assert (stats == 0).all() and (g == 0).all()


def test_policy_loss_extremes():
    """A ratio that overflows is clipped where it gains, is nothing where the advantage is 0, and a NaN stays one."""
    lp = np.array([[0.0, 0.0, 0.0, -1.0, 0.0]], np.float32)
    old = np.array([[-200.0, -200.0, -200.0, -1.0, np.nan]], np.float32)
    adv = np.array([[1.0, 0.0, -1.0, 1.0, 1.0]], np.float32)
    for n, finite in ((4, True), (5, False)):
        stats, g = torch.empty(8, device="cuda"), torch.empty((1, n), device="cuda")
        cd.conduit_policy_loss(cd.policy_opts(dual_clip=3.0, reduction="sum"), _gpu(lp[:, :n]), _gpu(adv[:, :n]), stats, g,
                               old_logp=_gpu(old[:, :n]))
        s, d = host(stats), host(g)
        assert list(d[0, :4]) == [0.0, 0.0, 0.0, -1.0]
        assert (abs(s[1] - (-1.2 + 0.0 + 3.0 - 1.0)) <= 1e-6) == finite and np.isnan(s[1]) != finite


@pytest.mark.parametrize("dtype", [F32, BF16])
# short rows, a wavefront a row, workgroups of 256 and 1,024, one wider than the registers, split rows
@pytest.mark.parametrize("B,T,V", [(1, 300, 18), (2, 9, 3), (3, 40, 400), (3, 7, 700), (2, 150, 4097), (1, 260, 8193),
                                   (4, 65, 33001), (1, 257, 70001), (3, 3, 20001), (1, 1, 128000)])
def test_policy_loss_from_logits(B, T, V, dtype):
    rng = np.random.default_rng(V)
    big = B * T * V > 10_000_000
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn((B, T, V), generator=g, device="cuda").mul_(2).to(dtype)
    tok = rng.integers(0, V, (B, T)).astype(np.int32)
    x.scatter_add_(-1, _gpu(tok).long()[..., None], torch.full((B, T, 1), 4.0, device="cuda", dtype=dtype))
    if V < 1000:
        x[0, 0, (tok[0, 0] + 1) % V] = float("-inf")
    mask = _mask(rng, B, T)
    mask[0, 0] = 1
    tau = 1.25
    z = x.double() / tau
    lse = torch.logsumexp(z, -1)
    logq = z - lse[..., None]
    logp = logq.gather(-1, _gpu(tok).long()[..., None])[..., 0]
    p = logq.exp()
    plogp = torch.where(p > 0, p * logq, torch.zeros_like(p))
    ent = -plogp.sum(-1)
    on = torch.from_numpy(mask != 0).cuda()
    q = _policy_inputs(rng, B, T)
    shift = q["old"] - q["logp"]
    lp64 = host(torch.where(on, logp, 0.0 * logp))
    en64 = host(torch.where(on, ent, 0.0 * ent))
    old, rf = (lp64 + shift).astype(np.float32), (lp64 + (q["ref"] - q["logp"])).astype(np.float32)
    tol = 2.0 ** -24 * (8 * 3 * 1.4427 * float(z[torch.isfinite(z)].abs().max()) + 128)
    for ec in (0.0, 0.02):
        for reduction in ("token_mean", "sequence_mean"):
            kw = dict(dual_clip=3.0, kl_coef=0.05, entropy_coef=ec, reduction=reduction)
            stats = torch.full((8,), 9.0, device="cuda")
            lpo, eno = torch.full((B, T), 9.0, device="cuda"), torch.full((B, T), 9.0, device="cuda")
            dx = x.clone()  # in place
            cd.conduit_policy_loss_logits(cd.policy_opts(**kw), dx, _gpu(tok), _gpu(q["adv"]), stats, dx, lpo, eno,
                                          old_logp=_gpu(old), ref_logp=_gpu(rf), mask=_gpu(mask), temperature=tau)
            _close(host(lpo), lp64, tol)
            _close(host(eno), en64, 2 * tol)
            ws, wg, wh = ref.policy_loss(lp64, q["adv"], old, rf, en64, mask, **kw)
            _close(host(stats)[:4], ws[:4], 40 * tol)
            _close(host(stats)[4:], ws[4:], 40 * tol * np.maximum(1, np.abs(ws[4:])))
            if big and (ec or reduction != "token_mean"):
                continue
            gg, hh = torch.from_numpy(wg).cuda()[..., None], torch.from_numpy(wh).cuda()[..., None]
            w = -gg * p - hh * (plogp + p * ent[..., None])
            w.scatter_add_(-1, _gpu(tok).long()[..., None], gg)
            w = torch.where(on[..., None], w / tau, torch.zeros_like(w))
            # relative to the token's weight: its slope (a ratio and a KL term, each a few times as sensitive as logp)
            wt = 1.0 / max(1, int((mask != 0).sum())) if reduction == "token_mean" else 1.0
            bound = 16 * tol * wt * 8 + (2.0 ** -8 * w.abs() if dtype == BF16 else 0.0)
            bad = ~((dx.double() - w).abs() <= bound)
            assert not bool(bad.any()), (bad.nonzero()[:4], dx[bad][:4], w[bad][:4])
    assert cd.conduit_sync_check() == cd.OK, cd.last_error()


# ---------------------------------------------------------------------------
# preference loss
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("P,T", [(1, 1), (1, 3), (3, 64), (2, 4096), (2, 4097), (1, 40001), (140, 33), (200, 5000)])
def test_preference_loss(P, T):
    rng = np.random.default_rng(P + T)
    ws = cd.workspace(cd.preference_loss_workspace(P, T))
    logp = (-rng.exponential(1.0, (2 * P, T))).astype(np.float32)
    rf = (logp + 0.1 * rng.standard_normal((2 * P, T))).astype(np.float32)
    for kw in (dict(), dict(label_smoothing=0.2, beta=0.3), dict(loss="squared", length_norm=True, scale=0.25),
               dict(length_norm=True, beta=2.0)):
        for masked in (False, True):
            mask = _mask(rng, 2 * P, T) if masked else None
            lp, r = _gpu(logp), _gpu(rf)
            if masked:
                off = torch.from_numpy(mask == 0).cuda()
                lp, r = lp.masked_fill(off, float("nan")), r.masked_fill(off, float("inf"))
            use_ref = kw.get("beta") != 2.0
            out = [torch.full((P,), 9.0, device="cuda") for _ in range(3)]
            stats, g = torch.full((4,), 9.0, device="cuda"), torch.full((2 * P, T), 9.0, device="cuda")
            cd.conduit_preference_loss(cd.preference_opts(**kw), lp, out[0], stats, g, ref_logp=r if use_ref else None,
                                       mask=None if mask is None else _gpu(mask), chosen=out[1], rejected=out[2], workspace=ws)
            w = ref.preference_loss(logp, rf if use_ref else None, mask, **kw)
            # sums in 64 bits, one rounding to 32 at the end of each value
            for got, want in zip([*out, stats, g], w):
                _close(host(got), want, 2.0 ** -23 * np.abs(want) + 1e-9 * np.abs(want).max())


def test_preference_loss_far_margins_and_none():
    lp = torch.zeros((2, 2), device="cuda")
    for margin, loss, q in ((1e4, 0.0, 0.0), (-1e4, 1e4, -1.0)):
        lp[0, 0] = margin
        out, stats, g = torch.empty(1, device="cuda"), torch.empty(4, device="cuda"), torch.empty((2, 2), device="cuda")
        cd.conduit_preference_loss(cd.preference_opts(beta=1.0), lp, out, stats, g)
        assert host(out)[0] == loss and host(g)[0, 0] == q and host(g)[1, 1] == -q
    stats = torch.full((4,), 9.0, device="cuda")
    cd.conduit_preference_loss(cd.preference_opts(), torch.empty((0, 4), device="cuda"), torch.empty(0, device="cuda"), stats)
    assert (stats == 0).all()


# ---------------------------------------------------------------------------
# workspaces, streams, graphs
# ---------------------------------------------------------------------------
def test_one_workspace_for_every_call():
    """Calls of every kind and of growing and shrinking sizes leave a workspace as they found it."""
    rng = np.random.default_rng(5)
    ws = cd.workspace(1 << 20)
    for B, T, V in [(2, 30, 2000), (300, 40, 18), (3, 2, 50000), (1, 20000, 4), (40, 7, 600)]:
        x, z = _logits(rng, B, T, V, F32)
        tok = rng.integers(0, V, (B, T)).astype(np.int32)
        mask = _mask(rng, B, T)
        q = _policy_inputs(rng, B, T)
        dev = {k: _gpu(v) for k, v in q.items()}
        f = lambda: torch.empty((B, T), device="cuda")  # noqa: E731
        for w in (ws, None):
            res = []
            lp, en, stats, dx = f(), f(), torch.empty(8, device="cuda"), torch.empty_like(x)
            opts = cd.policy_opts(kl_coef=0.1, reduction="sequence_mean")
            cd.conduit_token_logprobs(x, _gpu(tok), lp, mask=_gpu(mask), workspace=w)
            res += [lp.clone()]
            cd.conduit_policy_loss_logits(opts, x, _gpu(tok), dev["adv"], stats, dx, lp, en, old_logp=dev["old"],
                                          ref_logp=dev["ref"], mask=_gpu(mask), workspace=w)
            res += [lp.clone(), en, stats.clone(), dx]
            g = f()
            cd.conduit_policy_loss(opts, dev["logp"], dev["adv"], stats, g, old_logp=dev["old"], mask=_gpu(mask), workspace=w)
            res += [stats.clone(), g]
            if B % 2 == 0:
                loss, s4, pg = torch.empty(B // 2, device="cuda"), torch.empty(4, device="cuda"), f()
                cd.conduit_preference_loss(cd.preference_opts(), dev["logp"], loss, s4, pg, ref_logp=dev["ref"],
                                           mask=_gpu(mask), workspace=w)
                res += [loss, s4, pg]
            if w is not None:
                first = res
        for a, b in zip(first, res):
            assert torch.equal(a, b)


def test_calls_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(9)
    B, T, V = 6, 40, 9000
    x, z = _logits(rng, B, T, V, BF16)
    tok, mask = _gpu(rng.integers(0, V, (B, T)).astype(np.int32)), _gpu(_mask(rng, B, T))
    dev = {k: _gpu(v) for k, v in _policy_inputs(rng, B, T).items()}
    opts = cd.policy_opts(kl_coef=0.1, entropy_coef=0.01)
    ws = cd.workspace(cd.policy_loss_logits_workspace(x))
    lp, en, stats, dx = (torch.empty((B, T), device="cuda"), torch.empty((B, T), device="cuda"),
                         torch.empty(8, device="cuda"), torch.empty_like(x))

    def call(stream=None):
        cd.conduit_policy_loss_logits(opts, x, tok, dev["adv"], stats, dx, lp, en, old_logp=dev["old"], ref_logp=dev["ref"],
                                      mask=mask, workspace=ws, stream=stream)

    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in (lp, en, stats, dx)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    side.synchronize()
    for a, b in zip((lp, en, stats, dx), want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(3):
        dev["adv"].mul_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (lp, en, stats, dx)]
        call()
        torch.cuda.synchronize()
        for a, b in zip(got, (lp, en, stats, dx)):
            assert torch.equal(a, b), k


@pytest.mark.parametrize("n", [600, 20000])
def test_ratios_and_divergences_beyond_the_type(n):
    """exp of every argument past 88.73 is infinity, never NaN: a clipped token's loss and gradient stay finite, and
    the means of the ratio and of the divergence say infinity.  (Both sizes, so that both kernels of the loss run.)"""
    rng = np.random.default_rng(n)
    x = np.concatenate([rng.uniform(88.8, 1e3, n // 2), rng.uniform(1e3, 1e6, n - n // 2)]).astype(np.float32)[None]
    adv = rng.integers(-1, 2, (1, n)).astype(np.float32)
    zero = torch.zeros((1, n), device="cuda")
    stats, g = torch.empty(8, device="cuda"), torch.empty((1, n), device="cuda")
    cd.conduit_policy_loss(cd.policy_opts(dual_clip=3.0, reduction="sum"), _gpu(x), _gpu(adv), stats, g, old_logp=zero)
    s = host(stats)
    want = -1.2 * (adv > 0).sum() + 3.0 * (adv < 0).sum()
    assert abs(s[1] - want) <= 2.0 ** -20 * 3.0 * n and abs(s[0] - want) <= 2.0 ** -20 * 3.0 * n
    assert s[6] == np.inf and not host(g).any()
    cd.conduit_policy_loss(cd.policy_opts(kl_coef=0.1, reduction="sum"), zero, zero, stats, g, ref_logp=_gpu(x))
    s = host(stats)
    assert s[1] == 0.0 and s[2] == np.inf and s[0] == np.inf and (host(g) == -np.inf).all()


def test_ratios_up_to_the_type_s_largest():
    """Below the overflow exp is right to a few units of the last place, whatever the argument (2^-21: the instruction's
    unit, the two products', and half of one for the sum's)."""
    x = np.random.default_rng(5).uniform(-87.0, 88.7, 4000).astype(np.float32)
    stats, one = torch.empty((len(x), 8), device="cuda"), torch.ones((1, 1), device="cuda")
    lp = _gpu(x)
    opts, zero, g = cd.policy_opts(reduction="sum"), torch.zeros((1, 1), device="cuda"), torch.empty((1, 1), device="cuda")
    for i in range(len(x)):
        cd.conduit_policy_loss(opts, lp[i].view(1, 1), one, stats[i], g, old_logp=zero)
    want = np.exp(x.astype(np.float64))
    assert (np.abs(host(stats)[:, 6] - want) <= 2.0 ** -21 * want).all()
