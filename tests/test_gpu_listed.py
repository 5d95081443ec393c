"""Top alternatives, log-probabilities of listed choices, their gradient and the
distillation loss through the Python binding against the 64-bit forms of
oracle/losses.py: every kernel a row's width and the batch's size select, ties,
masks, entries that are no choices, numbers listed twice, strides, in-place
gradients, workspaces handed on, graphs and streams.

Tolerances.  As in test_gpu_losses.py, 2^-24 (8 R + 128) =: e bounds a
log-probability of rows with scores spread over R powers of two, a listed one as
well as that of the rest (the same sums and logarithms).  The divergence is a sum
of a (exp s - 1 - s) with s = log(b / a): its derivative by s is b - a, of absolute
sum at most 2, s is off by at most 2 e, and each term is rounded to 2^-22 (b + a (1 +
|s|)), so with U the largest |s|, 4 e (1 + U) bounds it.  A gradient of the
divergence is w / temperature times p (1 + exp u_rest) or q (1 + U) to first order
in u, so 8 e (1 + U) (p (1 + exp u_rest) + q) w / temperature.  bf16 adds half a
step, 2^-8 of the value."""
import numpy as np
import pytest
import torch

from gpu_util import host
from oracle import losses as ref

pytestmark = pytest.mark.gpu

from paper_2609_24456_amd import conduit as cd  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
NAN = float("nan")


def _gpu(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def _f(a):
    return _gpu(np.asarray(a, np.float32))


def _logits(rng, B, T, V, dtype, spread=3.0):
    """(device tensor, the same values in 64 bits)"""
    x = torch.from_numpy((spread * rng.standard_normal((B, T, V))).astype(np.float32)).to(dtype)
    return x.cuda(), x.double().numpy()


def _mask(rng, B, T):
    m = (rng.random((B, T)) < 0.7).astype(np.uint8) * rng.integers(1, 256, (B, T)).astype(np.uint8)
    if B > 1:
        m[B // 2] = 0
    return m


def _bound(z, temperature=1.0):
    fin = np.where(np.isfinite(z), z, 0.0) / temperature * 1.4427
    return 2.0 ** -24 * (8 * (fin.max() - fin.min() + np.abs(fin).max()) + 128)


def _close(got, want, tol):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        bad = ~same & ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


def _step(dtype, want):
    return 2.0 ** -8 * np.abs(np.where(np.isfinite(want), want, 0.0)) if dtype == BF16 else 0.0


# one choice, rows of a wavefront (8 and 32 elements a lane) and their edges, of a workgroup with and without elements
# after the last vector, wide enough to be split where there are few of them
WIDTHS = [1, 2, 3, 16, 17, 18, 32, 33, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1000, 2047, 2048, 2049, 4095, 4097, 4103, 5001, 16385, 33001]


def _shape(V):
    """Fewer rows than compute units where wide (these are split), else more."""
    return (3, 7) if V > 6000 else (4, 81)


# ---------------------------------------------------------------------------
# alternatives
# ---------------------------------------------------------------------------
def _alternatives(x, K, mask=None, temperature=1.0, tokens=None, values=True, **kw):
    shape = tuple(x.shape[:-1])
    ids = torch.full(shape + (K,), -7, dtype=torch.int32, device="cuda")
    logps = torch.full(shape + (K,), NAN, device="cuda")
    out = [torch.full(shape, NAN, device="cuda") if values and (tokens is not None or i) else None for i in range(3)]
    cd.conduit_token_alternatives(x, ids, logps, tokens=tokens, logp=out[0], lse=out[1], entropy=out[2], mask=mask,
                                  temperature=temperature, **kw)
    return host(ids), host(logps), [None if o is None else host(o) for o in out]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", WIDTHS)
def test_alternatives(V, dtype):
    rng = np.random.default_rng(V)
    B, T = _shape(V)
    tau = 0.7
    x, z = _logits(rng, B, T, V, dtype)
    mask, tok = _mask(rng, B, T), rng.integers(0, V, (B, T)).astype(np.int32)
    tol = _bound(z, tau)
    scores = ref.token_logprobs(z, tok, mask, tau)
    for K in (1, 5, 64, 128):
        want = ref.alternatives(z, K, mask, tau)
        ids, logps, out = _alternatives(x, K, _gpu(mask), tau, _gpu(tok))
        assert (ids == want[0]).all()
        _close(logps, want[1], tol)
        for g, w, k in zip(out, scores, (1, 1, 2)):
            _close(g, w, k * tol)
    ids, logps, _ = _alternatives(x, 5, _gpu(mask), tau, values=False)  # nothing but the choices
    assert (ids == ref.alternatives(z, 5, mask, tau)[0]).all()


def _hard_rows(rng, V, dtype):
    """[rows, V]: ties, orders and places that the candidates of a row may be too many for."""
    j = np.arange(V, dtype=np.float64)
    low = float(torch.finfo(dtype).min)
    r = [np.zeros(V), np.full(V, -np.inf), np.full(V, low), j / V, -j / V, rng.integers(0, 3, V), -rng.integers(0, 40, V) / 8.0,
         np.where(j % 512 < 8, 5.0 + j / V, rng.standard_normal(V)),          # in few lanes
         np.where(j % 2048 < 64, 9.0, rng.standard_normal(V)),                # the same, equal
         np.where(j >= V - 200, 3.0, rng.standard_normal(V) - 9),             # equal at the end
         np.where(j < V - 1, -np.inf, 2.0), np.where(j > 0, -np.inf, 2.0),
         np.where(rng.random(V) < 0.99, -np.inf, rng.standard_normal(V)),
         np.where(rng.random(V) < 0.5, 0.0, -0.0), 30000.0 + 3 * rng.standard_normal(V), 1e-3 * rng.standard_normal(V) + 1,
         1e-39 * rng.standard_normal(V)]
    a = np.stack(r)
    x = torch.from_numpy(a.astype(np.float32)).to(dtype)
    return x, x.double().numpy()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [3, 18, 130, 300, 513, 700, 2048, 2049, 4103, 5000, 40000])
@pytest.mark.parametrize("rows", ["few", "many"])
def test_alternatives_of_equal_and_ordered_scores(rows, V, dtype):
    rng = np.random.default_rng(V)
    x, z = _hard_rows(rng, V, dtype)
    if rows == "many":
        if V == 40000:
            x, z = x[:10], z[:10]
        k = -(-300 // len(x))
        x, z = x.repeat(k, 1), np.tile(z, (k, 1))
    n = len(z) if rows == "few" else len(z) // k
    for K in (1, 20, 64, 128):
        want = ref.alternatives(z[:n], K)
        ids, logps, _ = _alternatives(x.cuda(), K)
        for b in range(0, len(z), n):  # (the rows repeat)
            bad = np.argwhere((ids[b:b + n] != want[0]).any(-1))
            assert not bad.size, (K, bad.ravel())
            for i in range(n):
                _close(logps[b + i], want[1][i], _bound(z[i]))


def test_alternatives_of_rows_without_a_ranking():
    """A NaN or +infinity: -1 and NaN, in every kernel and without a trace in other rows."""
    rng = np.random.default_rng(5)
    for V, T in ((7, 9), (300, 9), (1500, 9), (5000, 300), (40000, 9)):
        for dtype in (F32, BF16):
            x, z = _logits(rng, 1, T, V, dtype)
            x[0, 2, V // 3], x[0, 4, V - 1], x[0, 6] = NAN, float("inf"), NAN
            z = x.double().cpu().numpy()
            want = ref.alternatives(z, 6)
            ids, logps, out = _alternatives(x, 6, tokens=torch.zeros((1, T), dtype=torch.int32, device="cuda"))
            assert (ids == want[0]).all() and (np.isnan(logps) == np.isnan(want[1])).all()
            assert np.isnan(out[1][0, [2, 4, 6]]).all() and np.isfinite(out[1][0, [0, 1, 3, 5, 7, 8]]).all()


def _check_alternatives_on_device(x, K, ids, logps, rows):
    """Some rows of a large batch against torch's stable sort in 64 bits."""
    for b, t in rows:
        z = x[b, t].double()
        order = torch.sort(z, descending=True, stable=True).indices[:K]
        assert torch.equal(ids[b, t].long(), order), (b, t)
        want = (z - torch.logsumexp(z, -1))[order]
        tol = 2.0 ** -24 * (8 * 3 * 1.4427 * float(z.abs().max()) + 128)
        assert float((logps[b, t].double() - want).abs().max()) <= tol


@pytest.mark.parametrize("B,T,V,dtype", [(1, 1, 128001, BF16), (5, 1, 70002, F32), (1, 530, 131079, F32), (1, 3, 600001, BF16),
                                         (2, 129, 50003, BF16), (1, 2, 3000003, F32)])
def test_alternatives_of_wide_rows(B, T, V, dtype):
    """Split rows joined by their last workgroup, and, more than 512 of them, by a launch of its own."""
    x = torch.randn((B, T, V), generator=torch.Generator(device="cuda").manual_seed(V), device="cuda").mul_(3).to(dtype)
    x[0, 0, V - 1] = 50.0
    for K in (1, 50, 128):
        ids = torch.empty((B, T, K), dtype=torch.int32, device="cuda")
        logps = torch.empty((B, T, K), device="cuda")
        cd.conduit_token_alternatives(x, ids, logps)
        _check_alternatives_on_device(x, K, ids, logps, [(0, 0), (B - 1, T - 1), (B // 2, T // 2)])
    x[:] = 1.0  # all equal: the lowest numbers
    cd.conduit_token_alternatives(x, ids, logps)
    assert torch.equal(ids, torch.arange(K, dtype=torch.int32, device="cuda").expand(B, T, K))


# ---------------------------------------------------------------------------
# listed log-probabilities and their gradient
# ---------------------------------------------------------------------------
def _ids(rng, B, T, V, K):
    """Numbers with some twice, some negative, and rows of none, of one and of all different ones."""
    ids = rng.integers(0, V, (B, T, K)).astype(np.int32)
    ids[rng.random((B, T, K)) < 0.1] = -1
    ids[0, 0] = -3
    ids[0, -1] = V - 1
    n = min(K, V)
    ids[-1, 0, :n] = rng.permutation(V)[:n]
    return ids


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", WIDTHS)
def test_listed_logprobs_and_gradient(V, dtype):
    rng = np.random.default_rng(V + 1)
    B, T = _shape(V)
    tau = 0.7
    x, z = _logits(rng, B, T, V, dtype)
    mask = _mask(rng, B, T)
    tol = _bound(z, tau)
    for K in (1, 7, 64, 128):
        ids = _ids(rng, B, T, V, K)
        want = ref.listed_logprobs(z, ids, mask, tau)
        out = [torch.full(s, NAN, device="cuda") for s in ((B, T, K), (B, T), (B, T))]
        cd.conduit_listed_logprobs(x, _gpu(ids), out[0], rest=out[1], lse=out[2], mask=_gpu(mask), temperature=tau)
        for g, w in zip(out, want):
            _close(host(g), w, tol)
        if K == 64:
            continue
        g, h = rng.standard_normal((B, T, K)).astype(np.float32), rng.standard_normal((B, T)).astype(np.float32)
        g[ids < 0] = NAN  # (not read into anything)
        gz = np.where(ids < 0, 0.0, g)
        logp = np.where(np.isfinite(z), z, -np.inf) / tau - want[2][..., None]
        for hh in (None, h):
            dx = torch.full_like(x, NAN)
            cd.conduit_listed_logprobs_backward(x, _gpu(ids), _f(want[2]), _gpu(g), dx, rest=None if hh is None else _f(want[1]),
                                                drest=None if hh is None else _gpu(hh), mask=_gpu(mask), temperature=tau)
            w = ref.listed_gradient(z, ids, gz, None if hh is None else hh, mask, tau)
            size = (np.abs(gz).sum(-1) + (0 if hh is None else np.abs(hh)))[..., None] * (np.exp(logp) + 2.0 ** -24)
            if hh is not None:
                size += np.abs(hh)[..., None] * np.exp(np.minimum(logp - np.where(np.isfinite(want[1]), want[1], 0.0)[..., None], 0))
            for k in range(K):
                np.add.at(size, (*np.indices((B, T)), np.maximum(ids[..., k], 0)), np.abs(gz[..., k]))
            _close(host(dx.float()), w, 4 * tol * size / tau + _step(dtype, w))


def test_rows_with_a_nan_or_infinity():
    """NaN in every output of the row, whether the list holds it or not or the row is nothing else; the others as ever."""
    rng = np.random.default_rng(8)
    for V, B, T in ((18, 1, 9), (300, 1, 9), (2100, 1, 9), (9000, 1, 300), (40000, 1, 9)):
        for dtype in (F32, BF16):
            x, _ = _logits(rng, B, T, V, dtype)
            ids, y = _teacher(rng, x.double().cpu().numpy(), 5)
            inside, outside = int(ids[0, 1, 2]), next(j for j in range(V) if j not in ids[0, 2])
            x[0, 1, inside], x[0, 2, outside], x[0, 3, int(ids[0, 3, 0])], x[0, 4], x[0, 5, V - 1] = NAN, NAN, float("inf"), NAN, float("inf")
            bad = np.zeros((B, T), bool)
            bad[0, 1:6] = True
            out = [torch.zeros(s, device="cuda") for s in ((B, T, 5), (B, T), (B, T))]
            cd.conduit_listed_logprobs(x, _gpu(ids), out[0], rest=out[1], lse=out[2])
            assert (np.isnan(host(out[0])).all(-1) == bad).all() and (np.isnan(host(out[0])).any(-1) == bad).all()
            assert (np.isnan(host(out[2])) == bad).all()
            dx = torch.zeros_like(x)
            cd.conduit_listed_logprobs_backward(x, _gpu(ids), out[2], _gpu(y), dx)
            assert (np.isnan(host(dx.float())).all(-1) == bad).all() and (np.isnan(host(dx.float())).any(-1) == bad).all()
            for opts in FORMS:
                dx.zero_()
                loss, stats = _distill(cd.distill_opts(**opts), x, ids, y, dx)
                assert (np.isnan(loss) == bad).all() and np.isnan(stats[:2]).all() and stats[2] == B * T
                assert (np.isnan(host(dx.float())).all(-1) == bad).all() and (np.isnan(host(dx.float())).any(-1) == bad).all()
                assert (np.isnan(_distill(cd.distill_opts(**opts), x, ids, y)[0]) == bad).all()


def test_rest_far_below_the_listed():
    """A rest of 1e-8 to 1e-30 of the row keeps its digits, in every kernel; nothing left is -infinity."""
    for V in (40, 700, 5000, 40000):
        for dtype in (F32, BF16):
            rng = np.random.default_rng(V)
            x, z = _logits(rng, 2, 5, V, dtype, spread=1.0)
            ids = np.stack([rng.permutation(V)[:9] for _ in range(10)]).reshape(2, 5, 9).astype(np.int32)
            for i, lead in enumerate((18.0, 30.0, 45.0, 60.0, 80.0)):
                for b in range(2):
                    x[b, i, torch.from_numpy(ids[b, i].astype(np.int64)).cuda()] += lead
            x[1, 4] = -np.inf
            x[1, 4, int(ids[1, 4, 3])] = 1.0
            z = x.double().cpu().numpy()
            want = ref.listed_logprobs(z, ids)
            out = [torch.empty(s, device="cuda") for s in ((2, 5, 9), (2, 5), (2, 5))]
            cd.conduit_listed_logprobs(x, _gpu(ids), out[0], rest=out[1], lse=out[2])
            for g, w in zip(out, want):
                _close(host(g), w, _bound(z))
            assert want[1][1, 4] == -np.inf
            g, h = rng.standard_normal((2, 5, 9)).astype(np.float32), rng.standard_normal((2, 5)).astype(np.float32)
            dx = torch.full_like(x, NAN)
            cd.conduit_listed_logprobs_backward(x, _gpu(ids), _f(want[2]), _gpu(g), dx, rest=_f(want[1]), drest=_gpu(h))
            w = ref.listed_gradient(z, ids, g, h)
            _close(host(dx.float()), w, 4 * _bound(z) * (np.abs(g).sum(-1) + np.abs(h))[..., None] + _step(dtype, w))


# ---------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------
def _teacher(rng, z, K, noise=1.0):
    """A teacher's K best choices and log-probabilities: the student's scores with noise."""
    y = z + noise * rng.standard_normal(z.shape)
    ids = np.argsort(-y, -1, kind="stable")[..., :K]
    lse = np.log(np.exp(y - y.max(-1, keepdims=True)).sum(-1, keepdims=True)) + y.max(-1, keepdims=True)
    logq = (np.take_along_axis(y, ids, -1) - lse).astype(np.float32)
    if ids.shape[-1] < K:  # fewer choices: entries without one
        pad = [(0, 0)] * (ids.ndim - 1) + [(0, K - ids.shape[-1])]
        ids, logq = np.pad(ids, pad, constant_values=-1), np.pad(logq, pad)
    return ids.astype(np.int32), logq


def _distill(opts, x, ids, y, dx=None, **kw):
    loss, stats = torch.full(ids.shape[:-1], NAN, device="cuda"), torch.full((3,), NAN, device="cuda")
    cd.conduit_distill_loss(opts, x, _gpu(ids), _gpu(y), loss, stats, dlogits=dx, **kw)
    return host(loss), host(stats)


def _check_distill(x, z, ids, y, mask, weight, tau, dtype, opts, in_place=False, **kw):
    sizes = []
    want = ref.distill_loss(z, ids, y, mask=mask, weight=weight, temperature=tau, sizes=sizes, **opts)
    dx = x.clone() if in_place else torch.full_like(x, NAN)
    loss, stats = _distill(cd.distill_opts(**opts), dx if in_place else x, ids, y, dx, mask=None if mask is None else _gpu(mask),
                           weight=None if weight is None else _gpu(weight), temperature=tau, **kw)
    e = _bound(z, tau)
    tol, size, mean = np.zeros(loss.shape), np.zeros(z.shape), 0.0
    for at, w, p, js, q, U, rest in sizes:
        tol[at] = 4 * e * (1 + U)
        size[at] = p * (1 + rest)
        size[at][js] += q
        size[at] *= 8 * e * (1 + U) * abs(w) / tau
        mean += abs(w) * tol[at]
    _close(loss, want[0], tol)
    _close(stats[0], want[1][0], mean + 2.0 ** -23 * abs(want[1][0]))
    _close(stats[1], want[1][1], tol.max() + 2.0 ** -23 * abs(want[1][1]))
    assert stats[2] == want[1][2]
    _close(host(dx.float()), want[2], abs(opts.get("scale", 1.0)) * size + 1e-44 + _step(dtype, want[2]))
    return loss, stats


FORMS = [dict(loss="forward", teacher_temperature=2.0), dict(loss="forward", rest=True, reduction="sequence_mean", scale=1.5),
         dict(loss="reverse", rest=True, reduction="sum", scale=0.01)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", WIDTHS)
def test_distill_loss(V, dtype):
    rng = np.random.default_rng(V + 2)
    B, T = _shape(V)
    tau = 0.8
    x, z = _logits(rng, B, T, V, dtype)
    mask = _mask(rng, B, T)
    weight = rng.random((B, T)).astype(np.float32)
    weight[mask == 0] = NAN  # (not read)
    weight[0, 0] = 0.0
    for i, opts in enumerate(FORMS):
        ids, y = _teacher(rng, z, (1, 40, 128)[i])
        loss, stats = _check_distill(x, z, ids, y, mask, weight if i else None, tau, dtype, opts, in_place=i == 1)
        again = _distill(cd.distill_opts(**opts), x, ids, y, mask=_gpu(mask), weight=_gpu(weight) if i else None, temperature=tau)
        _close(again[0], loss, 8 * _bound(z, tau) * (1 + np.abs(loss)) + 8 * _bound(z, tau) * 20)  # without the gradient


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [1, 2, 5, 16, 17, 33, 63, 64])
def test_rows_that_share_a_wavefront(V, dtype):
    """Many rows of few choices: a part of a wavefront each, some of them masked, empty, with numbers twice or not finite."""
    rng = np.random.default_rng(V)
    B, T, tau = 6, 119, 0.8
    x, _ = _logits(rng, B, T, V, dtype)
    x[1, 5], x[1, 6, V // 2], x[2, 7] = -np.inf, -np.inf, -np.inf
    z = x.double().cpu().numpy()
    mask = _mask(rng, B, T)
    for K in (1, 16, 17, 32, 33):
        ids = _ids(rng, B, T, V, K)
        want = ref.listed_logprobs(z, ids, mask, tau)
        out = [torch.full(s, NAN, device="cuda") for s in ((B, T, K), (B, T), (B, T))]
        cd.conduit_listed_logprobs(x, _gpu(ids), out[0], rest=out[1], lse=out[2], mask=_gpu(mask), temperature=tau)
        for g, w in zip(out, want):
            _close(host(g), w, _bound(z, tau))
    weight = rng.random((B, T)).astype(np.float32)
    weight[mask == 0] = NAN
    for i, opts in enumerate(FORMS):
        ids, y = _teacher(rng, np.where(np.isfinite(z), z, -20.0), (3, 20, 32)[i])
        ids[0, ::3] = np.where(rng.random(ids[0, ::3].shape) < 0.3, ids[0, ::3, :1], ids[0, ::3])
        y[3, ::4, 0] = -np.inf
        ids[4, ::5] = -1
        if opts["loss"] == "reverse":  # (a teacher's choice at -inf of the student's would be infinite only forward)
            ids[1, 6] = -1
        for m in (mask, None):
            loss, stats = _check_distill(x, z, ids, y, m, np.nan_to_num(weight, nan=0.5) if m is None else weight, tau, dtype, opts,
                                         in_place=i == 1)


def test_many_rows_that_share_a_wavefront():
    """The same bits from one large batch as from its halves."""
    rows, V, K = 36000, 18, 7
    g = torch.Generator(device="cuda").manual_seed(2)
    for dtype in (F32, BF16):
        x = torch.randn((1, rows, V), generator=g, device="cuda").mul_(2).to(dtype)
        ids = torch.randint(-1, V, (1, rows, K), generator=g, device="cuda", dtype=torch.int32)
        y = torch.log_softmax(torch.randn((1, rows, K), generator=g, device="cuda"), -1) - 0.1
        mask = (torch.rand((1, rows), generator=g, device="cuda") < 0.6).to(torch.uint8)
        outs = [[torch.full_like(t, 9) for t in (x, y[..., 0], y, y[..., 0])] for _ in range(2)]
        stats = torch.empty((3, 3), device="cuda")
        opts = cd.distill_opts(rest=True, reduction="sum")
        parts = [slice(0, rows), slice(0, rows // 2), slice(rows // 2, rows)]
        for i, h in enumerate(parts):
            dx, loss, logps, rest = outs[min(i, 1)]
            cd.conduit_distill_loss(opts, x[:, h], ids[:, h], y[:, h], loss[:, h], stats[i], dlogits=dx[:, h], mask=mask[:, h])
            cd.conduit_listed_logprobs(x[:, h], ids[:, h], logps[:, h], rest=rest[:, h], mask=mask[:, h])
        for a, b in zip(*outs):
            assert torch.equal(a, b)
        s = host(stats).astype(np.float64)
        _close(s[0, 0], s[1, 0] + s[2, 0], 2.0 ** -22 * s[0, 0])
        assert s[0, 2] == s[1, 2] + s[2, 2] == int(mask.sum())


@pytest.mark.parametrize("V", [6, 50, 900, 5000, 40000])
@pytest.mark.parametrize("opts", FORMS)
def test_distill_entries_that_do_not_count(V, opts):
    """Numbers twice, negative ones, values of -infinity; a token without entries, one with all choices listed; rows of
    -infinity alone and with choices at -infinity."""
    for dtype in (F32, BF16):
        rng = np.random.default_rng(V)
        T, K = 9, 12
        x, _ = _logits(rng, 2, T, V, dtype)
        x[0, 3, :V // 2] = -np.inf
        x[1, 5] = -np.inf
        x[1, 6, 1:] = -np.inf
        z = x.double().cpu().numpy()
        ids, y = _teacher(rng, np.where(np.isfinite(z), z, -20.0), K)
        ids[0, 0, 3:6] = ids[0, 0, 0]
        ids[0, 1, 1] = -5
        y[0, 2, 0] = -np.inf
        ids[0, 2, 1], y[0, 2, 1] = ids[0, 2, 0], -2.0  # the first of its number that has a value
        ids[0, 4] = -1
        y[0, 5] = -np.inf
        ids[1, 0] = ids[1, 0, 0]
        ids[1, 6] = np.where(np.arange(K) == 0, 0, -1)
        ids[1, 7], y[1, 7] = rng.permutation(max(V, K))[:K] % V, np.float32(np.log(1 / 13))
        if opts["loss"] == "reverse":
            ids[0, 3] = np.where(ids[0, 3] < V // 2, -1, ids[0, 3])
        _check_distill(x, z, ids, y, None, None, 1.0, dtype, opts)


def test_distill_of_near_and_far_students():
    """Students at the teacher (divergences far below the scores' rounding), close to it, and far away."""
    for V in (30, 1000, 5000):
        for opts in FORMS:
            rng = np.random.default_rng(V)
            x, z = _logits(rng, 2, 20, V, F32)
            for noise in (0.0, 1e-3, 0.1, 5.0):
                ids, y = _teacher(rng, z, min(V - 1, 24), noise)
                _check_distill(x, z, ids, y, None, None, 1.0, F32, dict(opts, teacher_temperature=1.0))


@pytest.mark.parametrize("V", [30, 300, 3000, 30000])
def test_distill_from_logits_far_from_zero(V):
    """A teacher's values may be logits of any offset: their differences count, not their size."""
    rng = np.random.default_rng(V)
    x, z = _logits(rng, 2, 10, V, F32)
    ids, y = _teacher(rng, z, 20)
    for offset, tau in ((3e4, 2.0), (-1e5, 0.7)):
        _check_distill(x, z, ids, (y + np.float32(offset)).astype(np.float32), None, None, 1.0, F32,
                       dict(loss="forward", teacher_temperature=tau))


@pytest.mark.parametrize("B,T,V,dtype", [(1, 530, 70001, F32), (3, 2, 140003, BF16), (2, 300, 9001, BF16), (700, 1, 2049, F32),
                                         (1, 300, 4096, F32), (1, 300, 8001, F32), (2, 150, 8203, BF16), (7, 171, 2050, BF16), (4, 512, 700, F32), (1, 2049, 700, F32), (1, 300, 16385, F32),
                                         (1, 300, 20001, BF16), (3, 100, 30003, F32), (1, 300, 50001, BF16), (1, 300, 40005, F32),
                                         (1, 300, 100007, BF16), (1, 520, 131072, BF16)])
def test_distill_of_many_and_wide_rows(B, T, V, dtype):
    """Rows of every number of wavefronts and wider than a workgroup's registers (more than 512 of these joined by a launch
    of its own), sums of many rows."""
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn((B, T, V), generator=g, device="cuda").mul_(3).to(dtype)
    mask = (torch.rand((B, T), generator=g, device="cuda") < 0.3).to(torch.uint8)
    mask[0, 0] = mask[-1, -1] = 1
    best, ids = torch.topk(x.float() + torch.randn((B, T, V), generator=g, device="cuda"), 30, dim=-1)
    ids, y = ids.int(), torch.log_softmax(best, -1) - 0.1
    dx, loss, stats = torch.full_like(x, NAN), torch.empty((B, T), device="cuda"), torch.empty(3, device="cuda")
    for opts in FORMS:
        opts = dict(opts, teacher_temperature=1.0)
        dx.fill_(NAN)
        cd.conduit_distill_loss(cd.distill_opts(**opts), x, ids, y, loss, stats, dlogits=dx, mask=mask)
        total = 0.0
        n = int(mask.sum())
        rows = int((mask != 0).any(1).sum())
        for b, t in [(0, 0), (B - 1, T - 1)] + np.argwhere(host(mask)).tolist()[:6]:
            z = x[b, t].double().cpu().numpy()[None, None]
            o = dict(opts, reduction="sum")
            sizes = []
            want = ref.distill_loss(z, host(ids[b, t])[None, None], host(y[b, t])[None, None], sizes=sizes, **o)
            w = {"token_mean": 1 / n, "sequence_mean": 1 / (rows * max(1, int(mask[b].sum()))), "sum": 1.0}[opts.get("reduction", "token_mean")]
            _, _, p, js, q, U, rest = sizes[0]
            e = 4 * _bound(z) * (1 + U)
            _close(host(loss[b, t]), want[0][0, 0], e)
            size = p * (1 + rest)
            size[js] += q
            d = want[2][0, 0] * w
            _close(host(dx[b, t].float()), d, 2 * e * w * opts.get("scale", 1.0) * size + 1e-44 + _step(dtype, d))
        on = host(mask) != 0
        assert (host(loss)[~on] == 0).all() and float(dx[mask == 0].abs().max()) == 0 and not bool(dx.isnan().any())
        per = on.sum(1, keepdims=True)
        wt = {"token_mean": on / n, "sequence_mean": on / (rows * np.maximum(per, 1)), "sum": on * 1.0}[opts.get("reduction", "token_mean")]
        l64 = host(loss).astype(np.float64)
        _close(host(stats), [opts.get("scale", 1.0) * (wt * l64).sum(), l64.sum() / n, n], 2.0 ** -23 * np.abs(host(stats)))


@pytest.mark.parametrize("V,dtype", [(700, F32), (2101, BF16), (9001, BF16), (20001, BF16), (30001, F32), (50001, BF16), (50001, F32), (100001, BF16), (140003, F32)])
def test_batches_larger_than_the_caches(V, dtype):
    """Their logits are read and gradients written another way: the same bits as from two calls of half the rows."""
    size = 4 if dtype == F32 else 2
    rows = (410 << 20) // (V * size) // 2 * 2
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn((1, rows, V), generator=g, device="cuda", dtype=dtype).mul_(3)
    ids = torch.randint(0, V, (1, rows, 20), generator=g, device="cuda", dtype=torch.int32)
    y = torch.log_softmax(torch.randn((1, rows, 20), generator=g, device="cuda"), -1) - 0.1
    mask = (torch.rand((1, rows), generator=g, device="cuda") < 0.6).to(torch.uint8)
    one, two = torch.full_like(x, NAN), torch.full_like(x, NAN)
    loss, stats, lse = torch.empty((1, rows), device="cuda"), torch.empty(3, device="cuda"), torch.empty((1, rows), device="cuda")
    halves = [slice(0, rows // 2), slice(rows // 2, rows)]
    outs = [[torch.full_like(t, 9) for t in (ids, y, lse, lse, y, lse)] for _ in range(2)]
    for parts, (top, lp, entropy, rest, logps, z) in zip(([slice(0, rows)], halves), outs):
        for h in parts:
            cd.conduit_token_alternatives(x[:, h], top[:, h], lp[:, h], entropy=entropy[:, h], mask=mask[:, h])
            cd.conduit_listed_logprobs(x[:, h], ids[:, h], logps[:, h], rest=rest[:, h], lse=z[:, h])
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    lse = z
    opts = cd.distill_opts(rest=True, reduction="sum")
    cd.conduit_distill_loss(opts, x, ids, y, loss, stats, dlogits=one, mask=mask)
    for h in halves:
        cd.conduit_distill_loss(opts, x[:, h], ids[:, h], y[:, h], loss[:, h], stats, dlogits=two[:, h], mask=mask[:, h])
    assert torch.equal(one, two)
    one.fill_(NAN)
    cd.conduit_listed_logprobs_backward(x, ids, lse, y, one, mask=mask)
    for h in halves:
        cd.conduit_listed_logprobs_backward(x[:, h], ids[:, h], lse[:, h], y[:, h], two[:, h], mask=mask[:, h])
    assert torch.equal(one, two) and not bool(one.isnan().any())


# ---------------------------------------------------------------------------
# layouts, workspaces, graphs, streams
# ---------------------------------------------------------------------------
def _all_calls(x, tok, ids, y, mask, tau=0.9, **kw):
    """Every call's outputs, in the layout of the arguments."""
    like = lambda t: torch.full_like(t, -9 if t.dtype == torch.int32 else NAN)  # noqa: E731
    top, lp = like(ids), like(y)
    t = [torch.empty_strided(tok.shape, tok.stride(), device="cuda").fill_(NAN) for _ in range(6)]
    cd.conduit_token_alternatives(x, top, lp, tokens=tok, logp=t[0], lse=t[1], entropy=t[2], mask=mask, temperature=tau, **kw)
    listed, dx, ddx, stats = like(y), like(x), like(x), torch.empty(3, device="cuda")
    cd.conduit_listed_logprobs(x, ids, listed, rest=t[3], lse=t[4], mask=mask, temperature=tau, **kw)
    back = {k: v for k, v in kw.items() if k != "workspace"}
    cd.conduit_listed_logprobs_backward(x, ids, t[4], y, dx, rest=t[3], drest=t[4], mask=mask, temperature=tau, **back)
    cd.conduit_distill_loss(cd.distill_opts(rest=True), x, ids, y, t[5], stats, dlogits=ddx, mask=mask, temperature=tau, **kw)
    return [top, lp, *t[:5], listed, dx, t[5], ddx, stats]


def _batch(rng, B, T, V, K, dtype):
    x, z = _logits(rng, B, T, V, dtype)
    ids, y = _teacher(rng, z, K)
    return x, _gpu(rng.integers(0, V, (B, T)).astype(np.int32)), _gpu(ids), _gpu(y), _gpu(_mask(rng, B, T))


def _padded(t, wide):
    """The same values as columns [:, 1:] (per-token) or rows [:, :-1] (of several elements) of a larger array."""
    if t.dim() == 2:
        big = torch.full((t.shape[0], t.shape[1] + 1), 77, dtype=t.dtype, device="cuda")
        big[:, 1:] = t
        return big[:, 1:]
    big = torch.full((t.shape[0], t.shape[1] + 1, t.shape[2] + wide), 77, dtype=t.dtype, device="cuda")
    big[:, :-1, 1:1 + t.shape[2]] = t
    return big[:, :-1, 1:1 + t.shape[2]]


def _equal(a, b):
    a, b = a.contiguous(), b.contiguous()
    return torch.equal(a, b) or torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [18, 700, 5001, 40003])
def test_strided_views_give_the_same(V, dtype):
    """Columns and rows of larger arrays, at odd element alignment; what lies around them stays.  Rows are summed in another
    order where they start elsewhere: each side is off from the exact value by at most the bounds above, so they are apart
    by at most twice these.  p (1 + exp u_rest) + q is at most 3 in these (p exp u_rest is a part of
    q_rest), U at most the largest |log q| and |log p|; a gradient's size is at most twice the sum of the |dlogps| and
    |drest| of its row."""
    rng = np.random.default_rng(V)
    B, T = (3, 5) if V > 6000 else (5, 70)
    plain = _batch(rng, B, T, V, min(9, V), dtype)
    want = _all_calls(*plain)
    views = [_padded(t, 3) for t in plain]
    got = _all_calls(*views)
    x, tok, ids, y, mask = plain
    on = host(mask) != 0
    e = _bound(x.double().cpu().numpy(), 0.9)
    logp = [host(want[i])[on] for i in (5, 7)]
    U = max(np.abs(v[np.isfinite(v)]).max() for v in logp + [host(y)[on]]) + 16  # (16: log q of a rest held at 2^-23)
    g = np.where(on, np.abs(host(y)).sum(-1) + np.abs(host(want[6])), 0.0)[..., None]
    loss = 8 * e * (1 + U)
    tols = [0, 2 * e, 2 * e, 2 * e, 4 * e, 2 * e, 2 * e, 2 * e, 16 * e * g / 0.9, loss, 6 * loss / on.sum() / 0.9, loss]

    def check(i, a, b):
        if i == 0:
            assert _equal(a, b)
        else:
            a, b = host(a.float()), host(b.float())
            _close(a, b, tols[i] + (2.0 ** -7 if dtype == BF16 and i in (8, 10) else 2.0 ** -22) * np.abs(b))

    for i, (a, b) in enumerate(zip(got, want)):
        check(i, a, b)
    for v, t in zip(views, plain):
        assert torch.equal(v, t)
    # outputs written into a larger array
    x, tok, ids, y, mask = views
    out = torch.full((B, T + 1, V + 3), 55.0, device="cuda").to(dtype)
    loss, stats = torch.full((B, T + 1), 55.0, device="cuda")[:, 1:], torch.empty(3, device="cuda")
    cd.conduit_distill_loss(cd.distill_opts(rest=True), x, ids, y, loss, stats, dlogits=out[:, :-1, 1:V + 1], mask=mask, temperature=0.9)
    check(10, out[:, :-1, 1:V + 1], want[10])
    assert bool((out[:, -1] == 55).all()) and bool((out[:, :, 0] == 55).all()) and bool((out[:, :, V + 1:] == 55).all())
    one = [t[0] for t in plain]  # one sequence, [T] and [T, K]
    assert _equal(_all_calls(*one)[0], want[0][0])


def test_gradient_in_place_and_runs_alike():
    """dlogits in the logits' place, and the same bits on every run, in every kernel."""
    for V, B, T in ((18, 4, 50), (900, 4, 50), (5001, 4, 80), (40003, 2, 6), (140003, 2, 3)):
        for dtype in (F32, BF16):
            rng = np.random.default_rng(V)
            x, tok, ids, y, mask = b = _batch(rng, B, T, V, 12, dtype)
            want = _all_calls(*b)
            for _ in range(3):
                for g, w in zip(_all_calls(*b), want):
                    assert _equal(g, w)
            a, c = x.clone(), x.clone()
            cd.conduit_listed_logprobs_backward(a, ids, want[6], y, a, rest=want[5], drest=want[6], mask=mask, temperature=0.9)
            assert _equal(a, want[8])
            loss, stats = torch.empty_like(want[9]), torch.empty(3, device="cuda")
            cd.conduit_distill_loss(cd.distill_opts(rest=True), c, ids, y, loss, stats, dlogits=c, mask=mask, temperature=0.9)
            assert _equal(c, want[10]) and _equal(loss, want[9])


def _need(x, K):
    return max(cd.token_alternatives_workspace(x, K), cd.listed_logprobs_workspace(x, K), cd.distill_loss_workspace(x, K),
               cd.token_logprobs_workspace(x), cd.policy_loss_logits_workspace(x))


def test_one_workspace_for_all_calls_in_turn():
    """Calls of different kinds and sizes leave a shared workspace ready for each other."""
    rng = np.random.default_rng(3)
    batches = [_batch(rng, B, T, V, 10, dtype) for B, T, V, dtype in
               ((2, 3, 40003, BF16), (4, 50, 300, F32), (1, 600, 5001, F32), (2, 2, 140003, F32), (5, 70, 2500, BF16))]
    want = [_all_calls(*b) for b in batches]
    ws = cd.workspace(max(_need(b[0], 10) for b in batches))
    for _ in range(2):
        for b, w in zip(batches, want):
            lp, ent, adv, stats = [torch.zeros(b[1].shape, device="cuda") for _ in range(3)] + [torch.empty(8, device="cuda")]
            cd.conduit_policy_loss_logits(cd.policy_opts(), b[0], b[1], adv, stats, torch.empty_like(b[0]), lp, ent, mask=b[4],
                                          workspace=ws)
            for g, v in zip(_all_calls(*b, workspace=ws), w):
                assert _equal(g, v)


def test_captured_and_replayed():
    """All calls in one graph, replayed with new inputs and eager calls between, each replay against eager calls."""
    rng = np.random.default_rng(4)
    for V, B, T, dtype in ((300, 3, 20, F32), (5001, 3, 100, BF16), (40003, 2, 4, BF16), (140003, 1, 3, F32)):
        batches = [_batch(rng, B, T, V, 10, dtype) for _ in range(3)]
        want = [_all_calls(*b) for b in batches]
        static = [t.clone() for t in batches[0]]
        ws = cd.workspace(_need(static[0], 10))
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            _all_calls(*static, workspace=ws)
        torch.cuda.current_stream().wait_stream(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = _all_calls(*static, workspace=ws)
        for i in (1, 2, 0, 1):
            for a, b in zip(static, batches[i]):
                a.copy_(b)
            graph.replay()
            torch.cuda.synchronize()
            eager = _all_calls(*batches[i])
            for g, w, e in zip(out, want[i], eager):
                assert _equal(g, w) and _equal(e, w)


def test_on_another_stream():
    rng = np.random.default_rng(6)
    b = _batch(rng, 2, 5, 40003, 10, BF16)
    want = _all_calls(*b)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):  # as torch's current stream
        got = _all_calls(*b)
    s.synchronize()
    for g, w in zip(got, want):
        assert _equal(g, w)


def test_flagged_numbers_and_tokens():
    """Numbers and tokens beyond the vocabulary are flagged and count as nothing."""
    rng = np.random.default_rng(7)
    for V, B, T in ((18, 2, 5), (900, 2, 5), (5001, 4, 80), (40003, 2, 5)):
        x, tok, ids, y, mask = _batch(rng, B, T, V, 6, F32)
        mask.fill_(1)
        for call in range(4):
            bad, gone = ids.clone(), ids.clone()
            bad[1, 2, 3], gone[1, 2, 3] = V, -1
            if call == 0:
                t = tok.clone()
                t[1, 2] = V
                top, lp, ls = torch.empty_like(ids), torch.empty_like(y), torch.empty(tok.shape, device="cuda")
                cd.conduit_token_alternatives(x, top, lp, tokens=t, lse=ls)
                assert not bool(top[1, 2].any()) and float(ls[1, 2]) == 0 and float(lp[1, 2].abs().max()) == 0
            else:
                res = []
                for i in (bad, gone):
                    lse, rest = [torch.empty(tok.shape, device="cuda") for _ in range(2)]
                    out = torch.empty_like(x if call > 1 else y)
                    if call == 1:
                        cd.conduit_listed_logprobs(x, i, out, rest=rest, lse=lse)
                    elif call == 2:
                        cd.conduit_listed_logprobs_backward(x, i, torch.logsumexp(x, -1), y, out)
                    else:
                        cd.conduit_distill_loss(cd.distill_opts(), x, i, y, lse, torch.empty(3, device="cuda"), dlogits=out)
                    res.append(out)
                    if i is bad:
                        assert cd.conduit_sync_check() == cd.ESTATE
                        cd.conduit_clear_error()
                assert _equal(*res)
            assert cd.conduit_sync_check() == (cd.ESTATE if call == 0 else cd.OK)
            cd.conduit_clear_error()


def test_empty_batches():
    for shape in ((0, 5), (3, 0)):
        x = torch.empty(shape + (50,), device="cuda")
        ids, y = torch.empty(shape + (4,), dtype=torch.int32, device="cuda"), torch.empty(shape + (4,), device="cuda")
        t, stats = torch.empty(shape, device="cuda"), torch.full((3,), NAN, device="cuda")
        cd.conduit_token_alternatives(x, ids, y, lse=t)
        cd.conduit_listed_logprobs(x, ids, y, lse=t)
        cd.conduit_listed_logprobs_backward(x, ids, t, y, x)
        cd.conduit_distill_loss(cd.distill_opts(), x, ids, y, t, stats, dlogits=x)
        assert host(stats).tolist() == [0, 0, 0]
    # a mask that leaves nothing
    x, tok, ids, y, mask = _batch(np.random.default_rng(1), 3, 9, 700, 5, F32)
    x.fill_(NAN)
    mask.zero_()
    for o in _all_calls(x, tok, ids, y, mask):
        assert float(o.abs().max()) == 0
