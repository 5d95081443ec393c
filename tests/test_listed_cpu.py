"""The calls on listed choices without a GPU: their 64-bit oracle against differences and closed forms, what the library
refuses before anything is enqueued (addresses are never followed), and what the binding refuses before anything reaches
the library."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import losses as ref
from paper_2609_24456_amd import conduit as cd

EPS = 1e-6
TOL = 1e-8  # of a central difference of step 1e-6: its square times a third derivative, and 2^-52 / 1e-6 of the value


def _differences(f, x, picks):
    out = []
    for at in picks:
        hi, lo = x.copy(), x.copy()
        hi[at] += EPS
        lo[at] -= EPS
        out.append((f(hi) - f(lo)) / (2 * EPS))
    return np.array(out)


def _picks(rng, shape, n=30):
    return [tuple(int(rng.integers(0, s)) for s in shape) for _ in range(n)]


IDS = np.array([[[1, 4, 6], [0, 0, 3], [-1, 2, 5]], [[3, 3, 3], [6, 5, 4], [-2, -1, -9]]])
MASK = np.array([[1, 1, 1], [1, 0, 1]])


def test_oracle_alternatives_are_a_stable_order():
    x = np.array([[[0.0, -0.0, 2.0, 2.0, -np.inf], [np.nan, 1, 2, 3, 4], [-np.inf] * 5, [1.0, 2.0, np.inf, 0.0, 0.0]]])
    ids, logps = ref.alternatives(x, 7)
    assert ids[0, 0].tolist() == [2, 3, 0, 1, 4, -1, -1] and ids[0, 2].tolist() == [0, 1, 2, 3, 4, -1, -1]
    assert (ids[0, [1, 3]] == -1).all() and np.isnan(logps[0, [1, 3]]).all() and (logps[0, 2] == -np.inf).all()
    assert np.isclose(np.exp(logps[0, 0]).sum(), 1.0, rtol=0, atol=1e-15) and logps[0, 0, 0] == logps[0, 0, 1]


@pytest.mark.parametrize("tau", [1.0, 0.6])
def test_oracle_listed_gradient_is_the_difference(tau):
    rng = np.random.default_rng(0)
    x = 2 * rng.standard_normal((2, 3, 7))
    g, h = rng.standard_normal(IDS.shape), rng.standard_normal((2, 3))

    def f(v):
        logps, rest, _ = ref.listed_logprobs(v, IDS, MASK, tau)
        return (np.where(np.isfinite(logps), logps, 0) * g).sum() + (h * rest)[MASK != 0].sum()

    want = ref.listed_gradient(x, IDS, g, h, MASK, tau)
    picks = _picks(rng, x.shape)
    assert np.allclose(_differences(f, x, picks), [want[p] for p in picks], rtol=0, atol=TOL)


def test_oracle_rest_is_what_the_list_leaves():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((2, 3, 7))
    logps, rest, lse = ref.listed_logprobs(x, IDS)
    for at in np.ndindex(2, 3):
        p = np.exp(x[at] - lse[at])
        js = sorted({j for j in IDS[at] if j >= 0})
        assert np.isclose(np.exp(rest[at]), 1 - p[js].sum(), rtol=0, atol=1e-14)


FORMS = [dict(loss="forward", teacher_temperature=1.7), dict(loss="forward", rest=True, reduction="sequence_mean", scale=1.5),
         dict(loss="reverse", rest=True, reduction="sum", scale=0.3)]


@pytest.mark.parametrize("opts", FORMS)
def test_oracle_distill_gradient_is_the_difference(opts):
    rng = np.random.default_rng(1)
    x = 2 * rng.standard_normal((2, 3, 7))
    y, weight = np.log(rng.random(IDS.shape) / 4), rng.random((2, 3))
    kw = dict(opts, weight=weight, mask=MASK, temperature=0.8)
    want = ref.distill_loss(x, IDS, y, **kw)[2]
    picks = _picks(rng, x.shape)
    got = _differences(lambda v: ref.distill_loss(v, IDS, y, **kw)[1][0], x, picks)
    assert np.allclose(got, [want[p] for p in picks], rtol=0, atol=TOL)


def test_oracle_distill_by_hand():
    x = np.log(np.array([[[0.5, 0.25, 0.125, 0.125]]]))
    ids, y = np.array([[[1, 0]]]), np.log(np.array([[[0.5, 0.25]]]))
    q, p = [2 / 3, 1 / 3], [0.25, 0.5]
    assert np.allclose(ref.distill_loss(x, ids, y)[0], sum(a * np.log(a / b) for a, b in zip(q, p)))
    q, p = [0.5, 0.25, 0.25], [0.25, 0.5, 0.25]
    assert np.allclose(ref.distill_loss(x, ids, y, rest=True)[0], sum(a * np.log(a / b) for a, b in zip(q, p)))
    assert np.allclose(ref.distill_loss(x, ids, y, rest=True, loss="reverse")[0], sum(b * np.log(b / a) for a, b in zip(q, p)))
    # the teacher's whole row listed, the student at it: nothing, and no gradient
    same = ref.distill_loss(x, np.array([[[3, 1, 0, 2]]]), x[..., [3, 1, 0, 2]], rest=True)
    assert np.abs(same[0]).max() < 1e-15 and np.abs(same[2]).max() < 1e-15


# ---------------------------------------------------------------------------
# refusals of the library
# ---------------------------------------------------------------------------
def at(k, off=0):
    return C.c_void_p((k << 24) + off)


B, T, V, K = 3, 4, 8, 2
WS, BIG = at(99), 1 << 20


def rows(data=at(1), dtype=cd.F32, width=V, stride_b=None, stride_t=None):
    r = cd.Rows()
    r.data, r.dtype, r.width = data, dtype, width
    r.stride_t = width if stride_t is None else stride_t
    r.stride_b = T * width if stride_b is None else stride_b
    return C.byref(r)


def ids(data=at(2), dtype=cd.I32, width=K, **kw):
    return rows(data, dtype, width, **kw)


def vals(data=at(3), dtype=cd.F32, width=K, **kw):
    return rows(data, dtype, width, **kw)


def alternatives(x=None, i=None, lps=None, B=B, T=T, stride=4, tok=at(5), tau=1.0, logp=at(6), lse=at(7), ent=at(8), mask=None,
                 ws=WS, n=BIG):
    return cd.lib().conduit_token_alternatives(x or rows(), B, T, stride, tok, mask, tau, i or ids(), lps or vals(), logp, lse, ent,
                                               ws, n, None)


def listed(x=None, i=None, lps=None, B=B, T=T, stride=4, tau=1.0, rest=at(6), lse=at(7), mask=None, ws=WS, n=BIG):
    return cd.lib().conduit_listed_logprobs(x or rows(), B, T, stride, i or ids(), mask, tau, lps or vals(), rest, lse, ws, n, None)


def backward(x=None, i=None, lps=None, B=B, T=T, stride=4, tau=1.0, lse=at(6), rest=at(7), drest=at(8), mask=None, dx=None):
    return cd.lib().conduit_listed_logprobs_backward(x or rows(), B, T, stride, i or ids(), mask, tau, lse, rest, lps or vals(), drest,
                                                     dx or rows(at(4)), None)


def distill(x=None, i=None, lps=None, B=B, T=T, stride=4, tau=1.0, weight=at(6), loss=at(7), stats=at(8), mask=None, dx=None, ws=WS,
            n=BIG, **opts):
    o = cd.distill_opts()
    for k, v in opts.items():
        setattr(o, k, v)
    return cd.lib().conduit_distill_loss(C.byref(o), x or rows(), B, T, stride, i or ids(), lps or vals(), weight, mask, tau, loss,
                                         stats, rows(at(4)) if dx is None else dx or None, ws, n, None)


CALLS = [alternatives, listed, backward, distill]
SHARED = [
    (dict(B=-1), ">= 0"), (dict(T=-1), ">= 0"), (dict(B=1 << 20, T=1 << 11, stride=1 << 11), "2^31"), (dict(stride=3), "stride"),
    (dict(tau=0.0), "temperature"), (dict(tau=-1.0), "temperature"), (dict(tau=float("nan")), "temperature"),
    (dict(tau=float("inf")), "temperature"), (dict(tau=1e-39), "temperature"),
    (dict(x=rows(dtype=cd.I32)), "F32 or BF16"), (dict(x=rows(width=0)), "width"), (dict(x=rows(width=(1 << 28) + 1)), "width"),
    (dict(x=rows(stride_t=-8)), "strides"), (dict(x=rows(stride_b=1 << 41)), "strides"), (dict(x=rows(data=None)), "NULL data"),
    (dict(x=rows(data=at(1, 2))), "aligned"), (dict(x=rows(data=at(1, 1), dtype=cd.BF16)), "aligned"),
    (dict(i=ids(dtype=cd.F32)), "I32"), (dict(i=ids(dtype=cd.BF16)), "I32"), (dict(i=ids(width=0)), "[1, 128]"),
    (dict(i=ids(width=129), lps=vals(width=129)), "[1, 128]"), (dict(i=ids(data=None)), "NULL data"),
    (dict(i=ids(data=at(2, 2))), "aligned"), (dict(lps=vals(dtype=cd.I32)), "F32"), (dict(lps=vals(dtype=cd.BF16)), "F32"),
    (dict(lps=vals(width=3)), "as many"), (dict(lps=vals(data=None)), "NULL data"), (dict(lps=vals(data=at(3, 1))), "aligned"),
    (dict(lps=vals(stride_t=-2)), "strides"),
    (dict(x=rows(stride_b=1 << 40), B=(1 << 16) + 1), "end within 2^56"), (dict(i=ids(stride_b=1 << 40), B=(1 << 16) + 1), "end within 2^56"),
    (dict(stride=1 << 40, B=(1 << 16) + 1), "end within 2^56"),
]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("kw,msg", SHARED)
def test_shared_refusals(call, kw, msg):
    assert call(**kw) == cd.EINVAL and msg in cd.last_error(), cd.last_error()


@pytest.mark.parametrize("call", [alternatives, listed, distill])
@pytest.mark.parametrize("kw,msg", [(dict(ws=None), "workspace"), (dict(ws=at(99, 16)), "aligned"), (dict(n=100), "smaller")])
def test_workspaces_that_do_not_do(call, kw, msg):
    assert call(**kw) == cd.EINVAL and msg in cd.last_error(), cd.last_error()


LAP = dict(stride_t=1)  # rows that share elements
ON = 4 * (T * K * B - 1)  # the last element of a listed array


@pytest.mark.parametrize("kw,msg", [
    (dict(i=ids(**LAP)), "rows must not overlap"), (dict(lps=vals(**LAP)), "rows must not overlap"),
    (dict(tok=None), "tokens"), (dict(lse=at(6)), "overlap"), (dict(lse=at(6, 44)), "overlap"), (dict(ent=at(5)), "tokens"),
    (dict(logp=at(6, 2)), "aligned"), (dict(lps=vals(at(2))), "ids must be apart"), (dict(lps=vals(at(2, ON))), "ids must be apart"),
    (dict(i=ids(at(1, 8))), "ids must be apart"), (dict(lps=vals(at(1))), "logps must be apart"),
    (dict(i=ids(at(5))), "ids must be apart"), (dict(lps=vals(at(7))), "logps must be apart"), (dict(lse=at(1)), "overlaps an input"),
    (dict(mask=at(2, ON)), "ids must be apart"), (dict(mask=at(3)), "logps must be apart"), (dict(mask=at(8)), "overlaps the mask"),
])
def test_alternatives_refusals(kw, msg):
    assert alternatives(**kw) == cd.EINVAL and msg in cd.last_error(), cd.last_error()


@pytest.mark.parametrize("kw,msg", [
    (dict(lps=vals(**LAP)), "rows must not overlap"), (dict(lse=at(6)), "overlap"), (dict(lps=vals(at(2, ON))), "logps must be apart"),
    (dict(lps=vals(at(1))), "logps must be apart"), (dict(lps=vals(at(6))), "logps must be apart"), (dict(rest=at(2)), "overlaps an input"),
    (dict(lse=at(1, 12)), "overlaps an input"), (dict(rest=at(6, 1)), "aligned"), (dict(mask=at(3)), "logps must be apart"),
    (dict(mask=at(7, 40)), "overlaps the mask"),
])
def test_listed_refusals(kw, msg):
    assert listed(**kw) == cd.EINVAL and msg in cd.last_error(), cd.last_error()


@pytest.mark.parametrize("kw,msg", [
    (dict(lse=None), "lse"), (dict(rest=None), "needs the rest"), (dict(dx=rows(at(4), dtype=cd.BF16)), "dtype and width"),
    (dict(dx=rows(at(4), width=7)), "dtype and width"), (dict(dx=rows(at(4), stride_t=1)), "rows must not overlap"),
    (dict(dx=rows(at(1, 4))), "apart from them"), (dict(dx=rows(at(2))), "dlogits must be apart"), (dict(dx=rows(at(3, 4))), "dlogits must be apart"),
    (dict(dx=rows(at(6))), "dlogits must be apart"), (dict(dx=rows(at(8))), "dlogits must be apart"), (dict(drest=at(8, 1)), "aligned"),
    (dict(mask=at(4)), "dlogits must be apart"),
])
def test_listed_gradient_refusals(kw, msg):
    assert backward(**kw) == cd.EINVAL and msg in cd.last_error(), cd.last_error()


@pytest.mark.parametrize("kw,msg", [
    (dict(loss=None), "loss"), (dict(stats=None), "stats"), (dict(stats=at(8, 2)), "aligned"), (dict(loss=at(6)), "apart from the inputs"),
    (dict(loss=at(6, 4)), "overlaps an input"), (dict(loss=at(3)), "overlaps an input"), (dict(loss=at(1)), "overlaps an input"),
    (dict(dx=rows(at(4), dtype=cd.BF16)), "dtype and width"), (dict(dx=rows(at(1, 4))), "apart from them"),
    (dict(dx=rows(at(7))), "dlogits must be apart"), (dict(dx=rows(at(2))), "dlogits must be apart"), (dict(mask=at(4)), "dlogits must be apart"),
    (dict(stats=at(1, 4)), "stats must be apart"), (dict(stats=at(2)), "stats must be apart"), (dict(stats=at(3)), "stats must be apart"),
    (dict(stats=at(4)), "stats must be apart"), (dict(stats=at(6)), "stats must be apart"), (dict(stats=at(7)), "stats must be apart"),
    (dict(mask=at(8)), "stats must be apart"), (dict(mask=at(7)), "overlaps the mask"),
    (dict(reduction=3), "reduction"), (dict(reduction=-1), "reduction"), (dict(scale=float("inf")), "scale"),
    (dict(scale=float("nan")), "scale"), (dict(teacher_temperature=0.0), "temperature"), (dict(teacher_temperature=float("nan")), "temperature"),
    (dict(rest=1, teacher_temperature=2.0), "teacher_temperature 1"),
])
def test_distill_refusals(kw, msg):
    assert distill(**kw) == cd.EINVAL and msg in cd.last_error(), cd.last_error()


def test_divergences_that_are_not_there():
    o = cd.distill_opts()
    for kind, rest, msg in ((2, 1, "unknown divergence"), (-1, 0, "unknown divergence"), (1, 0, "needs the rest")):
        o.loss, o.rest = kind, rest
        assert cd.lib().conduit_distill_loss(C.byref(o), rows(), B, T, 4, ids(), vals(), None, None, 1.0, at(7), at(8), None, WS, BIG,
                                             None) == cd.EINVAL and msg in cd.last_error()
    with pytest.raises(KeyError):
        cd.distill_opts(loss="sideways")


def test_null_arguments_empty_batches_and_sizes():
    L, n = cd.lib(), C.c_uint64()
    for f in (L.conduit_token_alternatives_workspace, L.conduit_listed_logprobs_workspace, L.conduit_distill_loss_workspace):
        assert f(B, T, None, K, C.byref(n)) == cd.EINVAL and f(B, T, rows(), K, None) == cd.EINVAL
        assert f(B, T, rows(), 0, C.byref(n)) == cd.EINVAL and f(B, T, rows(), 129, C.byref(n)) == cd.EINVAL
        assert f(-1, T, rows(), K, C.byref(n)) == cd.EINVAL and f(1 << 20, 1 << 20, rows(), K, C.byref(n)) == cd.EINVAL
        for b, t, v in ((0, 5, 9), (3, 0, 9), (1, 1, 1 << 28), (1, (1 << 31) - 1, 1 << 28), ((1 << 31) - 1, 1, 3), (3, 4, 50001)):
            for dtype in (cd.F32, cd.BF16):
                assert f(b, t, rows(dtype=dtype, width=v), 128, C.byref(n)) == cd.OK and n.value % 256 == 0 and n.value > 0
    assert L.conduit_distill_loss(None, rows(), B, T, 4, ids(), vals(), None, None, 1.0, at(7), at(8), None, WS, BIG, None) == cd.EINVAL
    assert L.conduit_token_alternatives(None, B, T, 4, None, None, 1.0, ids(), vals(), None, None, None, WS, BIG, None) == cd.EINVAL
    assert L.conduit_token_alternatives(rows(), B, T, 4, None, None, 1.0, None, vals(), None, None, None, WS, BIG, None) == cd.EINVAL
    assert L.conduit_token_alternatives(rows(), B, T, 4, None, None, 1.0, ids(), None, None, None, None, WS, BIG, None) == cd.EINVAL
    assert L.conduit_listed_logprobs_backward(rows(), B, T, 4, ids(), None, 1.0, at(6), None, vals(), None, None, None) == cd.EINVAL
    for call in (alternatives, listed, backward):
        assert call(B=0) == cd.OK and call(T=0, stride=0) == cd.OK
    L.conduit_distill_opts_default(None)


# ---------------------------------------------------------------------------
# refusals of the binding
# ---------------------------------------------------------------------------
def test_binding_checks(monkeypatch):
    monkeypatch.setattr(cd, "_on_device", lambda t: True)
    monkeypatch.setattr(cd, "_native_batch", None)
    monkeypatch.setattr(cd, "_native_rows", None)
    x, i, y = torch.zeros(2, 5, 16), torch.zeros(2, 5, 3, dtype=torch.int32), torch.zeros(2, 5, 3)
    t, stats = torch.zeros(2, 5), torch.zeros(3)
    for call in (lambda x, i, y, t: cd.conduit_token_alternatives(x, i, y, lse=t),
                 lambda x, i, y, t: cd.conduit_listed_logprobs(x, i, y, lse=t),
                 lambda x, i, y, t: cd.conduit_listed_logprobs_backward(x, i, t, y, torch.zeros_like(x)),
                 lambda x, i, y, t: cd.conduit_distill_loss(cd.distill_opts(), x, i, y, t, stats)):
        with pytest.raises(ValueError, match="logits must be"):
            call(x[:, :4], i, y, t)
        with pytest.raises(ValueError, match="logits must be"):
            call(x[0], i, y, t)
        with pytest.raises(TypeError, match="logits must be torch.float32 or torch.bfloat16"):
            call(x.half(), i, y, t)
        with pytest.raises(ValueError, match="next to each other"):
            call(torch.zeros(2, 16, 5).transpose(1, 2), i, y, t)
        with pytest.raises(TypeError, match="ids must be torch.int32"):
            call(x, i.long(), y, t)
        with pytest.raises(TypeError, match="ids must be a torch tensor"):
            call(x, [1], y, t)
        with pytest.raises(ValueError, match="must have the shape of ids"):
            call(x, i, y[..., :2], t)
        with pytest.raises(TypeError, match="float32"):
            call(x, i, y.bfloat16(), t)
        with pytest.raises(ValueError, match="must have shape"):
            call(x, i, y, t[:, :4])
        with pytest.raises(TypeError):
            call(x, i, y, t.double())
        with pytest.raises(ValueError):
            call(x, i[0, 0], y[0, 0], t[0])
    with pytest.raises(ValueError, match="dlogits must be"):
        cd.conduit_distill_loss(cd.distill_opts(), x, i, y, t, stats, dlogits=x[:1])
    with pytest.raises(ValueError):
        cd.conduit_distill_loss(cd.distill_opts(), x, i, y, t, torch.zeros(2), workspace=torch.zeros(1 << 16, dtype=torch.uint8))
    monkeypatch.setattr(cd, "_on_device", lambda t: False)
    with pytest.raises(ValueError, match="on a HIP device"):
        cd.conduit_listed_logprobs(x, i, y)


def test_native_calls_leave_everything_else_to_python():
    from paper_2609_24456_amd import _tensor_check
    x, i, y = torch.zeros(2, 5, 16), torch.zeros(2, 5, 3, dtype=torch.int32), torch.zeros(2, 5, 3)
    args = [1, 16, None, 1.0, 0, torch.zeros(256, dtype=torch.uint8), None, x, i, y, None, None, None, None, None, None]
    assert _tensor_check.listed(*args) is None  # (host tensors: no call)
    for at_, bad in ((0, 7), (0, "1"), (1, None), (3, "warm"), (4, "s"), (7, None), (8, 3), (9, [1])):
        assert _tensor_check.listed(*(args[:at_] + [bad] + args[at_ + 1:])) is None
    with pytest.raises(TypeError):
        _tensor_check.listed(*args[:15])
