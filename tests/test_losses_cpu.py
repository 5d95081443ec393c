"""The loss calls without a GPU: their 64-bit oracle against differences and
closed forms, what the library refuses before anything is enqueued, and what the
binding refuses before anything reaches the library."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import losses as ref
from paper_2609_24456_amd import conduit as cd

EPS = 1e-6


def _differences(f, x, picks):
    """Central differences of f at some elements of x."""
    out = []
    for at in picks:
        hi, lo = x.copy(), x.copy()
        hi[at] += EPS
        lo[at] -= EPS
        out.append((f(hi) - f(lo)) / (2 * EPS))
    return np.array(out)


# a difference of step h has an error of h^2 times a third derivative (at most a
# few units here) and of rounding, 2^-52 / h of the value: 1e-9 covers both
TOL = 1e-8


def _picks(rng, shape, n=25):
    return [tuple(int(rng.integers(0, s)) for s in shape) for _ in range(n)]


@pytest.mark.parametrize("tau", [1.0, 0.6])
def test_oracle_logits_gradient_is_the_difference(tau):
    rng = np.random.default_rng(0)
    x = 2 * rng.standard_normal((2, 3, 7))
    tok = rng.integers(0, 7, (2, 3))
    mask = np.array([[1, 0, 1], [1, 1, 1]])
    g, h = rng.standard_normal((2, 3)), rng.standard_normal((2, 3))

    def f(v):
        logp, _, ent = ref.token_logprobs(v, tok, mask, tau)
        return (g * logp + h * ent)[mask != 0].sum()

    want = ref.logits_gradient(x, tok, g, h, mask, tau)
    picks = _picks(rng, x.shape)
    assert np.allclose(_differences(f, x, picks), [want[p] for p in picks], rtol=0, atol=TOL)


@pytest.mark.parametrize("reduction", ["token_mean", "sequence_mean", "sum"])
def test_oracle_policy_gradient_is_the_difference(reduction):
    rng = np.random.default_rng(1)
    logp = -rng.exponential(1.0, (3, 5))
    old, rf = logp - 0.5 * rng.standard_normal((3, 5)), logp + 0.2 * rng.standard_normal((3, 5))
    adv, ent = 3 * rng.standard_normal((3, 5)), rng.random((3, 5))
    mask = np.array([[1, 1, 0, 1, 1], [0, 0, 0, 0, 0], [1, 0, 1, 1, 1]])
    kw = dict(dual_clip=1.5, kl_coef=0.3, entropy_coef=0.2, scale=0.7, reduction=reduction)
    for which in (0, 1):
        def f(v):
            return ref.policy_loss(v if which == 0 else logp, adv, old, rf, v if which else ent, mask, **kw)[0][0]
        x = ent if which else logp
        want = ref.policy_loss(logp, adv, old, rf, ent, mask, **kw)[1 + which]
        picks = _picks(rng, x.shape)
        assert np.allclose(_differences(f, x, picks), [want[p] for p in picks], rtol=0, atol=TOL)


def test_oracle_policy_terms_by_hand():
    lp, old = np.log([[0.6, 0.6, 0.2, 0.2, 0.9]]), np.log([[0.4, 0.4, 0.4, 0.4, 0.2]])
    adv = np.array([[1.0, -1.0, 1.0, -1.0, -2.0]])
    # ratios 1.5, 1.5, 0.5, 0.5, 4.5: clipped at 1.2; free; free; clipped at 0.8; ceiling 2 * 3
    s, g, _ = ref.policy_loss(lp, adv, old, dual_clip=3.0, reduction="sum")
    assert np.allclose(s[1], -1.2 + 1.5 - 0.5 + 0.8 + 6.0)
    assert np.allclose(g[0], [0, 1.5, -0.5, 0, 0])
    assert s[4] == 3 / 5 and s[7] == 5


@pytest.mark.parametrize("kw", [dict(), dict(label_smoothing=0.2), dict(loss="squared"), dict(length_norm=True, beta=0.7)])
def test_oracle_preference_gradient_is_the_difference(kw):
    rng = np.random.default_rng(2)
    lp, rf = -rng.exponential(1.0, (4, 6)), -rng.exponential(1.0, (4, 6))
    mask = (rng.random((4, 6)) < 0.7).astype(int)
    mask[3] = 0
    want = ref.preference_loss(lp, rf, mask, **kw)[4]
    picks = _picks(rng, lp.shape)
    got = _differences(lambda v: ref.preference_loss(v, rf, mask, **kw)[3][0], lp, picks)
    assert np.allclose(got, [want[p] for p in picks], rtol=0, atol=1e-6 if kw.get("loss") == "squared" else TOL)


# ---------------------------------------------------------------------------
# refusals of the library (addresses are never followed: every call fails first)
# ---------------------------------------------------------------------------
def at(k, off=0):
    return C.c_void_p((k << 24) + off)


def rows(data=at(1), dtype=cd.F32, width=8, stride_b=32, stride_t=8):
    r = cd.Rows()
    r.data, r.dtype, r.width, r.stride_b, r.stride_t = data, dtype, width, stride_b, stride_t
    return C.byref(r)


WS, BIG = at(99), 1 << 20
B, T = 3, 4


def logprobs(x=None, B=B, T=T, stride=4, tok=at(2), tau=1.0, logp=at(3), lse=at(4), ent=at(5), ws=WS, n=BIG):
    return cd.lib().conduit_token_logprobs(rows() if x is None else x, B, T, stride, tok, None, tau, logp, lse, ent, ws, n, None)


BAD_ROWS = [(dict(dtype=cd.U8), "dtype"), (dict(width=0), "width"), (dict(width=(1 << 28) + 1), "width"),
            (dict(stride_t=-8), "strides"), (dict(stride_b=1 << 41), "strides"), (dict(data=None), "NULL data"),
            (dict(data=at(1, 2)), "aligned"), (dict(dtype=cd.BF16, data=at(1, 1)), "aligned")]


@pytest.mark.parametrize("kw,msg", [
    (dict(B=-1), ">= 0"), (dict(T=-1), ">= 0"), (dict(B=1 << 20, T=1 << 11, stride=1 << 11), "2^31"), (dict(stride=3), "stride"),
    (dict(tok=None), "tokens"), (dict(tau=0.0), "temperature"), (dict(tau=-1.0), "temperature"),
    (dict(tau=float("nan")), "temperature"), (dict(tau=float("inf")), "temperature"), (dict(tau=1e-39), "temperature"),
    (dict(lse=at(3)), "overlap"), (dict(lse=at(3, 44)), "overlap"), (dict(lse=at(3, -44)), "overlap"),
    (dict(logp=at(3, 2)), "aligned"), (dict(ws=None), "workspace"), (dict(ws=at(99, 16)), "aligned"), (dict(n=100), "smaller"),
] + [(dict(x=rows(**r)), m) for r, m in BAD_ROWS])
def test_logprobs_refusals(kw, msg):
    assert logprobs(**kw) == cd.EINVAL and msg in cd.last_error(), cd.last_error()


def test_null_arguments_and_empty_batches():
    L = cd.lib()
    n = C.c_uint64()
    assert L.conduit_token_logprobs(None, B, T, 4, at(2), None, 1.0, at(3), None, None, WS, BIG, None) == cd.EINVAL
    assert L.conduit_token_logprobs_workspace(B, T, None, C.byref(n)) == cd.EINVAL
    assert L.conduit_token_logprobs_workspace(B, T, rows(), None) == cd.EINVAL
    assert L.conduit_policy_loss_workspace(B, T, None) == cd.EINVAL
    assert L.conduit_preference_loss_workspace(1 << 62, 1, C.byref(n)) == cd.EINVAL
    assert L.conduit_workspace_init(None, 256, None) == cd.EINVAL
    assert L.conduit_workspace_init(at(9, 8), 256, None) == cd.EINVAL
    assert L.conduit_workspace_init(at(9), 255, None) == cd.EINVAL
    assert logprobs(B=0) == cd.OK and logprobs(T=0, stride=0) == cd.OK
    L.conduit_policy_opts_default(None)
    L.conduit_preference_opts_default(None)


def backward(x=None, dx=None, lse=at(4), ent=at(5), g=at(6), h=at(7), tok=at(2), tau=1.0, stride=4):
    return cd.lib().conduit_token_logprobs_backward(rows() if x is None else x, B, T, stride, tok, None, tau, lse, ent, g, h,
                                                    rows(data=at(8)) if dx is None else dx, None)


@pytest.mark.parametrize("kw,msg", [
    (dict(lse=None), "lse"), (dict(tok=None), "tokens"), (dict(ent=None), "entropy"), (dict(tau=0.0), "temperature"),
    (dict(dx=rows(data=at(8), dtype=cd.BF16)), "dtype and width"), (dict(dx=rows(data=at(8), width=4)), "dtype and width"),
    (dict(dx=rows(data=at(8), stride_t=0)), "rows must not overlap"), (dict(dx=rows(data=at(8), stride_b=8)), "rows must not overlap"),
    (dict(dx=rows(data=at(1, 4))), "apart"), (dict(dx=rows(stride_t=9, stride_b=64)), "apart"),
    (dict(dx=rows(data=None)), "NULL data"), (dict(g=at(6, 1)), "aligned"),
])
def test_backward_refusals(kw, msg):
    assert backward(**kw) == cd.EINVAL and msg in cd.last_error(), cd.last_error()


def policy(opts=None, B=B, T=T, stride=4, logp=at(1), old=at(2), ref=at(3), adv=at(4), ent=at(5), stats=at(6), g=at(7), h=at(8),
           ws=WS, n=BIG):
    o = cd.policy_opts() if opts is None else opts
    return cd.lib().conduit_policy_loss(C.byref(o), B, T, stride, logp, old, ref, adv, ent, None, stats, g, h, ws, n, None)


def _opts(**kw):
    o = cd.policy_opts()
    for k, v in kw.items():
        setattr(o, k, v)
    return o


BAD_POLICY = [(dict(clip_low=-0.1), "clip_low"), (dict(clip_low=1.1), "clip_low"), (dict(clip_high=-1.0), "clip_high"),
              (dict(clip_high=float("inf")), "clip_high"), (dict(dual_clip=1.0), "dual_clip"), (dict(dual_clip=-2.0), "dual_clip"),
              (dict(kl_coef=float("nan")), "finite"), (dict(scale=float("inf")), "finite"), (dict(reduction=3), "reduction"),
              (dict(reduction=-1), "reduction")]


@pytest.mark.parametrize("kw,msg", [(dict(opts=o), m) for o, m in [(_opts(**k), m) for k, m in BAD_POLICY]] + [
    (dict(stats=None), "stats"), (dict(logp=None), "logp"), (dict(adv=None), "adv"), (dict(stride=2), "stride"),
    (dict(g=at(1, 4)), "overlaps an input"), (dict(h=at(7)), "outputs overlap"), (dict(h=at(7, 16)), "outputs overlap"),
    (dict(ws=None), "workspace"), (dict(n=256), "smaller")])
def test_policy_refusals(kw, msg):
    assert policy(**kw) == cd.EINVAL and msg in cd.last_error(), cd.last_error()


def policy_logits(opts=None, x=None, dx=None, stride=4, tok=at(2), old=at(3), ref=at(4), adv=at(5), tau=1.0, logp=at(6),
                  ent=at(7), stats=at(9), ws=WS, n=BIG):
    o = cd.policy_opts() if opts is None else opts
    return cd.lib().conduit_policy_loss_logits(C.byref(o), rows() if x is None else x, B, T, stride, tok, old, ref, adv, None, tau,
                                               logp, ent, stats, rows(data=at(8)) if dx is None else dx, ws, n, None)


@pytest.mark.parametrize("kw,msg", [(dict(opts=o), m) for o, m in [(_opts(**k), m) for k, m in BAD_POLICY]] + [
    (dict(x=rows(**r)), m) for r, m in BAD_ROWS] + [
    (dict(tok=None), "tokens"), (dict(adv=None), "adv"), (dict(logp=None), "logp"), (dict(ent=None), "entropy"),
    (dict(stats=None), "stats"), (dict(logp=at(3)), "apart"), (dict(ent=at(5, 4)), "overlaps an input"), (dict(tau=0.0), "temperature"),
    (dict(dx=rows(data=at(1, 4))), "apart"), (dict(n=256), "smaller")])
def test_policy_logits_refusals(kw, msg):
    assert policy_logits(**kw) == cd.EINVAL and msg in cd.last_error(), cd.last_error()


def preference(P=2, T=T, stride=4, logp=at(1), ref=at(2), loss=at(3), stats=at(6), g=at(7), ws=WS, n=BIG, **kw):
    o = cd.preference_opts()
    for k, v in kw.items():
        setattr(o, k, v)
    return cd.lib().conduit_preference_loss(C.byref(o), P, T, stride, logp, ref, None, loss if "form" not in kw else loss, at(4),
                                            at(5), stats, g, ws, n, None)


@pytest.mark.parametrize("kw,msg", [
    (dict(beta=0.0), "beta"), (dict(beta=float("nan")), "beta"), (dict(label_smoothing=1.0), "label_smoothing"),
    (dict(label_smoothing=-0.1), "label_smoothing"), (dict(scale=float("nan")), "scale"), (dict(P=-1), ">= 0"),
    (dict(P=1 << 30, T=2, stride=2), "2^31"), (dict(logp=None), "logp"), (dict(loss=None), "loss"), (dict(stats=None), "stats"),
    (dict(stride=3), "stride"), (dict(g=at(1, 8)), "overlaps an input"), (dict(n=256), "smaller")])
def test_preference_refusals(kw, msg):
    assert preference(**kw) == cd.EINVAL and msg in cd.last_error(), cd.last_error()


def test_columns_between_each_others_rows_are_apart():
    """Per-token arrays may be columns of one wider array (rows 16 apart, 4 wide), but share no element.  The calls
    here pass that check and stop at the workspace."""
    col = lambda k: at(1, 16 * k)  # noqa: E731
    kw = dict(stride=16, logp=col(0), old=col(1), adv=col(2), ref=None, ent=None, h=None, n=0)
    assert policy(g=col(3), **kw) == cd.EINVAL and "smaller" in cd.last_error()
    assert policy(g=at(1, 44), **kw) == cd.EINVAL and "overlaps an input" in cd.last_error()


# ---------------------------------------------------------------------------
# refusals of the binding
# ---------------------------------------------------------------------------
class _NoLibrary:
    def __getattr__(self, name):
        def call(*args):
            if name.endswith(("_workspace", "_default")):
                return cd.OK
            pytest.fail(f"{name} was called although an argument check should have raised")
        return call


@pytest.fixture
def host_tensors(monkeypatch):
    monkeypatch.setattr(cd, "_on_device", lambda t: True)
    monkeypatch.setattr(cd, "lib", lambda: _NoLibrary())


def test_binding_checks(host_tensors):
    f = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)  # noqa: E731
    i32 = torch.int32
    ws = f(4096, dtype=torch.uint8)
    x, tok, lp = f(2, 5, 9), f(2, 5, dtype=i32), f(2, 5)
    kw = dict(workspace=ws)
    with pytest.raises(ValueError, match="logits must be"):
        cd.conduit_token_logprobs(f(2, 4, 9), tok, lp, **kw)
    with pytest.raises(TypeError, match="logits"):
        cd.conduit_token_logprobs(f(2, 5, 9, dtype=torch.float16), tok, lp, **kw)
    with pytest.raises(ValueError, match="next to each other"):
        cd.conduit_token_logprobs(f(2, 5, 18)[..., ::2], tok, lp, **kw)
    with pytest.raises(TypeError, match="tokens"):
        cd.conduit_token_logprobs(x, tok.long(), lp, **kw)
    with pytest.raises(ValueError, match="logp"):
        cd.conduit_token_logprobs(x, tok, f(2, 4), **kw)
    with pytest.raises(ValueError, match="logp must"):
        cd.conduit_token_logprobs(x, tok, f(2, 6)[:, 1:], **kw)
    with pytest.raises(ValueError, match="logp must have rows"):
        cd.conduit_token_logprobs(x, f(2, 6, dtype=i32)[:, 1:], lp, **kw)
    with pytest.raises(ValueError, match="tokens must"):
        cd.conduit_token_logprobs(x, f(5, 2, dtype=i32).t(), lp, **kw)
    with pytest.raises(TypeError, match="mask"):
        cd.conduit_token_logprobs(x, tok, lp, mask=f(2, 5), **kw)
    with pytest.raises(ValueError, match="dlogits must be"):
        cd.conduit_token_logprobs_backward(x, tok, lp, lp, f(1, 5, 9))
    with pytest.raises(ValueError, match="stats holds"):
        cd.conduit_policy_loss(cd.PolicyOpts(), lp, lp, f(7), **kw)
    with pytest.raises(TypeError, match="adv"):
        cd.conduit_policy_loss(cd.PolicyOpts(), lp, f(2, 5, dtype=torch.float64), f(8), **kw)
    with pytest.raises(ValueError, match="must be a"):
        cd.conduit_policy_loss(cd.PolicyOpts(), f(2, 5, 1), lp, f(8), **kw)
    with pytest.raises(TypeError, match="workspace"):
        cd.conduit_policy_loss(cd.PolicyOpts(), lp, lp, f(8), workspace=f(64))
    with pytest.raises(ValueError, match="2 P"):
        cd.conduit_preference_loss(cd.PreferenceOpts(), f(3, 5), f(1), f(4), **kw)
    with pytest.raises(ValueError, match="loss holds"):
        cd.conduit_preference_loss(cd.PreferenceOpts(), f(4, 5), f(1), f(4), **kw)
    with pytest.raises(KeyError):
        cd.policy_opts(reduction="mean")
    with pytest.raises(TypeError, match="unknown option"):
        cd.policy_opts(clip=0.2)
    with pytest.raises(KeyError):
        cd.preference_opts(loss="hinge")


def test_struct_layouts():
    assert (C.sizeof(cd.Rows), C.sizeof(cd.PolicyOpts), C.sizeof(cd.PreferenceOpts)) == (40, 56, 32)
    o = cd.policy_opts()
    assert (o.clip_low, o.clip_high, o.dual_clip, o.kl_coef, o.entropy_coef, o.scale, o.reduction) == (0.2, 0.2, 0, 0, 0, 1, 0)
    p = cd.PreferenceOpts()
    cd.lib().conduit_preference_opts_default(C.byref(p))
    assert (p.beta, p.label_smoothing, p.scale, p.loss, p.length_norm) == (0.1, 0, 1, 0, 0)
