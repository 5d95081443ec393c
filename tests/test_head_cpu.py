"""What the projection head's calls and their binding refuse, on the host (addresses are never followed)."""
import ctypes as C

import pytest
import torch

from paper_2609_24456_amd import conduit as cd


def at(k, off=0):
    return C.c_void_p((k << 36) + off)


def rows(data=at(1), dtype=cd.BF16, width=8, stride_b=32, stride_t=8):
    r = cd.Rows()
    r.data, r.dtype, r.width, r.stride_b, r.stride_t = data, dtype, width, stride_b, stride_t
    return C.byref(r)


B, T, V = 3, 4, 50
WS, BIG = at(99), 1 << 34


def forward(x=None, w=None, V=V, B=B, T=T, stride=4, tok=at(3), tau=1.0, logp=at(4), lse=at(5), ent=at(6), ws=WS, n=BIG):
    return cd.lib().conduit_head_logprobs(rows() if x is None else x, rows(data=at(2)) if w is None else w, V, B, T, stride, tok,
                                          None, tau, logp, lse, ent, ws, n, None)


def backward(x=None, w=None, V=V, B=B, T=T, stride=4, tok=at(3), tau=1.0, lse=at(4), ent=at(5), g=at(6), h=at(7), dx=None,
             dw=None, ws=WS, n=BIG):
    return cd.lib().conduit_head_logprobs_backward(
        rows() if x is None else x, rows(data=at(2)) if w is None else w, V, B, T, stride, tok, None, tau, lse, ent, g, h,
        rows(data=at(8)) if dx is None else dx, rows(data=at(9)) if dw is None else dw, ws, n, None)


SHARED = [
    (dict(B=-1), ">= 0"), (dict(stride=3), "stride"), (dict(tok=None), "tokens"), (dict(tau=0.0), "temperature"),
    (dict(tau=float("nan")), "temperature"), (dict(V=0), "choices"), (dict(V=(1 << 22) + 1), "choices"),
    (dict(B=1 << 11, T=1 << 11, stride=1 << 11), "2^21"), (dict(x=rows(dtype=cd.F32)), "BF16"),
    (dict(w=rows(data=at(2), dtype=cd.F32)), "BF16"), (dict(w=rows(data=at(2), width=16)), "same width"),
    (dict(x=rows(width=1 << 17, stride_t=1 << 17, stride_b=1 << 20), w=rows(data=at(2), width=1 << 17, stride_t=1 << 17)), "2^16"),
    (dict(x=rows(data=None)), "NULL data"), (dict(w=rows(data=None)), "NULL data"), (dict(x=rows(data=at(1, 1))), "aligned"),
    (dict(ws=None), "workspace"), (dict(ws=at(99, 16)), "aligned"), (dict(n=64), "smaller"),
]


@pytest.mark.parametrize("kw,msg", SHARED + [(dict(lse=at(4)), "overlap"), (dict(logp=at(4, 2)), "aligned")])
def test_head_refusals(kw, msg):
    assert forward(**kw) == cd.EINVAL and msg in cd.last_error(), cd.last_error()


@pytest.mark.parametrize("kw,msg", SHARED + [
    (dict(lse=None), "lse"), (dict(ent=None), "entropy"), (dict(dx=rows(data=at(8), dtype=cd.F32)), "BF16"),
    (dict(dw=rows(data=at(9), width=4)), "hidden width"), (dict(dx=rows(data=at(8), stride_t=4)), "rows must not overlap"),
    (dict(dw=rows(data=at(9), stride_t=4)), "rows must not overlap"), (dict(dx=rows()), "apart"),
    (dict(dw=rows(data=at(2))), "apart"), (dict(dw=rows(data=at(8))), "apart"), (dict(dx=rows(data=at(2, 16))), "apart"),
])
def test_head_gradient_refusals(kw, msg):
    assert backward(**kw) == cd.EINVAL and msg in cd.last_error(), cd.last_error()


def test_head_null_arguments_and_empty_batches():
    L, n = cd.lib(), C.c_uint64()
    for f in (L.conduit_head_logprobs_workspace, L.conduit_head_logprobs_backward_workspace):
        assert f(B, T, rows(), rows(data=at(2)), V, None) == cd.EINVAL
        assert f(B, T, None, rows(data=at(2)), V, C.byref(n)) == cd.EINVAL
        assert f(B, T, rows(), None, V, C.byref(n)) == cd.EINVAL
        assert f(B, T, rows(), rows(data=at(2)), V, C.byref(n)) == cd.OK and n.value % 256 == 0 and n.value > 0
    assert forward(B=0) == cd.OK and forward(T=0, stride=0) == cd.OK


def test_head_binding_checks(monkeypatch):
    monkeypatch.setattr(cd, "_on_device", lambda t: True)
    monkeypatch.setattr(cd, "_native_batch", None)
    monkeypatch.setattr(cd, "_native_rows", None)
    b = torch.bfloat16
    x, w, tok = torch.zeros(2, 5, 16, dtype=b), torch.zeros(9, 16, dtype=b), torch.zeros(2, 5, dtype=torch.int32)
    lp, ws = torch.zeros(2, 5), torch.zeros(1 << 16, dtype=torch.uint8)
    with pytest.raises(ValueError, match="hidden must be"):
        cd.conduit_head_logprobs(x[:, :4], w, tok, lp, workspace=ws)
    with pytest.raises(ValueError, match="weight must be"):
        cd.conduit_head_logprobs(x, w[0], tok, lp, workspace=ws)
    with pytest.raises(TypeError, match="weight"):
        cd.conduit_head_logprobs(x, w.half(), tok, lp, workspace=ws)
    with pytest.raises(ValueError, match="next to each other"):
        cd.conduit_head_logprobs(x, torch.zeros(16, 9, dtype=b).t(), tok, lp, workspace=ws)
    with pytest.raises(TypeError, match="tokens"):
        cd.conduit_head_logprobs(x, w, tok.long(), lp, workspace=ws)
    with pytest.raises(ValueError, match="dweight must have"):
        cd.conduit_head_logprobs_backward(x, w, tok, lp, lp, x, w[:8], workspace=ws)
    with pytest.raises(ValueError, match="dhidden must be"):
        cd.conduit_head_logprobs_backward(x, w, tok, lp, lp, x[:1], w, workspace=ws)
