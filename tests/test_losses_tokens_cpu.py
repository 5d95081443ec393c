"""Outputs of the loss calls that would stand in the tokens' place: refused, since the tokens are read again after the
first outputs are written, and are no float input that an output may be (addresses are never followed)."""
import ctypes as C

import pytest

from paper_2609_24456_amd import conduit as cd

B, T, V = 3, 4, 50
WS, BIG = C.c_void_p(99 << 36), 1 << 34


def at(k, off=0):
    return C.c_void_p((k << 36) + off)


def rows(k, dtype=cd.F32, width=8):
    r = cd.Rows()
    r.data, r.dtype, r.width, r.stride_b, r.stride_t = at(k), dtype, width, 32, 8
    return C.byref(r)


TOK = [at(2), at(2, 4), at(2, -8)]


@pytest.mark.parametrize("out", TOK)
@pytest.mark.parametrize("which", [0, 1, 2])
def test_log_probabilities(out, which):
    L = cd.lib()
    o = [at(3), at(4), at(5)]
    o[which] = out
    assert L.conduit_token_logprobs(rows(1), B, T, 4, at(2), None, 1.0, *o, WS, BIG, None) == cd.EINVAL
    assert "overlaps the tokens" in cd.last_error()
    assert L.conduit_head_logprobs(rows(1, cd.BF16), rows(6, cd.BF16), V, B, T, 4, at(2), None, 1.0, *o, WS, BIG, None) == cd.EINVAL
    assert "overlaps the tokens" in cd.last_error()


@pytest.mark.parametrize("out", TOK)
@pytest.mark.parametrize("which", [0, 1])
def test_the_loss_from_logits(out, which):
    o = [at(3), at(4)]
    o[which] = out
    assert cd.lib().conduit_policy_loss_logits(C.byref(cd.policy_opts()), rows(1), B, T, 4, at(2), None, None, at(5), None, 1.0, *o,
                                               at(9), rows(8), WS, BIG, None) == cd.EINVAL
    assert "overlaps the tokens" in cd.last_error()
