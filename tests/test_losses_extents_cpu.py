"""Loss calls whose arrays would reach further than 64 bits of bytes: refused before any extent is formed, so that no
check of overlaps works on a wrapped one (addresses are never followed)."""
import ctypes as C

import pytest

from paper_2609_24456_amd import conduit as cd

F, TOP = 1 << 40, 1 << 63


def at(k):
    return C.c_void_p(k << 24)


def rows(data, stride_b, stride_t, width=8, dtype=cd.F32):
    r = cd.Rows()
    r.data, r.dtype, r.width, r.stride_b, r.stride_t = data, dtype, width, stride_b, stride_t
    return C.byref(r)


WS, BIG = at(99), 1 << 40

# B, stride_b, T, stride_t: the products wrap to 0, to a negative number, to a small one; and one just past the limit
FAR = [((1 << 24) + 1, F, 1, 8), ((1 << 23) + 1, F, 1, 8), (1, 8, (1 << 24) + 1, F), ((1 << 25) + 1, F, 4, 8),
       ((1 << 16) + 1, F, 1, 8)]


@pytest.mark.parametrize("B,sb,T,st", FAR)
def test_rows_that_reach_too_far(B, sb, T, st):
    L = cd.lib()
    x, dx = rows(at(1), sb, st), rows(at(8), sb, st)
    near = rows(at(1), 8 * T, 8)
    calls = [L.conduit_token_logprobs(x, B, T, T, at(2), None, 1.0, at(300), None, None, WS, BIG, None),
             L.conduit_token_logprobs_backward(x, B, T, T, at(2), None, 1.0, at(3), None, at(4), None, dx, None),
             L.conduit_token_logprobs_backward(near, B, T, T, at(2), None, 1.0, at(3), None, at(4), None, dx, None),
             L.conduit_policy_loss_logits(C.byref(cd.policy_opts()), x, B, T, T, at(2), None, None, at(5), None, 1.0, at(300),
                                          at(600), at(9), dx, WS, BIG, None)]
    for k, st_ in enumerate(calls):
        assert st_ == cd.EINVAL, k
    assert "end within 2^56" in cd.last_error()


@pytest.mark.parametrize("B", [(1 << 16) + 1, (1 << 23) + 1, (1 << 24) + 1, (1 << 31) - 1])
def test_per_token_arrays_that_reach_too_far(B):
    o = cd.policy_opts()
    assert cd.lib().conduit_policy_loss(C.byref(o), B, 1, F, at(1), None, None, at(2), None, None, at(3), at(4), None, WS, BIG,
                                        None) == cd.EINVAL and "end within 2^56" in cd.last_error()
    p = cd.preference_opts()
    assert cd.lib().conduit_preference_loss(C.byref(p), (B + 1) // 2, 1, F, at(1), None, None, at(2), None, None, at(3), at(4), WS,
                                            BIG, None) == cd.EINVAL and ("end within 2^56" in cd.last_error()
                                                                         or "2^31" in cd.last_error())


@pytest.mark.parametrize("V", [-TOP, -1, (1 << 22) + 1, TOP - 1])
def test_the_head_s_numbers_of_choices_at_the_ends_of_64_bits(V):
    x, w = rows(at(1), 64, 8, dtype=cd.BF16), rows(at(2), 0, F, dtype=cd.BF16)
    n = C.c_uint64()
    assert cd.lib().conduit_head_logprobs_workspace(1, 1, x, w, V, C.byref(n)) == cd.EINVAL


@pytest.mark.parametrize("P", [-TOP, -(1 << 62), -1])
def test_negative_numbers_of_pairs(P):
    n = C.c_uint64()
    assert cd.lib().conduit_preference_loss_workspace(P, 4, C.byref(n)) == cd.EINVAL and ">= 0" in cd.last_error()
    o = cd.preference_opts()
    assert cd.lib().conduit_preference_loss(C.byref(o), P, 4, 4, at(1), None, None, at(2), None, None, at(3), at(4), WS, BIG,
                                            None) == cd.EINVAL and ">= 0" in cd.last_error()


def test_rows_just_within_reach_pass_the_check():
    """(The calls stop at the workspace.)"""
    B = 1 << 16
    x = rows(at(1), F - 8, 8)
    assert cd.lib().conduit_token_logprobs(x, B, 1, 1, at(2), None, 1.0, at(300), None, None, WS, 1, None) == cd.EINVAL
    assert "smaller" in cd.last_error()
