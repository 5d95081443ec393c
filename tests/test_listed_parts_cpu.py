"""Batches of listed choices whose rows have too many parts for one launch are refused before anything is enqueued, so
that a workspace stays as it was.  (Addresses are never followed.)"""
import ctypes as C

import pytest

from paper_2609_24456_amd import conduit as cd

WIDE, K = 1 << 28, 2
HUGE = (1 << 63) - 1


def at(k):
    return C.c_void_p(k << 56)


def rows(k, dtype, width, step):
    r = cd.Rows()
    r.data, r.dtype, r.width, r.stride_b, r.stride_t = at(k), dtype, width, 0, step
    return C.byref(r)


def _common(T, dtype):
    return rows(1, dtype, WIDE, 0), T, rows(2, cd.I32, K, K), rows(3, cd.F32, K, K)


def alternatives(T, dtype, gradient):
    x, T, i, y = _common(T, dtype)
    return cd.lib().conduit_token_alternatives(x, 1, T, T, None, at(5), 1.0, i, y, None, at(6), None, at(9), HUGE, None)


def listed(T, dtype, gradient):
    x, T, i, y = _common(T, dtype)
    return cd.lib().conduit_listed_logprobs(x, 1, T, T, i, at(5), 1.0, y, at(6), None, at(9), HUGE, None)


def backward(T, dtype, gradient):
    x, T, i, y = _common(T, dtype)
    return cd.lib().conduit_listed_logprobs_backward(x, 1, T, T, i, at(5), 1.0, at(6), None, y, None, rows(4, dtype, WIDE, WIDE), None)


def distill(T, dtype, gradient):
    x, T, i, y = _common(T, dtype)
    dx = rows(4, dtype, WIDE, WIDE) if gradient else None
    o = cd.distill_opts()
    return cd.lib().conduit_distill_loss(C.byref(o), x, 1, T, T, i, y, None, at(5), 1.0, at(6), at(7), dx, at(9), HUGE, None)


@pytest.mark.parametrize("dtype", [cd.F32, cd.BF16])
@pytest.mark.parametrize("call,gradient", [(alternatives, False), (listed, False), (backward, True), (distill, False), (distill, True)])
def test_rows_of_too_many_parts(call, gradient, dtype):
    assert call(1 << 22, dtype, gradient) == cd.EINVAL and "2^31 parts" in cd.last_error(), cd.last_error()
