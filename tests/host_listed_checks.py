"""Host paths of the calls on listed choices, run against the library's AddressSanitizer + UndefinedBehaviorSanitizer
build (test_host_sanitizer_listed.py builds it and runs this file in a child process): argument checks and workspace
layouts over the ends of their ranges (addresses are never followed: validation fails first, or the batch is empty).
Usage: python host_listed_checks.py <library path>
"""
import ctypes as C
import importlib.util
import itertools
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("abi", os.path.join(ROOT, "paper_2609_24456_amd", "abi.py"))
abi = importlib.util.module_from_spec(spec)
spec.loader.exec_module(abi)
L = abi.load(sys.argv[1])


def at(k):
    return C.c_void_p(k << 24)


def rows(k, dtype=abi.F32, width=8, stride_b=32, stride_t=8):
    r = abi.Rows()
    r.data, r.dtype, r.width, r.stride_b, r.stride_t = at(k), dtype, width, stride_b, stride_t
    return C.byref(r)


def expect(st, want, what):
    if st not in want:
        raise SystemExit(f"{what}: status {st}, expected {want} ({L.conduit_last_error().decode()})")


ENDS = [-(1 << 63), -1, 0, 1, 128, 129, (1 << 31) - 1, 1 << 31, 1 << 40, (1 << 63) - 1]
n = C.c_uint64()
for f in (L.conduit_token_alternatives_workspace, L.conduit_listed_logprobs_workspace, L.conduit_distill_loss_workspace):
    for B, T, K in itertools.product(ENDS, ENDS, ENDS):
        for V in (0, 1, 2049, 1 << 28, (1 << 28) + 1):
            good = 0 <= B < 1 << 31 and 0 <= T < 1 << 31 and B * T < 1 << 31 and 1 <= K <= 128 and 1 <= V <= 1 << 28
            for dtype in (abi.F32, abi.BF16):
                expect(f(B, T, rows(1, dtype, V), K, C.byref(n)), (abi.OK,) if good else (abi.EINVAL,), f"{f.__name__} {B} {T} {K} {V}")

o = abi.DistillOpts()
L.conduit_distill_opts_default(C.byref(o))
for B, T, stride in itertools.product(ENDS, ENDS, ENDS):
    for sb, st in itertools.product((-1, 0, 8, 1 << 40, (1 << 63) - 1), repeat=2):
        x, i, y = rows(1, stride_b=sb, stride_t=st), rows(2, abi.I32, 2, sb, st), rows(3, abi.F32, 2, sb, st)
        any_ = (abi.OK, abi.EINVAL) if B == 0 or T == 0 else (abi.EINVAL,)
        # no workspace, or what it cannot do without missing: nothing but an empty batch passes
        expect(L.conduit_token_alternatives(x, B, T, stride, at(4), None, 1.0, i, y, at(5), at(6), at(7), None, 0, None), any_, "top")
        expect(L.conduit_listed_logprobs(x, B, T, stride, i, None, 1.0, y, at(5), at(6), None, 0, None), any_, "listed")
        expect(L.conduit_listed_logprobs_backward(x, B, T, stride, i, None, 1.0, None, None, y, None, rows(8, stride_b=sb, stride_t=st), None),
               any_, "backward")
        expect(L.conduit_distill_loss(C.byref(o), x, B, T, stride, i, y, at(4), at(9), 1.0, at(5), at(6), rows(8, stride_b=sb, stride_t=st),
                                      None, 0, None), (abi.EINVAL,), "distill")
print("listed checks ok", flush=True)
