"""Top alternatives of finite logits over the whole range of the scores: small temperatures, large logits, choices
forbidden by a large finite value, in every kernel, whole rows and rows in parts, against the 64-bit forms of
oracle/losses.py.

Tolerances.  A log-probability is ((x - max x) c - log2 s) ln2: the difference, c, the product, the subtraction, ln2 and
the last product are each off by at most 2^-24 of it, 6 roundings, counted as 8.  log s is off by the exponents' errors,
4 roundings of each distance d weighted by its share, sum p |d| <= log2 V <= 17, and by sums of at most 64 elements a
lane (40,000 choices in 4 parts: 40) and 12 steps of joins, whose errors are relative: together below 4 x 17 x ln2 + 76 <
128 of 2^-24.  The log-normaliser adds one rounding of max x / temperature and one of itself.  The entropy goes by sum p d:
its errors are those of log s, once more for each weight times the distance, at most L (L + 1) roundings of 4 with L = log2
V, and the weighted sum's own 76 times its value, at most L."""
import numpy as np
import pytest
import torch

from gpu_util import host
from oracle import losses as ref

pytestmark = pytest.mark.gpu

from paper_2609_24456_amd import conduit as cd  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
STEP = 2.0 ** -24
# by V: rows that share a wavefront, a wavefront each (by elements and in vectors), a workgroup each or in parts
WIDTHS = [40, 300, 513, 1000, 4100, 5000, 40000]


def _rows_of(a, dtype):
    x = torch.from_numpy(np.asarray(a, np.float64).astype(np.float32)).to(dtype)
    return x, x.double().numpy()


def _large_rows(rng, V):
    """Scores with large finite values: a few choices allowed, a block of the vocabulary forbidden, whole rows."""
    j, out = np.arange(V), []
    few = rng.permutation(V)[:5]
    for v in (-1e9, -1e10, -1e12, -1e20, -1e30):
        a = np.full(V, v)
        a[few] = 3 * rng.standard_normal(5)
        out.append(a)
        out.append(np.where(j < V // 2, v, 3 * rng.standard_normal(V)))
        out.append(np.where(j >= V // 3, v, 3 * rng.standard_normal(V)))
    out += [np.full(V, -1e10), 1e10 + 3 * rng.standard_normal(V), np.where(j % 2 == 0, 1e12, -1e12), np.where(j < V // 2, 1e10, -1e10),
            np.linspace(-1e30, 1e30, V)]
    out += [s * 3 * rng.standard_normal(V) for s in (1e6, 1e9, 1e15, 1e29)]
    return np.stack(out)


def _check(x, z, tau, tiles, Ks=(5, 64)):
    """`tiles` copies of the rows below each other."""
    n, V = z.shape
    tok = np.arange(n) * 7 % V
    logp, lse, ent = ref.token_logprobs(z, tok, None, tau)
    L = np.log2(V) + 1
    y = x.cuda().repeat(tiles, 1)
    t = torch.from_numpy(tok.astype(np.int32)).cuda().repeat(tiles)
    for K in Ks:
        want = ref.alternatives(z, K, None, tau)
        ids = torch.full((n * tiles, K), -7, dtype=torch.int32, device="cuda")
        logps = torch.full((n * tiles, K), float("nan"), device="cuda")
        out = [torch.full((n * tiles,), float("nan"), device="cuda") for _ in range(3)]
        cd.conduit_token_alternatives(y, ids, logps, tokens=t, logp=out[0], lse=out[1], entropy=out[2], temperature=tau)
        ids, logps, out = host(ids), host(logps).astype(np.float64), [host(o).astype(np.float64) for o in out]
        for b in range(0, n * tiles, n):  # (the rows repeat)
            s = slice(b, b + n)
            for got, exact, tol in ((logps[s], want[1], lambda e: STEP * (8 * np.abs(e) + 128)),
                                    (out[0][s], logp, lambda e: STEP * (8 * np.abs(e) + 128)),
                                    (out[1][s], lse, lambda e: STEP * (2 * np.abs(e) + 128)),
                                    (out[2][s], ent, lambda e: STEP * (4 * L * (L + 1) + 76 * L + 128))):
                with np.errstate(invalid="ignore", over="ignore"):
                    same = got == exact.astype(np.float32)  # (infinities: past the largest float)
                    bad = ~same & ~(np.abs(got - exact) <= tol(np.where(np.isfinite(exact), exact, 0.0)))
                assert not bad.any(), (K, b, np.argwhere(bad)[:6].tolist(), got[bad][:6], exact[bad][:6])
            assert (ids[s] == want[0]).all(), (K, b, np.argwhere((ids[s] != want[0]).any(-1)).ravel())


def _tiles(n, V, many):
    """Copies that make more rows than compute units of wide rows (whole ones), or one (parts)."""
    return -(-300 // n) if many and V > 4103 else 1


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", WIDTHS)
@pytest.mark.parametrize("many", [False, True])
def test_alternatives_of_large_finite_scores(many, V, dtype):
    x, z = _rows_of(_large_rows(np.random.default_rng(V), V), dtype)
    for tau in (1.0, 2.0):
        _check(x, z, tau, _tiles(len(z), V, many))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", WIDTHS)
@pytest.mark.parametrize("many", [False, True])
def test_alternatives_at_small_temperatures(many, V, dtype):
    rng = np.random.default_rng(V + 1)
    x, z = _rows_of(np.concatenate([3 * rng.standard_normal((8, V)), 30 + 3 * rng.standard_normal((2, V)), 1e-3 * rng.standard_normal((2, V)),
                                    rng.integers(-2, 3, (2, V))]), dtype)
    for tau in (1e-4, 1e-6, 1e-8, 1e-9, 1e-10, 1e-20):
        _check(x, z, tau, _tiles(len(z), V, many), Ks=(20,))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_alternatives_of_large_scores_joined_by_a_launch(dtype):
    """More than 512 rows in parts."""
    V = (1 << 17) + 3000 if dtype == F32 else (1 << 18) + 3000
    rng = np.random.default_rng(9)
    a = 3 * rng.standard_normal((4, V))
    a[1] *= 1e9
    a[2, : V // 2] = -1e10
    a[3, 5000:] = -1e12
    x, z = _rows_of(a, dtype)
    _check(x, z, 1.0, 130, Ks=(20,))
