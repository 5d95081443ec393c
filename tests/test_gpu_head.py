"""Log-probabilities through the projection head and their gradients against 64
bits: tile edges in tokens, choices and hidden units, rows that have to be packed,
masks, chunks of choices, split sums.

Tolerances.  A score is a sum of H exact products of bf16, rounded to 32 bits H
times at most while no partial sum passes Z = 2 max |z|; of random signs:
4 sqrt(H) 2^-24 Z, beside what a log-probability of given scores may lose,
2^-24 (8 R + 128) for a spread of R powers of two.  The gradients sum the
logits' gradient d after one rounding to bf16 (8 bits: at most 2^-8 of it, of
random sign), so their error is that of a sum of independent terms, 4 times
2^-8 sqrt(sum (d w)^2), and their own rounding, 2^-8."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2609_24456_amd import conduit as cd  # noqa: E402

BF16 = torch.bfloat16


class Batch:
    def __init__(self, B, T, H, V, seed=0, mask=True, spread=2.0):
        g = torch.Generator(device="cuda").manual_seed(seed + V)
        rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.B, self.T, self.H, self.V = B, T, H, V
        self.hidden = rn(B, T, H).to(BF16)
        self.weight = (rn(V, H) * (spread / H ** 0.5)).to(BF16)
        self.tokens = torch.randint(0, V, (B, T), generator=g, device="cuda", dtype=torch.int32)
        self.mask = (torch.rand((B, T), generator=g, device="cuda") < 0.6).to(torch.uint8) if mask else None
        if mask and B > 1:
            self.mask[0] = 0
        self.g, self.h = rn(B, T), rn(B, T)

    def on(self):
        return self.mask != 0 if self.mask is not None else torch.ones((self.B, self.T), dtype=torch.bool, device="cuda")

    def scores(self, tau):
        return (self.hidden.double().reshape(-1, self.H) @ self.weight.double().t()) / tau

    def tolerance(self, z):
        Z = 2 * float(z.abs().max())
        R = 1.4427 * float(z.max() - z.min())
        return 2.0 ** -24 * (4 * self.H ** 0.5 * Z + 8 * R + 128)

    def forward(self, tau, **kw):
        out = [torch.full((self.B, self.T), float("nan"), device="cuda") for _ in range(3)]
        cd.conduit_head_logprobs(kw.pop("hidden", self.hidden), kw.pop("weight", self.weight), self.tokens, out[0], lse=out[1],
                                 entropy=out[2], mask=self.mask, temperature=tau, **kw)
        return out


def _wanted(b, tau):
    z = b.scores(tau)
    lse = torch.logsumexp(z, -1)
    logq = z - lse[:, None]
    logp = logq.gather(1, b.tokens.reshape(-1, 1).long())[:, 0]
    ent = -(logq.exp() * logq).sum(-1)
    on = b.on().reshape(-1)
    return z, [torch.where(on, v, torch.zeros_like(v)).reshape(b.B, b.T) for v in (logp, lse, ent)]


def _close(got, want, tol, what):
    err = (got.double() - want).abs()
    bad = ~(err <= tol)
    assert not bool(bad.any()), (what, bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist(),
                                 int(bad.sum()), float(err[bad].max()))


def _check_gradients(b, tau, dh, dw, lse, entropy, h):
    z = b.scores(tau)
    logq = z - lse.double().reshape(-1, 1)
    p = logq.exp()
    g = b.g.double().reshape(-1, 1)
    d = -g * p
    d.scatter_add_(1, b.tokens.reshape(-1, 1).long(), g)
    if h is not None:
        d -= h.double().reshape(-1, 1) * p * (logq + entropy.double().reshape(-1, 1))
    d = torch.where(b.on().reshape(-1, 1), d / tau, torch.zeros_like(d))
    x, w = b.hidden.double().reshape(-1, b.H), b.weight.double()
    tz = b.tolerance(z)
    for got, a, o, what in ((dh.reshape(-1, b.H), d, w, "dhidden"), (dw, d.t().contiguous(), x, "dweight")):
        want = a @ o
        # (a score's error moves p, and with it d, by that much of (|g| + |h|) p at most)
        tol = 4 * 2.0 ** -8 * torch.sqrt((a * a) @ (o * o)) + 2.0 ** -8 * want.abs() + 4 * tz * (a.abs() @ o.abs()) + 1e-12
        _close(got, want, tol, what)


# one token, one choice, tiles of 256 and their edges, steps of 64 hidden units and their edges, rows that have to be
# packed (H not a multiple of 8), more tokens than a round of the list
SHAPES = [(1, 1, 8, 1), (1, 1, 64, 2), (2, 3, 72, 300), (1, 5, 100, 257), (1, 7, 1, 9), (4, 65, 256, 1000),
          (1, 256, 128, 256), (1, 257, 192, 255), (3, 171, 520, 513), (1, 16, 2048, 5000), (3, 100, 63, 20001), (70, 5, 136, 2050)]


@pytest.mark.parametrize("B,T,H,V", SHAPES)
@pytest.mark.parametrize("mask", [False, True])
def test_head_logprobs_and_gradients(B, T, H, V, mask):
    print(B, T, H, V, mask, flush=True)
    b = Batch(B, T, H, V, mask=mask)
    tau = 0.8
    z, want = _wanted(b, tau)
    tol = b.tolerance(z)
    got = b.forward(tau)
    for g, w, k in zip(got, want, (1, 1, 2)):
        _close(g, w, k * tol, "forward")
    lse, ent = want[1].float(), want[2].float()
    for h in (None, b.h):
        dh, dw = torch.full_like(b.hidden, 9.0), torch.full_like(b.weight, 9.0)
        cd.conduit_head_logprobs_backward(b.hidden, b.weight, b.tokens, lse, b.g, dh, dw, entropy=ent if h is not None else None,
                                          dentropy=h, mask=b.mask, temperature=tau)
        _check_gradients(b, tau, dh, dw, lse, ent, h)
    assert cd.conduit_sync_check() == cd.OK, cd.last_error()


def test_views_and_unaligned_rows():
    """Positions [:, :-1] of longer sequences, hidden states inside wider rows, rows off a 16-byte boundary, a
    projection with padded rows; masked places that nothing may read."""
    for off in (0, 3):
        B, T, H, V = 3, 50, 264, 777
        b = Batch(B, T, H, V)
        want = b.forward(1.0)
        lse, ent = want[1].clone(), want[2].clone()
        dh, dw = torch.empty_like(b.hidden), torch.empty_like(b.weight)
        cd.conduit_head_logprobs_backward(b.hidden, b.weight, b.tokens, lse, b.g, dh, dw, mask=b.mask)
        wide = torch.full((B, T + 1, 300), float("nan"), dtype=BF16, device="cuda")
        x = wide[:, :-1, off:off + H]
        x.copy_(b.hidden)
        x.masked_fill_((b.mask == 0)[..., None], float("nan"))
        wb = torch.full((V, 280), float("nan"), dtype=BF16, device="cuda")
        w = wb[:, off:off + H]
        w.copy_(b.weight)
        dirty = b.tokens.masked_fill(b.mask == 0, -100)
        keep, b.tokens = b.tokens, dirty
        for a, c in zip(b.forward(1.0, hidden=x, weight=w), want):
            assert torch.equal(a, c)
        dh2 = torch.full_like(wide, 5.0)
        dw2 = torch.full_like(wb, 5.0)
        cd.conduit_head_logprobs_backward(x, w, dirty, lse.masked_fill(b.mask == 0, float("nan")), b.g, dh2[:, :-1, off:off + H],
                                          dw2[:, off:off + H], mask=b.mask)
        assert torch.equal(dh2[:, :-1, off:off + H], dh) and torch.equal(dw2[:, off:off + H], dw)
        dh2[:, :-1, off:off + H] = 5.0
        dw2[:, off:off + H] = 5.0
        assert (dh2 == 5.0).all() and (dw2 == 5.0).all()  # nothing outside the views was written
        b.tokens = keep


def test_nothing_counts_and_no_tokens():
    b = Batch(2, 20, 64, 300)
    b.mask.zero_()
    assert all((o == 0).all() for o in b.forward(1.0))
    nan = torch.full((2, 20), float("nan"), device="cuda")
    dh, dw = torch.full_like(b.hidden, 9.0), torch.full_like(b.weight, 9.0)
    cd.conduit_head_logprobs_backward(b.hidden, b.weight, b.tokens, nan, nan, dh, dw, mask=b.mask)
    assert (dh == 0).all() and (dw == 0).all()
    e = torch.empty((0, 5), device="cuda")
    dw.fill_(9.0)
    cd.conduit_head_logprobs_backward(torch.empty((0, 5, 64), dtype=BF16, device="cuda"), b.weight, e.to(torch.int32), e, e,
                                      torch.empty((0, 5, 64), dtype=BF16, device="cuda"), dw)
    assert (dw == 0).all()


def test_tokens_outside_the_choices_are_flagged():
    for masked in (False, True):
        b = Batch(1, 40, 64, 300, mask=False)
        if masked:
            b.mask = torch.ones((1, 40), dtype=torch.uint8, device="cuda")
        b.tokens[0, 3], b.tokens[0, 9] = 300, -1
        out = b.forward(1.0)
        assert all((o[0, [3, 9]] == 0).all() and (o[0, 4] != 0) for o in out)
        assert cd.conduit_sync_check() == cd.ESTATE and "token outside" in cd.last_error()
        cd.conduit_clear_error()
        dh, dw = torch.full_like(b.hidden, 9.0), torch.full_like(b.weight, 9.0)
        cd.conduit_head_logprobs_backward(b.hidden, b.weight, b.tokens, out[1], b.g, dh, dw, mask=b.mask)
        assert (dh[0, [3, 9]] == 0).all() and (dh[0, 4] != 0).any()
        assert cd.conduit_sync_check() == cd.ESTATE
        cd.conduit_clear_error()


def test_gradient_in_chunks_of_choices():
    """So many tokens that the logits' gradient passes the workspace's 4 GiB: 69,632 tokens x 40,000 choices."""
    B, T, H, V = 17, 4096, 64, 40000
    b = Batch(B, T, H, V, mask=True)
    lse = b.forward(1.0)[1].clone()
    dh, dw = torch.full_like(b.hidden, 9.0), torch.full_like(b.weight, 9.0)
    cd.conduit_head_logprobs_backward(b.hidden, b.weight, b.tokens, lse, b.g, dh, dw, mask=b.mask)
    on, g, tok = b.on().reshape(-1), b.g.double().reshape(-1), b.tokens.reshape(-1).long()
    x, w = b.hidden.double().reshape(-1, H), b.weight.double()
    rows = torch.arange(0, B * T, 401, device="cuda")
    z = x[rows] @ w.t()
    d = -g[rows, None] * (z - lse.double().reshape(-1)[rows, None]).exp()
    d.scatter_add_(1, tok[rows, None], g[rows, None])
    d = torch.where(on[rows, None], d, torch.zeros_like(d))
    tol = 4 * 2.0 ** -8 * torch.sqrt((d * d) @ (w * w)) + 2.0 ** -8 * (d @ w).abs() + 4 * b.tolerance(z) * (d.abs() @ w.abs()) + 1e-12
    _close(dh.reshape(-1, H)[rows], d @ w, tol, "dhidden")
    picks = torch.arange(0, V, 399, device="cuda")
    z = x @ w[picks].t()
    d = -g[:, None] * (z - lse.double().reshape(-1, 1)).exp() + g[:, None] * (tok[:, None] == picks[None, :])
    d = torch.where(on[:, None], d, torch.zeros_like(d)).t().contiguous()
    tol = 4 * 2.0 ** -8 * torch.sqrt((d * d) @ (x * x)) + 2.0 ** -8 * (d @ x).abs() + 4 * b.tolerance(z) * (d.abs() @ x.abs()) + 1e-12
    _close(dw[picks], d @ x, tol, "dweight")


def test_results_do_not_change_from_run_to_run_and_in_a_graph():
    b = Batch(4, 200, 320, 3000)
    ws = cd.workspace(max(cd.head_logprobs_workspace(b.hidden, b.weight), cd.head_logprobs_backward_workspace(b.hidden, b.weight)))
    out = [torch.empty((b.B, b.T), device="cuda") for _ in range(3)]
    dh, dw = torch.empty_like(b.hidden), torch.empty_like(b.weight)

    def call():
        cd.conduit_head_logprobs(b.hidden, b.weight, b.tokens, out[0], lse=out[1], entropy=out[2], mask=b.mask, workspace=ws)
        cd.conduit_head_logprobs_backward(b.hidden, b.weight, b.tokens, out[1], b.g, dh, dw, entropy=out[2], dentropy=b.h,
                                          mask=b.mask, workspace=ws)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(3):
        b.hidden.mul_(0.5)
        b.mask.copy_(1 - b.mask)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*out, dh, dw)]
        call()
        torch.cuda.synchronize()
        for a, c in zip(got, (*out, dh, dw)):
            assert torch.equal(a, c), k




@pytest.mark.parametrize("N,H,V", [(1, 64, 300), (5, 200, 900), (31, 136, 2000), (33, 320, 700), (127, 64, 1000), (128, 256, 520)])
@pytest.mark.parametrize("mask", [False, True])
def test_gradients_of_few_tokens_are_rounded_once(N, H, V, mask):
    """Few tokens have few large elements in the logits' gradient, whose rounding would not average out: what is left
    is the outputs' own rounding to 8 bits, half a unit of the last place (2^-8 of the value at most), the halves'
    2^-16 of the terms summed, and what a probability may lose."""
    b = Batch(1, N, H, V, seed=N, mask=mask)
    if mask:
        b.mask[0, 0] = 1
    logp, lse, ent = b.forward(1.0)
    dh, dw = torch.empty_like(b.hidden), torch.empty_like(b.weight)
    cd.conduit_head_logprobs_backward(b.hidden, b.weight, b.tokens, lse, b.g, dh, dw, entropy=ent, dentropy=b.h, mask=b.mask)
    z = b.scores(1.0)
    logq = z - torch.logsumexp(z, -1, keepdim=True)
    p, on = logq.exp(), b.on().reshape(-1)
    e = -(p * logq).sum(-1, keepdim=True)
    g, h = b.g.double().reshape(-1, 1), b.h.double().reshape(-1, 1)
    d = -p * (g + h * (logq + e))
    d.scatter_add_(1, b.tokens.reshape(-1, 1).long(), g)
    d = torch.where(on[:, None], d, 0.0)
    x, w = b.hidden.double().reshape(N, H), b.weight.double()
    loss = 2.0 ** -16 + 4 * b.tolerance(z)
    for got, want, terms in ((dh.reshape(N, H), d @ w, d.abs() @ w.abs()), (dw, d.t() @ x, d.abs().t() @ x.abs())):
        err = (got.double() - want).abs()
        assert (err <= 2.0 ** -8 * want.abs() + loss * terms).all(), (err - 2.0 ** -8 * want.abs()).max()


@pytest.mark.parametrize("B,T,H,V", [(16, 1, 2056, 70001), (2, 6, 2056, 65537), (1, 16, 2048, 66000), (1, 3, 4104, 500)])
def test_few_tokens_by_rows_and_by_tiles(B, T, H, V):
    """Up to 16 tokens, both sides of the widths at which rows of the projection or tiles of it are multiplied."""
    b = Batch(B, T, H, V, mask=B == 2)
    z, want = _wanted(b, 1.0)
    tol = b.tolerance(z)
    got = b.forward(1.0)
    for name, g, w in zip(("logp", "lse", "entropy"), got, want):
        _close(g, w, 2 * tol, name)
    dh, dw = torch.full_like(b.hidden, float("nan")), torch.full_like(b.weight, float("nan"))
    cd.conduit_head_logprobs_backward(b.hidden, b.weight, b.tokens, got[1], b.g, dh, dw, entropy=got[2], dentropy=b.h, mask=b.mask)
    _check_gradients(b, 1.0, dh, dw, got[1], got[2], b.h)
