"""The calls on listed choices together, as a distillation uses them: a teacher scores a delivered batch and keeps its best
choices, a student is scored at them and drawn towards them, and the gradient goes on into its projection.  Against the
same in 64 bits, by torch's differentiation on the host; eagerly and as a captured graph; and as the example runs it.

Tolerances.  e = 2^-24 (8 R + 128) bounds a log-probability of scores spread over R powers of two (see
test_gpu_listed.py), 4 e (1 + U) a divergence with log ratios up to U.  The student's bf16 logits are the oracle's inputs
too; their gradient is off by half a step of bf16, 2^-8, and by 8 e (1 + U) of the sum of both sides' probabilities (at
most 2 a row), and the projection's sums over the tokens are taken in 64 bits from there on both sides."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

from gpu_util import host

pytestmark = pytest.mark.gpu

from paper_2609_24456_amd import conduit as cd  # noqa: E402

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "post_training.py")


def _example():
    spec = importlib.util.spec_from_file_location("post_training", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_example(capsys):
    out = _example().main(["--sequences", "6", "--max-len", "64", "--vocab", "3001", "--hidden", "96", "--steps", "3",
                           "--lr", "0.01", "--distill", "--choices", "12"])
    loss, mean, tokens = out["distill"]
    assert math.isfinite(loss) and loss == pytest.approx(mean, rel=1e-6) and loss > 0 and tokens > 0


def _delivered(n, T, V):
    ex = _example()
    buf = ex.record(4 * n, T, V, seed=3)
    batch = ex.Batch(n, T)
    batch.deliver(buf, torch.randint(-2 ** 63, 2 ** 63 - 1, (n,), dtype=torch.int64, device="cuda",
                                     generator=torch.Generator(device="cuda").manual_seed(5)))
    torch.cuda.synchronize()
    buf.close()
    return ex, batch


def _oracle(x, ids, y, mask):
    """(divergence of every token, mean, gradient) in 64 bits, forward with the rest, by torch's differentiation."""
    x = x.double().cpu().requires_grad_()
    logp = torch.log_softmax(x, -1)
    at, y = ids.long().cpu(), y.double().cpu()
    listed = logp.gather(-1, at)
    inside = torch.zeros_like(logp, dtype=torch.bool).scatter(-1, at, True)
    rest = torch.logsumexp(logp.masked_fill(inside, -math.inf), -1)
    q = y.exp()
    left = (1 - q.sum(-1)).clamp(min=2.0 ** -23)
    each = (q * (y - listed)).sum(-1) + left * (left.log() - rest)
    on = (mask != 0).cpu()
    each = torch.where(on, each, 0.0)
    loss = each.sum() / on.sum()
    loss.backward()
    listed, rest = listed.detach(), rest.detach()
    U = max(float((y - listed).abs()[on].max()), float((left.log() - rest).abs()[on].max()))
    return each.detach(), loss.detach(), x.grad, listed, rest, U


@pytest.mark.parametrize("V,H", [(257, 32), (3001, 64), (20011, 64)])
def test_teacher_to_the_students_projection(V, H):
    n, T, K = 5, 40, 12
    ex, batch = _delivered(n, T, V)
    g = torch.Generator(device="cuda").manual_seed(1)
    hidden = torch.randn((n, T, H), generator=g, device="cuda")
    w = torch.randn((V, H), generator=g, device="cuda") * (2 * H ** -0.5)
    scores = lambda weight: (hidden.reshape(-1, H) @ weight.t()).reshape(n, T, V).to(torch.bfloat16)  # noqa: E731
    student = w + 0.3 * H ** -0.5 * torch.randn((V, H), generator=g, device="cuda")
    mask = batch.mask[:, 1:]
    x = scores(student)
    zs = x[:, :-1].double()
    e = 2.0 ** -24 * (8 * 1.4427 * 3 * float(zs.abs().max()) + 128)

    def run():
        ids, y = ex.teacher_choices(batch, scores(w), K)
        stats, listed, rest, dx = ex.distill_step(batch, scores(student), ids, y, cd.distill_opts(rest=True))
        # (the gradient stands in the logits' place, where the last position has none and keeps its logits)
        return ids, y, stats, listed, rest, dx[:, :-1]

    def check(ids, y, stats, listed, rest, dx):
        on = host(mask) != 0
        order = torch.sort(scores(w)[:, :-1].double(), dim=-1, descending=True, stable=True).indices[..., :K]
        assert (host(ids)[on] == host(order)[on]).all()
        each, loss, grad, want, wrest, U = _oracle(x[:, :-1], ids, y, mask)
        tol = 4 * e * (1 + U)
        assert np.abs(host(listed.double()) - want.numpy())[on].max() <= e
        assert np.abs(host(rest.double()) - wrest.numpy())[on].max() <= e
        assert abs(float(stats[0]) - float(loss)) <= tol + 2.0 ** -23 * abs(float(loss)) and int(stats[2]) == on.sum()
        d = grad.numpy()
        got = host(dx.double())
        bound = 2.0 ** -8 * np.abs(d) + 2 * tol * 2 / on.sum()
        assert (np.abs(got - d) <= bound).all()
        # on into the projection: a row of dW is a sum over the tokens
        hid = hidden[:, :-1].double().cpu().reshape(-1, H).numpy()
        dw, dw_want = got.reshape(-1, V).T @ hid, d.reshape(-1, V).T @ hid
        assert (np.abs(dw - dw_want) <= bound.reshape(-1, V).T @ np.abs(hid) + 1e-15).all()

    check(*run())
    # the same in a graph, replayed with other weights and with eager calls in between
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    view = x[:, :-1]
    ids, y = [torch.empty((n, T - 1, K), dtype=t, device="cuda") for t in (torch.int32, torch.float32)]
    loss, stats, dx = torch.empty((n, T), device="cuda")[:, 1:], torch.empty(3, device="cuda"), torch.empty_like(view)
    teacher = scores(w)
    ws = cd.workspace(max(cd.token_alternatives_workspace(view, K), cd.distill_loss_workspace(view, K)))

    def both():
        cd.conduit_token_alternatives(teacher[:, :-1], ids, y, mask=mask, workspace=ws)
        cd.conduit_distill_loss(cd.distill_opts(rest=True), view, ids, y, loss, stats, dlogits=dx, mask=mask, workspace=ws)

    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for i in range(3):
        x.copy_(scores(student * (1 + 0.1 * i)))
        teacher.copy_(scores(w * (1 - 0.1 * i)))
        dx.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (ids, y, loss, stats, dx)]
        both()
        for a, b in zip(got, (ids, y, loss, stats, dx)):
            assert torch.equal(a, b)
        each, mean, grad, _, _, U = _oracle(view, ids, y, mask)
        tol = 4 * e * 1.5 * (1 + U)
        assert np.abs(host(loss.double()) - each.numpy()).max() <= tol
        assert (np.abs(host(dx.double()) - grad.numpy()) <= 2.0 ** -8 * np.abs(grad.numpy()) + 4 * tol / int(stats[2])).all()
