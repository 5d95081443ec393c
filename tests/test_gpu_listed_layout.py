"""The calls on listed choices: both ways of checking arguments give the same calls, offsets past 32 bits reach the right
elements, other streams have workspaces of their own, and more rows than one dimension of a launch takes."""
import ctypes as C

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2609_24456_amd import conduit as cd  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
FAR = (1 << 31) + 24  # elements: past 32 bits of elements and, at 2 and 4 bytes, of bytes


def _inputs(B, T, V, K, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((B, T, V), generator=g, device="cuda").mul_(3)
    y, ids = torch.topk(torch.log_softmax(x + torch.randn((B, T, V), generator=g, device="cuda"), -1), K, dim=-1)
    tok = torch.randint(0, V, (B, T), generator=g, device="cuda", dtype=torch.int32)
    mask = (torch.rand((B, T), generator=g, device="cuda") < 0.8).to(torch.uint8)
    mask[0, 0] = 1
    return x.to(dtype), tok, ids.int(), y, mask


def _calls(x, tok, ids, y, mask, outs=None, **kw):
    """Every call, into `outs` (made in the layout of the inputs without)."""
    like = lambda t: torch.full_like(t, 9)  # noqa: E731
    per = lambda: torch.full(tok.shape, 9.0, device="cuda")  # noqa: E731
    if outs is None:
        outs = [like(ids), like(y), per(), per(), per(), like(y), per(), per(), like(x), per(), torch.empty(3, device="cuda"), like(x),
                per(), torch.empty(3, device="cuda")]
    top, lp, a, b, c, listed, rest, lse, dx, loss, stats, ddx, loss2, stats2 = outs
    cd.conduit_token_alternatives(x, top, lp, tokens=tok, logp=a, lse=b, entropy=c, mask=mask, temperature=0.9, **kw)
    cd.conduit_listed_logprobs(x, ids, listed, rest=rest, lse=lse, mask=mask, temperature=0.9, **kw)
    back = {k: v for k, v in kw.items() if k != "workspace"}
    cd.conduit_listed_logprobs_backward(x, ids, lse, y, dx, rest=rest, drest=lse, mask=mask, temperature=0.9, **back)
    cd.conduit_distill_loss(cd.distill_opts(rest=True), x, ids, y, loss, stats, dlogits=ddx, weight=lse, mask=mask, temperature=0.9, **kw)
    cd.conduit_distill_loss(cd.distill_opts(reduction="sequence_mean"), x, ids, y, loss2, stats2, mask=mask, **kw)
    return outs


def test_both_ways_of_checking_arguments_are_the_same(monkeypatch):
    assert cd._native_batch is not None and cd._native_rows is not None
    for one in (False, True):
        args = _inputs(4, 9, 700, 6, BF16, 3)
        if one:
            args = [t[1] for t in args]
        a = _calls(*args)
        ws = cd.workspace(1 << 20)
        for gone in ((), ("_native_listed",), ("_native_listed", "_native_batch", "_native_rows")):
            with monkeypatch.context() as m:
                for name in gone:
                    m.setattr(cd, name, None)
                for kw in (dict(), dict(workspace=ws), dict(workspace=ws, stream=torch.cuda.current_stream()),
                           dict(workspace=ws, stream=torch.cuda.current_stream().cuda_stream)):
                    for mask in (args[4], args[4].bool()):
                        for i, (p, q) in enumerate(zip(a, _calls(*args[:4], mask, **kw))):
                            assert torch.equal(p, q), i


def test_native_calls_raise_the_library_s_errors():
    x, tok, ids, y, mask = _inputs(2, 5, 50, 4, F32, 1)
    ws, t, stats = cd.workspace(1 << 20), torch.empty((2, 5), device="cuda"), torch.empty(3, device="cuda")
    for call in (lambda: cd.conduit_listed_logprobs(x, ids, torch.empty_like(y), mask=mask, temperature=-1, workspace=ws),
                 lambda: cd.conduit_listed_logprobs(x, ids, torch.empty_like(y), workspace=ws[:256]),
                 lambda: cd.conduit_listed_logprobs_backward(x, ids, None, y, torch.empty_like(x)),
                 lambda: cd.conduit_token_alternatives(x, ids, y, logp=t, workspace=ws),
                 lambda: cd.conduit_distill_loss(cd.distill_opts(loss="reverse"), x, ids, y, t, stats, workspace=ws),
                 lambda: cd.conduit_distill_loss(cd.distill_opts(), x, ids, y, t, None, workspace=ws)):
        with pytest.raises(cd.ConduitError):
            call()
    with pytest.raises((TypeError, C.ArgumentError)):
        cd.conduit_listed_logprobs(x, ids, torch.empty_like(y), temperature="1", workspace=ws)
    with pytest.raises(ValueError, match="stats"):
        cd.conduit_distill_loss(cd.distill_opts(), x, ids, y, t, stats[:2], workspace=ws)
    with pytest.raises(ValueError, match="must have shape"):
        cd.conduit_listed_logprobs(x, ids, torch.empty_like(y), lse=t[:1], workspace=ws)
    with pytest.raises(ValueError):  # another step between rows
        cd.conduit_listed_logprobs(x, ids, torch.empty_like(y), lse=t, rest=torch.empty((2, 6), device="cuda")[:, 1:], workspace=ws)
    with pytest.raises(TypeError):
        cd.conduit_token_alternatives(x, ids, y, tokens=tok.long(), workspace=ws)


def test_shapes_that_do_not_fit_reach_nothing():
    """What the native check leaves to Python is refused there."""
    x, tok, ids, y, mask = _inputs(2, 5, 50, 4, F32, 1)
    out = torch.full_like(y, 9)
    with pytest.raises(ValueError, match="must have the shape of ids"):
        cd.conduit_listed_logprobs(x, ids, out[..., :3])
    with pytest.raises(ValueError, match="must have shape"):
        cd.conduit_listed_logprobs(x, ids, out, mask=mask[:, :4])
    with pytest.raises(ValueError, match="must have shape"):
        cd.conduit_listed_logprobs(x[:1], ids[:1], out[:1], mask=mask[0])
    with pytest.raises(ValueError, match="logits must be"):
        cd.conduit_listed_logprobs(x[0], ids, out)
    with pytest.raises(ValueError, match="next to each other"):
        cd.conduit_listed_logprobs(x, ids.transpose(0, 1).contiguous().transpose(0, 1)[..., ::2], out[..., :2])
    with pytest.raises(TypeError, match="int32"):
        cd.conduit_listed_logprobs(x, ids.long(), out)
    assert bool((out == 9).all())


def _far_rows(n, width, dtype):
    """n rows FAR elements apart (nothing between them is touched)."""
    return torch.empty((n - 1) * FAR + width, dtype=dtype, device="cuda").as_strided((1, n, width), (0, FAR, 1))


@pytest.mark.parametrize("V,dtype", [(18, BF16), (300, BF16), (700, BF16), (9000, BF16), (70000, BF16), (3001, F32)])
def test_rows_past_32_bits_of_elements(V, dtype):
    """The same results as from rows that follow each other: on a few lanes, a wavefront, a workgroup, in parts."""
    near = _inputs(1, 2, V, 6, dtype, V)
    want = _calls(*near)
    far = _far_rows(2, V, dtype)
    far.copy_(near[0])
    dx = _far_rows(2, V, dtype)
    outs = [torch.full_like(t, 9) for t in want]
    x, tok, ids, y, mask = far, *near[1:]
    outs[8] = outs[11] = dx  # (one after the other: the first is checked below)
    cd.conduit_listed_logprobs(x, ids, outs[5], rest=outs[6], lse=outs[7], mask=mask, temperature=0.9)
    cd.conduit_listed_logprobs_backward(x, ids, outs[7], y, dx, rest=outs[6], drest=outs[7], mask=mask, temperature=0.9)
    assert torch.equal(dx.contiguous(), want[8])
    _calls(x, tok, ids, y, mask, outs)
    for i, (a, b) in enumerate(zip(outs, want)):
        if i != 8:
            assert torch.equal(a.contiguous(), b), i


def test_listed_arrays_past_32_bits_of_elements():
    near = _inputs(1, 2, 500, 7, F32, 2)
    x, tok, ids, y, mask = near
    want = _calls(*near)
    far_ids, far_y, top, lp, listed = [_far_rows(2, 7, t) for t in (torch.int32, F32, torch.int32, F32, F32)]
    far_ids.copy_(ids)
    far_y.copy_(y)
    outs = [torch.full_like(t, 9) for t in want]
    outs[0], outs[1], outs[5] = top, lp, listed
    _calls(x, tok, far_ids, far_y, mask, outs)
    for i, (a, b) in enumerate(zip(outs, want)):
        assert torch.equal(a.contiguous(), b), i


@pytest.mark.parametrize("B,T,V", [(6, 40, 300), (6, 50, 5000), (2, 6, 40000)])
def test_calls_on_another_stream_make_their_own_workspace(B, T, V):
    args = _inputs(B, T, V, 9, BF16, V)
    outs = _calls(*args)
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    busy = torch.randn((2048, 2048), device="cuda")
    side = torch.cuda.Stream()
    x = args[0]
    sizes = [cd.token_alternatives_workspace(x, 9), cd.listed_logprobs_workspace(x, 9), cd.distill_loss_workspace(x, 9)]
    for stream in (side, side.cuda_stream):
        for _ in range(3):
            for t in outs:
                t.fill_(9)
            side.wait_stream(torch.cuda.current_stream())
            for n in sizes:  # memory of the workspaces' sizes, freed while the current stream has yet to write it
                t = torch.empty(n, dtype=torch.uint8, device="cuda")
                torch.mm(busy, busy)
                t.fill_(255)
                del t
            _calls(*args, outs=outs, stream=stream)
            side.synchronize()
            torch.cuda.synchronize()
            for i, (a, b) in enumerate(zip(outs, want)):
                assert torch.equal(a, b), i


def test_two_streams_at_once():
    """Calls that run beside each other, each with a workspace of its own."""
    args = [_inputs(2, 6, 40000, 9, BF16, s) for s in (1, 2)]
    want = [_calls(*a) for a in args]
    streams = [torch.cuda.Stream() for _ in args]
    ws = [cd.workspace(max(cd.token_alternatives_workspace(a[0], 9), cd.listed_logprobs_workspace(a[0], 9),
                           cd.distill_loss_workspace(a[0], 9))) for a in args]
    outs = [[torch.full_like(t, 9) for t in w] for w in want]
    torch.cuda.synchronize()
    for _ in range(20):
        for a, o, s, w in zip(args, outs, streams, ws):
            _calls(*a, outs=o, stream=s, workspace=w)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        for i, (a, b) in enumerate(zip(o, w)):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("rows,V", [((1 << 26) + 3, 70), ((1 << 24) + 3, 2100)])
def test_scores_of_many_rows(rows, V):
    """One row of logits for every token (a wavefront a row; a workgroup of 256): all as the first."""
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn((1, V), generator=g, device="cuda").to(BF16)
    ids, logps, lse = torch.empty((rows, 1), dtype=torch.int32, device="cuda"), torch.empty((rows, 1), device="cuda"), torch.empty(rows, device="cuda")
    cd.conduit_token_alternatives(x.expand(rows, V), ids, logps, lse=lse)
    z = x[0].double()
    assert int(ids[0]) == int(z.argmax()) and bool((ids == ids[0]).all()) and bool((logps == logps[0]).all()) and bool((lse == lse[0]).all())
    each = torch.arange(V, device="cuda", dtype=torch.int32)
    table = torch.empty((V, 1), device="cuda")
    cd.conduit_listed_logprobs(x.expand(V, V), each[:, None].contiguous(), table)
    want = torch.log_softmax(z, -1)
    assert float((table[:, 0].double() - want).abs().max()) <= 2.0 ** -24 * (8 * 3 * 1.4427 * float(z.abs().max()) + 128)
    ids.copy_(torch.randint(0, V, (rows, 1), generator=g, device="cuda", dtype=torch.int32))
    cd.conduit_listed_logprobs(x.expand(rows, V), ids, logps)
    assert torch.equal(logps[:, 0], table[:, 0][ids[:, 0].long()])


def test_gradients_and_divergences_of_more_rows_than_2_26():
    """67 million rows of two bf16 choices, the first listed: both have the same gradient with opposite signs."""
    T = (1 << 26) + 3
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((T, 2), generator=g, device="cuda", dtype=BF16)
    ids = torch.zeros((T, 1), dtype=torch.int32, device="cuda")
    lse, lp, one, dx = torch.empty(T, device="cuda"), torch.empty((T, 1), device="cuda"), torch.ones((T, 1), device="cuda"), torch.full_like(x, 9.0)
    cd.conduit_listed_logprobs(x, ids, lp, lse=lse)
    cd.conduit_listed_logprobs_backward(x, ids, lse, one, dx)
    loss, stats, ddx = torch.empty(T, device="cuda"), torch.empty(3, device="cuda"), torch.full_like(x, 9.0)
    cd.conduit_distill_loss(cd.distill_opts(reduction="sum"), x, ids, one, loss, stats, dlogits=ddx)
    total = 0.0
    for a in range(0, T, 1 << 24):
        s = slice(a, min(T, a + (1 << 24)))
        d = (x[s, 1].double() - x[s, 0].double())
        nll = torch.nn.functional.softplus(d)
        total += float(nll.sum())
        assert bool(((lp[s, 0].double() + nll).abs() <= 2.0 ** -24 * 256).all())
        assert bool(((loss[s].double() - nll).abs() <= 2.0 ** -24 * 1024).all())
        want = torch.sigmoid(d)
        tol = 2.0 ** -8 * want + 2.0 ** -24 * 256
        for got, sign in ((dx, 1), (ddx, -1)):
            assert bool(((got[s, 0].double() - sign * want).abs() <= tol).all())
            assert bool(((got[s, 1].double() + sign * want).abs() <= tol).all())
    assert abs(stats[0].item() - total) <= T * 2.0 ** -24 * 1024 + 2.0 ** -23 * total and stats[2].item() == float(torch.tensor(float(T)))


def test_listed_of_many_split_rows():
    """More than 512 rows in parts: joined by a launch of its own, with numbers twice and entries that are none."""
    B, T, V, K = 1, 520, 140001, 20
    x, tok, ids, y, mask = _inputs(B, T, V, K, F32, 4)
    ids[0, 0, 3:9] = ids[0, 0, 0]
    ids[0, 1, 4] = -1
    logps, rest, lse = torch.empty_like(y), torch.empty((B, T), device="cuda"), torch.empty((B, T), device="cuda")
    cd.conduit_listed_logprobs(x, ids, logps, rest=rest, lse=lse, mask=mask)
    for t in (0, 1, 2, 300, T - 1):
        if not int(mask[0, t]):
            assert float(rest[0, t]) == 0 and not bool(logps[0, t].any())
            continue
        if t == 1:
            assert float(logps[0, t, 4]) == -float("inf")
            continue
        z = torch.log_softmax(x[0, t].double(), -1)
        tol = 2.0 ** -24 * (8 * 3 * 1.4427 * float(x[0, t].abs().max()) + 128)
        assert float((logps[0, t].double() - z[ids[0, t].long()]).abs().max()) <= tol
        others = z.clone()
        others[ids[0, t].long()] = -float("inf")
        assert abs(float(rest[0, t]) - float(torch.logsumexp(others, 0))) <= tol
        assert abs(float(lse[0, t]) - float(torch.logsumexp(x[0, t].double(), 0))) <= tol
