"""Loss calls on a stream of their own that make their workspaces themselves, while torch's current stream still writes
memory that was freed on it."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2609_24456_amd import conduit as cd  # noqa: E402

BF16 = torch.bfloat16


def test_a_new_workspace_shares_nothing_with_memory_freed_on_another_stream():
    side = torch.cuda.Stream()
    n = 3 << 20
    gone = torch.empty(n, dtype=torch.uint8, device="cuda")
    at = gone.data_ptr()
    del gone
    ws = cd.workspace(n, stream=side)
    assert ws.data_ptr() + n <= at or at + n <= ws.data_ptr()
    side.synchronize()
    assert not bool(ws.any())


def test_calls_on_another_stream_make_their_own_workspace():
    g = torch.Generator(device="cuda").manual_seed(4)
    B, T, V, H = 6, 40, 9000, 128
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, adv, old = rn(B, T, V).to(BF16), rn(B, T), -rn(B, T).abs()
    hid, w = rn(B, T, H).to(BF16), rn(V, H).to(BF16)
    tok = torch.randint(0, V, (B, T), generator=g, device="cuda", dtype=torch.int32)
    mask = (torch.rand((B, T), generator=g, device="cuda") < 0.7).to(torch.uint8)
    opts = cd.policy_opts(kl_coef=0.1, entropy_coef=0.01)
    busy = rn(2048, 2048)

    f = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
    stats, lp, en, dx = f(8), f(B, T), f(B, T), torch.empty_like(x)
    loss, s4, hl, hs = f(B // 2), f(4), f(B, T), f(B, T)
    dh, dw = torch.empty_like(hid), torch.empty_like(w)
    outs = [stats, lp, en, dx, loss, s4, hl, hs, dh, dw]  # (made here: the current stream's memory too)

    def calls(stream):
        cd.conduit_policy_loss_logits(opts, x, tok, adv, stats, dx, lp, en, old_logp=old, mask=mask, stream=stream)
        cd.conduit_preference_loss(cd.preference_opts(), lp, loss, s4, mask=mask, stream=stream)
        cd.conduit_head_logprobs(hid, w, tok, hl, lse=hs, mask=mask, stream=stream)
        cd.conduit_head_logprobs_backward(hid, w, tok, hs, adv, dh, dw, mask=mask, stream=stream)

    calls(None)
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    sizes = [cd.policy_loss_logits_workspace(x), cd.preference_loss_workspace(B // 2, T), cd.head_logprobs_workspace(hid, w),
             cd.head_logprobs_backward_workspace(hid, w)]
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
            calls(stream)
            side.synchronize()
            torch.cuda.synchronize()
            for i, (a, b) in enumerate(zip(outs, want)):
                assert torch.equal(a, b), i
