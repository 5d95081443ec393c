"""Token losses: the binding's two ways of checking arguments give the same calls, and offsets past 32 bits reach
the right elements."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2609_24456_amd import conduit as cd  # noqa: E402

BF16 = torch.bfloat16


def _every_call(seed):
    """The outputs of all calls on views of columns [1, T) of one small batch."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    B, T, V, H = 4, 9, 700, 64
    per = lambda: torch.zeros((B, T), device="cuda")[:, 1:]  # noqa: E731
    tok = torch.randint(0, V, (B, T), generator=g, device="cuda", dtype=torch.int32)[:, 1:]
    mask = (torch.rand((B, T), generator=g, device="cuda") < 0.8).to(torch.uint8)[:, 1:]
    x, old, adv = rn(B, T, V).to(BF16)[:, :-1], rn(B, T)[:, 1:], rn(B, T)[:, 1:]
    hid, w = rn(B, T, H).to(BF16)[:, :-1], rn(V, H).to(BF16)
    lp, lse, ent, dl, dh = per(), per(), per(), per(), per()
    out = [lp, lse, ent, dl, dh]
    cd.conduit_token_logprobs(x, tok, lp, lse=lse, entropy=ent, mask=mask)
    stats = torch.empty(8, device="cuda")
    cd.conduit_policy_loss(cd.policy_opts(entropy_coef=0.01), lp, adv, stats, dl, old_logp=old, entropy=ent, dentropy=dh, mask=mask)
    dx = torch.empty((B, T - 1, V), dtype=BF16, device="cuda")
    cd.conduit_token_logprobs_backward(x, tok, lse, dl, dx, entropy=ent, dentropy=dh, mask=mask)
    out += [stats, dx]
    s2, lp2, en2, dx2 = torch.empty(8, device="cuda"), per(), per(), torch.empty_like(dx)
    cd.conduit_policy_loss_logits(cd.policy_opts(), x, tok, adv, s2, dx2, lp2, en2, old_logp=old, mask=mask)
    loss, s3, dp = torch.empty(B // 2, device="cuda"), torch.empty(4, device="cuda"), per()
    cd.conduit_preference_loss(cd.preference_opts(), lp, loss, s3, dp, mask=mask)
    hl, hs, he = per(), per(), per()
    cd.conduit_head_logprobs(hid, w, tok, hl, lse=hs, entropy=he, mask=mask)
    dhid, dw = torch.empty((B, T - 1, H), dtype=BF16, device="cuda"), torch.empty_like(w)
    cd.conduit_head_logprobs_backward(hid, w, tok, hs, dl, dhid, dw, entropy=he, dentropy=dh, mask=mask)
    return out + [s2, lp2, en2, dx2, loss, s3, dp, hl, hs, he, dhid, dw]


def test_both_ways_of_checking_arguments_are_the_same(monkeypatch):
    assert cd._native_batch is not None and cd._native_rows is not None
    a = _every_call(3)
    monkeypatch.setattr(cd, "_native_batch", None)
    monkeypatch.setattr(cd, "_native_rows", None)
    for i, (x, y) in enumerate(zip(a, _every_call(3))):
        assert torch.equal(x, y), i


FAR = (1 << 31) + 24  # elements: past 32 bits of elements and, at 2 and 4 bytes, of bytes


def _far_rows(n, width, dtype):
    """n rows FAR elements apart (nothing between them is touched)."""
    return torch.empty((n - 1) * FAR + width, dtype=dtype, device="cuda").as_strided((1, n, width), (0, FAR, 1))


@pytest.mark.parametrize("V", [300, 700, 9000, 70000])
def test_logits_past_32_bits_of_elements(V):
    """The same results as from rows that follow each other: a wavefront's part, a wavefront, a workgroup, parts."""
    g = torch.Generator(device="cuda").manual_seed(V)
    near = torch.randn((1, 2, V), generator=g, device="cuda").to(BF16)
    tok = torch.randint(0, V, (1, 2), generator=g, device="cuda", dtype=torch.int32)
    far, dfar, dnear = _far_rows(2, V, BF16), _far_rows(2, V, BF16), torch.empty_like(near)
    far.copy_(near)
    res = []
    for x, dx in ((near, dnear), (far, dfar)):
        lp, lse, ent = (torch.empty((1, 2), device="cuda") for _ in range(3))
        stats = torch.empty(8, device="cuda")
        cd.conduit_token_logprobs(x, tok, lp, lse=lse, entropy=ent)
        cd.conduit_token_logprobs_backward(x, tok, lse, torch.ones_like(lp), dx)
        first = dx.contiguous().clone()
        cd.conduit_policy_loss_logits(cd.policy_opts(), x, tok, torch.ones_like(lp), stats, dx, lp, ent)
        res.append([lp, lse, ent, stats, first, dx.contiguous()])
    for i, (a, b) in enumerate(zip(*res)):
        assert torch.equal(a, b), i


def test_token_arrays_past_32_bits_of_elements():
    g = torch.Generator(device="cuda").manual_seed(1)
    T, S = 40, (1 << 31) + 8
    near = [torch.randn((2, T), generator=g, device="cuda") for _ in range(2)] + [torch.zeros((2, T), device="cuda")]
    far = [torch.empty(S + T, device="cuda").as_strided((2, T), (S, 1)) for _ in near]
    for f, n in zip(far, near):
        f.copy_(n)
    res = []
    for lp, adv, d in (near, far):
        stats, s4, loss = torch.empty(8, device="cuda"), torch.empty(4, device="cuda"), torch.empty(1, device="cuda")
        cd.conduit_policy_loss(cd.policy_opts(reduction="sum"), lp, adv, stats, d)
        first = d.contiguous().clone()
        cd.conduit_preference_loss(cd.preference_opts(), lp, loss, s4, d)
        res.append([stats, first, s4, loss, d.contiguous()])
    for i, (a, b) in enumerate(zip(*res)):
        assert torch.allclose(a, b, rtol=2.0 ** -20, atol=0), i  # (statistics: another order of the sums)


def test_hidden_states_past_32_bits_of_elements():
    g = torch.Generator(device="cuda").manual_seed(2)
    H, V = 64, 500
    near = torch.randn((1, 20, H), generator=g, device="cuda").to(BF16)[:, :2]
    w = torch.randn((V, H), generator=g, device="cuda").to(BF16)
    tok = torch.randint(0, V, (1, 2), generator=g, device="cuda", dtype=torch.int32)
    far, dfar, dnear = _far_rows(2, H, BF16), _far_rows(2, H, BF16), torch.empty((1, 2, H), dtype=BF16, device="cuda")
    far.copy_(near)
    res = []
    for x, dx in ((near, dnear), (far, dfar)):
        lp, lse = torch.empty((1, 2), device="cuda"), torch.empty((1, 2), device="cuda")
        dw = torch.empty_like(w)
        cd.conduit_head_logprobs(x, w, tok, lp, lse=lse)
        cd.conduit_head_logprobs_backward(x, w, tok, lse, torch.ones_like(lp), dx, dw)
        res.append([lp, lse, dx.contiguous(), dw])
    for i, (a, b) in enumerate(zip(*res)):
        assert torch.equal(a, b), i
