"""The operators together, as a user runs them: a residual's addition and norm with 8-bit rows, weights
quantised once, rollouts scored under the 8-bit model and under the trained one, a clipped policy loss
against the first with an entropy bonus, and the gradients of the head; against float64 automatic
differentiation of the same sum."""
import pytest
import torch

import paper_2609_14306_amd as vp
import score_plain as sp

pytestmark = pytest.mark.gpu


def test_policy_step_against_an_8_bit_reference():
    T, d, rows, S = 600, 384, [700, 0, 901], 5
    g = torch.Generator(device="cuda").manual_seed(4)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    X, R = n(T, d), n(T, d)
    gamma = 1 + 0.1 * n(d)
    W = [n(r, d) / d ** 0.5 for r in rows]
    t = torch.randint(0, 1601, (T,), generator=g, device="cuda")
    t[::9] = -100
    start = torch.tensor([0, 100, 100, 350, 560, 590], dtype=torch.int32, device="cuda")
    adv, coef = n(S), 0.02

    # the reference model, in 8 bits
    sums, (h8, hk), _, _ = vp.add_norm(X, R, gamma, rms=True, f8=True)
    W8, Wk = map(list, zip(*[vp.quantize(w, 128) for w in W]))
    ref, _, _, ids, _ = vp.score_f8(h8, hk, W8, Wk, t, top=4)
    ref_y = sp.values(h8, hk, 1) @ torch.cat([sp.values(w, k, 128) for w, k in zip(W8, Wk)]).t().contiguous()
    live = t != -100
    want_ref = -torch.log_softmax(ref_y, 1).gather(1, torch.where(live, t, 0)[:, None])[:, 0] * live
    assert bool(((ref.double() - want_ref).abs() <= 1e-4).all())
    assert torch.equal(ids, torch.sort(ref_y, dim=1, descending=True, stable=True).indices[:, :4])

    # the trained one
    S2, Y, mean, rstd = vp.add_norm(X, R, gamma, rms=True)
    assert torch.equal(S2, sums)
    loss, lse, ent, _, _ = vp.score(Y, W, t)
    pol = vp.Policy(0.2, 0.3, 0.05)
    seq_loss, _, _, tokens = vp.policy_forward(loss, t, start, pol, adv, None, ref, mean=True)
    grad_loss = vp.policy_backward(loss, t, start, pol, adv, tokens, torch.full((S,), 1.0 / S, device="cuda"), None, ref, mean=True)
    grad_ent = torch.where(live, -coef / T, 0.0)
    dY, dW = vp.backward(Y, W, t, lse, grad_loss, entropy=ent, grad_entropy=grad_ent)
    dX, dgamma, _ = vp.add_norm_backward(S2, gamma, mean, rstd, dY, None, bias=False)

    # the same sum in float64
    x, ga = S2.double().requires_grad_(), gamma.double().requires_grad_()
    w = torch.cat(W).double().requires_grad_()
    logp = torch.log_softmax(x * ((x * x).mean(1, keepdim=True) + 1e-5).rsqrt() * ga @ w.t(), 1)
    nll = -logp.gather(1, torch.where(live, t, 0)[:, None])[:, 0]
    q = nll - ref.double()
    token = -torch.exp(nll.detach() - nll) * torch.repeat_interleave(torch.cat([adv, adv.new_zeros(1)]).double(),
        torch.cat([start.diff(), start.new_tensor([T - 590])]).long()) + 0.05 * (torch.exp(q) - q - 1)
    total = 0.0
    for a, b in zip(start.tolist()[:-1], start.tolist()[1:]):
        k = live[a:b]
        if k.any():
            total = total + token[a:b][k].mean() / S
    total = total - coef / T * (-(logp.exp() * logp).sum(1) * live).sum()
    gx, gg, gw = torch.autograd.grad(total, (x, ga, w))
    for got, want, what in ((dX, gx, "dX"), (dgamma, gg, "dgamma"), (torch.cat(dW), gw, "dW")):
        assert ((got.double() - want).norm() / want.norm()).item() <= 2e-5, what
