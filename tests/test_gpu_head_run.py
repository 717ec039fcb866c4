"""A whole head step on the GPU: layer norm, projection, a loss of whole sequences, and their
gradients back to the norm's input, against the same step in float64 with automatic
differentiation.

Bars as for the projection alone (tests/helpers.py), relative Frobenius errors of 1e-5 in float32
and 1e-2 in bfloat16: each gradient is a chain of the projection's, weighted per token.  Losses in
float32: a token's loss is within 1e-5 max(1, loss), a sequence's sum within n times that, and the
policy's ratios at most double it (they stay below 1.4 here, plus the KL's slope).  Losses in
bfloat16 are compared with the float64 step on the norm's own rounded output."""
import pytest
import torch

import helpers
import paper_2609_14306_amd as vp

pytestmark = pytest.mark.gpu
IGNORE = -100


def _setup(dtype, seed):
    T, d, rows = 203, 320, [700, 0, 301, 500]
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    X = (0.5 + 2 * n(T, d)).to(dtype)
    gamma, beta = (1 + 0.2 * n(d)).to(dtype), (0.2 * n(d)).to(dtype)
    Ws = [(n(r, d) * d ** -0.5).to(dtype) for r in rows]
    targets = torch.randint(0, sum(rows), (T,), generator=g)
    targets[torch.rand(T, generator=g) < 0.2] = IGNORE
    targets[40] = 5  # the sequence of one token
    start = torch.tensor([0, 40, 41, 120, 195], dtype=torch.int32)
    return X, gamma, beta, Ws, targets, start, g


class _Round(torch.autograd.Function):
    """The rounding of the norm's output to its type; gradients pass."""

    @staticmethod
    def forward(ctx, y, dtype):
        return y.to(dtype).double()

    @staticmethod
    def backward(ctx, g):
        return g, None


def _float64_nll(X, gamma, beta, Ws, targets, rms, eps, dtype):
    x, ga, be = (v.double().requires_grad_() for v in (X, gamma, beta))
    W = torch.cat(Ws).double().requires_grad_()
    mu = 0.0 if rms else x.mean(1, keepdim=True)
    y = (x - mu) / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + eps) * ga + be
    logits = _Round.apply(y.to(torch.float32), dtype) @ W.t()
    at = targets.clamp_min(0)
    nll = torch.logsumexp(logits, 1) - logits.gather(1, at[:, None])[:, 0]
    return torch.where(targets == IGNORE, 0.0, nll), (x, ga, be, W)


def _compare(dtype, got, leaves, what):
    name = "bf16" if dtype == torch.bfloat16 else "f32"
    dX, dWs, dgamma, dbeta = got
    x, ga, be, W = leaves
    for label, a, b in (("dX", dX, x.grad), ("dW", torch.cat(dWs), W.grad), ("dgamma", dgamma, ga.grad),
                        ("dbeta", dbeta, be.grad)):
        helpers.assert_grad_close(name, a.cpu(), b, f"{what} {label}")


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_policy_step(dtype, rms):
    X, gamma, beta, Ws, targets, start, g = _setup(dtype, 1)
    norm = vp.HeadNorm(gamma.cuda(), beta.cuda(), 1e-5, rms)
    Xd, Wd, td, sd = X.cuda(), [w.cuda() for w in Ws], targets.cuda(), start.cuda()
    loss, lse = vp.forward(Xd, Wd, td, norm=norm)
    nll, leaves = _float64_nll(X, gamma, beta, Ws, targets, rms, 1e-5, dtype)
    old = (nll.detach() + 0.6 * (torch.rand(203, generator=g) - 0.5)).clamp_min(0).float()
    # no ratio so near a bound that the projection's float error decides its side
    for b in (0.2, -0.2):
        edge = torch.log1p(torch.tensor(b, dtype=torch.float64))
        near = (old.double() - nll.detach() - edge).abs() < 0.01
        old[near] += 0.03
    ref = (nll.detach() + 0.4 * (torch.rand(203, generator=g) - 0.5)).clamp_min(0).float()
    adv = torch.tensor([1.0, -0.5, -2.0, 0.7])
    pol = vp.Policy(0.2, 0.2, 0.1)
    seq_loss, kl, clipped, tokens = vp.policy_forward(loss, td, sd, pol, adv.cuda(), old.cuda(), ref.cuda(), mean=True)
    up = torch.full((4,), 0.25)
    grad = vp.policy_backward(loss, td, sd, pol, adv.cuda(), tokens, up.cuda(), old.cuda(), ref.cuda(), mean=True)
    got = vp.backward(Xd, Wd, td, lse, grad, norm=norm)

    want, n_clip = [], []
    for s in range(4):
        at = [t for t in range(int(start[s]), int(start[s + 1])) if targets[t] != IGNORE]
        rho = torch.exp(old.double()[at] - nll[at])
        q = nll[at] - ref.double()[at]
        l = -torch.minimum(rho * adv[s], rho.clamp(0.8, 1.2) * adv[s]) + 0.1 * (torch.exp(q) - q - 1)
        want.append(l.mean())
        n_clip.append(int(((rho > 1.2) if adv[s] > 0 else (rho < 0.8)).sum()))
    want = torch.stack(want)
    (want.sum() * 0.25).backward()
    bar = 1e-5 if dtype == torch.float32 else 2e-3
    worst = float((loss.cpu().double() - nll.detach()).abs().max())
    assert worst <= bar * max(1.0, float(nll.detach().max()))
    # |d l / d nll| <= 1.4 |A| + 0.1 (e^0.4 - 1)
    assert bool(((seq_loss.cpu() - want).abs() <= (1.4 * adv.abs() + 0.1) * worst + 1e-6).all())
    assert clipped.tolist() == n_clip and sum(n_clip) > 0
    _compare(dtype, got, leaves, "policy")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_preference_step(dtype):
    X, gamma, beta, Ws, targets, start, g = _setup(dtype, 2)
    norm = vp.HeadNorm(gamma.cuda(), beta.cuda())
    Xd, Wd, td, sd = X.cuda(), [w.cuda() for w in Ws], targets.cuda(), start.cuda()
    loss, lse = vp.forward(Xd, Wd, td, norm=norm)
    nll, leaves = _float64_nll(X, gamma, beta, Ws, targets, False, 1e-5, dtype)
    ref = (nll.detach() + 0.2 * torch.randn(203, generator=g)).clamp_min(0).float()
    pref = vp.Preference("logistic", 0.2, 0.1, 0.05)
    pair, reward, coef = vp.preference_forward(loss, td, sd, pref, ref.cuda())
    grad = vp.preference_backward(td, sd, coef, torch.full((2,), 0.5, device="cuda"))
    dW = [torch.ones(w.shape, device="cuda") for w in Wd]
    dn = (torch.ones(320, device="cuda"), torch.ones(320, device="cuda"))
    got = vp.backward(Xd, Wd, td, lse, grad, norm=norm, dnorm=dn, dW_shards=dW, accumulate=True)
    assert got[2] is dn[0] and got[3] is dn[1]
    got = (got[0], [w - 1 for w in dW], dn[0] - 1, dn[1] - 1)

    R = []
    for s in range(4):
        at = [t for t in range(int(start[s]), int(start[s + 1])) if targets[t] != IGNORE]
        R.append(0.2 * (ref.double()[at] - nll[at]).sum())
    z = torch.stack([R[0] - R[1], R[2] - R[3]]) - 0.1
    want = 0.95 * torch.nn.functional.softplus(-z) + 0.05 * torch.nn.functional.softplus(z)
    (want.sum() * 0.5).backward()
    bar = 1e-5 if dtype == torch.float32 else 2e-3
    worst = bar * max(1.0, float(nll.detach().max())) * 203 * 0.2
    assert bool(((pair.cpu() - want).abs() <= worst).all())
    _compare(dtype, got, leaves, "preference")


def test_norm_of_the_projection_equals_its_parts():
    X, gamma, beta, Ws, targets, start, _ = _setup(torch.bfloat16, 3)
    norm = vp.HeadNorm(gamma.cuda(), None)
    Xd, Wd, td = X.cuda(), [w.cuda() for w in Ws], targets.cuda()
    Y, mean, rstd = vp.layer_norm(Xd, norm.gamma)
    a, b = vp.forward(Xd, Wd, td, norm=norm), vp.forward(Y, Wd, td)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    g = torch.rand(203, device="cuda")
    dX, dW, dgamma, dbeta = vp.backward(Xd, Wd, td, a[1], g, norm=norm)
    dH, dW2 = vp.backward(Y, Wd, td, a[1], g)
    want = vp.layer_norm_backward(Xd, norm.gamma, mean, rstd, dH, bias=False)
    assert dbeta is None and torch.equal(dX, want[0]) and torch.equal(dgamma, want[1])
    assert all(torch.equal(x, y) for x, y in zip(dW, dW2))
