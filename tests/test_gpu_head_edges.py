"""Calls at the edges of what the operators around the projection allow, on the GPU."""
import math
from fractions import Fraction

import pytest
import torch

import head_plain as hp
import paper_2609_14306_amd as vp
import test_gpu_norm as norms

pytestmark = pytest.mark.gpu


def test_squared_preference_with_a_smoothing_that_it_does_not_use():
    g = torch.Generator().manual_seed(4)
    loss, ref = (torch.rand(500, generator=g).cuda() for _ in range(2))
    targets = torch.zeros(500, dtype=torch.int64, device="cuda")
    start = torch.tensor([0, 100, 180, 300, 500], dtype=torch.int32, device="cuda")
    want = vp.preference_forward(loss, targets, start, vp.Preference("squared", 0.3, 0.1), ref)
    got = vp.preference_forward(loss, targets, start, vp.Preference("squared", 0.3, 0.1, 0.1), ref)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("S", [2, 2049, 2050, 4098, 40000])
def test_sequences_without_tokens(S):
    """No tokens at all, in more sequences than one workgroup takes: sums of 0 and the loss of a
    pair at -margin."""
    none, ids = torch.empty(0, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    start, adv = torch.zeros(S + 1, dtype=torch.int32, device="cuda"), torch.ones(S, device="cuda")
    for mean in (False, True):
        out = vp.policy_forward(none, ids, start, vp.Policy(kl_coef=0.1), adv, none, none, mean=mean)
        assert all(bool((v == 0).all()) for v in out)
        grad = vp.policy_backward(none, ids, start, vp.Policy(kl_coef=0.1), adv, out[3], adv, none, none, mean=mean)
        assert grad.numel() == 0
        if S % 2 == 0:
            pair, reward, coef = vp.preference_forward(none, ids, start, vp.Preference(beta=0.5, margin=0.75), none,
                                                       mean=mean)
            assert bool((reward == 0).all())
            want = math.log1p(math.exp(0.75))
            assert bool(((pair.double() - want).abs() <= want * 2.0 ** -24).all())
            # a sequence without tokens weighs 1, or 0 in the mean
            half = 0.0 if mean else 0.5 / (1 + math.exp(-0.75))
            sign = torch.tensor([-1.0, 1.0], device="cuda").repeat(S // 2)
            assert bool(((coef.double() * -sign - half).abs() <= half * 2.0 ** -24 * 1.01).all())
            assert vp.preference_backward(ids, start, coef, adv[:S // 2].contiguous()).numel() == 0


@pytest.mark.parametrize("what", ["dbeta missing", "dgamma's shape", "dbeta's type", "unaligned", "on the CPU"])
def test_wrong_norm_gradients_leave_dw_alone(what):
    """`backward` refuses a dnorm before it adds to anything."""
    d = 64
    f = lambda *s: torch.rand(*s, device="cuda")  # noqa: E731
    X, W, targets = f(20, d), [f(100, d)], torch.zeros(20, dtype=torch.int64, device="cuda")
    norm = vp.HeadNorm(f(d), f(d))
    lse = vp.forward(X, W, targets, norm=norm)[1]
    dW = [torch.full((100, d), 3.0, device="cuda")]
    dnorm = {"dbeta missing": (f(d), None), "dgamma's shape": (f(d + 8), f(d)), "dbeta's type": (f(d), f(d).double()),
             "unaligned": (f(d + 1)[1:], f(d)), "on the CPU": (f(d), f(d).cpu())}[what]
    with pytest.raises((ValueError, vp.VpError)):
        vp.backward(X, W, targets, lse, f(20), norm=norm, dW_shards=dW, accumulate=True, dnorm=dnorm)
    torch.cuda.synchronize()
    assert bool((dW[0] == 3).all())


def _kl(q):
    """e^q - q - 1 without a difference of nearly equal numbers."""
    if abs(q) > 1:
        return math.expm1(q) - q
    total, term = Fraction(0), Fraction(q)
    for k in range(2, 30):
        term = term * Fraction(q) / k
        total += term
    return float(total)


def test_small_log_ratios_keep_their_digits():
    """The KL term and its gradient of log ratios down to where float32 ends: each is one rounding
    of the exact value (2^-24), for which the float64 arithmetic has 2^-40 to spend."""
    q = [s * m * 10.0 ** -k for k in range(22) for m in (1.0, 3.4657, 3.466) for s in (1, -1)] + [7.5, -30.0, 80.0]
    loss = torch.tensor([max(v, 0.0) for v in q])
    ref = torch.tensor([max(-v, 0.0) for v in q])
    T = len(q)
    exact = [a - b for a, b in zip(loss.double().tolist(), ref.double().tolist())]
    targets = torch.zeros(T, dtype=torch.int64, device="cuda")
    start = torch.arange(T + 1, dtype=torch.int32, device="cuda")
    pol, adv, one = vp.Policy(kl_coef=0.5), torch.zeros(T, device="cuda"), torch.ones(T, device="cuda")
    seq_loss, kl, _, tokens = vp.policy_forward(loss.cuda(), targets, start, pol, adv, None, ref.cuda())
    grad = vp.policy_backward(loss.cuda(), targets, start, pol, adv, tokens, one, None, ref.cuda())
    for got, want in ((kl, [_kl(v) for v in exact]), (seq_loss, [0.5 * _kl(v) for v in exact]),
                      (grad, [0.5 * math.expm1(v) for v in exact])):
        want = torch.tensor(want, dtype=torch.float64)
        err = (got.double().cpu() - want).abs()
        bad = err > (2.0 ** -24 + 2.0 ** -40) * want.abs() + 2.0 ** -149
        assert not bool(bad.any()), [(exact[i], float(got[i]), float(want[i])) for i in bad.nonzero()[:4, 0].tolist()]


@pytest.mark.parametrize("T, d", [(50, 2880), (20, 7168), (9, 16384), (60, 1000), (300, 64), (40, 264)])
@pytest.mark.parametrize("dtype, offset", [(torch.bfloat16, 30.0), (torch.bfloat16, 3.9), (torch.float32, 1000.0),
                                           (torch.float32, 4.1), (torch.float32, -3.9)])
def test_offset_above_the_spread(T, d, dtype, offset):
    """Rows whose mean is up to 1000 times their spread (float32) or 30 times (bfloat16, whose
    values are 1/256 of the mean apart).  With u = 2^-24 and chains of at most DEPTH = 144
    additions: the mean of the first sum is off by e0 = 146 u mean|x|, the distances c from it by
    u |c|, and what is left of the mean in them, taken from their own sum where the mean is more
    than 4 spreads away, by e = 146 u mean|c|.  So Y does not depend on how far away the mean is:
    its centre is off by e (e0 within 4 spreads) + 2 u |c| and its rstd by 77 u, relative, and
    half of e0^2 / var where that is left in it; the mean by u |mean| and e or e0."""
    u, depth = 2.0 ** -24, 144
    g = torch.Generator().manual_seed(T + d)
    X = (offset + torch.randn(T, d, generator=g)).to(dtype)
    gamma, beta = (1 + 0.2 * torch.randn(d, generator=g)).to(dtype), torch.randn(d, generator=g).to(dtype)
    Y, mean, rstd = (v.double().cpu() for v in vp.layer_norm(X.cuda(), gamma.cuda(), beta.cuda(), 1e-5))
    y, mu, r = hp.norm_forward(X, gamma, beta, 1e-5, False)
    x, ga = X.double(), gamma.double().abs()
    e0 = (depth + 2) * u * x.abs().mean(1)
    c = (x - mu[:, None]).abs() + e0[:, None]
    far = mu ** 2 > 16.01 / r ** 2
    e = torch.where(far, (depth + 2) * u * c.mean(1), e0)
    e_r = 77 * u + torch.where(far, 0.0, 0.5 * e0 ** 2 * r ** 2)
    assert bool(((mean - mu).abs() <= 1.01 * (u * mu.abs() + e)).all())
    assert bool(((rstd - r).abs() <= e_r * r).all())
    xh = c * r[:, None]
    bound = ga * ((r * e)[:, None] + xh * (e_r + 8 * u)[:, None]) + 2 * u * (ga * xh + beta.double().abs())
    half = torch.finfo(dtype).eps / 2
    err = (Y - y).abs() - (bound * (1 + half) + half * y.abs())
    assert bool((err <= 0).all()), float(err.max())


@pytest.mark.parametrize("value", [0.1, 1000.1, -3e4])
@pytest.mark.parametrize("d", [40, 2880, 16384])
def test_constant_rows(value, d):
    """A row of one value v has nothing but its bias: what is left of its mean is at most
    e0 = 146 u |v| in front of the correction and 148 u e0 behind it, times eps^-1/2."""
    u = 2.0 ** -24
    X = torch.full((5, d), value, device="cuda")
    gamma, beta = torch.ones(d, device="cuda"), torch.full((d,), 0.25, device="cuda")
    Y, mean, rstd = vp.layer_norm(X, gamma, beta, 1e-5)
    left = 148 * u * 146 * u * abs(value)
    assert bool(((Y.double() - 0.25).abs() <= left * 1e-5 ** -0.5 * 1.01 + u).all())
    assert bool(((mean.double() - float(X[0, 0])).abs() <= 1.01 * (u * abs(value) + left)).all())
    assert bool(((rstd.double() - 1e-5 ** -0.5).abs() <= 1e-5 ** -0.5 * 80 * u).all())


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("d", [2056, 3448, 3456, 3464, 4088, 4096, 4104])
def test_widths_around_the_layouts_of_bfloat16(d, rms):
    X, gamma, beta, _ = norms._make(37, d, torch.bfloat16)
    norms._check_forward(X, gamma, beta, 1e-5, rms, vp.layer_norm(X, gamma, beta, 1e-5, rms))


@pytest.mark.parametrize("T, S", [(128, 2 ** 22), (700, 2 ** 20), (70000, 300000)])
def test_long_runs_of_empty_sequences(T, S):
    """Sequences of tokens with up to millions of empty ones between them: sums of whole numbers,
    exact, and the gradient of each token's own sequence."""
    g = torch.Generator().manual_seed(S)
    where = torch.randint(0, T + 1, (40,), generator=g).sort().values  # the offsets that there are
    start = where[torch.randint(0, 40, (S + 1,), generator=g).sort().values].int()
    start[0], start[-1] = 0, T
    loss = torch.randint(0, 64, (T,), generator=g).float()
    targets = torch.where(torch.rand(T, generator=g) < 0.3, -100, 5)
    seq = torch.searchsorted(start.long(), torch.arange(T), right=True) - 1
    keep, up = targets != -100, torch.randint(1, 100, (S,), generator=g).float()
    adv = torch.randint(-3, 4, (S,), generator=g).float()
    dev = [v.cuda() for v in (loss, targets, start)]
    out = vp.policy_forward(*dev, vp.Policy(), adv.cuda())
    n = torch.zeros(S).index_add_(0, seq[keep], torch.ones(int(keep.sum())))
    assert torch.equal(out[3].cpu(), n.int()) and torch.equal(out[0].cpu(), -adv * n)
    grad = vp.policy_backward(*dev, vp.Policy(), adv.cuda(), out[3], up.cuda())
    assert torch.equal(grad.cpu(), torch.where(keep, up[seq] * adv[seq], torch.zeros(T)))
    if S % 2 == 0:
        _, reward, coef = vp.preference_forward(*dev, vp.Preference(beta=1.0))
        total = torch.zeros(S).index_add_(0, seq[keep], loss[keep])
        assert torch.equal(reward.cpu(), -total)
