"""Plain float64 forms of the operators around the projection, on the CPU, one row or one
sequence at a time, for the tests."""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24  # half a step of float32, relative


def norm_forward(X, gamma, beta, eps, rms):
    x = X.double().cpu()
    mean = torch.zeros(x.shape[0], dtype=torch.float64) if rms else x.mean(1)
    c = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((c * c).mean(1) + eps)
    y = c * rstd[:, None] * gamma.double().cpu()
    return (y if beta is None else y + beta.double().cpu()), mean, rstd


def norm_backward(X, gamma, mean, rstd, dY):
    """From the mean (None: 0) and rstd that the forward left."""
    x, dy, r = X.double().cpu(), dY.double().cpu(), rstd.double().cpu()[:, None]
    xh = (x if mean is None else x - mean.double().cpu()[:, None]) * r
    g = dy * gamma.double().cpu()
    c1 = torch.zeros_like(r) if mean is None else g.mean(1, keepdim=True)
    c2 = (g * xh).mean(1, keepdim=True)
    return r * (g - c1 - xh * c2), (dy * xh).sum(0), dy.sum(0)


def spans(start, T):
    start = [int(v) for v in start]
    return list(zip(start[:-1], start[1:]))


def weight(n, mean):
    return 1.0 if not mean else (1.0 / n if n else 0.0)


def pref_forward(loss, targets, start, kind, beta, margin, smoothing, ref, ignore, mean):
    loss, targets = loss.double().cpu(), targets.cpu()
    ref = None if ref is None else ref.double().cpu()
    R, c = [], []
    for a, b in spans(start, len(loss)):
        keep = targets[a:b] != ignore
        ratio = (-loss[a:b] if ref is None else ref[a:b] - loss[a:b])[keep]
        c.append(weight(int(keep.sum()), mean))
        R.append(float(ratio.sum()) * c[-1] if len(ratio) else 0.0)
    reward = [beta * r for r in R]
    out = []
    for i in range(len(R) // 2):
        z = reward[2 * i] - reward[2 * i + 1] - margin
        if kind == "logistic":
            soft = lambda v: v + math.log1p(math.exp(-v)) if v > 0 else math.log1p(math.exp(v))  # noqa: E731
            out.append((1 - smoothing) * soft(-z) + smoothing * soft(z))
        else:
            out.append(((z - 0.5) / beta) ** 2)
    return torch.tensor(out, dtype=torch.float64), torch.tensor(reward, dtype=torch.float64), c


def pref_backward(loss, targets, start, kind, beta, margin, smoothing, ref, ignore, mean, grad_pair):
    _, reward, c = pref_forward(loss, targets, start, kind, beta, margin, smoothing, ref, ignore, mean)
    grad = torch.zeros(len(loss), dtype=torch.float64)
    targets = targets.cpu()
    for s, (a, b) in enumerate(spans(start, len(loss))):
        i = s // 2
        z = float(reward[2 * i] - reward[2 * i + 1]) - margin
        if kind == "logistic":
            sig = 1 / (1 + math.exp(-z)) if z > -700 else 0.0
            slope = sig - (1 - smoothing)
        else:
            slope = 2 * (z - 0.5) / beta ** 2
        sign = 1.0 if s % 2 else -1.0
        keep = targets[a:b] != ignore
        grad[a:b][keep] = sign * slope * beta * c[s] * float(grad_pair[i])
    return grad


def policy_tokens(loss, old, ref, adv, low, high, kl_coef):
    """l, kl, clipped, d l / d loss of tokens, float64."""
    x = torch.zeros_like(loss) if old is None else old - loss
    rho = torch.exp(x)
    clipped = ((adv > 0) & (rho > 1 + high)) | ((adv < 0) & (rho < 1 - low))
    l = -torch.minimum(rho * adv, rho.clamp(1 - low, 1 + high) * adv)
    slope = torch.where(clipped, 0.0, rho * adv)
    kl = torch.zeros_like(loss)
    if ref is not None:
        q = loss - ref
        kl = torch.expm1(q) - q
        l = l + kl_coef * kl
        slope = slope + kl_coef * torch.expm1(q)
    return l, kl, clipped, slope


def policy(loss, targets, start, adv, old, ref, ignore, mean, low, high, kl_coef, grad_seq=None, per_token=False):
    """(seq_loss, seq_kl, clipped, tokens) and, with grad_seq, the gradient."""
    d = lambda v: None if v is None else v.double().cpu()  # noqa: E731
    loss, old, ref, adv, targets = d(loss), d(old), d(ref), d(adv), targets.cpu()
    T, S = len(loss), len(start) - 1
    out = [torch.zeros(S, dtype=torch.float64) for _ in range(2)] + [torch.zeros(S, dtype=torch.int32) for _ in range(2)]
    grad = torch.zeros(T, dtype=torch.float64)
    for s, (a, b) in enumerate(spans(start, T)):
        at = torch.arange(a, b)[targets[a:b] != ignore]
        A = adv[at] if per_token else adv[s].expand(len(at))
        l, kl, clipped, slope = policy_tokens(loss[at], None if old is None else old[at],
                                              None if ref is None else ref[at], A, low, high, kl_coef)
        c = weight(len(at), mean)
        out[0][s], out[1][s], out[2][s], out[3][s] = c * l.sum(), c * kl.sum(), clipped.sum(), len(at)
        if grad_seq is not None:
            grad[at] = float(grad_seq[s]) * c * slope
    return out, grad
