"""Plain float64 forms of the scoring calls and of 8-bit quantisation, for the tests."""
from __future__ import annotations

import torch

U = 2.0 ** -24  # half a step of float32, relative


def score(H, W, targets, ignore, top=0):
    """(loss, lse, entropy, ids, top_loss, logits) from float64 H [T, d] and W [V, d]."""
    y = H @ W.t().contiguous()
    lse = torch.logsumexp(y, 1)
    logp = y - lse[:, None]
    entropy = -torch.where(logp == -torch.inf, 0.0, logp.exp() * logp).sum(1)
    t = targets.clone()
    bad = (t != ignore) & ((t < 0) | (t >= W.shape[0]))
    none = (t == ignore) | bad
    t[none] = 0
    loss = torch.where(targets == ignore, 0.0, -logp.gather(1, t[:, None])[:, 0])
    loss[bad] = torch.nan
    best = torch.sort(y, dim=1, descending=True, stable=True)
    ids = best.indices[:, :top]
    return loss, lse, entropy, ids, lse[:, None] - best.values[:, :top], y


def residual(H, W, targets, ignore, g, e):
    """d (sum_t g_t loss_t + e_t entropy_t) / d logits, in float64."""
    _, lse, entropy, _, _, y = score(H, W, targets, ignore)
    logp = y - lse[:, None]
    p = logp.exp()
    masked = logp == -torch.inf
    live = targets != ignore
    G = p * torch.where(live, g, 0.0)[:, None] - e[:, None] * torch.where(masked, 0.0, p * (logp + entropy[:, None]))
    rows = torch.arange(len(targets), device=H.device)[live]
    bad = live & ((targets < 0) | (targets >= W.shape[0]))
    G[rows[~bad[live]], targets[live & ~bad]] -= g[live & ~bad]
    G[bad] = torch.nan
    return G


def logit_bound(H, W):
    """How far a float32 sum of the d products of any token and id may be off: its worst order."""
    return (H.shape[1] + 2) * U * (H.abs() @ W.abs().t().contiguous()).amax(1)


def fold_bound(V):
    """Relative bound on a float32 sum of the exponentials of V logits: one chain of additions a lane
    takes at most V / 2 of them, and each exponential is off by a few units."""
    return (V / 2 + 80) * U


def grid(v):
    """|v| <= 448 (float64) to the nearest 8-bit value, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(v / step) * step


def quantize(X, rps):
    """(values, scale exponents) in float64, block by block; for tensors on the CPU."""
    x = X.double()
    r, c = x.shape
    out = torch.zeros_like(x)
    exps = torch.zeros(-(-r // rps), -(-c // 128), dtype=torch.float64)
    for i in range(exps.shape[0]):
        for j in range(exps.shape[1]):
            b = x[i * rps:(i + 1) * rps, 128 * j:128 * j + 128]
            fine = b.isfinite()
            m = b[fine].abs().max().item() if fine.any() else 0.0
            e = 0
            if m > 0:
                e = -127
                while m > 448.0 * 2.0 ** e:
                    e += 1
            exps[i, j] = e
            v = torch.full_like(b, torch.nan)
            v[fine] = grid(b[fine] / 2.0 ** e)
            out[i * rps:(i + 1) * rps, 128 * j:128 * j + 128] = v
    return out, exps


def values(x8, scale, rps):
    """What 8-bit values and scales stand for, in float64."""
    s = scale.double().repeat_interleave(rps, 0)[:x8.shape[0]].repeat_interleave(128, 1)[:, :x8.shape[1]]
    return x8.double() * s
