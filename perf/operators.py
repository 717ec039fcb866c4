"""The operators around the vocabulary projection, as cases that can be prepared and run.

* ``norm_forward`` / ``norm_backward``: the layer norm that makes the hidden states, and its
  gradients from the float32 dH of the projection's backward;
* ``preference``: a preference loss over pairs of packed sequences, from the per-token losses of
  ``vp_ce_forward`` to the per-token gradient that ``vp_ce_backward`` reads;
* ``policy``: a clipped policy loss with a KL term, between the same two.

With ``own`` false a case runs in elementary torch operations, with ``own`` true through the
library.  Widths and token counts are those of ``workloads.py`` where a workload has them.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

IGNORE = -100


def _norm(name, op, dtype, T, d, *, rms=False, bias=True):
    return {"name": name, "op": op, "dtype": dtype, "T": T, "d": d, "rms": rms, "bias": bias}


def _pref(name, T, pairs, *, kind="logistic", ref=True, mean=False, smoothing=0.0, margin=0.0, beta=0.1,
          prompt=0.4, skew=1.0):
    return {"name": name, "op": "preference", "T": T, "S": 2 * pairs, "kind": kind, "ref": ref, "mean": mean,
            "smoothing": smoothing, "margin": margin, "beta": beta, "prompt": prompt, "skew": skew}


def _policy(name, T, S, *, old=True, ref=True, mean=True, per_token=False, clip_low=0.2, clip_high=0.2,
            kl_coef=0.05, prompt=0.3, skew=1.0):
    return {"name": name, "op": "policy", "T": T, "S": S, "old": old, "ref": ref, "mean": mean,
            "per_token": per_token, "clip_low": clip_low, "clip_high": clip_high, "kl_coef": kl_coef,
            "prompt": prompt, "skew": skew}


def listed():
    return [
        # The final norm of one token in a serving loop (width of the stress workload): latency.
        _norm("norm_forward_token_bf16", "norm_forward", "bf16", 1, 4096),
        # The hidden states of the long-context workload.
        _norm("norm_forward_longctx_bf16", "norm_forward", "bf16", 32768, 2880),
        # The paper's float32 width, without a mean and a bias, at the wide workload's tokens.
        _norm("norm_forward_wide_f32", "norm_forward", "f32", 16384, 7168, rms=True, bias=False),
        # Packed tokens without padding, a small width that is no power of two.
        _norm("norm_backward_ragged_bf16", "norm_backward", "bf16", 1333, 1000),
        # The gradient of the long-context workload's hidden states.
        _norm("norm_backward_longctx_bf16", "norm_backward", "bf16", 32768, 2880),
        # The same for the paper's float32 width: the most bytes of all.
        _norm("norm_backward_wide_f32", "norm_backward", "f32", 16384, 7168, rms=True, bias=False),
        # A micro-batch of four short pairs.
        _pref("preference_4_pairs", 1111, 4),
        # One pair of very long documents, mean log-probabilities and a margin without a reference.
        _pref("preference_long_pair", 131071, 1, ref=False, mean=True, margin=0.5, beta=2.0, prompt=0.1),
        # A whole preference set in one pass, with label smoothing and lengths of a wide spread.
        _pref("preference_set", 4000003, 2500, smoothing=0.1, skew=1.5),
        # Eight short completions of one prompt, one advantage each.
        _policy("policy_8_completions", 1500, 8),
        # The long-context workload's tokens as 64 completions, one advantage each.
        _policy("policy_longctx", 32768, 64, clip_high=0.28),
        # A whole rollout buffer with one advantage per token and sums over sequences.
        _policy("policy_rollouts", 4194301, 4096, mean=False, per_token=True, skew=1.5),
    ]


_MOST_TOKENS = 4000003
_MOST_NORM = {"norm_forward": 16384 * 7168, "norm_backward": 16384 * 7168}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_forward", "norm_backward", "preference", "policy"])
    if op.startswith("norm"):
        d = _log_int(rng, 64, 16384) // 8 * 8
        # rows over the whole range and, as often, a few of them
        T = min(_log_int(rng, 1, 65536), _MOST_NORM[op] // d)
        return {"op": op, "dtype": rng.choice(["bf16", "bf16", "f32"]), "T": T, "d": d, "rms": rng.random() < 0.4,
                "bias": rng.random() < 0.5}
    T = _log_int(rng, 1, _MOST_TOKENS)
    S = _log_int(rng, 1, min(4096, max(1, T // 4)))
    case = {"op": op, "T": T, "mean": rng.random() < 0.5, "ref": rng.random() < 0.7,
            "prompt": rng.choice([0.0, 0.1, 0.4]), "skew": rng.choice([0.0, 1.0, 2.0])}
    if op == "preference":
        case.update(S=2 * ((S + 1) // 2), kind=rng.choice(["logistic", "logistic", "squared"]),
                    smoothing=rng.choice([0.0, 0.1]), margin=rng.choice([0.0, 0.5]),
                    beta=rng.choice([0.05, 0.1, 0.5]) if not case["mean"] else 2.0)
    else:
        case.update(S=S, old=rng.random() < 0.8, per_token=rng.random() < 0.4, clip_low=0.2,
                    clip_high=rng.choice([0.2, 0.28]), kl_coef=rng.choice([0.0, 0.05]))
    return case


# ---------------------------------------------------------------------------------------------
def _torch_dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _starts(case, seed):
    """Offsets [S + 1] of the sequences: lengths of a lognormal spread (some are empty), and up
    to a hundredth of the tokens behind the last one, as padding."""
    T, S = case["T"], case["S"]
    rng = np.random.default_rng([seed, 17])
    weight = np.exp(case["skew"] * rng.standard_normal(S)) + 1e-3
    packed = T - int(rng.integers(0, max(1, T // 100)))
    cut = np.floor(np.cumsum(weight) / weight.sum() * packed + 1e-6).astype(np.int64)
    cut[-1] = packed
    return np.concatenate([[0], cut]).astype(np.int32)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    if case["op"].startswith("norm"):
        T, d, dt = case["T"], case["d"], _torch_dtype(case)
        # hidden states with an offset and a few wide channels
        X = normal(T, d)
        X.mul_(0.5 + 2.0 * uniform(d) ** 8).add_(0.3)
        s = {"X": X.to(dt), "gamma": (1.0 + 0.1 * normal(d)).to(dt),
             "beta": (0.1 * normal(d)).to(dt) if case["bias"] else None}
        if case["op"] == "norm_backward":
            s["dY"] = normal(T, d) * 1e-3
            # what the forward left
            s["mean"] = None if case["rms"] else torch.empty(T, device="cuda")
            s["rstd"] = torch.empty(T, device="cuda")
            for a in range(0, T, 4096):
                x = s["X"][a:a + 4096].double()
                if not case["rms"]:
                    s["mean"][a:a + 4096] = x.mean(1)
                    x = x - x.mean(1, keepdim=True)
                s["rstd"][a:a + 4096] = ((x * x).mean(1) + 1e-5).rsqrt()
        return s

    T, S = case["T"], case["S"]
    start = _starts(case, seed)
    lens = np.diff(start)
    # the first part of every sequence is a prompt without loss, and so is the padding
    masked = np.ones(T, dtype=bool)
    seq = np.repeat(np.arange(S), lens)
    pos = np.arange(start[-1]) - start[:-1].astype(np.int64)[seq]
    masked[:start[-1]] = pos < np.floor(case["prompt"] * lens)[seq]
    mask = torch.from_numpy(masked).cuda()
    ids = torch.randint(0, 151936, (T,), generator=gen, device="cuda")
    s = {"start": torch.from_numpy(start).cuda(), "targets": torch.where(mask, IGNORE, ids)}
    # losses per token: mostly small, some large, exactly 0 on tokens without a target
    base = 6.0 * uniform(T) ** 3

    def losses(spread):
        return torch.where(mask, 0.0, (base + spread * normal(T)).clamp_min(0.0))

    s["loss"] = losses(0.15 if case["op"] == "policy" else 0.2)
    s["ref"] = losses(0.2) if case["ref"] else None
    if case["op"] == "preference":
        s["grad"] = torch.full((S // 2,), 2.0 / S, device="cuda")
    else:
        s["old"] = losses(0.15) if case["old"] else None
        s["adv"] = normal(T if case["per_token"] else S)
        s["grad"] = torch.full((S,), 1.0 / S, device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if not own:
        return s
    import paper_2609_14306_amd as vp

    s["vp"] = vp
    op = case["op"]
    f32 = {"dtype": torch.float32, "device": "cuda"}
    if op.startswith("norm"):
        T, d = case["T"], case["d"]
        s["prob"] = vp.Norm(T, d, vp.VP_BF16 if case["dtype"] == "bf16" else vp.VP_F32, eps=1e-5, rms=case["rms"])
        if op == "norm_forward":
            s["Y"], s["rstd"] = torch.empty_like(s["X"]), torch.empty(T, **f32)
            s["mean"] = None if case["rms"] else torch.empty(T, **f32)
        else:
            s["dX"], s["dgamma"] = torch.empty(T, d, **f32), torch.empty(d, **f32)
            s["dbeta"] = torch.empty(d, **f32) if case["bias"] else None
            s["ws"] = torch.empty(vp.vp_norm_workspace_size(s["prob"]), dtype=torch.uint8, device="cuda")
        return s
    T, S = case["T"], case["S"]
    s["seq"] = vp.Sequences(T, S, ignore_index=IGNORE, mean=case["mean"])
    s["ws"] = torch.empty(vp.vp_seq_workspace_size(s["seq"]), dtype=torch.uint8, device="cuda")
    s["grad_loss"] = torch.empty(T, **f32)
    if op == "preference":
        s["par"] = vp.Preference(case["kind"], beta=case["beta"], margin=case["margin"], smoothing=case["smoothing"])
        s["pair_loss"] = torch.empty(S // 2, **f32)
        s["reward"], s["coef"] = torch.empty(S, **f32), torch.empty(S, **f32)
    else:
        s["par"] = vp.Policy(clip_low=case["clip_low"], clip_high=case["clip_high"], kl_coef=case["kl_coef"],
                             per_token=case["per_token"])
        s["seq_loss"], s["seq_kl"] = torch.empty(S, **f32), torch.empty(S, **f32)
        s["clipped"], s["tokens"] = (torch.empty(S, dtype=torch.int32, device="cuda") for _ in range(2))
    return s


def _run_own(s):
    vp, op = s["vp"], s["case"]["op"]
    if op == "norm_forward":
        vp.vp_norm_forward(s["prob"], s["X"], s["gamma"], s["beta"], s["Y"], s["mean"], s["rstd"])
        return (s["Y"], s["rstd"]) if s["case"]["rms"] else (s["Y"], s["mean"], s["rstd"])
    if op == "norm_backward":
        vp.vp_norm_backward(s["prob"], s["X"], s["gamma"], s["mean"], s["rstd"], s["dY"], s["dX"], s["dgamma"],
                            s["dbeta"], s["ws"])
        return (s["dX"], s["dgamma"], s["dbeta"]) if s["case"]["bias"] else (s["dX"], s["dgamma"])
    if op == "preference":
        vp.vp_pref_forward(s["seq"], s["par"], s["start"], s["targets"], s["loss"], s["ref"], s["pair_loss"],
                           s["reward"], s["coef"], s["ws"])
        vp.vp_pref_backward(s["seq"], s["start"], s["targets"], s["coef"], s["grad"], s["grad_loss"])
        return s["pair_loss"], s["reward"], s["grad_loss"]
    vp.vp_policy_forward(s["seq"], s["par"], s["start"], s["targets"], s["loss"], s["old"], s["ref"], s["adv"],
                         s["seq_loss"], s["seq_kl"], s["clipped"], s["tokens"], s["ws"])
    vp.vp_policy_backward(s["seq"], s["par"], s["start"], s["targets"], s["loss"], s["old"], s["ref"], s["adv"],
                          s["tokens"], s["grad"], s["grad_loss"])
    return s["seq_loss"], s["seq_kl"], s["clipped"], s["tokens"], s["grad_loss"]


# The plain forms: elementary torch operations in float32; sums over sequences, and what decides
# on which side of a border a ratio lies, in float64.
def _plain_norm_forward(s):
    x, rms = s["X"].float(), s["case"]["rms"]
    if not rms:
        mean = x.mean(1)
        x = x - mean[:, None]
    rstd = ((x * x).mean(1) + 1e-5).rsqrt()
    y = x * rstd[:, None] * s["gamma"].float()
    if s["beta"] is not None:
        y = y + s["beta"].float()
    y = y.to(s["X"].dtype)
    return (y, rstd) if rms else (y, mean, rstd)


def _plain_norm_backward(s):
    x, rms = s["X"].float(), s["case"]["rms"]
    xh = (x if rms else x - s["mean"][:, None]) * s["rstd"][:, None]
    g = s["dY"] * s["gamma"].float()
    dx = g - xh * (g * xh).mean(1, keepdim=True)
    if not rms:
        dx = dx - g.mean(1, keepdim=True)
    dx = dx * s["rstd"][:, None]
    dgamma = (s["dY"] * xh).sum(0)
    return (dx, dgamma, s["dY"].sum(0)) if s["case"]["bias"] else (dx, dgamma)


def _plain_sequences(s):
    """Sequence of every token (S for none), and whether it counts."""
    case, start = s["case"], s["start"].long()
    t = torch.arange(case["T"], device=start.device)
    seq = torch.searchsorted(start, t, right=True) - 1
    valid = (s["targets"] != IGNORE) & (seq < case["S"])
    return seq, valid


def _plain_sum(values, s):
    """Sums over the sequences: differences of the running sum."""
    total = torch.cat([values.new_zeros(1, dtype=torch.float64), values.double().cumsum(0)])
    start = s["start"].long()
    return total[start[1:]] - total[start[:-1]]


def _plain_preference(s):
    case, S = s["case"], s["case"]["S"]
    seq, valid = _plain_sequences(s)
    ratio = -s["loss"].double() if s["ref"] is None else s["ref"].double() - s["loss"].double()
    total = _plain_sum(torch.where(valid, ratio, 0.0), s)
    scale = torch.ones_like(total)
    if case["mean"]:
        count = _plain_sum(valid.float(), s)
        scale = torch.where(count > 0, 1.0 / count, 0.0)
    reward = case["beta"] * scale * total
    z = reward[0::2] - reward[1::2] - case["margin"]
    if case["kind"] == "logistic":
        e = case["smoothing"]
        up, down = torch.log1p(torch.exp(-z.abs())) + (-z).clamp_min(0.0), torch.log1p(torch.exp(-z.abs())) + z.clamp_min(0.0)
        loss = (1.0 - e) * up + e * down
        slope = e / (1.0 + torch.exp(-z)) - (1.0 - e) / (1.0 + torch.exp(z))
    else:
        loss = ((z - 0.5) / case["beta"]) ** 2
        slope = 2.0 * (z - 0.5) / case["beta"] ** 2
    coef = torch.stack([-slope, slope], 1).reshape(-1) * case["beta"] * scale
    weight = coef * s["grad"].double().repeat_interleave(2)
    weight = torch.cat([weight, weight.new_zeros(1)])
    grad = torch.where(valid, weight[seq], 0.0)
    return loss.float(), reward.float(), grad.float()


def _plain_policy(s):
    case, S = s["case"], s["case"]["S"]
    seq, valid = _plain_sequences(s)
    adv = s["adv"] if case["per_token"] else torch.cat([s["adv"], s["adv"].new_zeros(1)])[seq]
    low, high = 1.0 - case["clip_low"], 1.0 + case["clip_high"]
    if s["old"] is None:
        exact, ratio = torch.ones(1, device=adv.device, dtype=torch.float64), torch.ones_like(s["loss"])
    else:
        exact = torch.exp(s["old"].double() - s["loss"].double())
        ratio = exact.float()
    clipped = valid & (((adv > 0) & (exact > high)) | ((adv < 0) & (exact < low)))
    token = -torch.minimum(ratio * adv, ratio.clamp(low, high) * adv)
    slope = torch.where(clipped, 0.0, ratio * adv)
    if s["ref"] is None:
        kl = torch.zeros_like(token)
    else:
        q = s["loss"].double() - s["ref"].double()
        kl = torch.exp(q) - q - 1.0  # two nearly equal terms for q near 0
        token = token + case["kl_coef"] * kl
        slope = slope + case["kl_coef"] * (torch.exp(q) - 1.0)
    count = _plain_sum(valid.float(), s)
    scale = torch.ones_like(count)
    if case["mean"]:
        scale = torch.where(count > 0, 1.0 / count, 0.0)
    loss = scale * _plain_sum(torch.where(valid, token, 0.0), s)
    kl = scale * _plain_sum(torch.where(valid, kl, 0.0), s)
    weight = scale * s["grad"].double()
    weight = torch.cat([weight, weight.new_zeros(1)])
    grad = torch.where(valid, weight[seq] * slope, 0.0)
    return loss.float(), kl.float(), _plain_sum(clipped.float(), s).int(), count.int(), grad.float()


def run(state):
    if own:
        return _run_own(state)
    return {"norm_forward": _plain_norm_forward, "norm_backward": _plain_norm_backward,
            "preference": _plain_preference, "policy": _plain_policy}[state["case"]["op"]](state)


# The definitions in float64, row by row and sequence by sequence.
def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"].startswith("norm"):
        return _exact_norm(case, s)
    start = s["start"].tolist()
    if case["op"] == "preference":
        return _exact_preference(case, s, start)
    return _exact_policy(case, s, start)


def _exact_norm(case, s):
    T, d = case["T"], case["d"]
    step = max(1, (1 << 25) // d)
    forward = case["op"] == "norm_forward"
    gamma = s["gamma"].double()
    rows, means, rstds = [], [], []
    dgamma = torch.zeros(d, dtype=torch.float64, device="cuda")
    dbeta = torch.zeros_like(dgamma)
    for a in range(0, T, step):
        x = s["X"][a:a + step].double()
        if forward:
            mu = torch.zeros(x.shape[0], 1, dtype=torch.float64, device="cuda") if case["rms"] else x.sum(1, keepdim=True) / d
            inv = 1.0 / torch.sqrt((x - mu).square().sum(1, keepdim=True) / d + 1e-5)
            y = torch.addcmul(torch.zeros_like(x) if s["beta"] is None else s["beta"].double().expand_as(x),
                              (x - mu) * inv, gamma.expand_as(x))
            rows.append(y)
            means.append(mu[:, 0])
            rstds.append(inv[:, 0])
            continue
        dy = s["dY"][a:a + step].double()
        inv = s["rstd"][a:a + step, None].double()
        xh = (x if case["rms"] else x.sub(s["mean"][a:a + step, None].double())).mul(inv)
        dxh = dy.mul(gamma)
        proj = torch.matmul(dxh.unsqueeze(1), xh.unsqueeze(2)).squeeze(2) / d
        cent = 0.0 if case["rms"] else dxh.sum(1, keepdim=True) / d
        rows.append(inv * (dxh - cent - xh * proj))
        dgamma += (dy * xh).sum(0)
        dbeta += dy.sum(0)
    if forward:
        return [torch.cat(v) for v in ((rows, rstds) if case["rms"] else (rows, means, rstds))]
    return [torch.cat(rows), dgamma] + ([dbeta] if case["bias"] else [])


def _exact_preference(case, s, start):
    nll = s["loss"].double()
    logratio = -nll + (0.0 if s["ref"] is None else s["ref"].double())
    keep = s["targets"].ne(IGNORE)
    S = case["S"]
    R, share = [], []
    for i in range(S):
        a, b = start[i], start[i + 1]
        n = keep[a:b].sum()
        c = 1.0 / n.clamp_min(1).double() if case["mean"] else torch.ones((), dtype=torch.float64, device="cuda")
        share.append(c)
        R.append(logratio[a:b][keep[a:b]].sum() * c)
    R, share = torch.stack(R) * case["beta"], torch.stack(share)
    margin = R.view(-1, 2)[:, 0] - R.view(-1, 2)[:, 1] - case["margin"]
    if case["kind"] == "logistic":
        e = case["smoothing"]
        soft = lambda v: torch.logaddexp(v, torch.zeros_like(v))
        loss = (1 - e) * soft(-margin) + e * soft(margin)
        d = torch.sigmoid(margin) - (1 - e)
    else:
        loss = torch.square(margin / case["beta"] - 0.5 / case["beta"])
        d = (2 * margin - 1) / case["beta"] ** 2
    grad = torch.zeros(case["T"], dtype=torch.float64, device="cuda")
    g = s["grad"].double()
    for i in range(S):
        a, b = start[i], start[i + 1]
        sign = -1.0 if i % 2 == 0 else 1.0
        grad[a:b] = keep[a:b] * (sign * case["beta"] * g[i // 2] * d[i // 2] * share[i])
    return loss, R, grad


def _exact_policy(case, s, start):
    keep = s["targets"].ne(IGNORE)
    T, S = case["T"], case["S"]
    grad = torch.zeros(T, dtype=torch.float64, device="cuda")
    out = [[], [], [], []]
    adv_all, g = s["adv"].double(), s["grad"].double()
    for i in range(S):
        a, b = start[i], start[i + 1]
        m = keep[a:b]
        logp = -s["loss"][a:b].double()
        A = adv_all[a:b] if case["per_token"] else adv_all[i].expand(b - a)
        r = torch.exp(logp + s["old"][a:b].double()) if case["old"] else torch.ones_like(logp)
        limit = torch.where(A >= 0, 1.0 + case["clip_high"], 1.0 - case["clip_low"])
        over = torch.where(A >= 0, r > limit, r < limit) & (A != 0)
        gain = torch.where(over, limit, r) * A
        if case["ref"]:
            lr = -s["ref"][a:b].double() - logp
            kl, dkl = torch.expm1(lr) - lr, torch.expm1(lr)
        else:
            kl = dkl = torch.zeros_like(logp)
        n = m.sum()
        c = 1.0 / n.clamp_min(1).double() if case["mean"] else 1.0
        out[0].append(((case["kl_coef"] * kl - gain) * m).sum() * c)
        out[1].append((kl * m).sum() * c)
        out[2].append((over & m).sum())
        out[3].append(n)
        d_nll = torch.where(over, 0.0, r * A) + case["kl_coef"] * dkl
        grad[a:b] = m * d_nll * c * g[i]
    loss, kl, over, n = (torch.stack(o) for o in out)
    return loss, kl, over.int(), n.int(), grad


def work(case):
    T = case["T"]
    if case["op"].startswith("norm"):
        d, e = case["d"], 2 if case["dtype"] == "bf16" else 4
        stats = 4 * T * (1 if case["rms"] else 2)
        vectors = d * e * (2 if case["bias"] else 1)
        if case["op"] == "norm_forward":
            return {"bytes": 2 * T * d * e + vectors + stats, "flops": 8 * T * d}
        return {"bytes": T * d * (e + 8) + d * e + 4 * d * (2 if case["bias"] else 1) + stats, "flops": 14 * T * d}
    S = case["S"]
    # targets, losses and the gradient of every token, the offsets, and per-sequence values
    token = 8 + 4 + 4 + (4 if case["ref"] else 0)
    if case["op"] == "preference":
        return {"bytes": T * token + 4 * (S + 1) + 4 * S + 4 * S, "flops": 4 * T}
    token += (4 if case["old"] else 0) + (4 if case["per_token"] else 0)
    return {"bytes": T * token + 4 * (S + 1) + (0 if case["per_token"] else 4 * S) + 20 * S, "flops": 30 * T}
