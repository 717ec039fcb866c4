"""Scoring around the vocabulary projection, as cases that can be prepared and run.

* ``score``: loss, normaliser, entropy and the most likely alternatives of every token;
* ``train``: a training step with an entropy term, the forward of ``score`` and its gradients;
* ``score_f8``: ``score`` of 8-bit hidden states and weights with block scales;
* ``add_norm`` / ``add_norm_backward``: a residual's addition and the norm of the sum, with the norm in
  8 bits, and its gradients;
* ``quantize``: 8-bit values and scales of weights or hidden states.

With ``own`` false a case runs in elementary torch operations, with ``own`` true through the
library.  Widths, vocabularies and token counts are those of ``workloads.py`` where a workload has
them.  8-bit values are float8_e4m3fn, scales float8_e8m0fnu (powers of two).
"""
from __future__ import annotations

import math

import torch

own = False

IGNORE = -100
BLOCK = 128


def _score(name, dtype, T, d, V, P, top, *, op="score", h_scale=2.0):
    return {"name": name, "op": op, "dtype": dtype, "T": T, "d": d, "V": V, "P": P, "top": top, "h_scale": h_scale}


def _norm(name, op, dtype, T, d, *, rms=True, bias=False, quant=True):
    return {"name": name, "op": op, "dtype": dtype, "T": T, "d": d, "rms": rms, "bias": bias, "quant": quant}


def _quantize(name, dtype, rows, cols, rows_per_scale):
    return {"name": name, "op": "quantize", "dtype": dtype, "rows": rows, "cols": cols, "rps": rows_per_scale}


def listed():
    return [
        # One new token in a serving loop, with the twenty alternatives that an interface offers
        # (width, vocabulary and shards of the stress workload): reading W.
        _score("score_token_bf16", "bf16", 1, 4096, 151936, 16, 20),
        # A batch of rollouts scored under the policy (the 4096-token workload), with alternatives.
        _score("score_4k_bf16", "bf16", 4096, 2880, 201088, 8, 8),
        # An evaluation in the paper's float32, the most likely token of each place beside the loss.
        _score("score_eval_f32", "f32", 1000, 7168, 32000, 8, 1),
        # A small ragged vocabulary in float32: a training step with an entropy term.
        _score("train_ragged_f32", "f32", 1333, 1000, 32003, 5, 0, op="train"),
        # The same for the 4096-token workload: policy training with an entropy bonus.
        _score("train_4k_bf16", "bf16", 4096, 2880, 201088, 8, 0, op="train"),
        # A short continuation under an 8-bit reference model: reading W.
        _score("score_f8_short", "f8", 40, 4096, 151936, 16, 5, op="score_f8"),
        # A long batch under the 8-bit reference model (the wide workload's projection).
        _score("score_f8_wide", "f8", 8192, 7168, 129280, 8, 0, op="score_f8"),
        # One token between two layers that take 8-bit rows: latency.
        _norm("add_norm_token", "add_norm", "bf16", 1, 4096),
        # The hidden states of the long-context workload, for an 8-bit product.
        _norm("add_norm_longctx", "add_norm", "bf16", 32768, 2880),
        # The gradient of such a norm at the wide workload's size.
        _norm("add_norm_backward_wide", "add_norm_backward", "bf16", 16384, 7168, quant=False),
        # A vocabulary shard's weights, once for each new set of them.
        _quantize("quantize_shard_bf16", "bf16", 25136, 2880, 128),
        # Hidden states that no norm of the library made.
        _quantize("quantize_tokens_f32", "f32", 16384, 7168, 1),
    ]


_MOST = {"score": 4096 * 2880 * 201088, "train": 4096 * 2880 * 201088, "score_f8": 8192 * 7168 * 129280}
_MOST_ELEMENTS = 16384 * 7168


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["score", "score", "train", "score_f8", "score_f8", "add_norm", "add_norm_backward", "quantize"])
    if op in _MOST:
        f8 = op == "score_f8"
        dtype = "f8" if f8 else rng.choice(["bf16", "bf16", "f32"])
        step = 16 if f8 else 8
        d = _log_int(rng, 64, 7168) // step * step
        V = _log_int(rng, 500, 201088)
        most = _MOST[op] if dtype != "f32" else _MOST[op] // 10
        if op == "train":
            most //= 4
        T = min(_log_int(rng, 1, 8192), max(1, most // (d * V)), (1 << 30) // V)
        P = rng.choice([1, 1, 2, 5, 8])
        top = 0 if op == "train" else rng.choice([0, 1, 5, 8, 20])
        return {"op": op, "dtype": dtype, "T": T, "d": d, "V": V, "P": P, "top": top,
                "h_scale": rng.choice([0.5, 2.0, 4.0])}
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "quantize":
        rows = _log_int(rng, 1, 65536)
        cols = max(16, min(_log_int(rng, 64, 16384), _MOST_ELEMENTS // rows) // 16 * 16)
        return {"op": op, "dtype": dtype, "rows": rows, "cols": cols, "rps": rng.choice([1, 128])}
    d = _log_int(rng, 64, 16384) // 8 * 8
    T = min(_log_int(rng, 1, 65536), _MOST_ELEMENTS // d)
    return {"op": op, "dtype": dtype, "T": T, "d": d, "rms": rng.random() < 0.7, "bias": rng.random() < 0.3,
            "quant": op == "add_norm" and rng.random() < 0.7}


# ---------------------------------------------------------------------------------------------
def _torch_dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _rows(case):
    """Rows of each vocabulary shard."""
    V, P = case["V"], case["P"]
    return [V // P + (p < V % P) for p in range(P)]


# Blocks of rps rows by 128 columns; those at the ends may be smaller.
def _blocks(x, rps):
    """x [r, c] padded with zeros to whole blocks: [r / rps, rps, c / 128, 128]."""
    r, c = x.shape
    x = torch.nn.functional.pad(x, (0, -c % BLOCK, 0, -r % rps))
    return x.reshape(x.shape[0] // rps, rps, x.shape[1] // BLOCK, BLOCK)


def _to_f8(x, rps):
    """(8-bit values [r, c], scales [r / rps, c / 128]): each block's scale is the smallest power of
    two with which its largest magnitude is at most 448."""
    b = _blocks(x.float(), rps)
    amax = b.abs().amax((1, 3))
    m, e = torch.frexp(amax)
    e = torch.where(amax == 0, 0, torch.where(m <= 0.875, e - 9, e - 8))
    v = torch.ldexp(b, -e[:, None, :, None]).reshape(-1, b.shape[2] * BLOCK)[:x.shape[0], :x.shape[1]]
    return v.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _from_f8(x, scale, rps):
    """The float32 values that 8-bit values and scales stand for."""
    s = scale.float().repeat_interleave(rps, 0).repeat_interleave(BLOCK, 1)
    return x.float() * s[:x.shape[0], :x.shape[1]]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    op = case["op"]
    if op == "quantize":
        # weights and activations with a few wide columns
        x = normal(case["rows"], case["cols"]) * (0.02 + 0.2 * uniform(case["cols"]) ** 8)
        return {"X": x.to(_torch_dtype(case))}
    if op.startswith("add_norm"):
        T, d, dt = case["T"], case["d"], _torch_dtype(case)
        wide = 0.5 + 2.0 * uniform(d) ** 8
        s = {"X": normal(T, d).mul_(0.3).to(dt), "R": normal(T, d).mul_(wide).add_(0.2).to(dt),
             "gamma": (1.0 + 0.1 * normal(d)).to(dt), "beta": (0.1 * normal(d)).to(dt) if case["bias"] else None}
        if op == "add_norm_backward":
            x = s.pop("X").add_(s.pop("R"))  # the sum that the forward left, and its statistics
            s["S"], s["dY"], s["dS"] = x, normal(T, d) * 1e-3, normal(T, d) * 1e-3
            s["mean"] = None if case["rms"] else torch.empty(T, device="cuda")
            s["rstd"] = torch.empty(T, device="cuda")
            for a in range(0, T, 4096):
                v = x[a:a + 4096].double()
                if not case["rms"]:
                    s["mean"][a:a + 4096] = v.mean(1)
                    v = v - v.mean(1, keepdim=True)
                s["rstd"][a:a + 4096] = ((v * v).mean(1) + 1e-5).rsqrt()
        return s
    T, d, V = case["T"], case["d"], case["V"]
    W = [normal(r, d).div_(math.sqrt(d)) for r in _rows(case)]
    targets = torch.randint(0, V, (T,), generator=gen, device="cuda")
    # hidden states with logits of a deviation of h_scale; half of the targets are likely ones
    H = normal(T, d).mul_(case["h_scale"])
    lean = 8.0 * uniform(T) * (torch.arange(T, device="cuda") % 2)
    first = 0
    for w in W:
        mine = (targets >= first) & (targets < first + w.shape[0])
        H[mine] += lean[mine, None] * w[targets[mine] - first]
        first += w.shape[0]
    targets[uniform(T) < 0.05] = IGNORE
    s = {"targets": targets}
    if op == "score_f8":
        s["H"], s["H_scale"] = _to_f8(H, 1)
        s["W"], s["W_scale"] = map(list, zip(*[_to_f8(w, BLOCK) for w in W]))
        return s
    s["H"], s["W"] = H.to(_torch_dtype(case)), [w.to(_torch_dtype(case)) for w in W]
    if op == "train":
        # what a policy loss gives each token, and the weight of its entropy
        s["grad_loss"] = torch.where(targets == IGNORE, 0.0, normal(T) / T)
        s["grad_entropy"] = torch.where(targets == IGNORE, 0.0, -0.05 / T * (0.5 + uniform(T)))
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
    code = {"bf16": vp.VP_BF16, "f32": vp.VP_F32, "f8": vp.VP_E4M3}[case["dtype"]]
    if op == "quantize":
        s["quant"] = vp.Quant(case["rows"], case["cols"], code, case["rps"])
        s["X8"], s["scale"] = vp.f8_buffers(case["rows"], case["cols"], case["rps"], "cuda")
    elif op.startswith("add_norm"):
        T, d = case["T"], case["d"]
        s["norm"] = vp.Norm(T, d, code, eps=1e-5, rms=case["rms"])
        if op == "add_norm":
            s["S"], s["rstd"] = torch.empty_like(s["X"]), torch.empty(T, **f32)
            s["mean"] = None if case["rms"] else torch.empty(T, **f32)
            s["Y"] = s["Y8"] = s["scale"] = None
            if case["quant"]:
                s["Y8"], s["scale"] = vp.f8_buffers(T, d, 1, "cuda")
            else:
                s["Y"] = torch.empty_like(s["X"])
        else:
            s["dX"], s["dgamma"] = torch.empty(T, d, **f32), torch.empty(d, **f32)
            s["dbeta"] = torch.empty(d, **f32) if case["bias"] else None
            s["ws"] = torch.empty(vp.vp_norm_workspace_size(s["norm"]), dtype=torch.uint8, device="cuda")
    else:
        T, top = case["T"], case["top"]
        s["prob"] = vp.Problem(T, case["d"], _rows(case), code, ignore_index=IGNORE)
        s["score"] = vp.Score(top)
        s["ws"] = torch.empty(vp.vp_score_workspace_size(s["prob"], s["score"]), dtype=torch.uint8, device="cuda")
        s["loss"], s["lse"], s["entropy"] = (torch.empty(T, **f32) for _ in range(3))
        s["top_ids"] = torch.empty(T, top, dtype=torch.int64, device="cuda") if top else None
        s["top_loss"] = torch.empty(T, top, **f32) if top else None
        if op == "train":
            s["ws_bwd"] = torch.empty(vp.vp_ce_workspace_size(s["prob"])[1], dtype=torch.uint8, device="cuda")
            s["dH"] = torch.empty(T, case["d"], **f32)
            s["dW"] = [torch.empty(r, case["d"], **f32) for r in _rows(case)]
    return s


def _run_own(s):
    vp, case = s["vp"], s["case"]
    op = case["op"]
    if op == "quantize":
        vp.vp_f8_quantize(s["quant"], s["X"], s["X8"], s["scale"])
        return s["X8"], s["scale"]
    if op == "add_norm":
        vp.vp_add_norm_forward(s["norm"], s["X"], s["R"], s["gamma"], s["beta"], s["S"], s["Y"], s["Y8"], s["scale"],
                               s["mean"], s["rstd"])
        return (s["S"], s["rstd"]) + ((s["Y8"], s["scale"]) if case["quant"] else (s["Y"],))
    if op == "add_norm_backward":
        vp.vp_add_norm_backward(s["norm"], s["S"], s["gamma"], s["mean"], s["rstd"], s["dY"], s["dS"], s["dX"],
                                s["dgamma"], s["dbeta"], s["ws"])
        return (s["dX"], s["dgamma"], s["dbeta"]) if case["bias"] else (s["dX"], s["dgamma"])
    if op == "score_f8":
        vp.vp_score_forward_f8(s["prob"], s["score"], s["H"], s["H_scale"], s["W"], s["W_scale"], s["targets"],
                               s["loss"], s["lse"], s["entropy"], s["top_ids"], s["top_loss"], s["ws"])
    else:
        vp.vp_score_forward(s["prob"], s["score"], s["H"], s["W"], s["targets"], s["loss"], s["lse"], s["entropy"],
                            s["top_ids"], s["top_loss"], s["ws"])
    out = (s["loss"], s["lse"], s["entropy"]) + ((s["top_ids"], s["top_loss"]) if case["top"] else ())
    if op != "train":
        return out
    vp.vp_score_backward(s["prob"], s["H"], s["W"], s["targets"], s["lse"], s["entropy"], s["grad_loss"],
                         s["grad_entropy"], s["dH"], s["dW"], s["ws_bwd"])
    # gradients in the type of what they are of
    return out + (s["dH"].to(s["H"].dtype), [w.to(s["H"].dtype) for w in s["dW"]])


# The plain forms: elementary torch operations in float32; the order of alternatives, which may lie
# closer than a rounding, from float64 logits of a few more candidates than are asked for.
def _plain_score(s, H, W):
    case = s["case"]
    y = H @ W.t()
    m = y.amax(1, keepdim=True)
    p = torch.exp(y - m)
    z = p.sum(1, keepdim=True)
    lse = m + torch.log(z)
    p /= z
    entropy = -(p * (y - lse)).sum(1)
    tg = s["targets"]
    valid = tg != IGNORE
    at = torch.where(valid, tg, 0)[:, None]
    loss = torch.where(valid, (lse - y.gather(1, at))[:, 0], 0.0)
    out = (loss, lse[:, 0], entropy)
    if case["top"]:
        some = torch.topk(y, min(case["top"] + 8, case["V"])).indices.sort(1).values
        exact = (H.double()[:, None, :] @ W[some].double().transpose(1, 2).contiguous())[:, 0]
        order = torch.sort(exact, dim=1, descending=True, stable=True).indices[:, :case["top"]]
        out += (some.gather(1, order), (lse - exact.gather(1, order)).float())
    return out, y, p


def _plain_train(s):
    H, W = s["H"].float(), torch.cat(s["W"]).float()
    out, y, p = _plain_score(s, H, W)
    _, lse, entropy = out
    G = p * (s["grad_loss"][:, None] - s["grad_entropy"][:, None] * (y - (lse - entropy)[:, None]))
    valid = s["targets"] != IGNORE
    at = torch.where(valid, s["targets"], 0)[:, None]
    G.scatter_add_(1, at, torch.where(valid, -s["grad_loss"], 0.0)[:, None])
    dW = (G.t() @ H).to(s["H"].dtype)
    return out + ((G @ W).to(s["H"].dtype), list(dW.split([w.shape[0] for w in s["W"]])))


def _plain_add_norm(s):
    case = s["case"]
    S = (s["X"].float() + s["R"].float()).to(s["X"].dtype)
    x = S.float()
    if not case["rms"]:
        x = x - x.mean(1, keepdim=True)
    rstd = ((x * x).mean(1) + 1e-5).rsqrt()
    y = x * rstd[:, None] * s["gamma"].float()
    if s["beta"] is not None:
        y = y + s["beta"].float()
    return (S, rstd) + (_to_f8(y, 1) if case["quant"] else (y.to(S.dtype),))


def _plain_add_norm_backward(s):
    x, rms = s["S"].float(), s["case"]["rms"]
    xh = (x if rms else x - s["mean"][:, None]) * s["rstd"][:, None]
    g = s["dY"] * s["gamma"].float()
    dx = g - xh * (g * xh).mean(1, keepdim=True)
    if not rms:
        dx = dx - g.mean(1, keepdim=True)
    dx = dx * s["rstd"][:, None] + s["dS"]
    dgamma = (s["dY"] * xh).sum(0)
    return (dx, dgamma, s["dY"].sum(0)) if s["case"]["bias"] else (dx, dgamma)


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    op = case["op"]
    if op == "quantize":
        return _to_f8(state["X"], case["rps"])
    if op == "add_norm":
        return _plain_add_norm(state)
    if op == "add_norm_backward":
        return _plain_add_norm_backward(state)
    if op == "train":
        return _plain_train(state)
    if op == "score":
        return _plain_score(state, state["H"].float(), torch.cat(state["W"]).float())[0]
    W = torch.cat([_from_f8(w, k, BLOCK) for w, k in zip(state["W"], state["W_scale"])])
    return _plain_score(state, _from_f8(state["H"], state["H_scale"], 1), W)[0]


# The definitions in float64, a few tokens or rows at a time.
def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "quantize":
        return _exact_f8(s["X"].double(), case["rps"])
    if case["op"] == "add_norm":
        return _exact_add_norm(case, s)
    if case["op"] == "add_norm_backward":
        return _exact_add_norm_backward(case, s)
    return _exact_score(case, s)


def _grid(v):
    """v, at most 448 in magnitude, to the nearest 8-bit value: steps of an eighth of the power of two
    below it, and of 2^-9 below 2^-6; ties to even."""
    low = torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6)))
    step = torch.exp2(low - 3)
    return torch.round(v / step) * step


def _exact_f8(x, rps):
    """Row groups one by one: the scale is searched from the largest magnitude down."""
    values, scales = [], []
    for a in range(0, x.shape[0], rps if rps > 1 else 4096):
        g = x[a:a + (rps if rps > 1 else 4096)]
        v, k = [], []
        for b in range(0, x.shape[1], BLOCK):
            part = g[:, b:b + BLOCK]
            most = part.abs().max() if rps > 1 else part.abs().max(1, keepdim=True).values
            e = torch.ceil(torch.log2(most / 448.0))
            e = torch.where(most > 448.0 * torch.exp2(e), e + 1, e)
            e = torch.where(most <= 448.0 * torch.exp2(e - 1), e - 1, e)
            e = torch.where(most > 0, e, torch.zeros_like(e))
            v.append(_grid(part / torch.exp2(e)))
            k.append(torch.exp2(e).reshape(-1, 1))
        values.append(torch.cat(v, 1))
        scales.append(torch.cat(k, 1))
    return torch.cat(values), torch.cat(scales)


def _exact_add_norm(case, s):
    sums, rstds, ys, ks = [], [], [], []
    for a in range(0, case["T"], 4096):
        # the sum as it is stored, which is what is normalised
        S = (s["X"][a:a + 4096].double() + s["R"][a:a + 4096].double()).to(s["X"].dtype).double()
        c = S - (0.0 if case["rms"] else S.sum(1, keepdim=True) / case["d"])
        inv = 1.0 / torch.sqrt(c.square().sum(1, keepdim=True) / case["d"] + 1e-5)
        y = c * inv * s["gamma"].double() + (0.0 if s["beta"] is None else s["beta"].double())
        sums.append(S)
        rstds.append(inv[:, 0])
        if case["quant"]:
            v, k = _exact_f8(y, 1)
            ys.append(v)
            ks.append(k)
        else:
            ys.append(y)
    return [torch.cat(v) for v in (sums, rstds, ys)] + ([torch.cat(ks)] if case["quant"] else [])


def _exact_add_norm_backward(case, s):
    d, rows = case["d"], []
    gamma = s["gamma"].double()
    dgamma, dbeta = (torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(2))
    for a in range(0, case["T"], 4096):
        part = slice(a, a + 4096)
        dy, inv = s["dY"][part].double(), s["rstd"][part, None].double()
        xh = s["S"][part].double() if case["rms"] else s["S"][part].double().sub(s["mean"][part, None].double())
        xh = xh.mul(inv)
        dxh = dy.mul(gamma)
        proj = torch.linalg.vecdot(dxh, xh)[:, None] / d
        cent = 0.0 if case["rms"] else dxh.sum(1, keepdim=True) / d
        rows.append(inv * (dxh - cent - xh * proj) + s["dS"][part].double())
        dgamma += (dy * xh).sum(0)
        dbeta += dy.sum(0)
    return [torch.cat(rows), dgamma] + ([dbeta] if case["bias"] else [])


def _exact_values(x, scale, rps):
    out = x.double()
    k = scale.double()
    for b in range(k.shape[1]):
        out[:, b * BLOCK:(b + 1) * BLOCK] *= k[:, b].repeat_interleave(rps)[:x.shape[0], None]
    return out


def _exact_score(case, s):
    f8, train, top = case["op"] == "score_f8", case["op"] == "train", case["top"]
    if f8:
        W = torch.cat([_exact_values(w, k, BLOCK) for w, k in zip(s["W"], s["W_scale"])])
    else:
        W = torch.cat([w.double() for w in s["W"]])
    out = [[] for _ in range(5)]
    dH, dW = [], torch.zeros_like(W) if train else None
    for a in range(0, case["T"], 512):
        part = slice(a, a + 512)
        H = _exact_values(s["H"][part], s["H_scale"][part], 1) if f8 else s["H"][part].double()
        logits = torch.mm(H, W.t())
        lse = torch.logsumexp(logits, 1)
        logp = logits - lse[:, None]
        prob = logp.exp()
        entropy = -torch.linalg.vecdot(prob, logp)
        keep = s["targets"][part] != IGNORE
        ids = s["targets"][part].clamp_min(0)
        row = torch.arange(ids.shape[0], device="cuda")
        out[0].append(-logp[row, ids] * keep)
        out[1].append(lse)
        out[2].append(entropy)
        if top:
            best = torch.sort(logp, dim=1, descending=True, stable=True)
            out[3].append(best.indices[:, :top].clone())
            out[4].append(-best.values[:, :top])
        if train:
            g, e = s["grad_loss"][part].double(), s["grad_entropy"][part].double()
            D = prob * g[:, None] - prob * (logp + entropy[:, None]) * e[:, None]
            D[row, ids] -= g * keep
            dH.append(torch.mm(D, W))
            dW += torch.mm(D.t(), H)
    got = [torch.cat(v) for v in out if v]
    return got + [torch.cat(dH), list(dW.split(_rows(case)))] if train else got


def work(case):
    op = case["op"]
    e = {"f8": 1, "bf16": 2, "f32": 4}[case["dtype"]]
    if op == "quantize":
        r, c = case["rows"], case["cols"]
        return {"bytes": r * c * (e + 1) + -(-r // case["rps"]) * -(-c // BLOCK), "flops": 2 * r * c}
    if op.startswith("add_norm"):
        T, d = case["T"], case["d"]
        vectors = d * e * (2 if case["bias"] else 1)
        stats = 4 * T * (1 if case["rms"] else 2)
        if op == "add_norm":
            y = 1 + 1 / BLOCK if case["quant"] else e
            return {"bytes": T * d * (3 * e + y) + vectors + stats, "flops": 8 * T * d}
        return {"bytes": T * d * (e + 12) + d * e + 4 * d * (2 if case["bias"] else 1) + stats, "flops": 15 * T * d}
    T, d, V, top = case["T"], case["d"], case["V"], case["top"]
    b = (T + V) * d * e + 8 * T + 12 * T + 12 * T * top
    if op == "score_f8":
        b += (T + V / BLOCK) * -(-d // BLOCK)
    if op == "train":
        return {"bytes": b + 8 * T + (T + V) * d * 4, "flops": 8 * T * V * d}
    return {"bytes": b, "flops": 2 * T * V * d}
