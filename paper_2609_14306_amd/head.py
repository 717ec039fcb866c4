"""Binding of the operators around the vocabulary projection: layer norm, preference loss and
clipped policy loss.  Argument marshalling only; the formulas and the conventions are those of
``include/vpce.h``.

Every tensor is checked against the problem before its pointer is taken, on the host, and a call
runs on the device of its tensors, on that device's current stream unless `stream` names one.
"""
from __future__ import annotations

import ctypes
from typing import Optional

from . import (VP_ACCUMULATE_DW, VP_ADV_PER_TOKEN, VP_ERR_WORKSPACE, VP_NORM_RMS, VP_PREF_LOGISTIC,
               VP_PREF_SQUARED, VP_SEQ_MEAN, _check, _dtype_code, _need, _need_ws, _same_device, _torch_dtype,
               load_library, vp_norm, vp_policy, vp_preference, vp_sequences)


class Norm:
    """A ``vp_norm``: rows, width, type and options of a layer norm."""

    def __init__(self, T: int, d: int, dtype: int, eps: float = 1e-5, rms: bool = False, accumulate: bool = False):
        flags = (VP_NORM_RMS if rms else 0) | (VP_ACCUMULATE_DW if accumulate else 0)
        self.c = vp_norm(T=int(T), d=int(d), dtype=int(dtype), flags=flags, eps=float(eps))
        self.ref = ctypes.byref(self.c)
        self.T, self.d, self.rms = int(T), int(d), bool(rms)


class Sequences:
    """A ``vp_sequences``: T packed tokens in S sequences; `mean` weights each sequence's sum by
    one over its counting tokens."""

    def __init__(self, T: int, S: int, ignore_index: int = -100, mean: bool = False):
        self.c = vp_sequences(T=int(T), S=int(S), ignore_index=int(ignore_index), flags=VP_SEQ_MEAN if mean else 0)
        self.ref = ctypes.byref(self.c)
        self.T, self.S, self.mean = int(T), int(S), bool(mean)


class Preference:
    """A ``vp_preference``: kind ("logistic" or "squared"), beta, margin and label smoothing."""

    def __init__(self, kind: str = "logistic", beta: float = 0.1, margin: float = 0.0, smoothing: float = 0.0):
        kinds = {"logistic": VP_PREF_LOGISTIC, "squared": VP_PREF_SQUARED}
        if kind not in kinds:
            raise ValueError(f"kind: {kind!r}, expected one of {sorted(kinds)}")
        self.c = vp_preference(kind=kinds[kind], beta=float(beta), margin=float(margin), smoothing=float(smoothing))
        self.ref = ctypes.byref(self.c)


class Policy:
    """A ``vp_policy``: clip bounds, KL weight, and whether the advantage is one value per token
    instead of one per sequence."""

    def __init__(self, clip_low: float = 0.2, clip_high: float = 0.2, kl_coef: float = 0.0, per_token: bool = False):
        self.c = vp_policy(clip_low=float(clip_low), clip_high=float(clip_high), kl_coef=float(kl_coef),
                           flags=VP_ADV_PER_TOKEN if per_token else 0)
        self.ref = ctypes.byref(self.c)
        self.per_token = bool(per_token)


class HeadNorm:
    """The layer norm in front of the projection, for ``forward(..., norm=)`` and
    ``backward(..., norm=)``: gamma [d] and beta [d] or None, of the hidden states' type."""

    def __init__(self, gamma, beta=None, eps: float = 1e-5, rms: bool = False):
        self.gamma, self.beta, self.eps, self.rms = gamma, beta, float(eps), bool(rms)


# ---------------------------------------------------------------------------
def _call(fn: str, head, named, ws, need, stream) -> None:
    """Checks `named` = (name, tensor, dtype, shape) and calls ``fn(*head, *pointers, stream)``.
    A name that ends in "?" may be None.  ws: the workspace of `need()` bytes, between the
    pointers and the stream; False for calls without one."""
    import torch
    args, dev, alike = list(head), -1, True
    for name, t, dtype, shape in named:
        if t is None and name[-1] == "?":
            args.append(None)
            continue
        try:
            good = t.dtype == dtype and t.shape == shape and t.is_contiguous()
        except AttributeError:  # not a tensor
            good = False
        if not good:
            _need(t, name.rstrip("?"), dtype, shape)
        at = t.get_device()
        alike &= at >= 0 and (dev < 0 or at == dev)
        dev = at if dev < 0 else dev
        args.append(t.data_ptr())
    if ws is not False:
        if not isinstance(ws, torch.Tensor) or not ws.is_contiguous():
            _need_ws(ws, 0)
        args += [ws.data_ptr(), ws.numel() * ws.element_size()]
        alike &= ws.get_device() == dev
    if not alike:
        if ws is not False:
            _need_ws(ws, need())
        _same_device([(n, t) for n, t, _, _ in named] + ([] if ws is False else [("ws", ws)]))
    lib = load_library()
    args.append(int(stream) if stream is not None else int(torch.cuda.current_stream(dev).cuda_stream))
    if torch.cuda.current_device() == dev:
        st = getattr(lib, fn)(*args)
    else:
        with torch.cuda.device(dev):
            st = getattr(lib, fn)(*args)
    if st == VP_ERR_WORKSPACE:
        _need_ws(ws, need())
    _check(st, fn)


def vp_norm_workspace_size(norm: Norm) -> int:
    """Bytes of the workspace of ``vp_norm_backward``."""
    n = ctypes.c_size_t(0)
    _check(load_library().vp_norm_workspace_size(norm.ref, ctypes.byref(n)), "vp_norm_workspace_size")
    return int(n.value)


def vp_norm_forward(norm: Norm, X, gamma, beta, Y, mean, rstd, stream=None) -> None:
    """Y and the row statistics of X.  beta may be None, and mean in the RMS form."""
    import torch
    f32, dt, Td, d, T = torch.float32, _torch_dtype(norm.c.dtype), (norm.T, norm.d), (norm.d,), (norm.T,)
    _call("vp_norm_forward", (norm.ref,),
          (("X", X, dt, Td), ("gamma", gamma, dt, d), ("beta?", beta, dt, d), ("Y", Y, dt, Td),
           ("mean?" if norm.rms else "mean", mean, f32, T), ("rstd", rstd, f32, T)), False, None, stream)


def vp_norm_backward(norm: Norm, X, gamma, mean, rstd, dY, dX, dgamma, dbeta, ws, stream=None) -> None:
    """dX (which may be dY), dgamma and dbeta (None: not computed)."""
    import torch
    f32, dt, Td, d, T = torch.float32, _torch_dtype(norm.c.dtype), (norm.T, norm.d), (norm.d,), (norm.T,)
    _call("vp_norm_backward", (norm.ref,),
          (("X", X, dt, Td), ("gamma", gamma, dt, d), ("mean?" if norm.rms else "mean", mean, f32, T),
           ("rstd", rstd, f32, T), ("dY", dY, f32, Td), ("dX", dX, f32, Td), ("dgamma", dgamma, f32, d),
           ("dbeta?", dbeta, f32, d)), ws, lambda: vp_norm_workspace_size(norm), stream)


def vp_seq_workspace_size(seq: Sequences) -> int:
    """Bytes of the workspace of ``vp_pref_forward`` and ``vp_policy_forward``."""
    n = ctypes.c_size_t(0)
    _check(load_library().vp_seq_workspace_size(seq.ref, ctypes.byref(n)), "vp_seq_workspace_size")
    return int(n.value)


def vp_pref_forward(seq: Sequences, pref: Preference, start, targets, loss, ref_loss, pair_loss, reward, coef, ws,
                    stream=None) -> None:
    """pair_loss [S/2], reward [S] and coef [S] of S/2 pairs.  ref_loss may be None."""
    import torch
    f32, T, S = torch.float32, (seq.T,), (seq.S,)
    _call("vp_pref_forward", (seq.ref, pref.ref),
          (("start", start, torch.int32, (seq.S + 1,)), ("targets", targets, torch.int64, T), ("loss", loss, f32, T),
           ("ref_loss?", ref_loss, f32, T), ("pair_loss", pair_loss, f32, (seq.S // 2,)), ("reward", reward, f32, S),
           ("coef", coef, f32, S)), ws, lambda: vp_seq_workspace_size(seq), stream)


def vp_pref_backward(seq: Sequences, start, targets, coef, grad_pair, grad_loss, stream=None) -> None:
    """grad_loss [T] from the forward's coef and the upstream gradient grad_pair [S/2]."""
    import torch
    f32, T = torch.float32, (seq.T,)
    _call("vp_pref_backward", (seq.ref,),
          (("start", start, torch.int32, (seq.S + 1,)), ("targets", targets, torch.int64, T),
           ("coef", coef, f32, (seq.S,)), ("grad_pair", grad_pair, f32, (seq.S // 2,)),
           ("grad_loss", grad_loss, f32, T)), False, None, stream)


def _policy_inputs(seq: Sequences, policy: Policy, start, targets, loss, old_loss, ref_loss, advantage):
    import torch
    f32, T = torch.float32, (seq.T,)
    return (("start", start, torch.int32, (seq.S + 1,)), ("targets", targets, torch.int64, T), ("loss", loss, f32, T),
            ("old_loss?", old_loss, f32, T), ("ref_loss?", ref_loss, f32, T),
            ("advantage", advantage, f32, T if policy.per_token else (seq.S,)))


def vp_policy_forward(seq: Sequences, policy: Policy, start, targets, loss, old_loss, ref_loss, advantage, seq_loss,
                      seq_kl, clipped, tokens, ws, stream=None) -> None:
    """seq_loss, seq_kl (float32) and clipped, tokens (int32) [S].  old_loss and ref_loss may be None."""
    import torch
    S = (seq.S,)
    _call("vp_policy_forward", (seq.ref, policy.ref),
          _policy_inputs(seq, policy, start, targets, loss, old_loss, ref_loss, advantage) +
          (("seq_loss", seq_loss, torch.float32, S), ("seq_kl", seq_kl, torch.float32, S),
           ("clipped", clipped, torch.int32, S), ("tokens", tokens, torch.int32, S)),
          ws, lambda: vp_seq_workspace_size(seq), stream)


def vp_policy_backward(seq: Sequences, policy: Policy, start, targets, loss, old_loss, ref_loss, advantage, tokens,
                       grad_seq, grad_loss, stream=None) -> None:
    """grad_loss [T] from the upstream gradient grad_seq [S]; tokens (from the forward) may be None
    without the mean."""
    import torch
    _call("vp_policy_backward", (seq.ref, policy.ref),
          _policy_inputs(seq, policy, start, targets, loss, old_loss, ref_loss, advantage) +
          (("tokens" if seq.mean else "tokens?", tokens, torch.int32, (seq.S,)),
           ("grad_seq", grad_seq, torch.float32, (seq.S,)), ("grad_loss", grad_loss, torch.float32, (seq.T,))),
          False, None, stream)


# ---------------------------------------------------------------------------
def _f32(*shape, like):
    import torch
    return torch.empty(*shape, dtype=torch.float32, device=like.device)


def _bytes(n: int, like):
    import torch
    return torch.empty(n, dtype=torch.uint8, device=like.device)


def layer_norm(X, gamma, beta=None, eps: float = 1e-5, rms: bool = False):
    """(Y, mean, rstd) of X [T, d]; mean is None in the RMS form."""
    import torch
    norm = Norm(X.shape[0], X.shape[1], _dtype_code(X), eps, rms)
    Y, mean, rstd = torch.empty_like(X), None if rms else _f32(norm.T, like=X), _f32(norm.T, like=X)
    vp_norm_forward(norm, X, gamma, beta, Y, mean, rstd)
    return Y, mean, rstd


def layer_norm_backward(X, gamma, mean, rstd, dY, bias: bool = True, dX=None, dgamma=None, dbeta=None,
                        accumulate: bool = False, ws=None):
    """(dX, dgamma, dbeta) float32 from dY float32 [T, d]; mean None means the RMS form, and
    `bias` False no dbeta (None).  dX may be dY; with `accumulate` the given dgamma and dbeta are
    added to."""
    if accumulate and (dgamma is None or (bias and dbeta is None)):
        raise ValueError("accumulate: dgamma (and dbeta) to add to are needed")
    norm = Norm(X.shape[0], X.shape[1], _dtype_code(X), 0.0, mean is None, accumulate)
    dX = _f32(norm.T, norm.d, like=X) if dX is None else dX
    dgamma = _f32(norm.d, like=X) if dgamma is None else dgamma
    dbeta = None if not bias else _f32(norm.d, like=X) if dbeta is None else dbeta
    ws = _bytes(vp_norm_workspace_size(norm), X) if ws is None else ws
    vp_norm_backward(norm, X, gamma, mean, rstd, dY, dX, dgamma, dbeta, ws)
    return dX, dgamma, dbeta


def preference_forward(loss, targets, start, pref: Preference, ref_loss=None, ignore_index: int = -100,
                       mean: bool = False, ws=None):
    """(pair_loss [S/2], reward [S], coef [S]) from the per-token loss of ``forward``; start:
    int32 [S + 1] offsets of the packed sequences, pairs one after the other."""
    seq = Sequences(loss.shape[0], start.shape[0] - 1, ignore_index, mean)
    pair_loss, reward, coef = (_f32(n, like=loss) for n in (seq.S // 2, seq.S, seq.S))
    ws = _bytes(vp_seq_workspace_size(seq), loss) if ws is None else ws
    vp_pref_forward(seq, pref, start, targets, loss, ref_loss, pair_loss, reward, coef, ws)
    return pair_loss, reward, coef


def preference_backward(targets, start, coef, grad_pair, ignore_index: int = -100):
    """grad_loss [T], for ``backward``, from the forward's coef and the gradient of each pair's loss."""
    seq = Sequences(targets.shape[0], start.shape[0] - 1, ignore_index)
    grad_loss = _f32(seq.T, like=targets)
    vp_pref_backward(seq, start, targets, coef, grad_pair, grad_loss)
    return grad_loss


def policy_forward(loss, targets, start, policy: Policy, advantage, old_loss=None, ref_loss=None,
                   ignore_index: int = -100, mean: bool = False, ws=None):
    """(seq_loss, seq_kl, clipped, tokens) [S] from the per-token loss of ``forward``; start: int32
    [S + 1] offsets of the packed sequences."""
    import torch
    seq = Sequences(loss.shape[0], start.shape[0] - 1, ignore_index, mean)
    seq_loss, seq_kl = _f32(seq.S, like=loss), _f32(seq.S, like=loss)
    clipped, tokens = (torch.empty(seq.S, dtype=torch.int32, device=loss.device) for _ in range(2))
    ws = _bytes(vp_seq_workspace_size(seq), loss) if ws is None else ws
    vp_policy_forward(seq, policy, start, targets, loss, old_loss, ref_loss, advantage, seq_loss, seq_kl, clipped,
                      tokens, ws)
    return seq_loss, seq_kl, clipped, tokens


def policy_backward(loss, targets, start, policy: Policy, advantage, tokens, grad_seq, old_loss=None, ref_loss=None,
                    ignore_index: int = -100, mean: bool = False):
    """grad_loss [T], for ``backward``, from the gradient grad_seq [S] of each sequence's loss."""
    seq = Sequences(loss.shape[0], start.shape[0] - 1, ignore_index, mean)
    grad_loss = _f32(seq.T, like=loss)
    vp_policy_backward(seq, policy, start, targets, loss, old_loss, ref_loss, advantage, tokens, grad_seq, grad_loss)
    return grad_loss
