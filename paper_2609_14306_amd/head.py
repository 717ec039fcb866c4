"""Binding of the operators around the vocabulary projection: layer norm, preference loss and
clipped policy loss.  Argument marshalling only; the formulas and the conventions are those of
``include/vpce.h``.

Every tensor is checked against the problem before its pointer is taken, on the host, and a call
runs on the device of its tensors, on that device's current stream unless `stream` names one.
"""
from __future__ import annotations

import ctypes
from functools import cached_property

from . import (VP_ACCUMULATE_DW, VP_ADV_PER_TOKEN, VP_ERR_ALIGN, VP_ERR_WORKSPACE, VP_NORM_RMS,
               VP_PREF_LOGISTIC, VP_PREF_SQUARED, VP_SEQ_MEAN, VpError, _check, _dtype_code, _need, _need_ws,
               _same_device, _torch_dtype, load_library, vp_norm, vp_policy, vp_preference, vp_sequences)


class Norm:
    """A ``vp_norm``: rows, width, type and options of a layer norm."""

    def __init__(self, T: int, d: int, dtype: int, eps: float = 1e-5, rms: bool = False, accumulate: bool = False):
        flags = (VP_NORM_RMS if rms else 0) | (VP_ACCUMULATE_DW if accumulate else 0)
        self.c = vp_norm(T=int(T), d=int(d), dtype=int(dtype), flags=flags, eps=float(eps))
        self.ref = ctypes.byref(self.c)
        self.T, self.d, self.rms = int(T), int(d), bool(rms)

    @cached_property
    def forward_spec(self):
        import torch
        f, x = torch.float32, _torch_dtype(self.c.dtype)
        Td, d, T = (self.T, self.d), (self.d,), (self.T,)
        return _spec(f"X gamma beta? Y {self._mean} rstd", (x, x, x, x, f, f), (Td, d, d, Td, T, T))

    @cached_property
    def backward_spec(self):
        import torch
        f, x = torch.float32, _torch_dtype(self.c.dtype)
        Td, d, T = (self.T, self.d), (self.d,), (self.T,)
        return _spec(f"X gamma {self._mean} rstd dY dX dgamma dbeta?", (x, x, f, f, f, f, f, f),
                     (Td, d, T, T, Td, Td, d, d))

    @cached_property
    def add_forward_spec(self):
        import torch
        f, x = torch.float32, _torch_dtype(self.c.dtype)
        Td, d, T = (self.T, self.d), (self.d,), (self.T,)
        return _spec(f"X R gamma beta? S Y? Y8? scale? {self._mean} rstd",
                     (x, x, x, x, x, x, torch.float8_e4m3fn, torch.float8_e8m0fnu, f, f),
                     (Td, Td, d, d, Td, Td, Td, (self.T, -(-self.d // 128)), T, T))

    @cached_property
    def add_backward_spec(self):
        import torch
        f, x = torch.float32, _torch_dtype(self.c.dtype)
        Td, d, T = (self.T, self.d), (self.d,), (self.T,)
        return _spec(f"S gamma {self._mean} rstd dY dS? dX dgamma dbeta?", (x, x, f, f, f, f, f, f, f),
                     (Td, d, T, T, Td, Td, Td, d, d))

    @property
    def _mean(self):
        return "mean?" if self.rms else "mean"


class Sequences:
    """A ``vp_sequences``: T packed tokens in S sequences; `mean` weights each sequence's sum by
    one over its counting tokens."""

    def __init__(self, T: int, S: int, ignore_index: int = -100, mean: bool = False):
        self.c = vp_sequences(T=int(T), S=int(S), ignore_index=int(ignore_index), flags=VP_SEQ_MEAN if mean else 0)
        self.ref = ctypes.byref(self.c)
        self.T, self.S, self.mean = int(T), int(S), bool(mean)

    def _spec(self, names, dtypes, shapes):
        import torch
        return _spec("start targets " + names, (torch.int32, torch.int64) + dtypes,
                     ((self.S + 1,), (self.T,)) + shapes)

    @cached_property
    def pref_forward_spec(self):
        import torch
        T, S, N = (self.T,), (self.S,), (self.S // 2,)
        return self._spec("loss ref_loss? pair_loss reward coef", (torch.float32,) * 5, (T, T, N, S, S))

    @cached_property
    def pref_backward_spec(self):
        import torch
        return self._spec("coef grad_pair grad_loss", (torch.float32,) * 3, ((self.S,), (self.S // 2,), (self.T,)))

    # by whether the advantage is one value per token
    @cached_property
    def policy_forward_spec(self):
        import torch
        f, i, T, S = torch.float32, torch.int32, (self.T,), (self.S,)
        return [self._spec("loss old_loss? ref_loss? advantage seq_loss seq_kl clipped tokens",
                           (f, f, f, f, f, f, i, i), (T, T, T, adv, S, S, S, S)) for adv in (S, T)]

    @cached_property
    def policy_backward_spec(self):
        import torch
        f, T, S = torch.float32, (self.T,), (self.S,)
        return [self._spec(f"loss old_loss? ref_loss? advantage {'tokens' if self.mean else 'tokens?'} grad_seq grad_loss",
                           (f, f, f, f, torch.int32, f, f), (T, T, T, adv, S, S, T)) for adv in (S, T)]


class Preference:
    """A ``vp_preference``: kind ("logistic" or "squared"), beta, margin and label smoothing (0..1/2;
    the squared form has none, and calls with it leave the value unused)."""

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
# A call's tensors, in the order of the C entry: names (one that ends in "?" may be None), dtypes
# and shapes.  The problems build each once, so that a call's checks are one pass of about 0.25 us
# a tensor; what a tensor is, and where, is looked up on every call.
def _spec(names, dtypes, shapes):
    return tuple((n, n[-1] == "?", dt, tuple(sh)) for n, dt, sh in zip(names.split(), dtypes, shapes))


def _raw_stream(dev: int) -> int:
    import torch
    get = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # 1 us less than a Stream object
    return int(get(dev) if get is not None else torch.cuda.current_stream(dev).cuda_stream)


def _refuse(spec, tensors, ws, need) -> None:
    for (name, may, dtype, shape), t in zip(spec, tensors):
        if not (may and t is None):
            _need(t, name.rstrip("?"), dtype, shape)
    if ws is not False:
        _need_ws(ws, need())
    _same_device([(n[0].rstrip("?"), t) for n, t in zip(spec, tensors)] + ([] if ws is False else [("ws", ws)]))


def _call(fn: str, head, spec, tensors, stream, ws=False, need=None) -> None:
    """Checks `tensors` against `spec` and calls ``fn(*head, *pointers, stream)``.  ws: the
    workspace of `need()` bytes, between the pointers and the stream; False for calls without."""
    import torch
    args = list(head)
    try:
        dev = tensors[0].get_device()
        good = dev >= 0
        for (_, may, dtype, shape), t in zip(spec, tensors):
            if may and t is None:
                args.append(None)
            elif t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous():
                args.append(t.data_ptr())
            else:
                good = False
                break
        if good and ws is not False:
            good = ws.get_device() == dev and ws.is_contiguous()
            args += (ws.data_ptr(), ws.numel() * ws.element_size())
    except AttributeError:  # not a tensor
        good = False
    if not good:
        _refuse(spec, tensors, ws, need)
        raise ValueError(f"{fn}: unsupported tensors")
    args.append(_raw_stream(dev) if stream is None else int(stream))
    call = getattr(load_library(), fn)
    if torch.cuda.current_device() == dev:
        st = call(*args)
    else:
        with torch.cuda.device(dev):
            st = call(*args)
    if st == VP_ERR_WORKSPACE:
        _refuse(spec, tensors, ws, need)
    _check(st, fn)


def vp_norm_workspace_size(norm: Norm) -> int:
    """Bytes of the workspace of ``vp_norm_backward``."""
    n = ctypes.c_size_t(0)
    _check(load_library().vp_norm_workspace_size(norm.ref, ctypes.byref(n)), "vp_norm_workspace_size")
    return int(n.value)


def vp_norm_forward(norm: Norm, X, gamma, beta, Y, mean, rstd, stream=None) -> None:
    """Y and the row statistics of X.  beta may be None, and mean in the RMS form."""
    _call("vp_norm_forward", (norm.ref,), norm.forward_spec, (X, gamma, beta, Y, mean, rstd), stream)


def vp_norm_backward(norm: Norm, X, gamma, mean, rstd, dY, dX, dgamma, dbeta, ws, stream=None) -> None:
    """dX (which may be dY), dgamma and dbeta (None: not computed)."""
    _call("vp_norm_backward", (norm.ref,), norm.backward_spec, (X, gamma, mean, rstd, dY, dX, dgamma, dbeta), stream,
          ws, lambda: vp_norm_workspace_size(norm))


def vp_add_norm_forward(norm: Norm, X, R, gamma, beta, S, Y, Y8, scale, mean, rstd, stream=None) -> None:
    """S = X + R (S may be X or R) and the norm of it: Y, or Y8 with scale, or both; what is not wanted is
    None, and so may be beta, and mean in the RMS form."""
    _call("vp_add_norm_forward", (norm.ref,), norm.add_forward_spec, (X, R, gamma, beta, S, Y, Y8, scale, mean, rstd),
          stream)


def vp_add_norm_backward(norm: Norm, S, gamma, mean, rstd, dY, dS, dX, dgamma, dbeta, ws, stream=None) -> None:
    """dX (which may be dY or dS), dgamma and dbeta (None: not computed); dS: the gradient that S has
    elsewhere, or None."""
    _call("vp_add_norm_backward", (norm.ref,), norm.add_backward_spec,
          (S, gamma, mean, rstd, dY, dS, dX, dgamma, dbeta), stream, ws, lambda: vp_norm_workspace_size(norm))


def vp_seq_workspace_size(seq: Sequences) -> int:
    """Bytes of the workspace of ``vp_pref_forward`` and ``vp_policy_forward``."""
    n = ctypes.c_size_t(0)
    _check(load_library().vp_seq_workspace_size(seq.ref, ctypes.byref(n)), "vp_seq_workspace_size")
    return int(n.value)


def _preference_ref(pref: Preference):
    """What the C entry takes for `pref`: with the squared form it accepts no smoothing but 0."""
    c = pref.c
    if c.kind == VP_PREF_SQUARED and 0.0 < c.smoothing <= 0.5:
        return ctypes.byref(vp_preference(kind=c.kind, beta=c.beta, margin=c.margin))
    return pref.ref


def vp_pref_forward(seq: Sequences, pref: Preference, start, targets, loss, ref_loss, pair_loss, reward, coef, ws,
                    stream=None) -> None:
    """pair_loss [S/2], reward [S] and coef [S] of S/2 pairs.  ref_loss may be None."""
    _call("vp_pref_forward", (seq.ref, _preference_ref(pref)), seq.pref_forward_spec,
          (start, targets, loss, ref_loss, pair_loss, reward, coef), stream, ws, lambda: vp_seq_workspace_size(seq))


def vp_pref_backward(seq: Sequences, start, targets, coef, grad_pair, grad_loss, stream=None) -> None:
    """grad_loss [T] from the forward's coef and the upstream gradient grad_pair [S/2]."""
    _call("vp_pref_backward", (seq.ref,), seq.pref_backward_spec, (start, targets, coef, grad_pair, grad_loss), stream)


def vp_policy_forward(seq: Sequences, policy: Policy, start, targets, loss, old_loss, ref_loss, advantage, seq_loss,
                      seq_kl, clipped, tokens, ws, stream=None) -> None:
    """seq_loss, seq_kl (float32) and clipped, tokens (int32) [S].  old_loss and ref_loss may be None."""
    _call("vp_policy_forward", (seq.ref, policy.ref), seq.policy_forward_spec[policy.per_token],
          (start, targets, loss, old_loss, ref_loss, advantage, seq_loss, seq_kl, clipped, tokens), stream, ws,
          lambda: vp_seq_workspace_size(seq))


def vp_policy_backward(seq: Sequences, policy: Policy, start, targets, loss, old_loss, ref_loss, advantage, tokens,
                       grad_seq, grad_loss, stream=None) -> None:
    """grad_loss [T] from the upstream gradient grad_seq [S]; tokens (from the forward) may be None
    without the mean."""
    _call("vp_policy_backward", (seq.ref, policy.ref), seq.policy_backward_spec[policy.per_token],
          (start, targets, loss, old_loss, ref_loss, advantage, tokens, grad_seq, grad_loss), stream)


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


def _check_norm_grads(X, bias, dgamma, dbeta, accumulate) -> None:
    """What a norm backward refuses of the given dgamma and dbeta (None: none given), for callers
    that have other work in front of it."""
    import torch
    if accumulate and (dgamma is None or (bias and dbeta is None)):
        raise ValueError("accumulate: dgamma (and dbeta) to add to are needed")
    named = [(n, t) for n, t in (("dgamma", dgamma), ("dbeta", dbeta if bias else None)) if t is not None]
    for name, t in named:
        _need(t, name, torch.float32, (X.shape[1],))
        if t.data_ptr() % 16 != 0:
            raise VpError(VP_ERR_ALIGN, name)
    if named:
        _same_device([("X", X)] + named)


def layer_norm_backward(X, gamma, mean, rstd, dY, bias: bool = True, dX=None, dgamma=None, dbeta=None,
                        accumulate: bool = False, ws=None):
    """(dX, dgamma, dbeta) float32 from dY float32 [T, d]; mean None means the RMS form, and
    `bias` False no dbeta (None).  dX may be dY; with `accumulate` the given dgamma and dbeta are
    added to."""
    _check_norm_grads(X, bias, dgamma, dbeta, accumulate)
    norm = Norm(X.shape[0], X.shape[1], _dtype_code(X), 0.0, mean is None, accumulate)
    dX = _f32(norm.T, norm.d, like=X) if dX is None else dX
    dgamma = _f32(norm.d, like=X) if dgamma is None else dgamma
    dbeta = None if not bias else _f32(norm.d, like=X) if dbeta is None else dbeta
    ws = _bytes(vp_norm_workspace_size(norm), X) if ws is None else ws
    vp_norm_backward(norm, X, gamma, mean, rstd, dY, dX, dgamma, dbeta, ws)
    return dX, dgamma, dbeta


def add_norm(X, R, gamma, beta=None, eps: float = 1e-5, rms: bool = False, f8: bool = False):
    """(S, Y, mean, rstd) with S = X + R [T, d] and Y its norm; mean is None in the RMS form.  With
    `f8`, Y is (Y8, scale) as ``score_f8`` takes them."""
    import torch
    from .scoring import f8_buffers
    norm = Norm(X.shape[0], X.shape[1], _dtype_code(X), eps, rms)
    S, mean, rstd = torch.empty_like(X), None if rms else _f32(norm.T, like=X), _f32(norm.T, like=X)
    Y8, scale = f8_buffers(norm.T, norm.d, 1, X.device) if f8 else (None, None)
    Y = None if f8 else torch.empty_like(X)
    vp_add_norm_forward(norm, X, R, gamma, beta, S, Y, Y8, scale, mean, rstd)
    return S, (Y8, scale) if f8 else Y, mean, rstd


def add_norm_backward(S, gamma, mean, rstd, dY, dS=None, bias: bool = True, dX=None, dgamma=None, dbeta=None,
                      accumulate: bool = False, ws=None):
    """(dX, dgamma, dbeta) float32: the gradient of X, which is that of R too, from dY and the gradient dS
    that S has elsewhere; the rest as for ``layer_norm_backward``."""
    _check_norm_grads(S, bias, dgamma, dbeta, accumulate)
    norm = Norm(S.shape[0], S.shape[1], _dtype_code(S), 0.0, mean is None, accumulate)
    dX = _f32(norm.T, norm.d, like=S) if dX is None else dX
    dgamma = _f32(norm.d, like=S) if dgamma is None else dgamma
    dbeta = None if not bias else _f32(norm.d, like=S) if dbeta is None else dbeta
    ws = _bytes(vp_norm_workspace_size(norm), S) if ws is None else ws
    vp_add_norm_backward(norm, S, gamma, mean, rstd, dY, dS, dX, dgamma, dbeta, ws)
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
