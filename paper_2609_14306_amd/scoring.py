"""Binding of the scoring calls: entropy and the most likely ids of every token beside its loss, in
the projection's types and in 8 bits, the gradients with an entropy term, and 8-bit operands.
Argument marshalling only; the formulas and the conventions are those of ``include/vpce.h``.

Every tensor is checked against the problem before its pointer is taken, on the host, and a call
runs on the device of its tensors, on that device's current stream unless `stream` names one.
8-bit values are ``torch.float8_e4m3fn``; scales are ``torch.float8_e8m0fnu`` (powers of two, the
bytes that the C entries describe).
"""
from __future__ import annotations

import ctypes
from functools import cached_property

from . import (VP_E4M3, VP_ERR_WORKSPACE, Problem, _check, _dtype_code, _need, _need_ws, _same_device, _torch_dtype,
               load_library, problem_for, vp_ce_workspace_size, vp_quant, vp_score)
from .head import _bytes, _call, _f32, _raw_stream, _spec, layer_norm


class Score:
    """A ``vp_score``: how many alternatives every token gets (0..32)."""

    def __init__(self, top: int = 0):
        self.c = vp_score(top=int(top))
        self.ref = ctypes.byref(self.c)
        self.top = int(top)


class Quant:
    """A ``vp_quant``: rows and columns, the type of what is quantised, and the rows of a block (1
    for hidden states, 128 for weights)."""

    def __init__(self, rows: int, cols: int, dtype: int, rows_per_scale: int = 1):
        self.c = vp_quant(rows=int(rows), cols=int(cols), dtype=int(dtype), rows_per_scale=int(rows_per_scale))
        self.ref = ctypes.byref(self.c)
        self.rows, self.cols, self.rows_per_scale = int(rows), int(cols), int(rows_per_scale)

    @cached_property
    def spec(self):
        import torch
        shape, step = (self.rows, self.cols), max(1, self.rows_per_scale)
        return _spec("X X8 scale", (_torch_dtype(self.c.dtype), torch.float8_e4m3fn, torch.float8_e8m0fnu),
                     (shape, shape, (-(-self.rows // step), -(-self.cols // 128))))


# ---------------------------------------------------------------------------
# A call's arguments in the order of the C entry.  Each is (name, may be None, dtype, shape, tensor),
# or for the shards a list of shapes and one of tensors, whose pointers go into one array.
def _shard_array(shapes, dtype, tensors, dev):
    out = []
    for t, shape in zip(tensors, shapes):
        if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
            return None
        out.append(t.data_ptr() if shape[0] else None)
    return (ctypes.c_void_p * len(shapes))(*out)


def _refuse(items, ws, need) -> None:
    named = []
    for name, may, dtype, shape, t in items:
        if isinstance(shape, list):
            if len(t) != len(shape):
                raise ValueError(f"{name}: {len(t)} shards, the problem has {len(shape)}")
            for p, (s, one) in enumerate(zip(shape, t)):
                _need(one, f"{name}[{p}]", dtype, s)
                named.append((f"{name}[{p}]", one))
        elif not (may and t is None):
            _need(t, name, dtype, shape)
            named.append((name, t))
    _need_ws(ws, need())
    _same_device(named + [("ws", ws)])


def _call_shards(fn: str, head, items, ws, need, stream) -> None:
    import torch
    args = list(head)
    try:
        dev = items[0][4].get_device()
        good = dev >= 0
        for _, may, dtype, shape, t in items:
            if isinstance(shape, list):
                a = _shard_array(shape, dtype, t, dev) if len(t) == len(shape) else None
                good = good and a is not None
                args.append(a)
            elif may and t is None:
                args.append(None)
            elif t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous():
                args.append(t.data_ptr())
            else:
                good = False
            if not good:
                break
        good = good and ws.get_device() == dev and ws.is_contiguous()
        if good:
            args += (ws.data_ptr(), ws.numel() * ws.element_size())
    except (AttributeError, TypeError):  # not a tensor, or no list of them
        good = False
    if not good:
        _refuse(items, ws, need)
        raise ValueError(f"{fn}: unsupported tensors")
    args.append(_raw_stream(dev) if stream is None else int(stream))
    call = getattr(load_library(), fn)
    if torch.cuda.current_device() == dev:
        st = call(*args)
    else:
        with torch.cuda.device(dev):
            st = call(*args)
    if st == VP_ERR_WORKSPACE:
        _refuse(items, ws, need)
    _check(st, fn)


def vp_score_workspace_size(prob: Problem, score: Score) -> int:
    """Bytes of the workspace of ``vp_score_forward`` and ``vp_score_forward_f8``."""
    n = ctypes.c_size_t(0)
    _check(load_library().vp_score_workspace_size(ctypes.byref(prob.c), score.ref, ctypes.byref(n)),
           "vp_score_workspace_size")
    return int(n.value)


def _outputs(prob: Problem, score: Score, loss, lse, entropy, top_ids, top_loss):
    import torch
    f, T, top = torch.float32, prob.shape_T, (prob.T, score.top)
    none = score.top == 0
    return [("loss", False, f, T, loss), ("lse", False, f, T, lse), ("entropy", True, f, T, entropy),
            ("top_ids", none, torch.int64, top, top_ids), ("top_loss", none, f, top, top_loss)]


def vp_score_forward(prob: Problem, score: Score, H, W_shards, targets, loss, lse, entropy, top_ids, top_loss, ws,
                     stream=None) -> None:
    """loss, lse, entropy [T], and with alternatives top_ids (int64) and top_loss [T, top].  entropy
    may be None; without alternatives top_ids and top_loss are None."""
    import torch
    dt = _torch_dtype(prob.c.dtype)
    items = [("H", False, dt, prob.shape_Td, H), ("W_shards", False, dt, prob.shapes_W, W_shards),
             ("targets", False, torch.int64, prob.shape_T, targets)]
    _call_shards("vp_score_forward", (ctypes.byref(prob.c), score.ref),
                 items + _outputs(prob, score, loss, lse, entropy, top_ids, top_loss), ws,
                 lambda: vp_score_workspace_size(prob, score), stream)


def vp_score_forward_f8(prob: Problem, score: Score, H, H_scale, W_shards, W_scales, targets, loss, lse, entropy,
                        top_ids, top_loss, ws, stream=None) -> None:
    """``vp_score_forward`` of 8-bit hidden states [T, d] with scales [T, ceil(d / 128)] and shards with
    scales [ceil(V_p / 128), ceil(d / 128)]; the problem's dtype is ``VP_E4M3``."""
    import torch
    v, s, nb = torch.float8_e4m3fn, torch.float8_e8m0fnu, -(-prob.d // 128)
    items = [("H", False, v, prob.shape_Td, H), ("H_scale", False, s, (prob.T, nb), H_scale),
             ("W_shards", False, v, prob.shapes_W, W_shards),
             ("W_scales", False, s, [(-(-r // 128), nb) for r in prob.shard_rows], W_scales),
             ("targets", False, torch.int64, prob.shape_T, targets)]
    _call_shards("vp_score_forward_f8", (ctypes.byref(prob.c), score.ref),
                 items + _outputs(prob, score, loss, lse, entropy, top_ids, top_loss), ws,
                 lambda: vp_score_workspace_size(prob, score), stream)


def vp_score_backward(prob: Problem, H, W_shards, targets, lse, entropy, grad_loss, grad_entropy, dH, dW_shards, ws,
                      stream=None) -> None:
    """dH and dW of a loss with an entropy term; ws: the backward's of ``vp_ce_workspace_size``."""
    import torch
    dt, f, T = _torch_dtype(prob.c.dtype), torch.float32, prob.shape_T
    items = [("H", False, dt, prob.shape_Td, H), ("W_shards", False, dt, prob.shapes_W, W_shards),
             ("targets", False, torch.int64, T, targets), ("lse", False, f, T, lse),
             ("entropy", False, f, T, entropy), ("grad_loss", False, f, T, grad_loss),
             ("grad_entropy", False, f, T, grad_entropy), ("dH", False, f, prob.shape_Td, dH),
             ("dW_shards", False, f, prob.shapes_W, dW_shards)]
    _call_shards("vp_score_backward", (ctypes.byref(prob.c),), items, ws, lambda: vp_ce_workspace_size(prob)[1],
                 stream)


def vp_f8_quantize(quant: Quant, X, X8, scale, stream=None) -> None:
    """X8 and scale of X (see ``f8_buffers``)."""
    _call("vp_f8_quantize", (quant.ref,), quant.spec, (X, X8, scale), stream)


# ---------------------------------------------------------------------------
def f8_buffers(rows: int, cols: int, rows_per_scale: int, device):
    """Empty 8-bit values [rows, cols] and scales of blocks of rows_per_scale x 128 on `device`."""
    import torch
    return (torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device=device),
            torch.empty(-(-rows // rows_per_scale), -(-cols // 128), dtype=torch.float8_e8m0fnu, device=device))


def quantize(X, rows_per_scale: int = 1):
    """(X8, scale) of X [rows, cols] in blocks of rows_per_scale (1 or 128) x 128."""
    quant = Quant(X.shape[0], X.shape[1], _dtype_code(X), rows_per_scale)
    if rows_per_scale not in (1, 128):
        raise ValueError(f"rows_per_scale: {rows_per_scale}, expected 1 or 128")
    X8, scale = f8_buffers(quant.rows, quant.cols, rows_per_scale, X.device)
    vp_f8_quantize(quant, X, X8, scale)
    return X8, scale


def _score_outputs(T: int, score: Score, like):
    import torch
    top = (torch.empty(T, score.top, dtype=torch.int64, device=like.device), _f32(T, score.top, like=like))
    return [_f32(T, like=like) for _ in range(3)] + (list(top) if score.top else [None, None])


def score(H, W_shards, targets, top: int = 0, ignore_index: int = -100, ws=None, norm=None):
    """(loss, lse, entropy, top_ids, top_loss) of hidden states H [T, d] and shards W_p [V_p, d]; the
    last two [T, top], or None without alternatives.

    With `norm` (a ``HeadNorm``, as ``forward`` and ``backward`` take it), H is what the norm takes."""
    import torch
    if norm is not None:
        with torch.cuda.device_of(H):  # the norm and the projection on one stream
            Y = layer_norm(H, norm.gamma, norm.beta, norm.eps, norm.rms)[0]
            return score(Y, W_shards, targets, top, ignore_index, ws)
    prob, sc = problem_for(H, W_shards, ignore_index), Score(top)
    ws = _bytes(vp_score_workspace_size(prob, sc), H) if ws is None else ws
    out = _score_outputs(prob.T, sc, H)
    vp_score_forward(prob, sc, H, W_shards, targets, *out, ws)
    return tuple(out)


def score_f8(H, H_scale, W_shards, W_scales, targets, top: int = 0, ignore_index: int = -100, ws=None):
    """``score`` of 8-bit operands, as ``quantize`` and ``add_norm`` make them."""
    prob = Problem(H.shape[0], H.shape[1], [w.shape[0] for w in W_shards], VP_E4M3, None, ignore_index)
    sc = Score(top)
    ws = _bytes(vp_score_workspace_size(prob, sc), H) if ws is None else ws
    out = _score_outputs(prob.T, sc, H)
    vp_score_forward_f8(prob, sc, H, H_scale, W_shards, W_scales, targets, *out, ws)
    return tuple(out)
