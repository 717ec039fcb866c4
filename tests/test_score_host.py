"""Host-side tests of the scoring calls, quantisation and the norm with a residual (no GPU): every
refusal is returned before any HIP call, the binding checks each tensor, and every call of the ranges
of perf/more_operators.py passes the host's checks; the plain gradients against differences."""
import ctypes
import os
import random

import pytest
import torch

import paper_2609_14306_amd as vp
import score_plain as sp
from perf import more_operators

pytestmark = pytest.mark.skipif(not os.path.exists(vp.LIB_PATH),
                                reason="libvpce.so not built (run __graft_entry__.build())")

FAKE = 0x100000  # an aligned pointer value that no call here dereferences


def _lib():
    return vp.load_library()


def _array(n, value=FAKE):
    return (ctypes.c_void_p * n)(*[value] * n)


def _problem(**over):
    kw = dict(T=10, d=64, shard_rows=[30, 50], dtype=vp.VP_BF16)
    kw.update(over)
    return vp.Problem(**kw)


def _forward(prob=None, score=None, ws=FAKE, ws_bytes=1 << 50, **over):
    prob, score = prob or _problem(), score or vp.Score(3)
    a = dict(H=FAKE, W=_array(prob.P), targets=FAKE, loss=FAKE, lse=FAKE, entropy=FAKE, top_ids=FAKE, top_loss=FAKE)
    a.update(over)
    return _lib().vp_score_forward(ctypes.byref(prob.c), score.ref, *a.values(), ws, ws_bytes, None)


def _forward_f8(prob=None, score=None, ws=FAKE, ws_bytes=1 << 50, **over):
    prob, score = prob or _problem(dtype=vp.VP_E4M3), score or vp.Score(3)
    a = dict(H=FAKE, H_scale=FAKE, W=_array(prob.P), W_scales=_array(prob.P), targets=FAKE, loss=FAKE, lse=FAKE,
             entropy=FAKE, top_ids=FAKE, top_loss=FAKE)
    a.update(over)
    return _lib().vp_score_forward_f8(ctypes.byref(prob.c), score.ref, *a.values(), ws, ws_bytes, None)


def _backward(prob=None, ws=FAKE, ws_bytes=1 << 50, **over):
    prob = prob or _problem()
    a = dict(H=FAKE, W=_array(prob.P), targets=FAKE, lse=FAKE, entropy=FAKE, grad_loss=FAKE, grad_entropy=FAKE, dH=FAKE,
             dW=_array(prob.P))
    a.update(over)
    return _lib().vp_score_backward(ctypes.byref(prob.c), *a.values(), ws, ws_bytes, None)


def _quantize(quant=None, **over):
    quant = quant or vp.Quant(10, 64, vp.VP_F32)
    a = dict(X=FAKE, X8=FAKE, scale=FAKE)
    a.update(over)
    return _lib().vp_f8_quantize(quant.ref, *a.values(), None)


def _add_fwd(norm=None, **over):
    norm = norm or vp.Norm(4, 64, vp.VP_BF16)
    a = dict(X=FAKE, R=FAKE, gamma=FAKE, beta=FAKE, S=FAKE, Y=FAKE, Y8=FAKE, scale=FAKE, mean=FAKE, rstd=FAKE)
    a.update(over)
    return _lib().vp_add_norm_forward(norm.ref, *a.values(), None)


def _add_bwd(norm=None, ws=FAKE, ws_bytes=1 << 40, **over):
    norm = norm or vp.Norm(4, 64, vp.VP_BF16)
    a = dict(S=FAKE, gamma=FAKE, mean=FAKE, rstd=FAKE, dY=FAKE, dS=FAKE, dX=FAKE, dgamma=FAKE, dbeta=FAKE)
    a.update(over)
    return _lib().vp_add_norm_backward(norm.ref, *a.values(), ws, ws_bytes, None)


@pytest.mark.parametrize("over, want", [
    (dict(T=-1), vp.VP_ERR_SHAPE), (dict(T=2 ** 23 - 255), vp.VP_ERR_SHAPE), (dict(d=4), vp.VP_ERR_SHAPE),
    (dict(d=60), vp.VP_ERR_SHAPE), (dict(shard_rows=[]), vp.VP_ERR_SHAPE), (dict(shard_rows=[0, 0]), vp.VP_ERR_SHAPE),
    (dict(shard_rows=[-1, 5]), vp.VP_ERR_SHAPE), (dict(order=[0, 0]), vp.VP_ERR_ORDER), (dict(dtype=7), vp.VP_ERR_DTYPE),
    (dict(shard_rows=[1 << 24, 1]), vp.VP_ERR_SHAPE)])
def test_problem_refused(over, want):
    prob = _problem(**over)
    assert _forward(prob) == want
    assert _lib().vp_score_workspace_size(ctypes.byref(prob.c), vp.Score(3).ref, None) == want
    if over.get("shard_rows") != [1 << 24, 1]:  # (a limit of the alternatives alone)
        assert _backward(prob) == want
    else:
        size = ctypes.c_size_t(0)
        assert _lib().vp_score_workspace_size(ctypes.byref(prob.c), vp.Score(0).ref, ctypes.byref(size)) == vp.VP_OK
        assert size.value < 1 << 20


def test_types_refused():
    assert _forward(_problem(dtype=vp.VP_E4M3)) == vp.VP_ERR_DTYPE
    assert _backward(_problem(dtype=vp.VP_E4M3)) == vp.VP_ERR_DTYPE
    assert _forward_f8(_problem()) == vp.VP_ERR_DTYPE
    for d in (8, 24, 14352):
        assert _forward_f8(_problem(dtype=vp.VP_E4M3, d=d)) == vp.VP_ERR_SHAPE, d
    prob = _problem(dtype=vp.VP_E4M3)  # the other calls of the library do not take 8 bits
    assert _lib().vp_ce_workspace_size(ctypes.byref(prob.c), None, None) == vp.VP_ERR_DTYPE
    assert _quantize(vp.Quant(10, 64, vp.VP_E4M3)) == vp.VP_ERR_DTYPE


@pytest.mark.parametrize("top", [-1, 33])
def test_number_of_alternatives_refused(top):
    assert _forward(score=vp.Score(top)) == vp.VP_ERR_VALUE
    assert _forward_f8(score=vp.Score(top)) == vp.VP_ERR_VALUE
    assert _lib().vp_score_workspace_size(ctypes.byref(_problem().c), vp.Score(top).ref, None) == vp.VP_ERR_VALUE


def test_null_pointers_refused():
    for call, names in ((_forward, "H W targets loss lse top_ids top_loss"),
                        (_forward_f8, "H H_scale W W_scales targets loss lse top_ids top_loss"),
                        (_backward, "H W targets lse entropy grad_loss grad_entropy dH dW"),
                        (_quantize, "X X8 scale"), (_add_fwd, "X R gamma S mean rstd Y8 scale"),
                        (_add_bwd, "S gamma mean rstd dY dX dgamma")):
        for name in names.split():
            assert call(**{name: None}) == vp.VP_ERR_NULL, (call, name)
    assert _add_fwd(Y=None, Y8=None, scale=None) == vp.VP_ERR_NULL
    for name in ("W", "W_scales"):
        assert _forward_f8(**{name: _array(2, None)}) == vp.VP_ERR_NULL
    n, p = [None] * 16, _problem()
    assert _lib().vp_score_forward(None, vp.Score().ref, None, None, *n[:7], 0, None) == vp.VP_ERR_NULL
    assert _lib().vp_score_forward(ctypes.byref(p.c), None, None, _array(2), *n[:7], 0, None) == vp.VP_ERR_NULL
    assert _lib().vp_f8_quantize(None, *n[:4]) == vp.VP_ERR_NULL
    assert _lib().vp_add_norm_forward(None, *n[:11]) == vp.VP_ERR_NULL
    assert _lib().vp_add_norm_backward(None, *n[:10], 0, None) == vp.VP_ERR_NULL


def test_misaligned_pointers_refused():
    for call, names in ((_forward, "H ws"), (_forward_f8, "H ws"), (_backward, "H dH ws"), (_quantize, "X X8"),
                        (_add_fwd, "X R gamma beta S Y Y8"), (_add_bwd, "S gamma dY dS dX dgamma dbeta ws")):
        for name in names.split():
            assert call(**{name: FAKE + 8}) == vp.VP_ERR_ALIGN, (call, name)
    assert _forward(W=_array(2, FAKE + 8)) == vp.VP_ERR_ALIGN
    assert _backward(dW=_array(2, FAKE + 8)) == vp.VP_ERR_ALIGN
    assert _add_fwd(mean=FAKE + 2) == vp.VP_ERR_ALIGN


def test_workspace_refused():
    size = ctypes.c_size_t(0)
    for prob, call in ((_problem(), _forward), (_problem(dtype=vp.VP_E4M3), _forward_f8)):
        assert call(ws=None) == vp.VP_ERR_WORKSPACE
        assert _lib().vp_score_workspace_size(ctypes.byref(prob.c), vp.Score(3).ref, ctypes.byref(size)) == vp.VP_OK
        assert call(ws_bytes=size.value - 1) == vp.VP_ERR_WORKSPACE
    assert _backward(ws_bytes=vp.vp_ce_workspace_size(_problem())[1] - 1) == vp.VP_ERR_WORKSPACE
    assert _add_bwd(ws_bytes=vp.vp_norm_workspace_size(vp.Norm(4, 64, vp.VP_BF16)) - 1) == vp.VP_ERR_WORKSPACE


@pytest.mark.parametrize("over, want", [
    (dict(rows=-1), vp.VP_ERR_SHAPE), (dict(rows=(1 << 30) + 1), vp.VP_ERR_SHAPE), (dict(cols=8), vp.VP_ERR_SHAPE),
    (dict(cols=72), vp.VP_ERR_SHAPE), (dict(cols=(1 << 22) + 16), vp.VP_ERR_SHAPE), (dict(dtype=3), vp.VP_ERR_DTYPE),
    (dict(rows_per_scale=0), vp.VP_ERR_VALUE), (dict(rows_per_scale=64), vp.VP_ERR_VALUE)])
def test_quantisation_refused(over, want):
    kw = dict(rows=10, cols=64, dtype=vp.VP_F32, rows_per_scale=1)
    kw.update(over)
    assert _quantize(vp.Quant(**kw)) == want


@pytest.mark.parametrize("over, want", [(dict(T=-1), vp.VP_ERR_SHAPE), (dict(d=16392), vp.VP_ERR_SHAPE),
                                        (dict(dtype=2), vp.VP_ERR_DTYPE), (dict(eps=-1.0), vp.VP_ERR_VALUE)])
def test_norm_refused(over, want):
    kw = dict(T=4, d=64, dtype=vp.VP_BF16)
    kw.update(over)
    assert _add_fwd(vp.Norm(**kw)) == want and _add_bwd(vp.Norm(**kw)) == want


def test_calls_without_work_need_no_arrays():
    assert _quantize(vp.Quant(0, 64, vp.VP_F32), X=None, X8=None, scale=None) == vp.VP_OK
    assert _add_fwd(vp.Norm(0, 64, vp.VP_F32), X=None, R=None, S=None, Y=None) == vp.VP_OK


def test_workspace_is_bounded():
    for top in (1, 32):
        big = vp.vp_score_workspace_size(_problem(T=100000, d=2880, shard_rows=[25136] * 8), vp.Score(top))
        assert big < (1 << 30) + (1 << 24)
    assert vp.vp_score_workspace_size(_problem(T=100000, d=2880, shard_rows=[25136] * 8), vp.Score()) < 1 << 26


# ---------------------------------------------------------------------------
def _tensors(**over):
    z = lambda *s: torch.zeros(*s)  # noqa: E731
    x = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    a = dict(H=x(10, 64), W_shards=[x(30, 64), x(50, 64)], targets=torch.zeros(10, dtype=torch.int64), loss=z(10), lse=z(10),
             entropy=z(10), top_ids=torch.zeros(10, 3, dtype=torch.int64), top_loss=z(10, 3),
             ws=torch.zeros(1 << 20, dtype=torch.uint8))
    a.update(over)
    return a


def _tensors_f8(**over):
    f = lambda *s: torch.zeros(*s, dtype=torch.uint8).view(torch.float8_e4m3fn)  # noqa: E731
    k = lambda *s: torch.zeros(*s, dtype=torch.uint8).view(torch.float8_e8m0fnu)  # noqa: E731
    a = _tensors()
    a = dict(H=f(10, 64), H_scale=k(10, 1), W_shards=[f(30, 64), f(50, 64)], W_scales=[k(1, 1), k(1, 1)],
             **{n: a[n] for n in list(a)[2:]})
    a.update(over)
    return a


@pytest.mark.parametrize("over, message", [
    (dict(H=torch.zeros(10, 64)), "H: dtype"), (dict(W_shards=[torch.zeros(30, 64, dtype=torch.bfloat16)]), "1 shards"),
    (dict(W_shards=[torch.zeros(r, 64, dtype=torch.bfloat16) for r in (30, 49)]), r"W_shards\[1\]: shape"),
    (dict(targets=torch.zeros(10)), "targets: dtype"), (dict(entropy=torch.zeros(9)), "entropy: shape"),
    (dict(top_ids=None), "top_ids"), (dict(top_ids=torch.zeros(10, 3, dtype=torch.int32)), "top_ids: dtype"),
    (dict(top_loss=torch.zeros(3, 10).t()), "top_loss: must be contiguous"), (dict(ws=None), "ws"),
    (dict(ws=torch.zeros(8, dtype=torch.uint8)), "ws: 8 bytes"), ({}, "must be on a GPU device")])
def test_binding_refuses_score_tensors(over, message):
    with pytest.raises(ValueError, match=message):
        vp.vp_score_forward(_problem(), vp.Score(3), **_tensors(**over))


@pytest.mark.parametrize("over, message", [
    (dict(H=torch.zeros(10, 64, dtype=torch.uint8)), "H: dtype"),
    (dict(H_scale=torch.zeros(10, 1, dtype=torch.uint8)), "H_scale: dtype"),
    (dict(W_scales=[torch.zeros(1, 1, dtype=torch.uint8).view(torch.float8_e8m0fnu)]), "W_scales: 1 shards"),
    ({}, "must be on a GPU device")])
def test_binding_refuses_f8_tensors(over, message):
    with pytest.raises(ValueError, match=message):
        vp.vp_score_forward_f8(_problem(dtype=vp.VP_E4M3), vp.Score(3), **_tensors_f8(**over))


def test_binding_refuses_the_rest():
    t = _tensors()
    z, x = torch.zeros, torch.zeros(10, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="grad_entropy: shape"):
        vp.vp_score_backward(_problem(), t["H"], t["W_shards"], t["targets"], z(10), z(10), z(10), z(11), z(10, 64),
                             [z(30, 64), z(50, 64)], torch.zeros(1 << 28, dtype=torch.uint8))
    with pytest.raises(ValueError, match="X8: dtype"):
        vp.vp_f8_quantize(vp.Quant(10, 64, vp.VP_BF16), x, z(10, 64), z(10, 1))
    with pytest.raises(ValueError, match="rows_per_scale"):
        vp.quantize(x, 64)
    norm, s = vp.Norm(10, 64, vp.VP_BF16), z(10)
    gamma = torch.ones(64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="R: shape"):
        vp.vp_add_norm_forward(norm, x, x[:9], gamma, None, x, x, None, None, s, s)
    with pytest.raises(ValueError, match="scale: dtype"):
        vp.vp_add_norm_forward(norm, x, x, gamma, None, x, x, x.to(torch.float8_e4m3fn), z(10, 1), s, s)
    with pytest.raises(ValueError, match="dS: dtype"):
        vp.vp_add_norm_backward(norm, x, gamma, s, s, z(10, 64), x, z(10, 64), z(64), None, torch.zeros(1 << 20, dtype=torch.uint8))
    with pytest.raises(ValueError, match="entropy and grad_entropy"):
        vp.backward(x, t["W_shards"], t["targets"], s, s, grad_entropy=s)


# ---------------------------------------------------------------------------
def _status(case):
    lib, op = _lib(), case["op"]
    code = {"bf16": vp.VP_BF16, "f32": vp.VP_F32, "f8": vp.VP_E4M3}[case["dtype"]]
    if op == "quantize":
        return _quantize(vp.Quant(case["rows"], case["cols"], code, case["rps"]), X=None), vp.VP_ERR_NULL
    if op == "add_norm":
        return _add_fwd(vp.Norm(case["T"], case["d"], code, rms=case["rms"]), X=None), vp.VP_ERR_NULL
    if op == "add_norm_backward":
        return _add_bwd(vp.Norm(case["T"], case["d"], code, rms=case["rms"]), ws=None), vp.VP_ERR_WORKSPACE
    prob = vp.Problem(case["T"], case["d"], more_operators._rows(case), code)
    if op == "train" and _backward(prob, ws=None) != vp.VP_ERR_WORKSPACE:
        return "backward", None
    call = _forward_f8 if op == "score_f8" else _forward
    assert lib.vp_score_workspace_size(ctypes.byref(prob.c), vp.Score(case["top"]).ref, None) == vp.VP_OK
    return call(prob, vp.Score(case["top"]), ws=None), vp.VP_ERR_WORKSPACE


def test_listed_and_drawn_cases_pass_the_checks():
    rng = random.Random(7)
    for case in more_operators.listed() + [more_operators.draw(rng) for _ in range(3000)]:
        got, want = _status(case)
        assert got == want, case


# ---------------------------------------------------------------------------
def test_plain_residual_against_differences():
    g = torch.Generator().manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    H, W, t = r(7, 6), r(11, 6), torch.tensor([3, -100, 0, 10, 5, 5, -100])
    gl, ge = r(7), r(7)

    def total(H, W):
        loss, _, entropy, _, _, _ = sp.score(H, W, t, -100)
        return float((gl * loss + ge * entropy).sum())

    G = sp.residual(H, W, t, -100, gl, ge)
    for at, grad in ((H, G @ W), (W, G.t() @ H)):
        for i in range(at.numel()):
            e = torch.zeros_like(at)
            e.view(-1)[i] = 1e-6
            up = total(*(v + e if v is at else v for v in (H, W)))
            dn = total(*(v - e if v is at else v for v in (H, W)))
            assert abs((up - dn) / 2e-6 - grad.reshape(-1)[i].item()) <= 1e-7


def test_plain_quantisation():
    x = torch.tensor([[448.0, 0.0, -1.0, 17.0], [449.0, 3.0, -1.0, 17.0]])
    v, e = sp.quantize(x, 1)
    assert e.tolist() == [[0.0], [1.0]]
    assert v.tolist() == [[448.0, 0.0, -1.0, 16.0], [224.0, 1.5, -0.5, 8.0]]  # (17 and 8.5: ties to even)
