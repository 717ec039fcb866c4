"""Host-side tests of the operators around the projection (no GPU): every refusal of the C
entries is returned before any HIP call, the binding checks each tensor, and empty calls do
nothing."""
import ctypes
import math
import os

import pytest
import torch

import paper_2609_14306_amd as vp

pytestmark = pytest.mark.skipif(not os.path.exists(vp.LIB_PATH),
                                reason="libvpce.so not built (run __graft_entry__.build())")

FAKE = 0x100000  # an aligned pointer value that no call here dereferences


def _lib():
    return vp.load_library()


def _norm_fwd(norm=None, **over):
    norm = norm or vp.Norm(4, 64, vp.VP_BF16)
    a = dict(X=FAKE, gamma=FAKE, beta=FAKE, Y=FAKE, mean=FAKE, rstd=FAKE)
    a.update(over)
    return _lib().vp_norm_forward(norm.ref, *a.values(), None)


def _norm_bwd(norm=None, ws=FAKE, ws_bytes=1 << 40, **over):
    norm = norm or vp.Norm(4, 64, vp.VP_BF16)
    a = dict(X=FAKE, gamma=FAKE, mean=FAKE, rstd=FAKE, dY=FAKE, dX=FAKE, dgamma=FAKE, dbeta=FAKE)
    a.update(over)
    return _lib().vp_norm_backward(norm.ref, *a.values(), ws, ws_bytes, None)


def _pref_fwd(seq=None, pref=None, ws=FAKE, ws_bytes=1 << 40, **over):
    seq, pref = seq or vp.Sequences(10, 4), pref or vp.Preference()
    a = dict(start=FAKE, targets=FAKE, loss=FAKE, ref=FAKE, pair_loss=FAKE, reward=FAKE, coef=FAKE)
    a.update(over)
    return _lib().vp_pref_forward(seq.ref, pref.ref, *a.values(), ws, ws_bytes, None)


def _pref_bwd(seq=None, **over):
    seq = seq or vp.Sequences(10, 4)
    a = dict(start=FAKE, targets=FAKE, coef=FAKE, grad_pair=FAKE, grad_loss=FAKE)
    a.update(over)
    return _lib().vp_pref_backward(seq.ref, *a.values(), None)


def _pol_fwd(seq=None, pol=None, ws=FAKE, ws_bytes=1 << 40, **over):
    seq, pol = seq or vp.Sequences(10, 3), pol or vp.Policy()
    a = dict(start=FAKE, targets=FAKE, loss=FAKE, old=FAKE, ref=FAKE, adv=FAKE, seq_loss=FAKE, seq_kl=FAKE,
             clipped=FAKE, tokens=FAKE)
    a.update(over)
    return _lib().vp_policy_forward(seq.ref, pol.ref, *a.values(), ws, ws_bytes, None)


def _pol_bwd(seq=None, pol=None, **over):
    seq, pol = seq or vp.Sequences(10, 3, mean=True), pol or vp.Policy()
    a = dict(start=FAKE, targets=FAKE, loss=FAKE, old=FAKE, ref=FAKE, adv=FAKE, tokens=FAKE, grad_seq=FAKE,
             grad_loss=FAKE)
    a.update(over)
    return _lib().vp_policy_backward(seq.ref, pol.ref, *a.values(), None)


BAD_NORMS = [
    (dict(T=-1), vp.VP_ERR_SHAPE), (dict(T=2 ** 23 - 255), vp.VP_ERR_SHAPE), (dict(d=0), vp.VP_ERR_SHAPE),
    (dict(d=4), vp.VP_ERR_SHAPE), (dict(d=60), vp.VP_ERR_SHAPE), (dict(d=16392), vp.VP_ERR_SHAPE),
    (dict(dtype=2), vp.VP_ERR_DTYPE), (dict(eps=-1e-6), vp.VP_ERR_VALUE), (dict(eps=math.nan), vp.VP_ERR_VALUE),
    (dict(eps=math.inf), vp.VP_ERR_VALUE),
]


@pytest.mark.parametrize("over, want", BAD_NORMS)
def test_norm_problem_refused(over, want):
    kw = dict(T=4, d=64, dtype=vp.VP_BF16)
    kw.update(over)
    norm = vp.Norm(**kw)
    assert _norm_fwd(norm) == want
    assert _norm_bwd(norm) == want
    assert _lib().vp_norm_workspace_size(norm.ref, None) == want


@pytest.mark.parametrize("call, names", [
    (_norm_fwd, ("X", "gamma", "Y", "mean", "rstd")),
    (_norm_bwd, ("X", "gamma", "mean", "rstd", "dY", "dX", "dgamma")),
    (_pref_fwd, ("start", "targets", "loss", "pair_loss", "reward", "coef")),
    (_pref_bwd, ("start", "targets", "coef", "grad_pair", "grad_loss")),
    (_pol_fwd, ("start", "targets", "loss", "adv", "seq_loss", "seq_kl", "clipped", "tokens")),
    (_pol_bwd, ("start", "targets", "loss", "adv", "tokens", "grad_seq", "grad_loss")),
])
def test_null_pointers_refused(call, names):
    for name in names:
        assert call(**{name: None}) == vp.VP_ERR_NULL, name


@pytest.mark.parametrize("call, names", [
    (_norm_fwd, {"X": 8, "gamma": 8, "beta": 8, "Y": 8, "mean": 2, "rstd": 2}),
    (_norm_bwd, {"X": 8, "gamma": 8, "mean": 2, "rstd": 2, "dY": 8, "dX": 8, "dgamma": 8, "dbeta": 8, "ws": 8}),
    (_pref_fwd, {"start": 2, "targets": 4, "loss": 2, "ref": 2, "pair_loss": 2, "reward": 2, "coef": 2, "ws": 8}),
    (_pref_bwd, {"start": 2, "targets": 4, "coef": 2, "grad_pair": 2, "grad_loss": 2}),
    (_pol_fwd, {"start": 2, "targets": 4, "loss": 2, "old": 2, "ref": 2, "adv": 2, "seq_loss": 2, "seq_kl": 2,
                "clipped": 2, "tokens": 2, "ws": 8}),
    (_pol_bwd, {"start": 2, "targets": 4, "loss": 2, "old": 2, "ref": 2, "adv": 2, "tokens": 2, "grad_seq": 2,
                "grad_loss": 2}),
])
def test_misaligned_pointers_refused(call, names):
    for name, by in names.items():
        assert call(**{name: FAKE + by}) == vp.VP_ERR_ALIGN, name


@pytest.mark.parametrize("call", [_norm_bwd, _pref_fwd, _pol_fwd])
def test_workspace_refused(call):
    assert call(ws=None) == vp.VP_ERR_WORKSPACE
    size = ctypes.c_size_t(0)
    if call is _norm_bwd:
        assert _lib().vp_norm_workspace_size(vp.Norm(4, 64, vp.VP_BF16).ref, ctypes.byref(size)) == vp.VP_OK
    else:
        S = 4 if call is _pref_fwd else 3
        assert _lib().vp_seq_workspace_size(vp.Sequences(10, S).ref, ctypes.byref(size)) == vp.VP_OK
    assert size.value > 0 and call(ws_bytes=size.value - 1) == vp.VP_ERR_WORKSPACE


@pytest.mark.parametrize("over", [dict(T=-1), dict(T=2 ** 23 - 255), dict(S=-2), dict(S=2 ** 22 + 2)])
def test_sequences_refused(over):
    kw = dict(T=10, S=4)
    kw.update(over)
    seq = vp.Sequences(**kw)
    for call in (_pref_fwd, _pref_bwd, _pol_fwd, _pol_bwd):
        assert call(seq) == vp.VP_ERR_SHAPE, call
    assert _lib().vp_seq_workspace_size(seq.ref, None) == vp.VP_ERR_SHAPE


def test_odd_number_of_preference_sequences_refused():
    assert _pref_fwd(vp.Sequences(10, 3)) == vp.VP_ERR_SHAPE
    assert _pref_bwd(vp.Sequences(10, 3)) == vp.VP_ERR_SHAPE


@pytest.mark.parametrize("over", [
    dict(beta=0.0), dict(beta=-1.0), dict(beta=math.nan), dict(beta=math.inf), dict(margin=math.inf),
    dict(margin=math.nan), dict(smoothing=-0.1), dict(smoothing=0.6), dict(smoothing=math.nan),
    dict(kind="squared", smoothing=0.1),
])
def test_preference_values_refused(over):
    assert _pref_fwd(pref=vp.Preference(**over)) == vp.VP_ERR_VALUE
    bad = vp.Preference()
    bad.c.kind = 2
    assert _pref_fwd(pref=bad) == vp.VP_ERR_VALUE


def test_preference_kind_name_refused():
    with pytest.raises(ValueError, match="kind"):
        vp.Preference("hinge")


@pytest.mark.parametrize("over", [
    dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_low=math.nan), dict(clip_high=-0.1), dict(clip_high=math.nan),
    dict(kl_coef=-0.1), dict(kl_coef=math.inf), dict(kl_coef=math.nan),
])
def test_policy_values_refused(over):
    pol = vp.Policy(**over)
    assert _pol_fwd(pol=pol) == vp.VP_ERR_VALUE
    assert _pol_bwd(pol=pol) == vp.VP_ERR_VALUE


def test_null_problems_refused():
    n = [None] * 16
    assert _lib().vp_norm_forward(None, *n[:7]) == vp.VP_ERR_NULL
    assert _lib().vp_norm_backward(None, *n[:9], 0, None) == vp.VP_ERR_NULL
    assert _lib().vp_pref_forward(None, None, *n[:8], 0, None) == vp.VP_ERR_NULL
    assert _lib().vp_pref_backward(None, *n[:6]) == vp.VP_ERR_NULL
    assert _lib().vp_policy_forward(None, None, *n[:11], 0, None) == vp.VP_ERR_NULL
    assert _lib().vp_policy_backward(None, None, *n[:10]) == vp.VP_ERR_NULL
    seq = vp.Sequences(10, 4)
    assert _pref_fwd(pref=type("P", (), {"ref": None})) == vp.VP_ERR_NULL
    assert _lib().vp_policy_backward(seq.ref, None, *n[:10]) == vp.VP_ERR_NULL


def test_calls_without_work_need_no_arrays():
    empty = vp.Sequences(0, 0)
    assert _norm_fwd(vp.Norm(0, 64, vp.VP_F32), X=None, gamma=None, Y=None, mean=None, rstd=None) == vp.VP_OK
    assert _pref_fwd(empty, start=None, targets=None, loss=None, pair_loss=None, reward=None, coef=None) == vp.VP_OK
    assert _pref_bwd(empty, start=None, targets=None, coef=None, grad_pair=None, grad_loss=None) == vp.VP_OK
    assert _pol_fwd(empty, start=None, targets=None, loss=None, adv=None, seq_loss=None, seq_kl=None, clipped=None,
                    tokens=None) == vp.VP_OK
    assert _pol_bwd(empty, start=None, targets=None, loss=None, adv=None, tokens=None, grad_seq=None,
                    grad_loss=None) == vp.VP_OK


def test_value_status_has_a_text():
    assert vp.vp_status_str(vp.VP_ERR_VALUE) == "a parameter is outside its range"


# ---------------------------------------------------------------------------
T, D, S = 6, 16, 4


def _norm_tensors(**over):
    x = torch.zeros(T, D, dtype=torch.bfloat16)
    a = dict(norm=vp.Norm(T, D, vp.VP_BF16), X=x, gamma=x[0].clone(), beta=x[0].clone(), Y=x.clone(),
             mean=torch.zeros(T), rstd=torch.zeros(T))
    a.update(over)
    return a


def _norm_grad_tensors(**over):
    x = torch.zeros(T, D, dtype=torch.bfloat16)
    a = dict(norm=vp.Norm(T, D, vp.VP_BF16), X=x, gamma=x[0].clone(), mean=torch.zeros(T), rstd=torch.zeros(T),
             dY=torch.zeros(T, D), dX=torch.zeros(T, D), dgamma=torch.zeros(D), dbeta=torch.zeros(D),
             ws=torch.zeros(1 << 20, dtype=torch.uint8))
    a.update(over)
    return a


def _pref_tensors(**over):
    a = dict(seq=vp.Sequences(T, S), pref=vp.Preference(), start=torch.zeros(S + 1, dtype=torch.int32),
             targets=torch.zeros(T, dtype=torch.int64), loss=torch.zeros(T), ref_loss=torch.zeros(T),
             pair_loss=torch.zeros(S // 2), reward=torch.zeros(S), coef=torch.zeros(S),
             ws=torch.zeros(1 << 20, dtype=torch.uint8))
    a.update(over)
    return a


def _policy_tensors(**over):
    a = dict(seq=vp.Sequences(T, S), policy=vp.Policy(), start=torch.zeros(S + 1, dtype=torch.int32),
             targets=torch.zeros(T, dtype=torch.int64), loss=torch.zeros(T), old_loss=torch.zeros(T),
             ref_loss=torch.zeros(T), advantage=torch.zeros(S), seq_loss=torch.zeros(S), seq_kl=torch.zeros(S),
             clipped=torch.zeros(S, dtype=torch.int32), tokens=torch.zeros(S, dtype=torch.int32),
             ws=torch.zeros(1 << 20, dtype=torch.uint8))
    a.update(over)
    return a


@pytest.mark.parametrize("fn, make, over, match", [
    (vp.vp_norm_forward, _norm_tensors, dict(X=torch.zeros(T, D)), "X: dtype"),
    (vp.vp_norm_forward, _norm_tensors, dict(X=None), "X: expected"),
    (vp.vp_norm_forward, _norm_tensors, dict(Y=torch.zeros(D, T, dtype=torch.bfloat16).t()), "Y: must be contiguous"),
    (vp.vp_norm_forward, _norm_tensors, dict(beta=torch.zeros(D)), "beta: dtype"),
    (vp.vp_norm_forward, _norm_tensors, dict(gamma=torch.zeros(D + 8, dtype=torch.bfloat16)), "gamma: shape"),
    (vp.vp_norm_forward, _norm_tensors, dict(mean=None), "mean: expected"),
    (vp.vp_norm_forward, _norm_tensors, dict(), "on a GPU device"),
    (vp.vp_norm_backward, _norm_grad_tensors, dict(dY=torch.zeros(T, D, dtype=torch.bfloat16)), "dY: dtype"),
    (vp.vp_norm_backward, _norm_grad_tensors, dict(dgamma=torch.zeros(D + 1)), "dgamma: shape"),
    (vp.vp_norm_backward, _norm_grad_tensors, dict(ws=None), "ws: expected"),
    (vp.vp_norm_backward, _norm_grad_tensors, dict(ws=torch.zeros(8, dtype=torch.uint8)), "ws: 8 bytes"),
    (vp.vp_norm_backward, _norm_grad_tensors, dict(), "on a GPU device"),
    (vp.vp_pref_forward, _pref_tensors, dict(start=torch.zeros(S + 1, dtype=torch.int64)), "start: dtype"),
    (vp.vp_pref_forward, _pref_tensors, dict(start=torch.zeros(S, dtype=torch.int32)), "start: shape"),
    (vp.vp_pref_forward, _pref_tensors, dict(targets=torch.zeros(T, dtype=torch.int32)), "targets: dtype"),
    (vp.vp_pref_forward, _pref_tensors, dict(loss=torch.zeros(2 * T)[::2]), "loss: must be contiguous"),
    (vp.vp_pref_forward, _pref_tensors, dict(ref_loss=torch.zeros(T + 1)), "ref_loss: shape"),
    (vp.vp_pref_forward, _pref_tensors, dict(pair_loss=torch.zeros(S)), "pair_loss: shape"),
    (vp.vp_pref_forward, _pref_tensors, dict(), "on a GPU device"),
    (vp.vp_policy_forward, _policy_tensors, dict(advantage=torch.zeros(T)), "advantage: shape"),
    (vp.vp_policy_forward, _policy_tensors, dict(policy=vp.Policy(per_token=True)), "advantage: shape"),
    (vp.vp_policy_forward, _policy_tensors, dict(clipped=torch.zeros(S)), "clipped: dtype"),
    (vp.vp_policy_forward, _policy_tensors, dict(old_loss=torch.zeros(T, dtype=torch.float64)), "old_loss: dtype"),
    (vp.vp_policy_forward, _policy_tensors, dict(), "on a GPU device"),
])
def test_tensors_refused(fn, make, over, match):
    with pytest.raises(ValueError, match=match):
        fn(**make(**over))


def test_accumulating_helper_needs_buffers():
    x = torch.zeros(T, D)
    with pytest.raises(ValueError, match="accumulate"):
        vp.layer_norm_backward(x, x[0], None, torch.zeros(T), x, accumulate=True)


def test_plain_gradients_against_differences():
    """The formulas that the GPU tests compare with: gradients against differences."""
    import head_plain as hp

    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.rand(*s, generator=g, dtype=torch.float64)  # noqa: E731
    n, start = 13, [0, 4, 4, 9, 12]
    targets = torch.randint(0, 50, (n,), generator=g)
    targets[[1, 6, 10]] = -100
    loss, ref, old = 3 * r(n), 3 * r(n), None
    old = loss + 0.4 * (r(n) - 0.5)
    h = 1e-5
    for kind, smoothing in (("logistic", 0.0), ("logistic", 0.2), ("squared", 0.0)):
        for mean in (False, True):
            args = (kind, 0.7, 0.1, smoothing, ref, -100, mean)
            grad = hp.pref_backward(loss, targets, start, *args, [0.5, -1.5])
            for t in range(n):
                up, down = loss.clone(), loss.clone()
                up[t] += h
                down[t] -= h
                diff = hp.pref_forward(up, targets, start, *args)[0] - hp.pref_forward(down, targets, start, *args)[0]
                assert abs(float(diff[0]) * 0.5 - float(diff[1]) * 1.5 - 2 * h * float(grad[t])) <= 1e-8 * h
    adv = r(4) * 2 - 1
    gs = r(4)
    for mean in (False, True):
        f = lambda v: hp.policy(v, targets, start, adv, old, ref, -100, mean, 0.1, 0.15, 0.3, gs)  # noqa: E731
        grad = f(loss)[1]
        for t in range(n):
            up, down = loss.clone(), loss.clone()
            up[t] += h
            down[t] -= h
            diff = ((f(up)[0][0] - f(down)[0][0]) * gs).sum()
            assert abs(float(diff) - 2 * h * float(grad[t])) <= 1e-8 * h
    X, gamma, dY = r(3, 8) * 4, 1 + r(8), r(3, 8) - 0.5
    for rms in (False, True):
        _, mean, rstd = hp.norm_forward(X, gamma, None, 1e-3, rms)
        dx, dg, _ = hp.norm_backward(X, gamma, None if rms else mean, rstd, dY)
        for k in range(24):
            e = torch.zeros(24, dtype=torch.float64)
            e[k] = h
            e = e.view(3, 8)
            diff = hp.norm_forward(X + e, gamma, None, 1e-3, rms)[0] - hp.norm_forward(X - e, gamma, None, 1e-3, rms)[0]
            assert abs(float((diff * dY).sum()) - 2 * h * float(dx.view(-1)[k])) <= 1e-8 * h
        for j in range(8):
            e = torch.zeros(8, dtype=torch.float64)
            e[j] = h
            diff = hp.norm_forward(X, gamma + e, None, 1e-3, rms)[0] - hp.norm_forward(X, gamma - e, None, 1e-3, rms)[0]
            assert abs(float((diff * dY).sum()) - 2 * h * float(dg[j])) <= 1e-8 * h


# ---------------------------------------------------------------------------
# How the kernels find the sequences of their tokens, in Python: 64 offsets at a time, whatever
# they are.  Reads outside start[0..S] and sequences outside -1..S raise.
class _Offsets:
    BEHIND = 2 ** 31 - 1

    def __init__(self, start):
        self.start, self.S = start, len(start) - 1

    def at(self, i):
        assert 0 <= i <= self.S
        return self.start[i]

    def window(self, base):
        assert base >= 0
        return [self.at(base + k) if base + k <= self.S and self.S > 0 else self.BEHIND for k in range(64)]

    def open(self, t):
        lo, n, rounds = 0, self.S + 1, 0
        while n > 64:
            step = (n + 63) // 64
            c = sum(lo + (k + 1) * step - 1 < lo + n and self.at(min(lo + (k + 1) * step - 1, self.S)) <= t
                    for k in range(64))
            lo, n, rounds = lo + c * step, min(step - 1, n - c * step), rounds + 1
            assert n >= 0 and rounds <= 4
        return lo, lo - 1 + sum(o <= t for o in self.window(lo))

    def walk(self, base, first, last):
        s, rounds = [base - 1] * (last - first + 1), 0
        while True:
            o = self.window(base)
            s = [v + sum(x <= first for x in o) + sum(first < x <= last and x <= first + k for x in o)
                 for k, v in enumerate(s)]
            if o[63] > last:
                return base, s
            base, rounds = base + 64, rounds + 1
            assert rounds <= self.S // 64 + 1


def _ordered(g, S, T):
    return sorted(int(v) for v in torch.randint(0, T + 1, (S + 1,), generator=g))


def _disordered(g, S, T):
    out = _ordered(g, S, T)
    for i in torch.randint(0, S + 1, (max(1, S // 3),), generator=g).tolist():
        out[i] = [-5, T + 9, 2 ** 31 - 1, -2 ** 31, 0, T // 2][int(torch.randint(0, 6, (1,), generator=g))]
    return out


@pytest.mark.parametrize("S", [0, 1, 2, 63, 64, 65, 200, 4096, 5000])
@pytest.mark.parametrize("make", [_ordered, _disordered])
def test_walk_over_offsets(S, make):
    T = 700
    for seed in range(3):
        start = make(torch.Generator().manual_seed(100 * S + seed), S, T)
        off = _Offsets(start)
        for chunk in (64, 128):
            slots = set()
            for c in range(-(-T // chunk)):
                t0, t1 = c * chunk, min(T, (c + 1) * chunk)
                base, s = off.open(t0)
                assert -1 <= s <= S
                seen = []
                for b in range(t0, t1, 64):
                    base, mine = off.walk(base, b, min(b + 64, t1) - 1)
                    assert all(-1 <= v <= S for v in mine)
                    seen += mine
                if make is _ordered and S > 0:
                    want = torch.searchsorted(torch.tensor(start), torch.arange(t0, t1), right=True) - 1
                    assert seen == want.tolist() and s == seen[0]
                    parts = {c + v for v in set(seen) if 0 <= v < S}
                    assert len(parts) == len({v for v in set(seen) if 0 <= v < S}) and not parts & slots
                    slots |= parts
            assert all(0 <= v < -(-T // chunk) + S for v in slots)


@pytest.mark.parametrize("T, S", [(0, 0), (1, 2), (700, 0), (2048, 40), (2049, 40), (2 ** 20, 8), (2 ** 23 - 256, 2 ** 22)])
def test_sequence_workspace_holds_every_part(T, S):
    """Three sums for each chunk of tokens and each sequence."""
    most = 16 if T <= 2048 else 16384
    chunk = 64 * max(1, -(-T // (64 * most)))
    assert vp.vp_seq_workspace_size(vp.Sequences(T, S)) >= 24 * (-(-T // chunk) + S)
