"""The preference loss and the clipped policy loss on the GPU against the plain float64 forms.

The kernels compute in float64 between float32 inputs and outputs, so an output is off by its own
rounding, 2^-24 relative, and by what float64 sums of differently ordered terms leave: 2^-40 of the
sum of the terms' magnitudes covers 2^13 roundings of 2^-53 each.  A gradient of the preference
loss is the product of two float32 values, one of them rounded: two roundings.
"""
import math

import pytest
import torch

import head_plain as hp
import paper_2609_14306_amd as vp

pytestmark = pytest.mark.gpu
U = hp.U
IGNORE = -100


def _offsets(lens, before=0):
    out = [before]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _make(lens, before=0, behind=0, seed=0, ignore=IGNORE, masked=0.3, junk=True):
    """Packed sequences with masked tokens (NaN, infinities and large values in their places)."""
    g = torch.Generator().manual_seed(seed + 31 * len(lens) + sum(lens))
    start = _offsets(lens, before)
    T = start[-1] + behind
    r = lambda: torch.rand(T, generator=g)  # noqa: E731
    targets = torch.randint(0, 1000, (T,), generator=g)
    mask = r() < masked
    mask[:before] = torch.rand(before, generator=g) < 0.5
    targets[mask] = ignore
    loss = 5 * r() ** 3
    old, ref = (loss + 0.3 * (r() - 0.5)).clamp_min(0), (loss + 0.4 * (r() - 0.5)).clamp_min(0)
    outside = torch.ones(T, dtype=torch.bool)
    outside[start[0]:start[-1]] = False
    if junk:
        for v in (loss, old, ref):
            pick = torch.randint(0, 4, (T,), generator=g)
            bad = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38])[pick]
            v[mask | outside] = bad[mask | outside]
    adv = torch.randn(T, generator=g)
    return {"T": T, "S": len(lens), "start": torch.tensor(start, dtype=torch.int32, device="cuda"),
            "targets": targets.cuda(), "loss": loss.cuda(), "old": old.cuda(), "ref": ref.cuda(),
            "adv_t": adv.cuda(), "adv_s": adv[:len(lens)].clone().cuda() if T >= len(lens) else
            torch.randn(len(lens), generator=g).cuda(), "mask": mask | outside, "ignore": ignore}


def _spread(n, total, seed):
    g = torch.Generator().manual_seed(seed)
    w = torch.exp(1.5 * torch.randn(n, generator=g))
    cut = (torch.cumsum(w, 0) / w.sum() * total).long().tolist()
    cut[-1] = total
    return [b - a for a, b in zip([0] + cut[:-1], cut)]


LAYOUTS = {
    "one token each": ([1, 1], 0, 0),
    "empty ones": ([0, 3, 0, 0, 1, 0], 0, 0),
    "all empty": ([0, 0], 0, 0),
    "all empty, tokens around": ([0, 0], 5, 9),
    "padding around": ([17, 250, 3, 64], 11, 300),
    "whole blocks": ([256, 512, 256, 1024], 0, 0),
    "one off whole blocks": ([255, 257, 1023, 1025], 0, 1),
    "single tokens": ([1] * 1200, 0, 3),
    "tens of tokens": (_spread(150, 4000, 1), 0, 17),
    "one workgroup": (_spread(8, 2048, 2), 0, 0),
    "just above": (_spread(8, 2049, 2), 0, 0),
    "4096 tokens": (_spread(8, 4096, 2), 0, 0),
    "4097 tokens": (_spread(8, 4097, 2), 0, 0),
    "a long one among short ones": ([3, 5, 150000, 1, 0, 40, 70001, 2], 2, 5),
    "many of a wide spread": (_spread(3000, 400000, 3), 0, 1000),
    "empty ones inside": ([5] + [0] * 700 + [900] + [0] * 3001 + [1, 2, 0], 0, 0),
    "two of a million": ([1000003, 999001], 0, 70),
}


def _close(got, want, slack, what):
    got, want = got.double().cpu(), want.double()
    assert got.shape == want.shape, what
    err = (got - want).abs()
    bound = U * want.abs() + slack + 1e-45
    assert bool((err <= bound).all()), (what, float((err - bound).max()), int((err - bound).argmax()))


def _magnitudes(values, m):
    """Per sequence: c_s sum |values| over the counting tokens."""
    out, t = [], m["targets"].cpu()
    for a, b in hp.spans(m["start"].cpu(), m["T"]):
        out.append(float(values[a:b][t[a:b] != m["ignore"]].abs().sum()))
    return torch.tensor(out, dtype=torch.float64)


@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("kind, ref, smoothing, margin", [("logistic", True, 0.0, 0.0), ("logistic", False, 0.1, 0.4),
                                                          ("squared", True, 0.0, 0.0)])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_preference(layout, kind, ref, smoothing, margin, mean):
    m = _make(*LAYOUTS[layout])
    beta = 1.5 if mean else 0.01
    pref = vp.Preference(kind, beta, margin, smoothing)
    r = m["ref"] if ref else None
    got = vp.preference_forward(m["loss"], m["targets"], m["start"], pref, r, IGNORE, mean)
    plain = (kind, beta, margin, smoothing, r, IGNORE, mean)
    loss, reward, c = hp.pref_forward(m["loss"], m["targets"], m["start"].cpu(), *plain)
    ratio = -m["loss"].double().cpu() if r is None else r.double().cpu() - m["loss"].double().cpu()
    e_reward = 2.0 ** -40 * beta * torch.tensor(c, dtype=torch.float64) * _magnitudes(ratio, m)
    _close(got[1], reward, e_reward, "reward")
    # the loss moves by at most |dL/dz| for a z that is off by both rewards' errors
    e_z = e_reward[0::2] + e_reward[1::2] + 2.0 ** -50 * (reward[0::2].abs() + reward[1::2].abs())
    steep = 1.0 if kind == "logistic" else 2 * loss.sqrt() / beta
    curve = 1.0 if kind == "logistic" else 2 / beta ** 2
    _close(got[0], loss, 1.01 * steep * e_z + 2.0 ** -48, "pair_loss")
    g = torch.linspace(-1, 2, m["S"] // 2)
    grad = vp.preference_backward(m["targets"], m["start"], got[2], g.cuda(), IGNORE)
    want = hp.pref_backward(m["loss"], m["targets"], m["start"].cpu(), *plain, g.tolist())
    e_grad = torch.zeros(m["T"], dtype=torch.float64)
    for s, (a, b) in enumerate(hp.spans(m["start"].cpu(), m["T"])):
        e_grad[a:b] = beta * c[s] * abs(float(g[s // 2])) * (1.01 * curve * float(e_z[s // 2]) + 2.0 ** -48)
    _close(grad, want, e_grad + U * 1.01 * want.abs(), "grad_loss")
    assert bool((grad.cpu()[m["mask"]] == 0).all())


def _policy_args(m, old, ref, per_token, mean):
    adv = m["adv_t"] if per_token else m["adv_s"]
    return adv, m["old"] if old else None, m["ref"] if ref else None


@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("old, ref, per_token, kl_coef", [(True, True, False, 0.1), (True, False, True, 0.0),
                                                          (False, True, True, 0.3), (True, True, True, 0.0)])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_policy(layout, old, ref, per_token, kl_coef, mean):
    m = _make(*LAYOUTS[layout])
    adv, o, r = _policy_args(m, old, ref, per_token, mean)
    pol = vp.Policy(0.08, 0.1, kl_coef, per_token)
    got = vp.policy_forward(m["loss"], m["targets"], m["start"], pol, adv, o, r, IGNORE, mean)
    g = torch.linspace(-1, 2, m["S"])
    want, grad = hp.policy(m["loss"], m["targets"], m["start"].cpu(), adv, o, r, IGNORE, mean, 0.08, 0.1, kl_coef, g,
                           per_token)
    n = want[3].double().clamp_min(1)
    c = 1 / n if mean else torch.ones_like(n)
    # |l_t| <= e^|x| |A| + kl_coef kl with |x|, |q| <= 0.2: below 2 |A| + 0.1, and kl below 0.1;
    # with no old loss and no clip the same
    A = (adv.double().cpu().abs() if per_token else adv.double().cpu().abs().repeat_interleave(
        torch.tensor([b - a for a, b in hp.spans(m["start"].cpu(), 0)])) if m["S"] else torch.zeros(0))
    if not per_token:
        A = torch.cat([torch.zeros(int(m["start"][0])), A, torch.zeros(m["T"] - int(m["start"][-1]))])
    mag = _magnitudes(2 * A + 0.1, m)
    _close(got[0], want[0], 2.0 ** -40 * c * mag, "seq_loss")
    _close(got[1], want[1], 2.0 ** -40 * c * mag, "seq_kl")
    assert torch.equal(got[2].cpu(), want[2]) and torch.equal(got[3].cpu(), want[3])
    back = vp.policy_backward(m["loss"], m["targets"], m["start"], pol, adv, got[3], g.cuda(), o, r, IGNORE, mean)
    _close(back, grad, 2.0 ** -45 * float(2 * adv.abs().max() + 1 if m["S"] and m["T"] else 1) * 2, "grad_loss")
    assert bool((back.cpu()[m["mask"]] == 0).all())


@pytest.mark.parametrize("S, T", [(35000, 200003), (40000, 1500), (2 ** 22, 70000), (8000, 2 ** 23 - 256)])
def test_many_sequences(S, T):
    """More sequences than wavefronts, and many more sequences than tokens; sums by sequence from
    the plain form of each token."""
    g = torch.Generator().manual_seed(S)
    start = torch.cat([torch.zeros(1, dtype=torch.int64), torch.randint(0, T + 1, (S - 1,), generator=g).sort().values,
                       torch.tensor([T])])
    loss, old, ref = [(3 * torch.rand(T, generator=g)) for _ in range(3)]
    targets = torch.where(torch.rand(T, generator=g) < 0.3, IGNORE, 5)
    adv, up = torch.randn(S, generator=g), torch.rand(S, generator=g)
    seq = torch.searchsorted(start, torch.arange(T), right=True) - 1
    keep = targets != IGNORE
    l, kl, clipped, slope = hp.policy_tokens(loss.double(), old.double(), ref.double(), adv.double()[seq], 0.2, 0.2, 0.1)

    def total(v):
        return torch.zeros(S, dtype=torch.float64).index_add_(0, seq[keep], v.double()[keep])

    dev = [v.cuda() for v in (loss, targets, start.int())]
    pol, more = vp.Policy(kl_coef=0.1), dict(old_loss=old.cuda(), ref_loss=ref.cuda())
    got = vp.policy_forward(*dev, pol, adv.cuda(), **more)
    # at most 2^15 tokens a sequence, each below e^3 |A| + 0.1 e^3
    _close(got[0], total(l), 2.0 ** -45 * total(21 * adv.double()[seq].abs() + 3), "seq_loss")
    _close(got[1], total(kl), 2.0 ** -45 * total(torch.full((T,), 21.0)), "seq_kl")
    assert torch.equal(got[2].cpu(), total(clipped).int()) and torch.equal(got[3].cpu(), total(keep).int())
    back = vp.policy_backward(*dev, pol, adv.cuda(), got[3], up.cuda(), **more)
    _close(back, torch.where(keep, up.double()[seq] * slope, 0.0), 2.0 ** -40, "policy grad_loss")
    pair, reward, coef = vp.preference_forward(*dev, vp.Preference("squared", 0.3), ref.cuda())
    R = 0.3 * total(ref.double() - loss.double())
    _close(reward, R, 2.0 ** -45 * 0.3 * total(torch.full((T,), 3.0)), "reward")
    z = R[0::2] - R[1::2]
    _close(pair, ((z - 0.5) / 0.3) ** 2, 2.0 ** -38 * (1 + z.abs()), "pair_loss")
    grad = vp.preference_backward(dev[1], dev[2], coef, up[:S // 2].cuda())
    sign = torch.where(seq % 2 == 0, -1.0, 1.0).double()  # (float32 would round 0.3 to 0.3 (1 + 4e-8))
    want = torch.where(keep, sign * 0.3 * (2 * (z - 0.5) / 0.09)[seq // 2] * up.double()[seq // 2], 0.0)
    _close(grad, want, 1.01 * U * want.abs() + 2.0 ** -36, "preference grad_loss")


def test_ratios_next_to_the_bounds():
    """Ratios one float32 step around each bound, and the bounds' neighbours in float64, fall on
    their side; a token without advantage has neither loss nor gradient."""
    hi, lo = math.log1p(0.2), math.log1p(-0.2)
    loss = torch.tensor([1.0, 2.0, 0.25, 0.5]).repeat_interleave(24)
    x = []
    for b in (hi, lo):
        f = torch.tensor(b, dtype=torch.float32)
        x += [float(f) + k * 2.0 ** -26 for k in range(-6, 6)]
    old = (loss.double() + torch.tensor(x, dtype=torch.float64).repeat(4)).float()
    T = loss.numel()
    for a in (1.0, -1.0, 0.0):
        adv = torch.full((T,), a)
        targets = torch.zeros(T, dtype=torch.int64)
        start = torch.arange(T + 1, dtype=torch.int32)
        pol = vp.Policy(0.2, 0.2, 0.0)
        dev = [v.cuda() for v in (loss, targets, start)]
        got = vp.policy_forward(*dev, pol, adv.cuda(), old.cuda())
        want, grad = hp.policy(loss, targets, start, adv, old, None, IGNORE, False, 0.2, 0.2, 0.0, torch.ones(T))
        assert torch.equal(got[2].cpu(), want[2])
        back = vp.policy_backward(*dev, pol, adv.cuda(), got[3], torch.ones(T, device="cuda"), old.cuda())
        _close(got[0], want[0], 2.0 ** -50, "seq_loss")
        _close(back, grad, 2.0 ** -50, "grad_loss")
    assert bool((got[0] == 0).all()) and bool((back == 0).all())


def test_extreme_tokens():
    """Infinite and very unlikely tokens: limits instead of NaN where the limit exists, and a NaN
    stays in its sequence."""
    inf, nan = float("inf"), float("nan")
    #         p -> 0, A>0  p -> 0, A<0  ratio e^200  the same, A<0  no A   ref p = 0  NaN    clean
    loss = [inf, inf, 0.0, 0.0, 0.0, 1.0, nan, 1.0]
    old = [1.0, 1.0, 200.0, 200.0, 200.0, 1.0, 1.0, 1.0]
    adv = [1.0, -1.0, 1.0, -1.0, 0.0, 0.0, 1.0, 2.0]
    ref = [1.0, 1.0, 0.0, 0.0, 0.0, inf, 1.0, 1.0]
    f = lambda v: torch.tensor(v, device="cuda")  # noqa: E731
    T = len(loss)
    start, targets = torch.arange(T + 1, dtype=torch.int32, device="cuda"), torch.zeros(T, dtype=torch.int64, device="cuda")
    pol = vp.Policy(0.2, 0.25, 0.0)
    out = vp.policy_forward(f(loss), targets, start, pol, f(adv), f(old))
    back = vp.policy_backward(f(loss), targets, start, pol, f(adv), out[3], torch.ones(T, device="cuda"), f(old))
    l, b = out[0].tolist(), back.tolist()
    assert l[0] == 0 and b[0] == 0
    assert abs(l[1] - 0.8) <= 2 ** -24 and b[1] == 0
    assert l[2] == -1.25 and b[2] == 0
    assert l[3] == inf and b[3] == -inf  # e^200 is beyond float32
    assert l[4] == 0 and b[4] == 0 and l[5] == 0 and b[5] == 0
    assert math.isnan(l[6]) and math.isnan(b[6])
    assert l[7] == -2 and b[7] == 2
    assert out[2].tolist() == [0, 1, 1, 0, 0, 0, 0, 0] and out[3].tolist() == [1] * T
    kl = vp.policy_forward(f(loss), targets, start, pol, f(adv), f(old), f(ref))[1].tolist()
    assert kl[0] == inf and kl[5] == inf and math.isnan(kl[6]) and kl[7] == 0 and kl[2] == 0
    no_old = vp.policy_forward(f(loss[5:]), targets[5:], start[:4], pol, f(adv[5:7] + [2.0]))[0].tolist()
    assert no_old[0] == 0 and math.isnan(no_old[1]) and no_old[2] == -2


def test_preference_extremes():
    """Saturated pairs, infinite log ratios, and a NaN token that stays in its pair."""
    inf, nan = float("inf"), float("nan")
    loss = torch.tensor([0.0, 3e4, 3e4, 0.0, inf, 1.0, 1.0, inf, nan, 1.0, 1.0, 1.0], device="cuda")
    start = torch.arange(13, dtype=torch.int32, device="cuda")
    targets = torch.zeros(12, dtype=torch.int64, device="cuda")
    pair, reward, coef = vp.preference_forward(loss, targets, start, vp.Preference(beta=1.0))
    grad = vp.preference_backward(targets, start, coef, torch.ones(6, device="cuda"))
    p, g = pair.tolist(), grad.tolist()
    assert p[0] == 0 and g[0] == g[1] == 0
    assert p[1] == 3e4 and g[2] == 1 and g[3] == -1
    assert p[2] == inf and g[4] == 1 and g[5] == -1
    assert p[3] == 0 and g[6] == g[7] == 0
    assert math.isnan(p[4]) and math.isnan(g[8]) and math.isnan(g[9])
    assert abs(p[5] - math.log(2)) <= 2 ** -24 and g[10] == 0.5 and g[11] == -0.5


@pytest.mark.parametrize("ignore", [0, 7, -1, -2 ** 40])
def test_other_ignore_index(ignore):
    m = _make([40, 0, 300, 21], 0, 3, ignore=ignore)
    got = vp.policy_forward(m["loss"], m["targets"], m["start"], vp.Policy(kl_coef=0.1), m["adv_s"], m["old"], m["ref"],
                            ignore, True)
    want, _ = hp.policy(m["loss"], m["targets"], m["start"].cpu(), m["adv_s"], m["old"], m["ref"], ignore, True, 0.2,
                        0.2, 0.1)
    assert torch.equal(got[3].cpu(), want[3])
    _close(got[0], want[0], 2.0 ** -45, "seq_loss")


def test_everything_masked():
    m = _make([30, 700, 5, 9], masked=1.1)
    for mean in (False, True):
        out = vp.policy_forward(m["loss"], m["targets"], m["start"], vp.Policy(kl_coef=0.1), m["adv_s"], m["old"],
                                m["ref"], IGNORE, mean)
        assert all(bool((v == 0).all()) for v in out)
        back = vp.policy_backward(m["loss"], m["targets"], m["start"], vp.Policy(kl_coef=0.1), m["adv_s"], out[3],
                                  torch.full((4,), float("nan"), device="cuda"), m["old"], m["ref"], IGNORE, mean)
        assert bool((back == 0).all())
        pair, reward, coef = vp.preference_forward(m["loss"], m["targets"], m["start"], vp.Preference(), m["ref"],
                                                   IGNORE, mean)
        assert bool((reward == 0).all())
        _close(pair, torch.full((2,), math.log(2), dtype=torch.float64), 0.0, "pair_loss")
        grad = vp.preference_backward(m["targets"], m["start"], coef, torch.full((2,), float("nan"), device="cuda"))
        assert bool((grad == 0).all())


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_arrays_at_any_element(shift):
    """Per-token arrays that start at any element of a larger buffer."""
    m = _make([700, 2, 0, 5000, 90, 1], 3, 40)

    def at(v):
        big = torch.empty(v.numel() + 8, dtype=v.dtype, device="cuda")
        big[shift:shift + v.numel()] = v
        return big[shift:shift + v.numel()]

    want = vp.policy_forward(m["loss"], m["targets"], m["start"], vp.Policy(kl_coef=0.1), m["adv_s"], m["old"], m["ref"])
    args = [at(m[k]) for k in ("loss", "targets", "start")]
    got = vp.policy_forward(*args, vp.Policy(kl_coef=0.1), at(m["adv_s"]), at(m["old"]), at(m["ref"]))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.linspace(1, 2, 6, device="cuda")
    bw = vp.policy_backward(m["loss"], m["targets"], m["start"], vp.Policy(kl_coef=0.1), m["adv_s"], want[3], g, m["old"],
                            m["ref"])
    bg = vp.policy_backward(*args, vp.Policy(kl_coef=0.1), at(m["adv_s"]), at(want[3]), at(g), at(m["old"]), at(m["ref"]))
    assert torch.equal(bw, bg)
    pw = vp.preference_forward(m["loss"], m["targets"], m["start"], vp.Preference(), m["ref"])
    pg = vp.preference_forward(*args, vp.Preference(), at(m["ref"]))
    assert all(torch.equal(a, b) for a, b in zip(pw, pg))


@pytest.mark.parametrize("starts", [
    [0, 10, 5, 12], [0, -7, 4, 12], [0, 4, 99, 12], [-3, 4, 6, 8], [4, 4, 4, 40], [2 ** 31 - 1, -2 ** 31, 0, 5],
])
@pytest.mark.parametrize("T", [12, 9000])
def test_wrong_offsets_stay_inside(starts, T):
    """Offsets that decrease or leave the tokens: NaN for the sequences that they bound, and
    nothing outside the arrays is touched."""
    guard = torch.full((T + 64,), 5.0, device="cuda")
    loss, grad = torch.ones(T, device="cuda"), guard[32:32 + T]
    targets = torch.zeros(T, dtype=torch.int64, device="cuda")
    start = torch.tensor(starts, dtype=torch.int32, device="cuda")
    adv = torch.ones(3, device="cuda")
    seq_loss, kl, clipped, tokens = vp.policy_forward(loss, targets, start, vp.Policy(), adv, None, loss, IGNORE, True)
    for s in range(3):
        a, b = starts[s], starts[s + 1]
        if not 0 <= a <= b <= T:
            assert math.isnan(seq_loss[s].item()) and math.isnan(kl[s].item())
    seq = vp.Sequences(T, 3, mean=True)
    vp.vp_policy_backward(seq, vp.Policy(), start, targets, loss, None, None, adv, tokens, adv, grad)
    assert bool((guard[:32] == 5).all()) and bool((guard[32 + T:] == 5).all())
    pair = vp.preference_forward(loss, targets, torch.cat([start, start[-1:]]), vp.Preference())[0]
    if not all(0 <= a <= b <= T for a, b in zip(starts[:2], starts[1:3])):
        assert math.isnan(pair[0].item())


def test_no_sequences():
    loss, targets = torch.ones(700, device="cuda"), torch.zeros(700, dtype=torch.int64, device="cuda")
    start, none = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    assert vp.preference_forward(loss, targets, start, vp.Preference())[0].numel() == 0
    assert bool((vp.preference_backward(targets, start, none, none) == 0).all())
    out = vp.policy_forward(loss, targets, start, vp.Policy(), none)
    assert bool((vp.policy_backward(loss, targets, start, vp.Policy(), none, out[3], none) == 0).all())


@pytest.mark.parametrize("lens", [[100, 50, 0, 3], _spread(40, 60000, 5)])
def test_captured_and_replayed(lens):
    """Both losses in two graphs on one workspace, replayed in turn with eager calls between, on
    new values and new offsets; and the same bits every time."""
    m, other = _make(lens, 0, 9, seed=1), _make(lens[::-1], 0, 9, seed=2)
    T, S = m["T"], m["S"]
    seq = vp.Sequences(T, S, mean=True)
    ws = torch.empty(vp.vp_seq_workspace_size(seq), dtype=torch.uint8, device="cuda")
    pol, pref = vp.Policy(kl_coef=0.1), vp.Preference(beta=0.5)
    f = lambda n, dt=torch.float32: torch.empty(n, dtype=dt, device="cuda")  # noqa: E731
    a = [f(S), f(S), f(S, torch.int32), f(S, torch.int32)]
    ga, b, gb = f(T), [f(S // 2), f(S), f(S)], f(T)
    up_a, up_b = torch.rand(S, device="cuda"), torch.rand(S // 2, device="cuda")

    def policy():
        vp.vp_policy_forward(seq, pol, m["start"], m["targets"], m["loss"], m["old"], m["ref"], m["adv_s"], *a, ws)
        vp.vp_policy_backward(seq, pol, m["start"], m["targets"], m["loss"], m["old"], m["ref"], m["adv_s"], a[3], up_a, ga)

    def preference():
        vp.vp_pref_forward(seq, pref, m["start"], m["targets"], m["loss"], m["ref"], *b, ws)
        vp.vp_pref_backward(seq, m["start"], m["targets"], b[2], up_b, gb)

    policy()
    preference()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    for run in (policy, preference):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run()
        graphs.append(graph)
    for step in range(4):
        for k in ("start", "targets", "loss", "old", "ref", "adv_s"):
            keep = m[k].clone()
            m[k].copy_(other[k])
            other[k].copy_(keep)
        if step % 2:
            m["loss"].mul_(0.75)
        graphs[step % 2].replay()
        want = vp.policy_forward(m["loss"], m["targets"], m["start"], pol, m["adv_s"], m["old"], m["ref"], IGNORE, True)
        graphs[1 - step % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a, want))
        assert torch.equal(ga, vp.policy_backward(m["loss"], m["targets"], m["start"], pol, m["adv_s"], want[3], up_a,
                                                  m["old"], m["ref"], IGNORE, True))
        pw = vp.preference_forward(m["loss"], m["targets"], m["start"], pref, m["ref"], IGNORE, True)
        assert all(torch.equal(x, y) for x, y in zip(b, pw))
        assert torch.equal(gb, vp.preference_backward(m["targets"], m["start"], pw[2], up_b))


def test_two_streams():
    """Calls on two streams with workspaces of their own."""
    ms = [_make(_spread(50, 90000, k), seed=k) for k in range(2)]
    args = lambda m: (m["loss"], m["targets"], m["start"], vp.Policy(kl_coef=0.1), m["adv_s"], m["old"], m["ref"])  # noqa: E731
    want = [vp.policy_forward(*args(m)) for m in ms]
    streams = [torch.cuda.Stream() for _ in ms]
    torch.cuda.synchronize()
    got = []
    for m, s in zip(ms, streams):
        with torch.cuda.stream(s):
            got.append(vp.policy_forward(*args(m)))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
