"""8-bit scoring where the matrix unit's cut of small products shows: likely ids have their exact logits in lse and
entropy whatever the alternatives need, alternatives are looked for whatever the likely ids need, the same token has
the same bits, and wide rows are held to root mean squares.

``built``: one token, as often as wanted.  A pair of products of +-P in one group of eight cuts the group's six others,
which are below 2^-13 P: an id's product is 0 short by c = 1 to 6 of them, exactly (every number here is exact in 8
bits, and its sums in float32)."""
import pytest
import torch

import paper_2609_14306_amd as vp
import score_plain as sp

pytestmark = pytest.mark.gpu
U = sp.U


def built(T, levels, short, big, d=128, step=8, V=2500):
    """levels: the ids' logits without what is cut; short: how many small products each has (0: no pair either);
    big: P = big^2.  Ids lie `step` apart from 16 on; the rest have logits of -24."""
    small = {8.0: (0.125, 0.0546875), 32.0: (1.0, 0.109375)}[big]  # products of 0.0068 < 2^-13 64, 0.109 < 2^-13 1024
    H, W = torch.zeros(1, d), torch.zeros(V, d)
    H[0, :2], H[0, 2:8], H[0, 16] = big, small[0], 1.0
    W[:, 16] = -24.0
    for k, (level, n) in enumerate(zip(levels, short)):
        v = 16 + step * k
        W[v, 16] = level
        if n:
            W[v, 0], W[v, 1], W[v, 2:2 + n] = big, -big, small[1]
    H = H.expand(T, d).contiguous().cuda()
    h8, hs = vp.quantize(H)
    w8, ws = vp.quantize(W.cuda(), 128)
    h, w = sp.values(h8, hs, 1), sp.values(w8, ws, 128)
    assert torch.equal(h, H.double()) and torch.equal(w, W.cuda().double())
    t = torch.full((T,), -100, dtype=torch.int64, device="cuda")
    return (h8, hs, [w8], [ws], t), sp.score(h[:1], w, t[:1], -100, 8)


def one_value(x):
    x = x.view(torch.int32) if x.dtype == torch.float32 else x
    assert bool((x == x[:1]).all()), x.unique()[:4]


# float32's roundings of the correction: p of e^z with z = m - lse (u |lse|), its sums, the logarithm, lse itself
def held(got, want):
    lse, S = float(want[1]), float(want[2])
    assert abs(float(got[1][0]) - lse) <= 16 * U * (1 + abs(lse)), (float(got[1][0]), lse)
    assert abs(float(got[2][0]) - S) <= 32 * U * (1 + abs(lse)) * (1 + S), (float(got[2][0]), S)


T = [1, 30, 100, 600, 2100]


@pytest.mark.parametrize("T", T)
@pytest.mark.parametrize("big", [8.0, 32.0])
@pytest.mark.parametrize("top", [0, 2])
def test_likely_ids_beside_many_near_alternatives(top, big, T):
    """An id of 0.30, thirty of 0.009 (above 2^-7) and sixty of 0.0071: with alternatives more ids than there is room
    for lie near the second one, and the thirty alone have room."""
    ops, want = built(T, [3.5] + [0.0] * 30 + [-0.25] * 60, [0] + [6] * 3 + [1 + k % 6 for k in range(27)] + [0] * 60, big)
    got = vp.score_f8(*ops, top=top)
    held(got, want)
    if top:
        assert torch.equal(got[3], want[3][:, :top].expand(T, top))


@pytest.mark.parametrize("T", T)
def test_near_alternatives_beside_many_likely_ids(T):
    """Ninety-five ids above 2^-7, more than there is room for; the largest logit is the last of five that the
    product does not tell apart."""
    ops, want = built(T, [1.0] * 5 + [0.0] * 90, [1, 2, 3, 4, 5] + [0] * 90, 8.0)
    got = vp.score_f8(*ops, top=1)
    assert torch.equal(got[3], want[3][:, :1].expand(T, 1))


@pytest.mark.parametrize("T", [30, 600, 2100])
@pytest.mark.parametrize("big", [8.0, 32.0])
@pytest.mark.parametrize("top", [0, 1, 8])
def test_equal_tokens_have_equal_bits(top, big, T):
    """Forty likely ids with corrections of many sizes, in the shares of many wavefronts."""
    ops, want = built(T, [(k % 7) / 8 for k in range(40)], [1 + (5 * k) % 6 for k in range(40)], big, step=1096, V=50000)
    got = vp.score_f8(*ops, top=top)
    held(got, want)
    for x in got[:3] + (got[3:] if top else ()):
        one_value(x)


@pytest.mark.parametrize("top", [0, 3])
@pytest.mark.parametrize("d", [4096, 14336])
@pytest.mark.parametrize("T, rows", [(40, [3001, 0, 700]), (128, [30000]), (2100, [1500, 601])])
def test_wide_rows_with_scales_that_vary(T, rows, d, top):
    """As test_gpu_f8.py's test_likely_ids_have_their_exact_logits, with the same 3e-5 of the sums' root mean square
    for a logit, on wide rows whose scales differ from block to block."""
    from test_gpu_f8 import make
    H, Hs, W, Ws, t = make(T, d, rows, seed=3)
    got = vp.score_f8(H, Hs, W, Ws, t, top=top)
    h, w = sp.values(H, Hs, 1), torch.cat([sp.values(a, b, 128) for a, b in zip(W, Ws)])
    want = sp.score(h, w, t, -100, top)
    y, lse, S = want[5], want[1], want[2]
    logp = y - lse[:, None]
    p = logp.exp()
    e = 3e-5 * (h.square() @ w.square().t().contiguous()).mean(1).sqrt()
    rms = lambda v: float(v.square().mean().sqrt())  # noqa: E731
    left = 4 * rms(e * p.square().sum(1).sqrt())
    assert rms(got[1].double() - lse) <= left + 4 * U * rms(lse)
    left = 4 * rms(e * (p * (logp + S[:, None])).square().sum(1).sqrt())
    assert rms(got[2].double() - S) <= left + 4 * U * rms(lse + 1)
    if top:
        assert torch.equal(got[3], want[3])
