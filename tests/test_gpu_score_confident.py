"""Entropies of confident tokens, whose probability one id holds but for 1e-2 to 1e-9 of it: to a relative
bound, and never negative.

The logits are sums of a few small integers and halves, exact in every type, so what is left are the roundings of
the sums: with d = y - max exact, d log2e is off by u |d log2e| and the exponential by that times ln2 and a unit of
its own, i.e. by (|d| + 2) u; a state is rescaled once in a lane's fold and at most twice where states are joined,
each time by such an exponential; products and the sums of up to eight terms (the others are 0) take 12 u more, the
logarithm and the quotient 6 u.  So S is held to (4 (|d| + 2) + 18) u of itself, with the largest |d| that is there,
27.  Of one id alone nothing is left."""
import math

import pytest
import torch

import paper_2609_14306_amd as vp
import score_plain as sp

pytestmark = pytest.mark.gpu
U = sp.U
# (four significant bits: every type holds them)
TOP = [208.0, 8.0, 16.0, 24.0, 32.0, 40.0, 48.0, 64.0, 80.0, 96.0, 112.0, 128.0, 144.0, 160.0, 176.0, 192.0, 52.0]
GAP = [18.0, 4.0, 5.0, 6.0, 7.0, 8.0, 9.0, 10.0, 11.0, 12.0, 13.0, 14.0, 15.0, 16.0]
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(T, rows, far, d=64):
    """H, W in float32: logits of b_t for one id, b_t - g_t and b_t - 1.5 g_t for `far` others, b_t - 240 for
    the rest; the others lie in the four of the first, in its tile, or in other tiles and shards."""
    V = sum(rows)
    top = V // 3 // 4 * 4
    others = {"four": [top + 1, top + 3], "tile": [top + 4, top + 8, top + 37, top + 64],
              "all": [0, 5, top - 300, top + 300, V - 1]}[far]
    H, W = torch.zeros(T, d, device="cuda"), torch.zeros(V, d, device="cuda")
    W[:, 0] = 1.0
    W[:, 16] = -240.0
    W[[top] + others, 16] = 0.0
    for k, v in enumerate(others):
        W[v, 32] = -1.5 if k % 2 else -1.0
    t = torch.arange(T, device="cuda")
    H[:, 0] = torch.tensor(TOP, device="cuda")[t % len(TOP)]
    H[:, 16] = 1.0
    H[:, 32] = torch.tensor(GAP, device="cuda")[t % len(GAP)]
    return H, W, torch.full((T,), -100, dtype=torch.int64, device="cuda")


def held(got, h, w, t, top):
    want = sp.score(h, w, t, -100, top)
    S = want[2]
    assert float(S.min()) < 1e-6 < 1e-2 < float(S.max())
    assert bool((got[2] >= 0).all())
    rel = ((got[2].double() - S) / S).abs()
    assert float(rel.max()) <= (4 * 29 + 18) * U, (float(rel.max()), float(S[rel.argmax()]))
    assert bool(((got[1].double() - want[1]).abs() <= 2 * U * want[1].abs() + 1e-9).all())
    if top:
        assert torch.equal(got[3], want[3])


@pytest.mark.parametrize("top", [0, 2])
@pytest.mark.parametrize("far", ["four", "tile", "all"])
@pytest.mark.parametrize("T, rows", [(14, [3001]), (40, [2000, 3001]), (90, [20000, 10001]), (300, [5000, 501]),
                                     (700, [4000, 3001, 9]), (2100, [3000, 1, 2001])])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_confident_tokens(dtype, T, rows, far, top):
    H, W, t = make(T, rows, far)
    H, W = H.to(DT[dtype]), W.to(DT[dtype])
    held(vp.score(H, list(W.split(rows)), t, top=top), H.double(), W.double(), t, top)


@pytest.mark.parametrize("top", [0, 2])
@pytest.mark.parametrize("far", ["four", "tile", "all"])
@pytest.mark.parametrize("T, rows", [(14, [3001]), (90, [20000, 10001]), (2100, [3000, 128, 2001])])
def test_confident_tokens_in_8_bits(T, rows, far, top):
    H, W, t = make(T, rows, far, d=128)
    h8, hs = vp.quantize(H)
    W8, Ws = map(list, zip(*[vp.quantize(w.contiguous(), 128) for w in W.split(rows)]))
    h, w = sp.values(h8, hs, 1), torch.cat([sp.values(a, b, 128) for a, b in zip(W8, Ws)])
    assert torch.equal(h, H.double()) and torch.equal(w, W.double())
    held(vp.score_f8(h8, hs, W8, Ws, t, top=top), h, w, t, top)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 40, 300, 2100])
def test_one_id_alone(dtype, T):
    """One live id: an entropy of 0, and lse its logit."""
    H, W, t = make(T, [1999], "four")
    W[:, 32] = -240.0
    W[1999 // 3 // 4 * 4, 32] = 0.0
    H, W = H.to(DT[dtype]), W.to(DT[dtype])
    _, lse, S, _, _ = vp.score(H, [W], t)
    assert bool((S == 0).all())
    assert bool((lse == H[:, 0].float()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [5, 300, 2100])
def test_two_equal_ids_and_all_equal(dtype, T):
    """log 2 and log V, with nothing lost to the ones."""
    H, W, t = make(T, [1999], "tile")
    W[:, 32] = -240.0
    W[[660, 700], 32] = W[[660, 700], 16] = 0.0
    H, W = H.to(DT[dtype]), W.to(DT[dtype])
    S = vp.score(H, [W], t)[2].double()
    assert bool(((S - math.log(2)).abs() <= 4 * U).all())
    W[:] = W[660]
    S = vp.score(H, [W], t)[2].double()
    assert bool(((S - math.log(1999)).abs() <= 4 * U * 7.6).all())
