"""lse and entropy of bfloat16 and float32 operands to what float32 sums are off by on average (test_gpu_score.py's
bounds are those of the worst order, which a wide row never comes near).

A sum of d products is rounded d times at most, each time by no more than u of the partial sum.  Partial sums of
random products grow as a walk, S_k^2 = k / d of the whole's sum of squares q, and roundings are independent: a logit
is off by e = u sqrt(q d / 2) at most as a root mean square.  lse = sum p y is off by e sqrt(sum p^2) then, and the
entropy by e sqrt(sum p^2 (log p + S)^2).  Held to twice that (the largest of the products enters more than one
sum), and what the exponentials' sums and the result are rounded by: 4 u of lse, and 4 u of lse + 1 in the entropy,
whose terms are log p.  A logit rounded to bfloat16 is off by 2^-9 of itself, 80 times e at d = 4096."""
import pytest
import torch

import paper_2609_14306_amd as vp
import score_plain as sp
from test_gpu_score import make

pytestmark = pytest.mark.gpu
U = sp.U


@pytest.mark.parametrize("top", [0, 1])
@pytest.mark.parametrize("scale", [2.0, 5.0])
@pytest.mark.parametrize("T, d, rows", [(20, 1000, [9001]), (40, 4096, [3001, 700]), (100, 2880, [30000]), (300, 7168, [2500]),
                                        (700, 1000, [4000, 3001, 9]), (2100, 4096, [2000, 77])])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rounding_of_wide_rows(dtype, T, d, rows, scale, top):
    H, W, t = make(dtype, T, d, rows, seed=4, scale=scale)
    got = vp.score(H, W, t, top=top)
    h, w = H.double(), torch.cat(W).double()
    want = sp.score(h, w, t, -100, top)
    y, lse, S = want[5], want[1], want[2]
    logp = y - lse[:, None]
    p = logp.exp()
    e = U * ((h.square() @ w.square().t().contiguous()).mean(1) * d / 2).sqrt()
    rms = lambda v: float(v.square().mean().sqrt())  # noqa: E731
    assert rms(got[1].double() - lse) <= 2 * rms(e * p.square().sum(1).sqrt()) + 4 * U * rms(lse)
    left = 2 * rms(e * (p * (logp + S[:, None])).square().sum(1).sqrt())
    assert rms(got[2].double() - S) <= left + 4 * U * rms(lse + 1)
    live = t != -100
    assert rms((got[0].double() - want[0])[live]) <= 2 * rms(e * p.square().sum(1).sqrt()) + 4 * U * rms(lse) + 2 * U * rms(want[0])
    if top:
        assert torch.equal(got[3], want[3])
