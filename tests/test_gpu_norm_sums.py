"""dgamma and dbeta over many rows, bit for bit: with whole numbers, whose float32 sums below 2^24
have no rounding, every row has to arrive exactly once, whatever the order."""
import pytest
import torch

import paper_2609_14306_amd as vp

pytestmark = pytest.mark.gpu

# rows side by side in a workgroup, one row to several wavefronts, one workgroup alone, a last
# round that is not full, more partial rows than the join has wavefronts
SIZES = [(1, 64), (4, 4096), (5, 4096), (128, 64), (129, 64), (1333, 1000), (20011, 320), (33000, 136), (4099, 2880),
         (2051, 7168), (1030, 16384), (300007, 64), (70001, 512), (70001, 40), (50021, 1032)]


def _signs(g, *shape):
    return torch.randint(0, 2, shape, generator=g, device="cuda").float() * 2 - 1


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T, d", SIZES + [(2 ** 23 - 256, 8)])
def test_every_row_once(T, d, dtype, rms):
    """No entry of dY or of X is 0, so a row left out or taken twice shows in every column."""
    g = torch.Generator(device="cuda").manual_seed(T + d)
    X, dY = _signs(g, T, d), _signs(g, T, d)
    if T < 100000:  # (|sums| stay below 2^24)
        X *= torch.randint(1, 9, (T, d), generator=g, device="cuda")
        dY *= torch.randint(1, 9, (T, d), generator=g, device="cuda")
    X = X.to(dtype)
    gamma, one = torch.ones(d, device="cuda").to(dtype), torch.ones(T, device="cuda")
    mean = None if rms else torch.zeros(T, device="cuda")
    base = torch.arange(2 * d, device="cuda").float().view(2, d)
    want = torch.zeros(2, d, dtype=torch.float64, device="cuda")
    step = max(1, 2 ** 25 // d)
    for a in range(0, T, step):
        dy = dY[a:a + step].double()
        want += torch.stack([(X[a:a + step].double() * dy).sum(0), dy.sum(0)])
    got = vp.layer_norm_backward(X, gamma, mean, one, dY)
    assert torch.equal(torch.stack(got[1:]).double(), want)
    acc = base.clone()
    vp.layer_norm_backward(X, gamma, mean, one, dY, dX=dY, dgamma=acc[0], dbeta=acc[1], accumulate=True)
    assert torch.equal(acc.double(), want + base)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T, d", [(1333, 1000), (33000, 136), (20011, 320), (4099, 2880), (300007, 64)])
def test_one_row_alone(T, d, dtype):
    """The gradient in one row: the first and the last ones of a round, of a walk and of all."""
    g = torch.Generator(device="cuda").manual_seed(3)
    X = (_signs(g, T, d) * torch.randint(1, 9, (T, d), generator=g, device="cuda")).to(dtype)
    gamma, one, zero = torch.ones(d, device="cuda").to(dtype), torch.ones(T, device="cuda"), torch.zeros(T, device="cuda")
    dY = torch.zeros(T, d, device="cuda")
    rows = {0, 1, 31, 32, 255, 256, 257, 511, 512, 1023, 1024, 8191, 8192, 16384, T // 2, T - 257, T - 33, T - 2, T - 1}
    for t in sorted(r for r in rows if 0 <= r < T):
        dY[t] = 2.0
        dX, dgamma, dbeta = vp.layer_norm_backward(X, gamma, zero, one, dY)
        assert torch.equal(dgamma, 2 * X[t].float()) and bool((dbeta == 2).all()), t
        dX[t] = 0
        assert not bool(dX.any()), t
        dY[t] = 0
