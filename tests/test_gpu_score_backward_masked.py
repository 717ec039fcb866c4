"""Gradients with an entropy term where a token has neither a loss nor an entropy gradient: nothing of it is in dH or
dW, whatever its lse and entropy are (a token whose mask leaves no id, entries that were never written)."""
import pytest
import torch

import paper_2609_14306_amd as vp
from test_gpu_score import make

pytestmark = pytest.mark.gpu


def gradients(H, W, t, g, e, lse, entropy):
    dH, dW = vp.backward(H, W, t, lse, g, entropy=entropy, grad_entropy=e)
    return dH, torch.cat(dW)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T, d, rows", [(5, 64, [300]), (300, 128, [700, 900]), (2100, 200, [1000, 513])])
@pytest.mark.parametrize("how", ["masked", "unwritten"])
def test_tokens_without_any_gradient(dtype, T, d, rows, how):
    H, W, t = make(dtype, T, d, rows)
    H[:, -1] = 0.0
    gone = torch.arange(T, device="cuda") % 5 == 3
    t[gone] = -100
    gen = torch.Generator(device="cuda").manual_seed(T)
    g, e = torch.randn(T, generator=gen, device="cuda"), torch.randn(T, generator=gen, device="cuda")
    e[gone] = 0.0
    _, lse, entropy, _, _ = vp.score(H, W, t)
    want = gradients(H, W, t, g, e, lse, entropy)
    assert bool((want[0][gone] == 0).all())
    if how == "masked":  # every logit of these tokens is the type's lowest value
        H[gone] = 0.0
        H[gone, -1] = 1.0
        for w in W:
            w[:, -1] = torch.finfo(w.dtype).min
        _, lse, entropy, _, _ = vp.score(H, W, t)
        got = gradients(H, W, t, g, e, lse, entropy)
        # (the last column of W enters dH of the other tokens, and the last one of H dW nowhere)
        assert bool((got[0][gone] == 0).all())
        assert torch.equal(got[0][~gone, :-1], want[0][~gone, :-1])
        assert bool(got[1].isfinite().all())
    else:
        lse[gone], entropy[gone] = torch.nan, torch.nan
        lse[gone.nonzero()[::2, 0]] = torch.inf
        got = gradients(H, W, t, g, e, lse, entropy)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
