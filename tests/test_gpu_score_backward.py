"""Gradients of a loss with an entropy term on the GPU, against the plain float64 ones, on every tile
class of the backward; at the projection's bars (1e-5 relative in float32, 1e-2 in bfloat16, whose
residual is held in bfloat16: half a step, 2^-8, of every element)."""
import pytest
import torch

import paper_2609_14306_amd as vp
import score_plain as sp
import tile_cases
from test_gpu_score import make

pytestmark = pytest.mark.gpu
BAR = {torch.float32: 1e-5, torch.bfloat16: 1e-2}


def upstream(T, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(T, generator=g, device="cuda"), torch.randn(T, generator=g, device="cuda")


def reference(H, W, t, g, e, ignore=-100):
    W64 = torch.cat(W).double()
    dH, dW = torch.empty(H.shape, dtype=torch.float64, device="cuda"), torch.zeros_like(W64)
    for a in range(0, H.shape[0], 1024):
        s = slice(a, a + 1024)
        H64 = H[s].double()
        G = sp.residual(H64, W64, t[s], ignore, g[s].double(), e[s].double())
        dH[s] = G @ W64
        dW += G.t().contiguous() @ H64
    return dH, dW


def close(got, want, dtype, what):
    rel = ((got.double() - want).norm() / want.norm()).item()
    assert rel <= BAR[dtype], (what, rel)


@pytest.mark.parametrize("cls, dtype, T, d, rows, strip", tile_cases.BACKWARD)
def test_every_tile_class(cls, dtype, T, d, rows, strip):
    H, W, t = make(dtype, T, d, rows)
    g, e = upstream(T)
    _, lse, ent, _, _ = vp.score(H, W, t)
    dH, dW = vp.backward(H, W, t, lse, g, strip_elems=strip, entropy=ent, grad_entropy=e)
    want = reference(H, W, t, g, e)
    close(dH, want[0], H.dtype, "dH")
    close(torch.cat(dW), want[1], H.dtype, "dW")


@pytest.mark.parametrize("dtype, T, d, rows", [
    ("f32", 1, 8, [1]), ("f32", 1, 64, [3, 0, 500]), ("bf16", 1, 4096, [2000]), ("f32", 77, 72, [255, 256, 257]),
    ("bf16", 300, 200, [4, 3000, 100]), ("f32", 2100, 128, [600, 700]), ("bf16", 2100, 320, [3000])])
@pytest.mark.parametrize("part", ["both", "entropy", "loss"])
def test_sizes_and_terms(dtype, T, d, rows, part):
    H, W, t = make(dtype, T, d, rows)
    g, e = upstream(T)
    if part == "entropy":
        g.zero_()
    if part == "loss":
        e.zero_()
    _, lse, ent, _, _ = vp.score(H, W, t)
    dH, dW = vp.backward(H, W, t, lse, g, entropy=ent, grad_entropy=e)
    want = reference(H, W, t, g, e)
    if float(want[1].norm()) == 0 or sum(rows) == 1:  # (one id: no gradient, but for roundings)
        assert float(dH.abs().max()) <= 1e-5 and float(torch.cat(dW).abs().max()) <= 1e-4
        return
    close(dH, want[0], H.dtype, "dH")
    close(torch.cat(dW), want[1], H.dtype, "dW")


def test_entropy_of_ignored_tokens_keeps_its_gradient():
    H, W, t = make("f32", 200, 64, [300, 50])
    t[:] = -100
    g, e = upstream(200)
    _, lse, ent, _, _ = vp.score(H, W, t)
    dH, dW = vp.backward(H, W, t, lse, g, entropy=ent, grad_entropy=e)
    want = reference(H, W, t, torch.zeros_like(g), e)
    close(dH, want[0], H.dtype, "dH")
    close(torch.cat(dW), want[1], H.dtype, "dW")


def test_out_of_range_targets_are_nan_rows():
    H, W, t = make("f32", 90, 64, [300, 50])
    t[4] = 350
    g, e = upstream(90)
    _, lse, ent, _, _ = vp.score(H, W, t)
    dH, _ = vp.backward(H, W, t, lse, g, entropy=ent, grad_entropy=e)
    assert bool(dH[4].isnan().all()) and not bool(dH[torch.arange(90, device="cuda") != 4].isnan().any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [40, 1333])
def test_masked_rows(dtype, T):
    """Logits of minus infinity have no probability and no gradient, not NaN."""
    H, W, t = make(dtype, T, 128, [512, 300])
    H[:, -1] = 1.0
    t[:] = 20
    W[0][100:200] = 0.0
    W[0][100:200, -1] = -torch.inf
    W[1][290:] = 0.0
    W[1][290:, -1] = -torch.inf
    g, e = upstream(T)
    _, lse, ent, _, _ = vp.score(H, W, t)
    dH, dW = vp.backward(H, W, t, lse, g, entropy=ent, grad_entropy=e)
    live = torch.ones(812, dtype=torch.bool, device="cuda")
    live[100:200] = live[802:] = False
    want = reference(H, [torch.cat(W)[live]], t, g, e)
    dW = torch.cat(dW)
    assert bool((dW[~live] == 0).all())
    close(dW[live], want[1], H.dtype, "dW")
    close(dH[:, :-1], want[0][:, :-1], H.dtype, "dH")  # (the last column meets minus infinity itself)


def test_accumulates_and_refuses():
    H, W, t = make("f32", 300, 64, [700, 800])
    g, e = upstream(300)
    _, lse, ent, _, _ = vp.score(H, W, t)
    dH, dW = vp.backward(H, W, t, lse, g, entropy=ent, grad_entropy=e)
    base = [torch.randn_like(w) for w in dW]
    acc = [b.clone() for b in base]
    vp.backward(H, W, t, lse, g, dW_shards=acc, accumulate=True, entropy=ent, grad_entropy=e)
    for a, b, w in zip(acc, base, dW):
        assert bool(((a - b - w).abs() <= 4 * sp.U * (a.abs() + b.abs())).all())
    with pytest.raises(ValueError, match="grad_entropy"):
        vp.backward(H, W, t, lse, g, entropy=ent)


def test_with_a_norm_in_front():
    X = torch.randn(200, 64, device="cuda")
    gamma = 1 + 0.1 * torch.randn(64, device="cuda")
    norm = vp.HeadNorm(gamma, None, rms=True)
    _, W, t = make("f32", 200, 64, [300, 50])
    Y = vp.layer_norm(X, gamma, None, norm.eps, True)[0]
    g, e = upstream(200)
    loss, lse, ent, ids, top_loss = vp.score(Y, W, t, top=3)
    for a, b in zip(vp.score(X, W, t, top=3, norm=norm), (loss, lse, ent, ids, top_loss)):
        assert torch.equal(a, b)
    dX, dW, dgamma, _ = vp.backward(X, W, t, lse, g, norm=norm, entropy=ent, grad_entropy=e)
    x, ga = X.double().requires_grad_(), gamma.double().requires_grad_()
    y = x * ((x * x).mean(1, keepdim=True) + norm.eps).rsqrt() * ga
    logp = torch.log_softmax(y @ torch.cat(W).double().t(), 1)
    live = t != -100
    nll = -logp.gather(1, torch.where(live, t, 0)[:, None])[:, 0] * live
    total = (nll * g.double()).sum() + (-(logp.exp() * logp).sum(1) * e.double()).sum()
    gx, gg = torch.autograd.grad(total, (x, ga))
    close(dX, gx, torch.float32, "dX")
    close(dgamma, gg, torch.float32, "dgamma")


def test_graph_replays_with_an_eager_graph_alive():
    H, W, t = make("bf16", 300, 320, [900, 500])
    g, e = upstream(300)
    _, lse, ent, _, _ = vp.score(H, W, t)
    prob = vp.problem_for(H, W)
    ws = torch.empty(vp.vp_ce_workspace_size(prob)[1], dtype=torch.uint8, device="cuda")
    dH, dW = torch.empty(300, 320, device="cuda"), [torch.empty(w.shape, device="cuda") for w in W]
    run = lambda: vp.vp_score_backward(prob, H, W, t, lse, ent, g, e, dH, dW, ws)  # noqa: E731
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    want = [dH.clone()] + [w.clone() for w in dW]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for o in [dH] + dW:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip([dH] + dW, want))
        vp.score(H, W, t, top=1)
        torch.cuda.synchronize()
