"""Layer norm and its gradients on the GPU against the plain float64 form.

Bounds, with u = 2^-24 and sums of a row in chains of at most DEPTH additions (a lane's
elements, then the lanes), so that a float32 sum of x_k is off by at
most DEPTH u sum |x_k|:
* mean: DEPTH u mean|x|; the variance around a mean that is off by e gains e^2, and its own sum
  and squares (DEPTH + 4) u, so rstd is off by half of that and 3 u, relative;
* y: what mean and rstd make of gamma xh, 6 u for its own operations, and half a step of its type;
* dX from the given mean and rstd: the two row means, and 10 u of each of its terms;
* dgamma, dbeta: a chain of at most ROWS(T) tokens, 3 u for each product.
"""
import pytest
import torch

import head_plain as hp
import paper_2609_14306_amd as vp

pytestmark = pytest.mark.gpu
U = hp.U
DEPTH = 144


def ROWS(T):
    return min(T, 8192) + 32


def _make(T, d, dtype, bias=True, seed=0, scale=1.0, offset=0.3):
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + 7 * T + d)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    X = (offset + scale * n(T, d) * (0.5 + n(d).abs())).to(dtype)
    gamma, beta = (1 + 0.2 * n(d)).to(dtype), (0.3 * n(d)).to(dtype) if bias else None
    return X, gamma, beta, n(T, d)


def _within(got, want, bound, what):
    err = (got.double().cpu() - want).abs()
    worst = (err - bound).argmax()
    assert bool((err <= bound).all()), (what, err.view(-1)[worst].item(), bound.expand_as(err).reshape(-1)[worst].item())


def _check_forward(X, gamma, beta, eps, rms, got):
    Y, mean, rstd = got
    y, mu, r = hp.norm_forward(X, gamma, beta, eps, rms)
    x, ga = X.double().cpu(), gamma.double().cpu().abs()
    e_mean = torch.zeros_like(mu) if rms else (DEPTH + 2) * U * x.abs().mean(1)
    var = 1 / r ** 2
    e_r = (0.5 * (DEPTH + 4) + 3) * U + 0.5 * e_mean ** 2 / var
    if rms:
        assert mean is None
    else:
        _within(mean, mu, e_mean, "mean")
    _within(rstd, r, r * e_r, "rstd")
    xh = ((x - mu[:, None]) * r[:, None]).abs()
    half = torch.finfo(X.dtype).eps / 2
    b = 0.0 if beta is None else beta.double().cpu().abs()
    bound = ga * ((r * e_mean)[:, None] + xh * (e_r + 6 * U)[:, None]) + 2 * U * (ga * xh + b)
    _within(Y, y, bound * (1 + half) + half * y.abs() + 1e-44, "Y")


def _check_backward(X, gamma, mean, rstd, dY, got, base=None):
    dX, dgamma, dbeta = got
    dx, dg, db = hp.norm_backward(X, gamma, mean, rstd, dY)
    x, dy, r = X.double().cpu(), dY.double().cpu(), rstd.double().cpu()[:, None]
    xh = (x if mean is None else x - mean.double().cpu()[:, None]) * r
    g = dy * gamma.double().cpu()
    m1 = torch.zeros_like(r) if mean is None else g.abs().mean(1, keepdim=True)
    m2 = (g * xh).abs().mean(1, keepdim=True)
    _within(dX, dx, r * U * ((DEPTH + 10) * (m1 + xh.abs() * m2) + 10 * g.abs()) + 1e-44, "dX")
    T = X.shape[0]
    old = [0.0, 0.0] if base is None else [v.double().cpu() for v in base]
    if dgamma is None:
        return
    _within(dgamma, dg + old[0], (ROWS(T) + 4) * U * ((dy * xh).abs().sum(0) + (abs(old[0]))) + 1e-44, "dgamma")
    if dbeta is not None:
        _within(dbeta, db + old[1], (ROWS(T) + 1) * U * (dy.abs().sum(0) + abs(old[1])) + 1e-44, "dbeta")


# every layout of a row, its widest and a width that leaves part of it empty
SIZES = [(1, 8), (1, 4096), (2, 16384), (3, 40), (5, 1000), (37, 2880), (130, 264), (257, 512), (64, 7168),
         (9, 16384), (700, 1032), (4100, 64), (1500, 2056), (33, 8200), (2049, 128), (70, 256), (45, 776), (19, 1024), (23, 2048), (31, 3336),
         (3, 5000), (6, 8192), (150, 72), (5, 9000)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("T, d", SIZES)
def test_against_float64(T, d, dtype, rms):
    bias = (T + d) % 3 != 0
    X, gamma, beta, dY = _make(T, d, dtype, bias)
    out = vp.layer_norm(X, gamma, beta, 1e-5, rms)
    _check_forward(X, gamma, beta, 1e-5, rms, out)
    grads = vp.layer_norm_backward(X, gamma, out[1], out[2], dY, bias=bias)
    assert (grads[2] is None) == (not bias)
    _check_backward(X, gamma, out[1], out[2], dY, grads)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T, d", [(20011, 320), (33000, 136)])
def test_many_rows(T, d, dtype):
    X, gamma, beta, dY = _make(T, d, dtype)
    out = vp.layer_norm(X, gamma, beta)
    _check_forward(X, gamma, beta, 1e-5, False, out)
    _check_backward(X, gamma, out[1], out[2], dY, vp.layer_norm_backward(X, gamma, out[1], out[2], dY))


@pytest.mark.parametrize("T, d", [(1, 64), (7, 2880), (900, 1000), (40, 16384)])
def test_accumulate_and_in_place(T, d):
    X, gamma, beta, dY = _make(T, d, torch.bfloat16)
    _, mean, rstd = vp.layer_norm(X, gamma, beta)
    plain = vp.layer_norm_backward(X, gamma, mean, rstd, dY)
    base = torch.randn(2, d, device="cuda")
    acc, buf = [b.clone() for b in base], dY.clone()
    got = vp.layer_norm_backward(X, gamma, mean, rstd, buf, dX=buf, dgamma=acc[0], dbeta=acc[1], accumulate=True)
    assert got[0] is buf and torch.equal(buf, plain[0])
    _check_backward(X, gamma, mean, rstd, dY, (got[0], acc[0], acc[1]), base)


def test_no_rows():
    X = torch.empty(0, 64, device="cuda")
    gamma = torch.ones(64, device="cuda")
    Y, mean, rstd = vp.layer_norm(X, gamma, gamma)
    assert Y.shape == (0, 64) and mean.shape == rstd.shape == (0,)
    dg, db = torch.full((64,), 3.0, device="cuda"), torch.full((64,), 4.0, device="cuda")
    vp.layer_norm_backward(X, gamma, mean, rstd, torch.empty(0, 64, device="cuda"), dgamma=dg, dbeta=db,
                           accumulate=True)
    assert bool((dg == 3).all()) and bool((db == 4).all())
    vp.layer_norm_backward(X, gamma, mean, rstd, torch.empty(0, 64, device="cuda"), dgamma=dg, dbeta=db)
    assert bool((dg == 0).all()) and bool((db == 0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rms", [False, True])
def test_rows_apart(dtype, rms):
    """A row of NaN or infinities leaves the other rows as they are; a constant row has rstd
    eps^-1/2; the same call gives the same bits."""
    X, gamma, beta, dY = _make(300, 1000, dtype)
    clean = vp.layer_norm(X, gamma, beta, 1e-3, rms)
    grads = vp.layer_norm_backward(X, gamma, clean[1], clean[2], dY)
    again = vp.layer_norm_backward(X, gamma, clean[1], clean[2], dY)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    Z = X.clone()
    Z[17, 3], Z[18], Z[40] = float("nan"), float("inf"), 0.5
    out = vp.layer_norm(Z, gamma, beta, 1e-3, rms)
    keep = torch.ones(300, dtype=torch.bool, device="cuda")
    keep[[17, 18, 40]] = False
    assert torch.equal(out[0][keep], clean[0][keep]) and torch.equal(out[2][keep], clean[2][keep])
    assert bool(out[0][17].isnan().all())
    _check_forward(Z[40:41], gamma, beta, 1e-3, rms, [v if v is None else v[40:41] for v in out])
    dx = vp.layer_norm_backward(Z, gamma, out[1], out[2], dY)[0]
    assert torch.equal(dx[keep], grads[0][keep])


def test_large_offset_keeps_the_spread():
    """A mean 1000 times the spread: the variance is taken around the mean, not from squares."""
    X, gamma, beta, dY = _make(50, 2880, torch.float32, offset=1000.0)
    out = vp.layer_norm(X, gamma, beta, 1e-5)
    _check_forward(X, gamma, beta, 1e-5, False, out)
    _check_backward(X, gamma, out[1], out[2], dY, vp.layer_norm_backward(X, gamma, out[1], out[2], dY))


@pytest.mark.parametrize("T, d, dtype", [
    (300007, 8192, torch.bfloat16),   # more than 2^31 elements
    (1048597, 4104, torch.float32),   # more rows than one launch of 2^30 threads has
    (2 ** 23 - 256, 8, torch.bfloat16),  # the most rows
])
def test_large(T, d, dtype):
    """Rows at the beginning, in the middle and at the end, and the sums over all rows, taken in
    float64 on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(5)
    X = torch.empty(T, d, dtype=dtype, device="cuda").normal_(0.2, 1.0, generator=g)
    gamma, beta = torch.linspace(0.5, 1.5, d, device="cuda").to(dtype), torch.linspace(-1, 1, d, device="cuda").to(dtype)
    out = vp.layer_norm(X, gamma, beta)
    rows = torch.cat([torch.arange(3), torch.arange(T // 2, T // 2 + 3), torch.arange(min(T, 2 ** 20) - 3, min(T, 2 ** 20 + 3)),
                      torch.arange(T - 3, T)]).cuda()
    _check_forward(X[rows], gamma, beta, 1e-5, False, [v[rows] for v in out])
    mean, rstd = out[1:]
    del out
    dY = torch.empty(T, d, device="cuda").normal_(0.0, 1.0, generator=g)
    dX, dgamma, dbeta = vp.layer_norm_backward(X, gamma, mean, rstd, dY)
    want, mag = torch.zeros(2, d, dtype=torch.float64, device="cuda"), torch.zeros(2, d, dtype=torch.float64, device="cuda")
    step = max(1, 2 ** 27 // d)
    for a in range(0, T, step):
        dy = dY[a:a + step].double()
        p = (X[a:a + step].double() - mean[a:a + step, None]) * rstd[a:a + step, None] * dy
        want += torch.stack([p.sum(0), dy.sum(0)])
        mag += torch.stack([p.abs().sum(0), dy.abs().sum(0)])
    # chains of at most 1024 rows of a lane, 32 rows side by side and 2^13 / 16 + 16 workgroups
    bound = (1024 + 32 + 528 + 4) * U * mag
    assert bool(((torch.stack([dgamma, dbeta]) - want).abs() <= bound).all())
    _check_backward(X[rows], gamma, mean[rows], rstd[rows], dY[rows], (dX[rows], None, None))


@pytest.mark.parametrize("T", [1, 300])
def test_captured_and_replayed(T):
    """Two graphs that share a workspace, replayed in turn with eager work between, on new inputs."""
    d = 1000
    X, gamma, beta, dY = _make(T, d, torch.bfloat16)
    norm = vp.Norm(T, d, vp.VP_BF16)
    ws = torch.empty(vp.vp_norm_workspace_size(norm), dtype=torch.uint8, device="cuda")
    f = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    out = [torch.empty_like(X), f(T), f(T)]
    grads = [[f(T, d), f(d), f(d)] for _ in range(2)]

    def run(k):
        vp.vp_norm_forward(norm, X, gamma, beta, *out)
        vp.vp_norm_backward(norm, X, gamma, out[1], out[2], dY, *grads[k], ws)

    run(0)
    graphs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for k in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run(k)
        graphs.append(graph)
    for step in range(3):
        X.copy_(_make(T, d, torch.bfloat16, seed=step + 1)[0])
        dY.mul_(-0.5)
        for k in range(2):
            graphs[k].replay()
            want = vp.layer_norm(X, gamma, beta)
            want_g = vp.layer_norm_backward(X, gamma, want[1], want[2], dY)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want))
            assert all(torch.equal(a, b) for a, b in zip(grads[k], want_g))


def test_another_stream():
    X, gamma, beta, dY = _make(500, 2880, torch.bfloat16)
    want = vp.layer_norm(X, gamma, beta)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = vp.layer_norm(X, gamma, beta)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
