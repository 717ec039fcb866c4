"""The norm with the residual's addition on the GPU.

The sum is one float32 addition and one rounding: compared bit for bit.  Its norm and gradients are
held to the bounds of test_gpu_norm.py (at the sum); dX gains one rounding of the sum with dS.  An 8-bit
value is y over its block's scale to the nearest: off by half a step of the value (2^-4) or of the
smallest step of the scale (2^-10), on top of what y may be off by; a scale may differ from that of the
exact y only where the largest magnitude lies within y's bound of a border."""
import pytest
import torch

import head_plain as hp
import paper_2609_14306_amd as vp
import score_plain as sp
from test_gpu_norm import DEPTH, SIZES, U, _check_backward, _check_forward, _make, _within

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


def make(T, d, dtype, bias, seed=0):
    X, gamma, beta, dY = _make(T, d, dtype, bias, seed)
    g = torch.Generator(device="cuda").manual_seed(T + d)
    R = (torch.randn(T, d, generator=g, device="cuda") * 2).to(dtype)
    return X, R, gamma, beta, dY


def check_f8(S, gamma, beta, rms, y8, scale):
    """8-bit rows against the float64 norm of S."""
    y, mu, r = hp.norm_forward(S, gamma, beta, 1e-5, rms)
    x, ga = S.double().cpu(), gamma.double().cpu().abs()
    e_mean = torch.zeros_like(mu) if rms else (DEPTH + 2) * U * x.abs().mean(1)
    e_r = (0.5 * (DEPTH + 4) + 3) * U + 0.5 * e_mean ** 2 * r ** 2
    xh = ((x - mu[:, None]) * r[:, None]).abs()
    b = 0.0 if beta is None else beta.double().cpu().abs()
    off = ga * ((r * e_mean)[:, None] + xh * (e_r + 6 * U)[:, None]) + 2 * U * (ga * xh + b)
    s = scale.double().cpu().repeat_interleave(128, 1)[:, :S.shape[1]]
    _within(sp.values(y8, scale, 1).cpu(), y, off * 1.1 + torch.maximum(y.abs() * 2.0 ** -4, s * 2.0 ** -10), "Y8")
    # scales: those of a largest magnitude within the bound
    T, d = S.shape
    pad = lambda v: torch.nn.functional.pad(v, (0, -d % 128)).view(T, -1, 128).amax(2)  # noqa: E731
    top, slack = pad(y.abs()), pad(off)
    k = scale.double().cpu()
    zero = top == 0
    assert bool((k[zero] == 1).all())
    assert bool(((top - slack <= 448 * k) & ((top + slack > 224 * k) | (k == 2.0 ** -127)))[~zero].all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("T, d", SIZES)
def test_against_float64(T, d, dtype, rms):
    bias = (T + d) % 3 != 0
    X, R, gamma, beta, dY = make(T, d, dtype, bias)
    S, Y, mean, rstd = vp.add_norm(X, R, gamma, beta, 1e-5, rms)
    assert torch.equal(S, (X.float() + R.float()).to(dtype))
    _check_forward(S, gamma, beta, 1e-5, rms, (Y, mean, rstd))
    S8, (y8, scale), mean8, rstd8 = vp.add_norm(X, R, gamma, beta, 1e-5, rms, f8=True)
    assert torch.equal(S8, S) and torch.equal(rstd8, rstd) and (rms or torch.equal(mean8, mean))
    check_f8(S, gamma, beta, rms, y8, scale)
    dS = torch.randn(T, d, device="cuda")
    dX, dgamma, dbeta = vp.add_norm_backward(S, gamma, mean, rstd, dY, dS, bias=bias)
    alone = vp.layer_norm_backward(S, gamma, mean, rstd, dY, bias=bias)
    _check_backward(S, gamma, mean, rstd, dY, alone)
    # dX = fl(p + dS) of a product p of which `alone` is fl(p), where the compiler joins product and
    # addition into one operation: two roundings of u between them
    p = alone[0].double()
    assert bool(((dX.double() - (p + dS.double())).abs() <= 1.01 * U * (p.abs() + dX.double().abs())).all())
    assert torch.equal(dgamma, alone[1]) and (not bias or torch.equal(dbeta, alone[2]))
    none = vp.add_norm_backward(S, gamma, mean, rstd, dY, None, bias=bias)
    assert torch.equal(none[0], alone[0])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, d", [(1, 64), (7, 2880), (300, 1000), (5, 16384)])
def test_in_place_and_both_results(T, d, dtype):
    X, R, gamma, beta, dY = make(T, d, dtype, True)
    S, Y, mean, rstd = vp.add_norm(X, R, gamma, beta)
    _, (y8, scale), _, _ = vp.add_norm(X, R, gamma, beta, f8=True)
    norm = vp.Norm(T, d, vp.VP_BF16 if dtype == torch.bfloat16 else vp.VP_F32)
    for target in (0, 1):
        xr = [X.clone(), R.clone()]
        Y2, m2, r2 = torch.empty_like(X), torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        z8, k = vp.f8_buffers(T, d, 1, "cuda")
        vp.vp_add_norm_forward(norm, xr[0], xr[1], gamma, beta, xr[target], Y2, z8, k, m2, r2)
        assert torch.equal(xr[target], S) and torch.equal(xr[1 - target], (X, R)[1 - target])
        assert torch.equal(Y2, Y) and torch.equal(m2, mean) and torch.equal(r2, rstd)
        assert torch.equal(z8.view(torch.uint8), y8.view(torch.uint8)) and torch.equal(k.view(torch.uint8), scale.view(torch.uint8))
    dS = torch.randn(T, d, device="cuda")
    want = vp.add_norm_backward(S, gamma, mean, rstd, dY, dS)
    for buf in (0, 1):
        io = [dY.clone(), dS.clone()]
        got = vp.add_norm_backward(S, gamma, mean, rstd, io[0], io[1], dX=io[buf])
        assert got[0] is io[buf] and all(torch.equal(a, b) for a, b in zip(got, want))
    base = torch.randn(2, d, device="cuda")
    acc = [b.clone() for b in base]
    vp.add_norm_backward(S, gamma, mean, rstd, dY, dS, dgamma=acc[0], dbeta=acc[1], accumulate=True)
    for a, b, w in zip(acc, base, want[1:]):
        assert bool(((a - b - w).abs() <= 4 * U * (a.abs() + b.abs() + w.abs())).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, d", [(1, 64), (3, 64), (30, 264), (513, 1000)])
def test_gradients_against_differences(T, d, dtype):
    """The gradient along one direction against a central difference of the plain float64 forward."""
    X, R, gamma, beta, dY = make(T, d, dtype, True, seed=3)
    S, Y, mean, rstd = vp.add_norm(X, R, gamma, beta)
    dS = torch.randn(T, d, device="cuda")
    dX, dgamma, dbeta = vp.add_norm_backward(S, gamma, mean, rstd, dY, dS)
    to, h = torch.randn(T, d, dtype=torch.float64), 1e-4
    f = lambda x: (hp.norm_forward(x, gamma, beta, 1e-5, False)[0] * dY.double().cpu()).sum() + (x.double().cpu() * dS.double().cpu()).sum()  # noqa: E731
    diff = ((f(S.double().cpu() + h * to) - f(S.double().cpu() - h * to)) / (2 * h)).item()
    along = (dX.double().cpu() * to).sum().item()
    size = (dX.double().cpu().abs() * to.abs()).sum().item()
    # the difference's own error is h^2 of third derivatives (a row's spread is above 0.5), 1e-6 of the size
    assert abs(diff - along) <= 1e-5 * size


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_apart(dtype):
    """NaN and infinite rows, rows of zeros and constant rows; every other row as without them."""
    X, R, gamma, beta, _ = make(40, 520, dtype, False)
    clean = vp.add_norm(X, R, gamma, None, rms=True, f8=True)
    X[3, 5], R[7, 9] = torch.nan, torch.inf
    X[11], R[11] = 0.0, 0.0
    X[12] = -R[12]
    out = vp.add_norm(X, R, gamma, None, rms=True, f8=True)
    rest = [i for i in range(40) if i not in (3, 7, 11, 12)]
    for a, b in ((clean[0], out[0]), (clean[1][0].view(torch.uint8), out[1][0].view(torch.uint8)),
                 (clean[1][1].view(torch.uint8), out[1][1].view(torch.uint8)), (clean[3], out[3])):
        assert torch.equal(a[rest], b[rest])
    v, k = out[1][0].float(), out[1][1].float()
    assert bool(v[3].isnan().all()) and bool(v[7, 9].isnan())
    assert bool((v[11:13] == 0).all()) and bool((k[11:13] == 1).all())


def test_no_rows_many_rows_and_streams():
    e = torch.empty(0, 64, device="cuda")
    S, (y8, k), mean, rstd = vp.add_norm(e, e, torch.ones(64, device="cuda"), f8=True)
    assert S.shape == y8.shape == (0, 64) and k.shape == (0, 1) and rstd.shape == (0,)
    X, R, gamma, beta, dY = make(30001, 136, torch.bfloat16, True)
    S, (y8, k), mean, rstd = vp.add_norm(X, R, gamma, beta, f8=True)
    check_f8(S, gamma, beta, False, y8, k)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        T2 = vp.add_norm(X, R, gamma, beta, f8=True)
    s.synchronize()
    assert torch.equal(T2[1][0].view(torch.uint8), y8.view(torch.uint8))


def test_graph():
    X, R, gamma, beta, dY = make(900, 1000, torch.bfloat16, True)
    norm = vp.Norm(900, 1000, vp.VP_BF16)
    S, mean, rstd = torch.empty_like(X), torch.empty(900, device="cuda"), torch.empty(900, device="cuda")
    y8, k = vp.f8_buffers(900, 1000, 1, "cuda")
    dS, dX = torch.randn(900, 1000, device="cuda"), torch.empty(900, 1000, device="cuda")
    dg, db = torch.empty(1000, device="cuda"), torch.empty(1000, device="cuda")
    ws = torch.empty(vp.vp_norm_workspace_size(norm), dtype=torch.uint8, device="cuda")

    def run():
        vp.vp_add_norm_forward(norm, X, R, gamma, beta, S, None, y8, k, mean, rstd)
        vp.vp_add_norm_backward(norm, S, gamma, mean, rstd, dY, dS, dX, dg, db, ws)

    outs = [S, y8.view(torch.uint8), k.view(torch.uint8), dX, dg, db]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        vp.add_norm(X[:5], R[:5], gamma)
        torch.cuda.synchronize()
