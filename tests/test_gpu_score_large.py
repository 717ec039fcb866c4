"""Scoring, quantisation and the norm with a residual on operands of more than 2^32 bytes and of more than
2^31 elements, where a 32-bit offset would wrap to other rows, and two calls at once on two streams."""
import pytest
import torch

import paper_2609_14306_amd as vp
import score_plain as sp

pytestmark = pytest.mark.gpu
U = sp.U
D = 2048


def gauss(*shape, seed, scale=1.0, dtype=torch.bfloat16):
    """Normal numbers, 64 Ki rows at a time."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.empty(*shape, dtype=dtype, device="cuda")
    for a in range(0, shape[0], 1 << 16):
        part = out[a:a + (1 << 16)]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * scale)
    return out


def logits64(H, rows_of, V):
    """Float64 logits [T, V] of float64 H, with W's rows a .. b given by rows_of(a, b), and max_v sum |h w|."""
    y, most = torch.empty(H.shape[0], V, dtype=torch.float64, device="cuda"), torch.zeros(H.shape[0], device="cuda").double()
    for a in range(0, V, 1 << 16):
        b = min(V, a + (1 << 16))
        w = rows_of(a, b).double()
        y[:, a:b] = H @ w.t().contiguous()
        most = torch.maximum(most, (H.abs() @ w.abs().t().contiguous()).amax(1))
    return y, most


def held(out, y, most, t, unit, top):
    """Against float64 logits: ids exactly, the rest within the bounds of test_gpu_score (unit: what a
    product's sum may be off by, of sum |h w|)."""
    loss, lse, entropy, ids, top_loss = out
    V = y.shape[1]
    want = torch.logsumexp(y, 1)
    b = unit * most + sp.fold_bound(V) + 2 * U * want.abs()
    p = (y - want[:, None]).exp()
    S = -(p * (y - want[:, None])).sum(1)
    assert bool(((lse.double() - want).abs() <= b).all())
    wl = want - y.gather(1, t[:, None])[:, 0]
    assert bool(((loss.double() - wl).abs() <= b + U * wl.abs()).all())
    assert bool(((entropy.double() - S).abs() <= 2 * unit * most * (S + 1) + (2 * sp.fold_bound(V) + 8 * U) * (S + 1) + 8 * U).all())
    order = torch.sort(y, dim=1, descending=True, stable=True)
    assert torch.equal(ids, order.indices[:, :top])
    wt = want[:, None] - order.values[:, :top]
    assert bool(((top_loss.double() - wt).abs() <= b[:, None] + U * wt.abs()).all())


@pytest.mark.parametrize("dtype, V", [(torch.bfloat16, 1_100_003), (torch.float32, 560_001)])
@pytest.mark.parametrize("T", [3, 300])
def test_weights_past_4_gib(dtype, V, T):
    W = gauss(V, D, seed=1, scale=D ** -0.5, dtype=dtype)
    assert W.numel() * W.element_size() > 1 << 32
    H = gauss(T, D, seed=2, scale=2.0, dtype=dtype)
    W[-1] = H[0] / 8  # the last id is the most likely one of a token, and another token's target
    t = torch.arange(T, device="cuda") * 17
    t[1] = V - 1
    t[2] = V - 70_000
    out = vp.score(H, [W], t, top=4)
    y, most = logits64(H[:40].double(), lambda a, b: W[a:b], V)
    held([x[:40] for x in out], y, most, t[:40], (D + 2) * U, 4)
    assert int(out[3][0, 0]) == V - 1


@pytest.mark.parametrize("T", [3, 100, 300])
def test_8_bit_weights_past_4_gib(T):
    V = 2_150_001
    g = torch.Generator(device="cuda").manual_seed(3)
    W8, scale = vp.f8_buffers(V, D, 128, "cuda")
    assert W8.numel() > 1 << 32
    step = 128 << 9
    for a in range(0, V, step):
        x = torch.randn(min(step, V - a), D, generator=g, device="cuda") * D ** -0.5
        w, s = vp.quantize(x, 128)
        W8.view(torch.uint8)[a:a + step].copy_(w.view(torch.uint8))
        scale.view(torch.uint8)[a // 128:(a + step) // 128].copy_(s.view(torch.uint8))
    H8, hs = vp.quantize(gauss(T, D, seed=4, scale=2.0))
    t = torch.arange(T, device="cuda") * 17
    t[1] = V - 1
    out = vp.score_f8(H8, hs, [W8], [scale], t, top=4)

    def rebuilt(v, s, per):
        e = torch.exp2(s.view(torch.uint8).double() - 127)
        return v.float().double() * e.repeat_interleave(per, 0)[:v.shape[0]].repeat_interleave(128, 1)

    H64 = rebuilt(H8[:40], hs[:40], 1)
    # (65536 rows a time: whole blocks)
    y, most = logits64(H64, lambda a, b: rebuilt(W8[a:b], scale[a // 128:-(-b // 128)], 128), V)
    # every product of eight may lose 2^-13 of the largest, which is no more than their sum: 2^-13 of sum |h w|
    # for each of the seven others, and float32 sums on top
    held([x[:40] for x in out], y, most, t[:40], 7 * 2.0 ** -13 + (D + 2) * U, 4)


def test_hidden_states_past_4_gib():
    T = 1_060_000
    H = gauss(T, D, seed=5)
    assert H.numel() * 2 > 1 << 32
    W = [gauss(40, D, seed=6, scale=D ** -0.5), gauss(25, D, seed=7, scale=D ** -0.5)]
    t = torch.arange(T, device="cuda") % 65
    out = vp.score(H, W, t, top=2)
    near = slice(T - 300, T)
    y, most = logits64(H[near].double(), lambda a, b: torch.cat(W)[a:b], 65)
    held([x[near] for x in out], y, most, t[near], (D + 2) * U, 2)


def test_quantise_and_add_norm_past_2_31_elements():
    T = 1_060_000
    X = gauss(T, D, seed=8)
    assert X.numel() > 1 << 31
    tail = slice(T - T % 128 - 256, T)
    for per in (1, 128):
        x8, s = vp.quantize(X, per)
        y8, z = vp.quantize(X[tail].clone(), per)
        assert torch.equal(x8[tail].view(torch.uint8), y8.view(torch.uint8))
        assert torch.equal(s[tail.start // per:].view(torch.uint8), z.view(torch.uint8))
        del x8, s
    R, gamma = gauss(T, D, seed=9), torch.linspace(0.5, 1.5, D, device="cuda").bfloat16()
    S, (Y8, scale), _, rstd = vp.add_norm(X, R, gamma, rms=True, f8=True)
    s2, (y8, z), _, r2 = vp.add_norm(X[tail].clone(), R[tail].clone(), gamma, rms=True, f8=True)
    assert torch.equal(S[tail], s2) and torch.equal(rstd[tail], r2)
    assert torch.equal(Y8[tail].view(torch.uint8), y8.view(torch.uint8)) and torch.equal(scale[tail].view(torch.uint8), z.view(torch.uint8))


def test_two_calls_at_once():
    """The same problem's calls on two streams, with a workspace each, between and over each other."""
    T, V = 200, 30_000
    H = [gauss(T, 512, seed=10 + i, scale=2.0) for i in range(2)]
    W = [gauss(V, 512, seed=12, scale=512 ** -0.5)]
    t = torch.arange(T, device="cuda")
    want = [vp.score(h, W, t, top=3) for h in H]
    prob, sc = vp.problem_for(H[0], W), vp.Score(3)
    ws = [torch.empty(vp.vp_score_workspace_size(prob, sc), dtype=torch.uint8, device="cuda") for _ in H]
    outs = [[torch.empty_like(x) for x in want[0]] for _ in H]
    streams = [torch.cuda.Stream() for _ in H]
    torch.cuda.synchronize()
    for _ in range(8):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                vp.vp_score_forward(prob, sc, H[i], W, t, *outs[i], ws[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i]))
