"""8-bit operands on the GPU: quantisation value for value against the plain form, and scoring of
such operands against float64 of the values that they stand for.

The matrix unit cuts eight products at a time off at 2^-13 of the largest one's power of two, i.e. each of
the seven others by less than 2^-13 of the largest: no more than 7 2^-13 of the eight magnitudes' sum. So a
logit is held to (7 2^-13 + (d + 2) u) sum |h w| (float32 sums alone, (d + 2) u, hold it only where many
products or ids average that out).  loss and top_loss have float64 logits, so only lse's error enters."""
import pytest
import torch

import paper_2609_14306_amd as vp
import score_plain as sp
from test_gpu_score import check

pytestmark = pytest.mark.gpu


def rebuilt(X, rps):
    x8, scale = vp.quantize(X, rps)
    return x8, scale, x8.double().cpu(), torch.log2(scale.double()).cpu()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rps", [1, 128])
@pytest.mark.parametrize("rows, cols", [(1, 16), (1, 4096), (3, 112), (127, 128), (128, 144), (129, 272), (300, 1008),
                                        (33, 16400), (260, 384)])
def test_quantize_value_for_value(rows, cols, rps, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    X = torch.randn(rows, cols, generator=g, device="cuda") * torch.exp2(
        torch.randint(-12, 12, (rows, cols), generator=g, device="cuda").float())
    X = X.to(dtype)
    _, _, v, e = rebuilt(X, rps)
    want, exps = sp.quantize(X.cpu(), rps)
    assert torch.equal(e, exps) and torch.equal(v, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rps", [1, 128])
def test_quantize_borders(rps, dtype):
    """Largest magnitudes at and next to 448 times a power of two, every value of the 8-bit grid with
    the halves between them, zeros, tiny and huge numbers, NaN and infinities."""
    one = torch.tensor(1.0, dtype=dtype)
    up = torch.nextafter(448 * one, torch.tensor(torch.inf, dtype=dtype)).item()
    down = torch.nextafter(448 * one, -one).item()
    grid = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    grid = grid[grid.isfinite() & (grid >= 0)].sort().values.unique()
    half = (grid[1:] + grid[:-1]) / 2
    rows = [[448.0], [up], [down], [448 * 2.0 ** 40], [up * 2.0 ** -60], [0.0], [2.0 ** -126, -2.0 ** -130], [3e38, -1e30, 5.0],
            [torch.nan, 1.0, 700.0], [torch.inf, 3.0, -900.0], [-torch.inf] * 3, [torch.nan], [448.0] + half.tolist()[:60],
            [448.0] + half.tolist()[60:], [-448.0] + (-grid).tolist()[:100], [2.0 ** -149], [1.0, 2.0 ** -10, -2.0 ** -10, 2.0 ** -9 * 1.5]]
    X = torch.zeros(len(rows), 256)
    for i, r in enumerate(rows):
        X[i, 128:128 + len(r)] = torch.tensor(r)
    X = X.to(dtype).repeat_interleave(rps, 0)  # (blocks of as many equal rows)
    _, _, v, e = rebuilt(X.cuda(), rps)
    want, exps = sp.quantize(X, rps)
    assert torch.equal(e, exps), (e - exps).nonzero()
    assert torch.equal(v.isnan(), want.isnan())
    assert torch.equal(v.nan_to_num(), want.nan_to_num())


def test_quantize_many_blocks_and_no_rows():
    X = torch.randn(70001, 80, device="cuda")
    x8, scale = vp.quantize(X)
    err = (sp.values(x8, scale, 1) - X.double()).abs()
    # half a step of the value, or of the smallest step 2^-9 of its block's scale
    assert bool((err <= torch.maximum(X.double().abs() * 2.0 ** -4, scale.double() * 2.0 ** -10)).all())
    x8, scale = vp.quantize(X[:0], 128)
    assert x8.shape == (0, 80) and scale.shape == (0, 1)


# ---------------------------------------------------------------------------
def make(T, d, rows, seed=0, spread=2.0):
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + 13 * T + d)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    wide = torch.exp2(spread * n(d))  # scales that differ from block to block
    H, Hs = vp.quantize(2.0 * n(T, d) * wide, 1)
    W, Ws = map(list, zip(*[vp.quantize(n(r, d) / d ** 0.5 / wide, 128) for r in rows]))
    t = torch.randint(0, sum(rows), (T,), generator=g, device="cuda")
    t[::7] = -100
    return H, Hs, W, Ws, t


def check_f8(H, Hs, W, Ws, t, got, top, ignore=-100):
    check(sp.values(H, Hs, 1), [sp.values(w, s, 128) for w, s in zip(W, Ws)], t, got, top, ignore,
          product=7 * 2.0 ** -13)


@pytest.mark.parametrize("T", [300, 2100])
@pytest.mark.parametrize("d", [16, 64, 112, 512, 4096])
def test_rounding_of_a_single_sum(T, d):
    """With one id lse is its logit: the sum of the products as the matrix unit rounds it, 1.5e-5 of the sums'
    root mean square (held to twice that), on the small tiles and the large one."""
    H, Hs, W, Ws, t = make(T, d, [1], spread=0.0)
    lse = vp.score_f8(H, Hs, W, Ws, t)[1].double()
    h, w = sp.values(H, Hs, 1), sp.values(W[0], Ws[0], 128)
    y = (h @ w.t().contiguous())[:, 0]
    assert bool(((lse - y).abs() <= (7 * 2.0 ** -13 + (d + 2) * sp.U) * (h.abs() @ w.abs().t().contiguous())[:, 0]).all())
    assert float((lse - y).square().mean().sqrt()) <= 3e-5 * float((h.square() @ w.square().t().contiguous()).mean().sqrt())


@pytest.mark.parametrize("top", [0, 1, 20])
@pytest.mark.parametrize("T, d, rows", [
    (1, 16, [1]), (1, 4096, [3001]), (3, 128, [127, 129, 0, 256]), (40, 2880, [700, 4097]), (64, 112, [300]),
    (65, 272, [1000]), (300, 640, [255, 3000]), (2100, 256, [1000, 513]), (2300, 400, [2001]), (2600, 1040, [1333, 4003]),
    (2049, 128, [256]), (2500, 384, [300, 5, 128, 129, 640]),
    # the tile of 128 tokens
    (100, 14336, [3001, 0, 500]), (128, 272, [40000]), (90, 1040, [20001, 127, 30000]), (127, 144, [60000])])
def test_score_of_8_bit_operands(T, d, rows, top):
    ops = make(T, d, rows, seed=top)
    check_f8(*ops, vp.score_f8(*ops, top=top), top)


def test_widest_rows():
    ops = make(2100, 14336, [300, 513], spread=1.0)
    check_f8(*ops, vp.score_f8(*ops, top=3), 3)
    ops = make(20, 14336, [30000], spread=1.0)  # (more tiles a workgroup than their scales have room for)
    check_f8(*ops, vp.score_f8(*ops, top=3), 3)


def test_many_tiles_a_workgroup():
    """Scales of a workgroup's vocabulary tiles are loaded some tiles at a time."""
    for T, d, V in [(2100, 14336, 6400), (2100, 2048, 80000), (10, 1024, 400000)]:
        ops = make(T, d, [V], spread=0.5)
        H, Hs, W, Ws, t = ops
        out = vp.score_f8(*ops, top=2)
        pick = torch.arange(0, T, max(1, T // 64), device="cuda")
        check_f8(H.view(torch.uint8)[pick].view(torch.float8_e4m3fn), Hs.view(torch.uint8)[pick].view(torch.float8_e8m0fnu),
                 W, Ws, t[pick], [o[pick] for o in out], 2)


@pytest.mark.parametrize("T", [7, 2100])
def test_nan_values_and_scales(T):
    H, Hs, W, Ws, t = make(T, 256, [700])
    clean = vp.score_f8(H, Hs, W, Ws, t, top=2)
    H.view(torch.uint8)[1, 3] = 0x7f
    Hs.view(torch.uint8)[4, 1] = 255
    out = vp.score_f8(H, Hs, W, Ws, t, top=2)
    for r in (1, 4):
        assert out[1][r].isnan() and out[2][r].isnan() and bool((out[3][r] == -1).all())
    rest = [i for i in range(T) if i not in (1, 4)]
    assert all(torch.equal(a[rest], b[rest]) for a, b in zip(clean, out))


def test_extreme_scales():
    """Blocks with scales of 2^-60 beside ones of 2^60, and products in between."""
    H, Hs, W, Ws, t = make(70, 512, [600], spread=0.0)
    Hs.view(torch.uint8)[:, 1] += 60
    Ws[0].view(torch.uint8)[:, 1] -= 60
    Hs.view(torch.uint8)[:, 2] -= 100
    Ws[0].view(torch.uint8)[:, 2] += 101
    Hs.view(torch.uint8)[:, 3], Ws[0].view(torch.uint8)[:, 3] = 0, 250  # 2^-127 and 2^123
    Hs.view(torch.uint8)[5, 3], Hs.view(torch.uint8)[6, 3] = 4, 8
    ops = (H, Hs, W, Ws, t)
    check_f8(*ops, vp.score_f8(*ops, top=4), 4)


def test_graph():
    ops = make(300, 640, [1000, 700])
    prob, sc = vp.Problem(300, 640, [1000, 700], vp.VP_E4M3), vp.Score(4)
    ws = torch.empty(vp.vp_score_workspace_size(prob, sc), dtype=torch.uint8, device="cuda")
    out = [torch.empty(300, device="cuda") for _ in range(3)]
    out += [torch.empty(300, 4, dtype=torch.int64, device="cuda"), torch.empty(300, 4, device="cuda")]
    X = torch.randn(300, 640, device="cuda")
    q, x8 = vp.Quant(300, 640, vp.VP_F32), vp.f8_buffers(300, 640, 1, "cuda")

    def run():
        vp.vp_f8_quantize(q, X, *x8)
        vp.vp_score_forward_f8(prob, sc, *x8, *ops[2:4], ops[4], *out, ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    want = [o.clone() for o in out]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for o in out:
            o.zero_()
        x8[0].view(torch.uint8).zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        vp.score_f8(*make(33, 128, [500]), top=1)
        torch.cuda.synchronize()


@pytest.mark.parametrize("top", [0, 1, 8])
@pytest.mark.parametrize("T, d, rows", [(1, 96, [527]), (7, 464, [9000, 772]), (90, 512, [3000]), (600, 128, [20000, 6264]),
                                        (2200, 512, [6000])])
def test_likely_ids_have_their_exact_logits(T, d, rows, top):
    """Logits of spread 4, where few ids hold the probability.  What is left of the matrix unit's rounding are
    the ids below 2^-7 and the ones that are not the largest of their four.  Their logits are off by e, 3e-5 of
    the sums' root mean square at most (test_rounding_of_a_single_sum), independently: lse by e sqrt(sum p^2) and
    the entropy by e sqrt(sum p^2 (log p + S)^2), as root mean squares over the tokens.  Held to four of these,
    and float32 roundings: 4 u of lse, and 4 u of lse + 1 in the entropy, whose terms are log p."""
    H, Hs, W, Ws, t = make(T, d, rows, seed=5, spread=0.0)
    Hs.view(torch.uint8).add_(1)  # twice the make's 2
    got = vp.score_f8(H, Hs, W, Ws, t, top=top)
    h, w = sp.values(H, Hs, 1), torch.cat([sp.values(a, b, 128) for a, b in zip(W, Ws)])
    want = sp.score(h, w, t, -100, top)
    y, lse, S = want[5], want[1], want[2]
    exact = torch.zeros_like(y, dtype=torch.bool)
    at = 0
    for r in rows:
        four = torch.nn.functional.pad(y[:, at:at + r], (0, -r % 4), value=-torch.inf).view(T, -1, 4)
        exact[:, at:at + r] = (four == four.amax(2, keepdim=True)).view(T, -1)[:, :r]
        at += r
    logp = y - lse[:, None]
    p = torch.where(exact & (logp > -7 * 0.6931), 0.0, logp.exp())
    e = 3e-5 * (h.square() @ w.square().t().contiguous()).mean(1).sqrt()
    rms = lambda v: float(v.square().mean().sqrt())  # noqa: E731
    left = 4 * rms(e * p.square().sum(1).sqrt())
    assert rms(got[1].double() - lse) <= left + 4 * sp.U * rms(lse)
    left = 4 * rms(e * (p * (logp + S[:, None])).square().sum(1).sqrt())
    assert rms(got[2].double() - S) <= left + 4 * sp.U * rms(lse + 1)
    if top:
        assert torch.equal(got[3], want[3])
