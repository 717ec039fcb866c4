"""Scoring on the GPU against the plain float64 form: loss, lse, entropy and alternatives, on every
tile, in bfloat16 and float32, and what the calls do with masked rows, ties, NaN and missing targets.

Bounds (score_plain): a float32 logit is off by at most e_y = (d + 2) u max_v sum_k |h_k w_k|; the
sum of V exponentials by e_s = (V / 2 + 80) u relative.  lse: e_y + e_s + 2 u |lse|.  loss and
top_loss: that, as the logit itself is a float64 one rounded with the result.  The entropy is
sum p (-log p): logits off by e_y change it by at most e_y sum p |log p + S| <= 2 e_y S, its two sums
by e_s of themselves and of S, each term is the product of an exponential (2 u of |x| + 2) and x.
"""
import pytest
import torch

import paper_2609_14306_amd as vp
import score_plain as sp
import tile_cases

pytestmark = pytest.mark.gpu
U = sp.U
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(dtype, T, d, rows, seed=0, scale=2.0):
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + 13 * T + d)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    H = (scale * n(T, d)).to(DT[dtype])
    W = [(n(r, d) / d ** 0.5).to(DT[dtype]) for r in rows]
    t = torch.randint(0, sum(rows), (T,), generator=g, device="cuda")
    t[::7] = -100
    return H, W, t


def check(H, W, t, got, top, ignore=-100, exact_ids=True, product=0.0):
    """got: (loss, lse, entropy, ids, top_loss) against float64, 512 tokens at a time.  product: what the
    products lose before they are summed, of sum_k |h_k w_k|."""
    loss, lse, entropy, ids, top_loss = got
    W64 = torch.cat(W).double()
    V = W64.shape[0]
    for a in range(0, H.shape[0], 512):
        s = slice(a, a + 512)
        H64 = H[s].double()
        want = sp.score(H64, W64, t[s], ignore, top)
        e_y = sp.logit_bound(H64, W64) * (1 + product / ((H64.shape[1] + 2) * U))
        b = e_y + sp.fold_bound(V) + 2 * U * want[1].abs()

        def within(x, y, bound, what):
            assert torch.equal(x.isnan(), y.isnan()), what
            err = (x.double() - y).abs()
            ok = (err <= bound) | y.isnan() | (x.double() == y)
            assert bool(ok.all()), (what, a, err[~ok][:4], bound.expand_as(err)[~ok][:4])

        within(lse[s], want[1], b, "lse")
        within(loss[s], want[0], b + U * want[0].abs(), "loss")
        S = want[2]
        within(entropy[s], S, 2 * e_y * (S + 1) + (2 * sp.fold_bound(V) + 8 * U) * (S + 1) + 8 * U,
               "entropy")
        assert bool((loss[s][t[s] == ignore] == 0).all())
        if top:
            k = min(top, V)
            if exact_ids:
                assert torch.equal(ids[s, :k], want[3]), (a, (ids[s, :k] != want[3]).nonzero()[:4])
            within(top_loss[s, :k], want[4], b[:, None] + U * want[4].abs(), "top_loss")
            assert bool((ids[s, k:] == -1).all()) and bool((top_loss[s, k:] == torch.inf).all())


@pytest.mark.parametrize("kind, dtype, T, d, rows", [(c[0],) + c[2:] for c in tile_cases.FORWARD])
def test_every_tile(kind, dtype, T, d, rows):
    H, W, t = make(dtype, T, d, rows)
    check(H, W, t, vp.score(H, W, t, top=8), 8)
    check(H, W, t, vp.score(H, W, t), 0)


SIZES = [("bf16", 1, 8, [1]), ("bf16", 1, 4096, [3001]), ("f32", 1, 72, [5, 0, 4]), ("bf16", 3, 64, [255, 256, 257]),
         ("f32", 64, 520, [1000]), ("bf16", 65, 200, [33] * 11), ("f32", 2300, 200, [1000, 513]),
         ("bf16", 2300, 64, [1000, 0, 2001]), ("bf16", 2600, 1000, [1333, 4003]), ("bf16", 300, 16, [4, 3, 2, 1]),
         # float32's tiles: 128 x 128, 128 x 64 and 128 x 32
         ("f32", 700, 200, [5000, 3001, 9]), ("f32", 100, 72, [20001, 5, 30000]), ("f32", 1100, 40, [12000, 5001]),
         ("f32", 1030, 72, [5000, 3001, 9]), ("f32", 64, 1000, [60000, 300]), ("f32", 20, 1000, [3001, 0, 129]),
         ("f32", 33, 104, [20001, 127]), ("f32", 32, 2880, [128, 70001])]


@pytest.mark.parametrize("top", [1, 5, 32])
@pytest.mark.parametrize("dtype, T, d, rows", SIZES)
def test_sizes(dtype, T, d, rows, top):
    H, W, t = make(dtype, T, d, rows, seed=top)
    check(H, W, t, vp.score(H, W, t, top=top), top)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [40, 2100])
def test_peaked_and_flat(dtype, T):
    """Distributions of nearly one id (entropy near 0) and of all of them (log V)."""
    H, W, t = make(dtype, T, 128, [700, 900], scale=60.0)
    check(H, W, t, vp.score(H, W, t, top=4), 4)
    H.zero_()
    out = vp.score(H, W, t, top=4)
    check(H, W, t, out, 4)
    assert torch.equal(out[3], torch.arange(4, device="cuda").expand(T, 4))


@pytest.mark.parametrize("T, V", [(1, 5000), (40, 40000), (2100, 9000)])
def test_equal_logits_go_to_the_lowest_ids(T, V):
    """Every logit is the same, or one of two values in long runs: ids from the front."""
    H = torch.ones(T, 64, dtype=torch.bfloat16, device="cuda")
    W = [torch.ones(V // 2, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(V - V // 2, 64, dtype=torch.bfloat16, device="cuda")]
    t = torch.full((T,), -100, dtype=torch.int64, device="cuda")
    out = vp.score(H, W, t, top=32)
    assert torch.equal(out[3], torch.arange(32, device="cuda").expand(T, 32))
    check(H, W, t, out, 32)
    W[0][:100] = 0.5
    W[1][3:9] = 2.0
    out = vp.score(H, W, t, top=32)
    first = V // 2 + torch.arange(3, 9, device="cuda")
    assert torch.equal(out[3], torch.cat([first, torch.arange(100, 126, device="cuda")]).expand(T, 32))


@pytest.mark.parametrize("T, V", [(3, 151936), (700, 30000)])
def test_tokens_of_zeros_and_few_distinct_logits(T, V):
    """Padding tokens (all logits 0) among others, and vocabularies with long runs of equal rows above,
    at and below the border."""
    H, W, t = make("bf16", T, 64, [V // 2, V - V // 2])
    H[::2] = 0.0
    check(H, W, t, vp.score(H, W, t, top=20), 20)
    for lo, hi, k in [(100, 20000, 3.0), (V // 2 - 60, V // 2, 5.0), (V // 2 - 3000, V // 2 - 2999, 9.0)]:
        W[0][lo:hi] = 0.0
        W[0][lo:hi, 0] = k
    H[:, 0] = 1.0
    check(H, W, t, vp.score(H, W, t, top=32), 32)


def test_large_logits_in_few_shares():
    """More logits above the first threshold than the lists take: every 64th tile's are large."""
    V = 64 * 1024
    H = torch.randn(600, 64, device="cuda")
    H[:, 0] = 40.0
    W = torch.randn(V, 64, device="cuda") / 8
    for tile in (128, 256):
        w = W.clone()
        w[:, 0] = (torch.arange(V, device="cuda") // tile % 64 < 3).float()
        t = torch.zeros(600, dtype=torch.int64, device="cuda")
        check(H, [w], t, vp.score(H, [w], t, top=8), 8)
        check(H[:9], [w], t[:9], vp.score(H[:9], [w], t[:9], top=8), 8)


@pytest.mark.parametrize("T", [1, 600, 2100])
@pytest.mark.parametrize("top", [1, 4, 32])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_closer_than_float32_holds(dtype, top, T):
    """Fifty ids with logits of 100 + k 2^-25, which no float32 sum tells apart, in scrambled order among
    others below 20: exact logits decide."""
    g = torch.Generator().manual_seed(top)
    d, rows, n = 64, [3000, 5000], 50
    H = torch.randn(T, d, generator=g).cuda()
    H[:, 0], H[:, 1] = 1.0, 2.0 ** -12
    W = torch.randn(sum(rows), d, generator=g).cuda() / d ** 0.5
    W[:, :2] = 0
    at = (torch.randperm(sum(rows) // 8, generator=g)[:n] * 8 + 3).cuda()  # groups of their own
    W[at] = 0
    W[at, 0] = 100.0
    W[at, 1] = torch.arange(n, device="cuda") * 2.0 ** -13
    H, W = H.to(DT[dtype]), W.to(DT[dtype])
    t = torch.zeros(T, dtype=torch.int64, device="cuda")
    out = vp.score(H, list(W.split(rows)), t, top=top)
    assert torch.equal(out[3], at.flip(0)[:top].expand(T, top))
    check(H, list(W.split(rows)), t, out, top)


def test_repeated_rows():
    """The same row under several ids, in several shards: the lower id first."""
    H, W, t = make("bf16", 300, 256, [600, 700, 800])
    for a, b in [((0, 17), (1, 400)), ((0, 17), (2, 5)), ((1, 3), (2, 799)), ((2, 100), (2, 101))]:
        W[b[0]][b[1]] = W[a[0]][a[1]]
    H[:100] = 8 * W[0][17]
    H[100:200] = 8 * W[1][3]
    H[200:] = 8 * W[2][100]
    check(H, W, t, vp.score(H, W, t, top=6), 6)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", ["inf", "lowest"])
@pytest.mark.parametrize("T", [1, 40, 300, 2100])
def test_masked_rows(dtype, value, T):
    """Vocabulary rows switched off by a last weight of minus infinity or the type's lowest value."""
    H, W, t = make(dtype, T, 128, [512, 300, 1100])
    H[:, -1] = 1.0
    low = -torch.inf if value == "inf" else torch.finfo(H.dtype).min
    off = torch.zeros(1912, dtype=torch.bool, device="cuda")
    off[0:64] = off[512:812] = off[1900:] = True
    t[:] = 100
    for w, m in zip(W, off.split([512, 300, 1100])):
        w[m] = 0.0
        w[m, -1] = low
    live = (~off).nonzero()[:, 0]
    W64 = torch.cat(W).double()[live]
    out = vp.score(H, W, t, top=8)
    want = sp.score(H.double(), W64, torch.full_like(t, 36), -100, 8)
    b = sp.logit_bound(H.double(), W64) + sp.fold_bound(1912) + 30 * U
    assert bool(((out[0].double() - want[0]).abs() <= 2 * b).all())
    assert bool(((out[2].double() - want[2]).abs() <= 2 * (b + 8 * U) * (want[2] + 1)).all())
    assert torch.equal(out[3], live[want[3]])
    # fewer live ids than asked for: the masked ones follow, lowest first, with infinite loss
    for w in W:
        w[:] = 0.0
        w[:, -1] = -torch.inf
    W[1][7] = W[2][9] = 0.0
    out = vp.score(H, W, t, top=8)
    ids = torch.tensor([519, 821, 0, 1, 2, 3, 4, 5], device="cuda")
    assert torch.equal(out[3], ids.expand(T, 8))
    assert bool((out[4][:, 2:] == torch.inf).all()) and bool(((out[4][:, :2] - 0.6931472).abs() < 1e-6).all())
    assert bool(((out[2] - 0.6931472).abs() < 1e-6).all())
    # none live
    W[1][7, -1] = W[2][9, -1] = -torch.inf
    out = vp.score(H, W, t, top=2)
    assert bool((out[3] == -1).all()) and bool(out[2].isnan().all()) and bool(out[4].isnan().all())


@pytest.mark.parametrize("T", [5, 300, 2100])
def test_tokens_of_nan_and_infinities_stand_apart(T):
    H, W, t = make("bf16", T, 200, [1000, 300])
    clean = vp.score(H, W, t, top=3)
    H[1, 5], H[3, 7] = torch.nan, torch.inf
    out = vp.score(H, W, t, top=3)
    for r in (1, 3):
        assert out[2][r].isnan() and out[1][r].isnan() and bool((out[3][r] == -1).all()) and bool(out[4][r].isnan().all())
    rest = [i for i in range(T) if i not in (1, 3)]
    for a, b in zip(clean, out):
        assert torch.equal(a[rest], b[rest])


def test_targets_that_are_ignored_or_out_of_range():
    H, W, t = make("f32", 130, 64, [77, 60])
    t[3], t[9], t[20] = -1, 137, 5
    prob, sc = vp.problem_for(H, W, 5), vp.Score(2)
    ws = torch.empty(vp.vp_score_workspace_size(prob, sc), dtype=torch.uint8, device="cuda")
    f = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    loss, lse, ent, ids, tl = f(130), f(130), f(130), torch.empty(130, 2, dtype=torch.int64, device="cuda"), f(130, 2)
    vp.vp_score_forward(prob, sc, H, W, t, loss, lse, ent, ids, tl, ws)
    bad = (t != 5) & ((t < 0) | (t >= 137))
    assert vp.vp_ce_check(ws) == int(bad.sum())
    assert torch.equal(loss.isnan(), bad)
    check(H, W, t, (loss, lse, ent, ids, tl), 2, ignore=5)
    # an entropy that is not asked for, and the library's own loss beside it
    loss2, lse2 = f(130), f(130)
    vp.vp_score_forward(prob, sc, H, W, t, loss2, lse2, None, ids, tl, ws)
    assert torch.equal(lse, lse2) and torch.equal(loss[~bad], loss2[~bad])


def test_visiting_order_is_not_used():
    H, W, t = make("bf16", 70, 64, [300, 200, 100])
    sc, outs = vp.Score(4), []
    for order in (None, [2, 0, 1]):
        prob = vp.problem_for(H, W, order=order)
        ws = torch.empty(vp.vp_score_workspace_size(prob, sc), dtype=torch.uint8, device="cuda")
        out = [torch.empty(70, device="cuda") for _ in range(3)]
        out += [torch.empty(70, 4, dtype=torch.int64, device="cuda"), torch.empty(70, 4, device="cuda")]
        vp.vp_score_forward(prob, sc, H, W, t, *out, ws)
        outs.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_no_tokens():
    H, W, t = make("bf16", 0, 64, [30])
    out = vp.score(H, W, t, top=3)
    assert [tuple(o.shape) for o in out] == [(0,), (0,), (0,), (0, 3), (0, 3)]


def test_tokens_in_chunks():
    """More tokens than the workspace holds maxima for: several chunks, the last one short."""
    T, V = 9001, 150001
    H, W, t = make("bf16", T, 16, [100000, 50001])
    prob = vp.problem_for(H, W)
    assert vp.vp_score_workspace_size(prob, vp.Score(3)) < (1 << 30) + (1 << 26)
    out = vp.score(H, W, t, top=3)
    plain = vp.score(H, W, t)
    for a, b in zip(out[:3], plain[:3]):  # (another plan of the tiles: other orders of the sums)
        assert bool(((a - b).abs() <= 1e-4).all())
    pick = torch.cat([torch.arange(0, T, 37), torch.arange(T - 40, T)]).cuda()
    check(H[pick], W, t[pick], [o[pick] for o in out], 3)


def test_largest_vocabulary_with_alternatives():
    V = 1 << 24
    H = torch.randn(2, 8, device="cuda")
    W = [torch.randn(V, 8, device="cuda")]
    t = torch.tensor([5, V - 1], device="cuda")
    out = vp.score(H, W, t, top=32)
    y = (H.double() @ W[0].double().t().contiguous())
    assert torch.equal(out[3], torch.sort(y, dim=1, descending=True, stable=True).indices[:, :32])
    with pytest.raises(vp.VpError, match="shape"):
        vp.score(H, [W[0], W[0][:1]], t, top=1)
    assert vp.score(H, [W[0], W[0][:1]], t)[3] is None


def test_graphs_on_one_workspace_and_another_stream():
    """Two captured calls that share a workspace, replayed in turn with eager work in between, and a
    call on a stream of its own, against the eager results bit for bit."""
    sc = vp.Score(5)
    sets = [make("bf16", T, 320, [900, 1000, 300], seed=T) for T in (60, 2200)]
    probs = [vp.problem_for(H, W) for H, W, _ in sets]
    ws = torch.empty(max(vp.vp_score_workspace_size(p, sc) for p in probs), dtype=torch.uint8, device="cuda")
    outs = [[torch.empty(H.shape[0], device="cuda") for _ in range(3)] +
            [torch.empty(H.shape[0], 5, dtype=torch.int64, device="cuda"), torch.empty(H.shape[0], 5, device="cuda")]
            for H, _, _ in sets]
    run = lambda i: vp.vp_score_forward(probs[i], sc, *sets[i], *outs[i], ws)  # noqa: E731
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run(0), run(1)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    want = [[o.clone() for o in out] for out in outs]
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(i)
        graphs.append(g)
    for rep in range(3):
        for out in outs:
            for o in out:
                o.zero_()
        for i in (1, 0):
            graphs[i].replay()
        torch.cuda.synchronize()
        for out, w in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(out, w)), rep
        vp.score(*make("f32", 33, 64, [500], seed=rep), top=2)
        torch.cuda.synchronize()
