"""Alternatives where the first groups that are looked at have logits that float32 holds, so that nothing is seen of
what the product's sums round, and a later id has the largest logit by less than that."""
import pytest
import torch

import paper_2609_14306_amd as vp

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def operands(T, top, level, d=64, V=9000):
    """top + 2 ids with a logit of `level`, and behind them one with level (1 + 2^-25), which float32 rounds to level;
    the rest far below."""
    H, W = torch.zeros(T, d), torch.zeros(V, d)
    H[:, 0], H[:, 1], H[:, 2] = level, level * 2.0 ** -12, 1.0
    W[:, 2] = -256.0
    at = [100 + 40 * k for k in range(top + 2)] + [V - 500]
    W[at, 2] = 0.0
    W[at, 0] = 1.0
    W[at[-1], 1] = 2.0 ** -13
    return H.cuda(), W.cuda(), at, torch.zeros(T, dtype=torch.int64, device="cuda")


@pytest.mark.parametrize("T", [1, 60, 300, 700, 2100])
@pytest.mark.parametrize("level", [1.0, 96.0, 2.0 ** -20, -3.0])
@pytest.mark.parametrize("top", [1, 4, 32])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_rounded_logit_behind_exact_ones(dtype, top, level, T):
    H, W, at, t = operands(T, top, level)
    if level < 0:
        W[at[-1], 1] *= -1.0  # (less far below 0)
    H, W = H.to(DT[dtype]), W.to(DT[dtype])
    y = H[:1].double() @ W.double().t().contiguous()
    want = torch.sort(y, dim=1, descending=True, stable=True).indices[:, :top]
    assert want[0, 0] == at[-1]
    assert torch.equal(vp.score(H, [W], t, top=top)[3], want.expand(T, top))


@pytest.mark.parametrize("T", [1, 60, 100, 700, 2100])
@pytest.mark.parametrize("top", [2, 5, 32])
def test_a_cut_product_behind_exact_ones_in_8_bits(top, T):
    """The matrix unit cuts a product of 2^-20 beside one of 1, in ids that are not likely beside one of nearly
    all probability."""
    H, W, at, t = operands(T, top - 1, 1.0, d=128)
    H[:, 1], W[at[-1], 1], W[:, 2] = 2.0 ** -8, 2.0 ** -12, torch.where(W[:, 2] < 0, -16.0, 0.0)
    W[5, 2] = 12.0
    h8, hs = vp.quantize(H)
    w8, ws = vp.quantize(W, 128)
    y = h8[:1].double() * hs[:1].double() @ (w8.double() * ws.double().repeat_interleave(128, 0)[:9000]).t().contiguous()
    want = torch.sort(y, dim=1, descending=True, stable=True).indices[:, :top]
    assert want[0, 0] == 5 and want[0, 1] == at[-1]
    assert torch.equal(vp.score_f8(h8, hs, [w8], [ws], t, top=top)[3], want.expand(T, top))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [3, 700])
def test_sums_that_cancel_to_nothing(dtype, T):
    """A logit of 2^-30 whose float32 sum is 0, behind logits of 0 with no products at all, for tokens that
    are not zeros; tokens of zeros beside them have the first ids."""
    H, W, at, t = operands(T, 1, 1.0)
    W[at, 0] = 0.0
    W[at[-1], 0], W[at[-1], 1], W[at[-1], 32] = 1.0, 2.0 ** -18, -1.0
    H[:, 32] = 1.0
    H[1::3] = 0.0
    H, W = H.to(DT[dtype]), W.to(DT[dtype])
    got = vp.score(H, [W], t, top=1)[3][:, 0]
    want = torch.full_like(got, at[-1])
    want[1::3] = 0
    assert torch.equal(got, want)
