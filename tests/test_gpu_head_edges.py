"""Calls at the edges of what the operators around the projection allow, on the GPU."""
import pytest
import torch

import paper_2609_14306_amd as vp

pytestmark = pytest.mark.gpu


def test_squared_preference_with_a_smoothing_that_it_does_not_use():
    g = torch.Generator().manual_seed(4)
    loss, ref = (torch.rand(500, generator=g).cuda() for _ in range(2))
    targets = torch.zeros(500, dtype=torch.int64, device="cuda")
    start = torch.tensor([0, 100, 180, 300, 500], dtype=torch.int32, device="cuda")
    want = vp.preference_forward(loss, targets, start, vp.Preference("squared", 0.3, 0.1), ref)
    got = vp.preference_forward(loss, targets, start, vp.Preference("squared", 0.3, 0.1, 0.1), ref)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
