"""`forward` and `backward` with a norm on the host (no GPU): wrong buffers for the norm's gradients
are refused in front of the projection, and both parts run on the device of the hidden states."""
import os

import pytest
import torch

import paper_2609_14306_amd as vp

pytestmark = pytest.mark.skipif(not os.path.exists(vp.LIB_PATH),
                                reason="libvpce.so not built (run __graft_entry__.build())")

T, D, V = 6, 16, 40


def _backward(bias=True, **kw):
    x, v = torch.zeros(T, D), torch.zeros(D)
    return vp.backward(x, [torch.zeros(V, D)], torch.zeros(T, dtype=torch.int64), torch.zeros(T), torch.zeros(T),
                       norm=vp.HeadNorm(v, v if bias else None), dW_shards=[torch.zeros(V, D)], **kw)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dnorm, match", [
    ((torch.zeros(D + 8), torch.zeros(D)), "dgamma: shape"),
    ((torch.zeros(D), torch.zeros(D, dtype=torch.float64)), "dbeta: dtype"),
    ((torch.zeros(D), torch.zeros(2 * D)[::2]), "dbeta: must be contiguous"),
    ((None, [0.0] * D), "dbeta: expected|accumulate"),
    ((torch.zeros(D),) * 3, "too many values"),
    # (right ones get as far as the device)
    ((torch.zeros(D), torch.zeros(D)), "on a GPU device"),
])
def test_wrong_buffers_are_refused_first(dnorm, match, accumulate):
    with pytest.raises(ValueError, match=match):
        _backward(dnorm=dnorm, accumulate=accumulate)


def test_unaligned_buffers_are_refused():
    at = torch.zeros(D + 8)
    first = 1 if at.data_ptr() % 16 == 0 else 4 - at.data_ptr() // 4 % 4 + 1
    with pytest.raises(vp.VpError) as e:
        _backward(dnorm=(at[first:first + D], torch.zeros(D)))
    assert e.value.status == vp.VP_ERR_ALIGN


def test_accumulation_needs_what_it_adds_to():
    for dnorm in ((torch.zeros(D), None), (None, torch.zeros(D)), (None, None)):
        with pytest.raises(ValueError, match="accumulate"):
            _backward(dnorm=dnorm, accumulate=True)
    # no beta: nothing to add its gradient to
    with pytest.raises(ValueError, match="on a GPU device"):
        _backward(bias=False, dnorm=(torch.zeros(D), None), accumulate=True)


def test_dnorm_without_a_norm_is_refused():
    with pytest.raises(ValueError, match="dnorm"):
        vp.backward(torch.zeros(T, D), [torch.zeros(V, D)], torch.zeros(T, dtype=torch.int64), torch.zeros(T),
                    torch.zeros(T), dnorm=(torch.zeros(D), torch.zeros(D)))


def test_norm_and_projection_run_on_one_device(monkeypatch):
    """The norm takes the stream of its tensors' device and the projection the current one: both
    calls are made with the hidden states' device as the current one."""
    current, seen = [None], []

    class Device:
        def __init__(self, t):
            self.t = t

        def __enter__(self):
            current[0] = self.t

        def __exit__(self, *_):
            current[0] = None

    def record(name):
        return lambda *a, **kw: seen.append((name, current[0] is x))

    x, v = torch.zeros(T, D), torch.zeros(D)
    W, t = [torch.zeros(V, D)], torch.zeros(T, dtype=torch.int64)
    monkeypatch.setattr(torch.cuda, "device_of", Device)
    monkeypatch.setattr(vp.head, "vp_norm_forward", record("norm"))
    monkeypatch.setattr(vp.head, "vp_norm_backward", record("norm backward"))
    monkeypatch.setattr(vp, "vp_ce_forward", record("projection"))
    monkeypatch.setattr(vp, "vp_ce_backward", record("projection backward"))
    norm = vp.HeadNorm(v, v)
    loss, lse = vp.forward(x, W, t, norm=norm)
    assert seen == [("norm", True), ("projection", True)]
    seen.clear()
    assert len(vp.backward(x, W, t, lse, loss, norm=norm)) == 4
    assert seen == [("norm", True), ("projection backward", True), ("norm backward", True)]
    assert current[0] is None
