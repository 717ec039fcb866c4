"""The eps of a layer norm, which the kernels hold in float32 (no GPU)."""
import os

import pytest

import paper_2609_14306_amd as vp

pytestmark = pytest.mark.skipif(not os.path.exists(vp.LIB_PATH),
                                reason="libvpce.so not built (run __graft_entry__.build())")
FAKE = 0x100000  # an aligned pointer value that no call here dereferences


def _status(eps):
    """Of a call without its input, the last refusal of all."""
    lib, norm = vp.load_library(), vp.Norm(4, 64, vp.VP_F32, eps=eps)
    return lib.vp_norm_forward(norm.ref, None, *[FAKE] * 5, None), lib.vp_norm_backward(norm.ref, *[FAKE] * 8, None, 0, None)


@pytest.mark.parametrize("eps", [5e-324, 1e-60, 1e-45, 1.17e-38, 3.41e38, 1e60])
def test_refused(eps):
    assert _status(eps) == (vp.VP_ERR_VALUE, vp.VP_ERR_VALUE)


@pytest.mark.parametrize("eps", [0.0, 1.18e-38, 1e-12, 1e-5, 1.0, 3.4e38])
def test_accepted(eps):
    assert _status(eps) == (vp.VP_ERR_NULL, vp.VP_ERR_WORKSPACE)
