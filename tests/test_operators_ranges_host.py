"""Every call of the ranges that perf/operators.py draws passes the host's checks (no GPU).

A call without a workspace, or without its input where it takes no workspace, is refused last of
all: that refusal is what a problem that passes every check of its values ends with here, before
any launch."""
import os
import random

import pytest

import paper_2609_14306_amd as vp
from paper_2609_14306_amd import head

from perf import operators

pytestmark = pytest.mark.skipif(not os.path.exists(vp.LIB_PATH),
                                reason="libvpce.so not built (run __graft_entry__.build())")

FAKE = 0x100000  # an aligned pointer value that no call here dereferences


def _preference(case):
    return vp.Preference(case["kind"], beta=case["beta"], margin=case["margin"], smoothing=case["smoothing"])


def _status(case):
    lib, op = vp.load_library(), case["op"]
    if op.startswith("norm"):
        norm = vp.Norm(case["T"], case["d"], vp.VP_BF16 if case["dtype"] == "bf16" else vp.VP_F32, rms=case["rms"])
        if op == "norm_forward":
            return lib.vp_norm_forward(norm.ref, None, *[FAKE] * 5, None), vp.VP_ERR_NULL
        return lib.vp_norm_backward(norm.ref, *[FAKE] * 8, None, 0, None), vp.VP_ERR_WORKSPACE
    seq = vp.Sequences(case["T"], case["S"], operators.IGNORE, case["mean"])
    if op == "preference":
        pref = head._preference_ref(_preference(case))
        return lib.vp_pref_forward(seq.ref, pref, *[FAKE] * 7, None, 0, None), vp.VP_ERR_WORKSPACE
    pol = vp.Policy(case["clip_low"], case["clip_high"], case["kl_coef"], case["per_token"])
    return lib.vp_policy_forward(seq.ref, pol.ref, *[FAKE] * 10, None, 0, None), vp.VP_ERR_WORKSPACE


def test_listed_cases_pass_the_checks():
    for case in operators.listed():
        got, want = _status(case)
        assert got == want, case


def test_drawn_cases_pass_the_checks():
    rng = random.Random(7)
    kinds = set()
    for _ in range(4000):
        case = operators.draw(rng)
        got, want = _status(case)
        assert got == want, case
        if case["op"] == "preference":
            kinds.add((case["kind"], case["smoothing"] > 0))
    assert len(kinds) == 4  # both kinds, each with a smoothing and without


@pytest.mark.parametrize("smoothing", [0.0, 0.1, 0.5])
def test_squared_form_does_not_use_a_smoothing(smoothing):
    pref = vp.Preference("squared", 0.3, 0.2, smoothing)
    c = head._preference_ref(pref)._obj
    assert (c.kind, c.beta, c.margin, c.smoothing) == (vp.VP_PREF_SQUARED, 0.3, 0.2, 0.0)
    assert pref.c.smoothing == smoothing
    pref.c.beta = 0.7  # (values set later are the ones that count)
    assert head._preference_ref(pref)._obj.beta == 0.7


@pytest.mark.parametrize("smoothing", [-0.1, 0.6, float("nan"), float("inf")])
@pytest.mark.parametrize("kind", ["logistic", "squared"])
def test_smoothing_outside_its_range_is_refused(kind, smoothing):
    seq, pref = vp.Sequences(10, 4), vp.Preference(kind, smoothing=smoothing)
    got = vp.load_library().vp_pref_forward(seq.ref, head._preference_ref(pref), *[FAKE] * 7, None, 0, None)
    assert got == vp.VP_ERR_VALUE
