"""Workspaces of the scoring calls on the CPU: 8-bit operands go through in the same chunks with and without
alternatives, whose maxima are the same."""
import pytest

import paper_2609_14306_amd as vp


@pytest.mark.parametrize("T, d, rows", [(8192, 7168, [16160] * 8), (6000, 4096, [9496] * 16), (100000, 2880, [25136] * 8),
                                        (9001, 1024, [100001, 30000]), (300, 1024, [16000000]), (40, 256, [999])])
def test_alternatives_do_not_cut_8_bit_tokens_further(T, d, rows):
    prob = vp.Problem(T, d, rows, vp.VP_E4M3)
    none, one, most = (vp.vp_score_workspace_size(prob, vp.Score(k)) for k in (0, 1, 32))
    assert none == one == most
    padded = sum(-(-r // 256) * 256 for r in rows)
    assert none < max(2 << 30, 320 * padded) + (1 << 26)
