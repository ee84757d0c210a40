"""griffin_verify_drafts refuses tokens that come out where drafted ones lie, also where only a part of them does (no GPU)."""
import pytest

import paper_2404_01365_amd as G
from test_layer_abi_cpu import FAKE
from test_q4_abi_cpu import verify

ROWS = 9                                          # of verify()


@pytest.mark.parametrize("by", [-(ROWS - 1), -1, 0, 1, 5, ROWS - 1])
def test_tokens_that_lie_over_drafted_ones_are_refused(by):
    # ... ahead of anything that a call without a workspace is refused for
    assert verify(drafted=FAKE + 4096, tokens=FAKE + 4096 + 4 * by, vocab=100000, ldp=100000, ldq=100000, ws=None) == G.EINVAL


@pytest.mark.parametrize("by", [-ROWS, ROWS, 1000])
def test_tokens_beside_drafted_ones_are_taken(by):
    assert verify(drafted=FAKE + 4096, tokens=FAKE + 4096 + 4 * by, vocab=100000, ldp=100000, ldq=100000, ws=None) == G.EWORKSPACE
