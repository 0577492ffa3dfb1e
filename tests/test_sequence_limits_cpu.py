"""Scales of the token scores that float32 cannot hold times log2(e): every logit, 0 too, would
give NaN. Refused on the host."""
import pytest

import paper_1711_03016_amd as dl
from test_sequence_cpu import SCORES, SCORESB, _call, built_library  # noqa: F401


@pytest.mark.parametrize("scale", [2.5e38, 3.4e38])
def test_scales_that_overflow_are_refused(scale):
    assert _call("dlvm_token_logprobs", SCORES, dict(scale=scale)) == dl.ERR_UNSUPPORTED
    assert _call("dlvm_token_logprobs_backward", SCORESB, dict(scale=scale)) == dl.ERR_UNSUPPORTED
