"""tkv_prompt_attn and tkv_quant_attn_decode_shared refuse a scale that is not finite in units of log 2, before any GPU work (no GPU needed)."""
import pytest

import test_prompt_refusals as prompt
import test_shared_prefix_refusals as shared
from test_prompt_refusals import L  # noqa: F401  (the library)


@pytest.mark.parametrize("sm,status", [(3.0e38, -1), (2.4e38, -1), (2.3e38, -4), (1e-44, -4)])
def test_scale(L, sm, status):  # noqa: F811
    """(A call that passes the check asks for its workspace, too small here.)"""
    assert prompt._call(L, sm=sm, ws=16) == status
    assert shared._call(L, sm=sm, ws=16) == status
