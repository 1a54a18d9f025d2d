"""How the backward norm's rows are shared among workgroups: by the tokens that there are, not by a group_len or a number of groups beyond them (no GPU)."""
import os

import pytest

from paper_2602_04789_amd import lf


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(lf.library_path()):
        from paper_2602_04789_amd import build
        build.build()
    return lf.load()


@pytest.mark.parametrize("channels", [8, 512, 1536, 2048, 5120, 8192])
@pytest.mark.parametrize("tokens", [1, 7, 300, 4680, 32760])
def test_the_scratch_follows_the_tokens(tokens, channels):
    """It holds the sums of every workgroup's share, so calls with the same shares ask for the same."""
    size = lf.lf_gate_norm_bwd_workspace_bytes
    one = size(tokens, channels, 1, tokens)
    assert one > 0
    for group_len in (tokens + 1, 2 * tokens, 32768, 1 << 20, 1 << 30, (1 << 31) - 1):
        if group_len >= tokens:
            assert size(tokens, channels, 1, group_len) == one, group_len
            assert size(tokens, channels, 81, group_len) == one, group_len
    for group_len in (1, 40, 1560):
        live = -(-tokens // group_len)
        assert size(tokens, channels, live + 60, group_len) == size(tokens, channels, live, group_len), group_len
