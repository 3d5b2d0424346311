"""The largest calls of the serving entry points, and what a refusal says, on the host (no GPU needed)."""
import pytest

from test_serving_abi import OK, PAGED, ROPE, ROWS, arr, b, caller  # noqa: F401


@pytest.mark.parametrize("scale", [0.0, -1.0, float("nan"), float("inf")])
def test_a_refused_scale_is_explained(b, scale):  # noqa: F811
    """attn_paged_fwd refuses a scale of 0, and the status text may not call that one fine."""
    assert caller(b, "attn_paged_fwd", PAGED)(scale=scale) == b.ATTN_ERR_SCALE
    text = b.attn_strerror(b.ATTN_ERR_SCALE)
    assert "> 0" in text and ">= 0" not in text


@pytest.mark.parametrize("entry, spec", [("attn_cache_write", ROWS), ("attn_cache_read_f16", ROWS), ("attn_paged_fwd", PAGED),
                                         ("attn_paged_fwd_f16", PAGED)])
def test_a_batch_that_the_lanes_cannot_count_is_refused(b, entry, spec):  # noqa: F811
    """The kernels step through the sequences by up to 1024 at a time: with B next to 2^31 the step's sum is negative, below B, and
    an index in front of kv_len.  (Arguments that are misaligned as well, so that nothing could be launched.)"""
    f = caller(b, entry, spec)
    for B in ((1 << 30) + 1, 2 ** 31 - 1025, 2 ** 31 - 64, 2 ** 31 - 2, 2 ** 31 - 1):
        assert f(B=B, start=OK + 2) == b.ATTN_ERR_SHAPE
        assert b.attn_paged_fwd_workspace_bytes(3, B, 4, 2, 64) == -1
    assert f(B=1 << 30, start=OK + 2) == b.ATTN_ERR_ALIGN
    assert b.attn_paged_fwd_workspace_bytes(3, 1 << 30, 4, 2, 64) > 0
