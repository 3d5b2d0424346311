"""The largest calls of the serving entry points, and what a refusal says, on the host (no GPU needed)."""
import pytest

from test_serving_abi import OK, PAGED, ROPE, ROWS, arr, b, caller  # noqa: F401


@pytest.mark.parametrize("scale", [0.0, -1.0, float("nan"), float("inf")])
def test_a_refused_scale_is_explained(b, scale):  # noqa: F811
    """attn_paged_fwd refuses a scale of 0, and the status text may not call that one fine."""
    assert caller(b, "attn_paged_fwd", PAGED)(scale=scale) == b.ATTN_ERR_SCALE
    text = b.attn_strerror(b.ATTN_ERR_SCALE)
    assert "> 0" in text and ">= 0" not in text
