"""Score factors that razer_attn_kv8 refuses on the host (no GPU needed)."""
import ctypes

import pytest

from test_i8_refusals import _attn, _cache, b  # noqa: F401


@pytest.mark.parametrize("scale", [2.0 ** 62 * 1.5, -2.0 ** 63, 3e38, -3e38, float("inf"), float("-inf"), float("nan")])
def test_scales_beyond_what_a_score_bears(b, scale):  # noqa: F811
    """Times log2 e and a row's power of two they would be infinite, and a score of 0 NaN."""
    assert _attn(b, _cache(b), scale=scale) == b.ERR_INVALID_ARG and "scale" in b.last_error()


def test_scales_up_to_that(b):  # noqa: F811
    """Looked at before the workspace, which is too small here."""
    for scale in (0.0, -1.0, 2.0 ** 62, -2.0 ** 62, 2.0 ** -149):
        assert _attn(b, _cache(b), scale=ctypes.c_float(scale), size=0) == b.ERR_WORKSPACE
