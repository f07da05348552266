"""Calls that the cache operators refuse before anything is launched: outputs in the way of inputs or of themselves."""
import ctypes

import pytest

from tests.test_cache_host import norm_args, sb  # noqa: F401  (sb: a fixture)

two, three = ctypes.c_int64 * 2, ctypes.c_int64 * 3


@pytest.mark.parametrize("change", [dict(q_out_stride=three(4096, 128, 1024)), dict(k_out_stride=three(4096, 520, 128)),
                                    dict(q_out_stride=three(8192, 512, 128), batch=2), dict(q_out=8192, k_out=1 << 20),
                                    dict(k_out=4096, q_out=1 << 20), dict(q_out=1 << 20, k_out=1 << 20)])
def test_norm_in_place_with_other_strides_or_the_others_place(sb, change):  # noqa: F811
    """q_out may be q with q's strides and k_out k, but neither the other's input or output: warps read and write heads on their own."""
    assert sb.lib().sol_attn_qk_norm_rope(ctypes.byref(norm_args(sb, **change))) == sb.SOL_ERR_INVALID_ARG
