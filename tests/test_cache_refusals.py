"""Calls that the cache operators refuse before anything is launched: outputs in the way of inputs or of themselves."""
import ctypes

import pytest
import torch

from tests.test_cache_host import P, attention_args, cache_of, norm_args, sb  # noqa: F401  (sb: a fixture)

two, three = ctypes.c_int64 * 2, ctypes.c_int64 * 3


@pytest.mark.parametrize("change", [dict(q_out_stride=three(4096, 128, 1024)), dict(k_out_stride=three(4096, 520, 128)),
                                    dict(q_out_stride=three(8192, 512, 128), batch=2), dict(q_out=8192, k_out=1 << 20),
                                    dict(k_out=4096, q_out=1 << 20), dict(q_out=1 << 20, k_out=1 << 20)])
def test_norm_in_place_with_other_strides_or_the_others_place(sb, change):  # noqa: F811
    """q_out may be q with q's strides and k_out k, but neither the other's input or output: warps read and write heads on their own."""
    assert sb.lib().sol_attn_qk_norm_rope(ctypes.byref(norm_args(sb, **change))) == sb.SOL_ERR_INVALID_ARG


def test_outputs_whose_rows_lie_on_one_another(sb):  # noqa: F811
    """Strides of 0, as of an expanded tensor, of a dimension with more than one entry; inputs may have them."""
    bad, c = sb.SOL_ERR_INVALID_ARG, cache_of(sb)
    for st in (two(0, 128), two(512, 0)):
        assert sb.lib().sol_attn_cache_attention(ctypes.byref(attention_args(sb, out_stride=st))) == bad
        assert sb.lib().sol_attn_cache_read(ctypes.byref(c), P(4096), P(1 << 20), st, two(256, 128), P(4096), 4, 0, None) == bad
        assert sb.lib().sol_attn_cache_read(ctypes.byref(c), None, P(1 << 20), None, st, P(4096), 4, 0, None) == bad
    for st in (three(0, 512, 128), three(4096, 0, 128), three(4096, 512, 0)):
        for side in ("q", "k"):
            for where in (4096 if side == "q" else 8192, 1 << 20):
                a = norm_args(sb, batch=2, **{side + "_out": where, side + "_stride": st, side + "_out_stride": st})
                assert sb.lib().sol_attn_qk_norm_rope(ctypes.byref(a)) == bad


@pytest.mark.parametrize("change", [dict(pages=5), dict(page_size=32), dict(heads=3), dict(d=128)])
def test_a_cache_that_is_changed_is_measured_again(sb, change):  # noqa: F811
    """Fields set after it was made: the buffer has to hold what they say."""
    cache = sb.make_cache(4, 16, 2, 64, device="cpu")
    cache.c(-1)                                                           # (-1: where tensors of the CPU are)
    for name, value in change.items():
        setattr(cache, name, value)
    with pytest.raises(ValueError):
        cache.c(-1)
    cache.data = torch.zeros(sb.sol_attn_cache_bytes(cache.pages, cache.page_size, cache.heads, cache.d), dtype=torch.uint8)
    assert cache.c(-1)[1:5] == (cache.pages, cache.page_size, cache.heads, cache.d) and cache.bytes == cache.data.numel()
    cache.page_size = 24
    with pytest.raises(sb.SolAttnError):
        cache.c(-1)


def test_a_step_without_queries(sb):  # noqa: F811
    """All requests idle: no rows, and a longest request of none."""
    f = sb.lib().sol_attn_cache_attention
    assert f(ctypes.byref(attention_args(sb, tokens=0, q=None, out=None, max_q=0))) == sb.SOL_OK
    assert f(ctypes.byref(attention_args(sb, tokens=0, q=None, out=None, max_q=-1))) == sb.SOL_ERR_INVALID_ARG
    assert f(ctypes.byref(attention_args(sb, max_q=0))) == sb.SOL_ERR_INVALID_ARG
    assert f(ctypes.byref(attention_args(sb, tokens=0, q=None, out=None, max_q=0, workspace=None))) == sb.SOL_ERR_WORKSPACE
