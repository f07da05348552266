"""The weights of the many-row kernels by what they do to lse, where a single key has nearly all of the weight."""
import math

import pytest
import torch

from tests.test_gpu_cache import ints, sb  # noqa: F401  (sb: a fixture)

pytestmark = pytest.mark.gpu
LN2 = math.log(2)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("column", [0, 1, 2, 3, 4, 5, 6, 7])
def test_weights_of_every_column_in_lse(sb, d, column):  # noqa: F811
    """Two steps of 128 keys: the first sets the maximum with a logit of 0, in the second one key lies 2^1 to 2^3.9 above it, too little for a
    new maximum; the others have no weight.  One item to a block, so that the steps are one block's.

    lse = ln2 (log2(2^11 + 2^x) - 11), x = 11 + u.  Errors: x, near 16, is rounded (2^-21), u = scale q k log2(e) has two factors rounded
    (2^-23 u); the weight 2^-22; three sums 2^-24 each; log2f is good to a unit (2^-20) and added to the maximum (2^-21); two products."""
    rows, blocks = 64, torch.cuda.get_device_properties(0).multi_processor_count
    cache = sb.make_cache(4, 64, 1, d)
    k = torch.zeros(256, 1, d, dtype=torch.float16)
    k[:, 0, 0] = -2688
    k[5, 0, 0], k[128 + 40 + column, 0, 0] = 0, 6                         # all are values that the cache has
    sb.sol_attn_cache_append(k.cuda(), torch.zeros_like(k).cuda(), torch.arange(256, dtype=torch.int32, device="cuda"), cache)
    q = torch.zeros(rows * blocks, 1, d, dtype=torch.float16)
    q[:, 0, 0] = 1 + 2.9 * torch.rand(rows * blocks, generator=torch.Generator().manual_seed(column))
    scale = torch.tensor(LN2 / 6).item()
    lse, out = torch.zeros(rows * blocks, 1, device="cuda"), torch.empty_like(q, device="cuda")
    sb.sol_attn_cache_attention(q.cuda(), ints([rows * b for b in range(blocks + 1)]), ints([256] * blocks), ints([[0, 1, 2, 3]] * blocks), cache, out, rows,
                                sb.make_cache_workspace(rows, 1, 1, d), lse=lse, causal=False, scale=scale)
    u = scale * q[:, 0, 0].double() * 6 / LN2
    want = torch.log1p(torch.exp2(u))
    bound = LN2 * (2.0 ** -21 + 2.0 ** -23 * u + 2.0 ** -20 + 2.0 ** -21) + 2.0 ** -22 + 3 * 2.0 ** -24 + 2 * 2.0 ** -24 * want
    error = (lse[:, 0].double().cpu() - want).abs()
    assert (error <= bound).all(), ((error / bound).max().item(), error.max().item())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [1, 12, 64])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("largest", [1.0, 1.5])
def test_small_elements_of_a_query_are_exact(sb, dtype, rows, d, largest):  # noqa: F811
    """An element with all of its type's bits, 2^-28 of the row's largest: a rounding in its last bit would move the logit, about 8, by 2^-12 of it.
    lse = log(1 + exp(x)), x with an error of three roundings (2^-22) and a subtraction of 16 at most (2^-21)."""
    cache = sb.make_cache(1, 16, 1, d)
    k = torch.zeros(2, 1, d, dtype=torch.float16)
    k[1, 0, 0] = 6
    sb.sol_attn_cache_append(k.cuda(), torch.zeros_like(k).cuda(), torch.arange(2, dtype=torch.int32, device="cuda"), cache)
    q = torch.zeros(rows, 1, d, dtype=dtype)
    q[:, 0, d - 1] = largest * 2.0 ** 15
    q[:, 0, 0] = 2.0 ** -13 * (2 - torch.finfo(dtype).eps)
    scale = torch.tensor(8 / 6 * 2.0 ** 12).item()
    lse, out = torch.zeros(rows, 1, device="cuda"), torch.empty_like(q, device="cuda")
    sb.sol_attn_cache_attention(q.cuda(), ints([0, rows]), ints([2]), ints([[0]]), cache, out, rows, sb.make_cache_workspace(rows, 1, 1, d),
                                lse=lse, causal=False, scale=scale)
    x = scale * q[:, 0, 0].double() * 6
    assert ((lse[:, 0].double().cpu() - torch.log1p(torch.exp(x))).abs() <= 2.0 ** -22 * x + 2.0 ** -18).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [1, 12, 64])
@pytest.mark.parametrize("keys", [3, 300, 5000])
def test_logits_outside_fp32(sb, d, rows, keys):  # noqa: F811
    """A logit of 1e40 makes its row NaN, one of -1e40 has no weight; the rows beside it are exact."""
    n, key = -(-keys // 64), keys * 2 // 3
    cache = sb.make_cache(n, 64, 1, d)
    k, v = torch.zeros(keys, 1, d, dtype=torch.bfloat16), torch.randn(keys, 1, d, generator=torch.Generator().manual_seed(1)).bfloat16()
    k[key, 0, 0], k[key, 0, 1] = 2688, -2688
    slots = torch.arange(keys, dtype=torch.int32, device="cuda")
    sb.sol_attn_cache_append(k.cuda(), v.cuda(), slots, cache)
    held = torch.empty_like(v, device="cuda")
    sb.sol_attn_cache_read(cache, slots, None, held)
    q = torch.zeros(rows, 3, d, dtype=torch.bfloat16)
    q[:, 1, 0], q[:, 2, 1] = 2.0 ** 126, 2.0 ** 126
    lse, out = torch.zeros(rows, 3, device="cuda"), torch.empty_like(q, device="cuda")
    sb.sol_attn_cache_attention(q.cuda(), ints([0, rows]), ints([keys]), ints([list(range(n))]), cache, out, rows,
                                sb.make_cache_workspace(rows, 3, 1, d), lse=lse, causal=False, scale=1.0)
    assert out[:, 1].isnan().all() and lse[:, 1].isnan().all()
    others = held[torch.arange(keys) != key].double()
    for head, values in ((0, held.double()), (2, others)):
        want = values.mean(0)
        # weights are all alike: what is left are the sum's, the products' and the result's roundings
        bound = 2.0 ** -8 * want.abs() + 2.0 ** -11 * values.abs().mean(0)
        assert ((out[:, head].double() - want).abs() <= bound).all(), head
        assert ((lse[:, head].double() - math.log(len(values))).abs() <= 2.0 ** -18).all(), head
