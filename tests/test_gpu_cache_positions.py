"""Causal attention where the buffers hold less than the lengths say: each query keeps its place."""
import pytest
import torch

from tests import cache_reference as ref
from tests.test_gpu_cache import batch, close, filled, held_values, ints, sb  # noqa: F401  (sb: a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, H, Hk, d", [(torch.bfloat16, 4, 2, 128), (torch.float16, 3, 1, 64)])
@pytest.mark.parametrize("new, tokens, columns", [([5, 6], 9, None), ([3, 8], 2, None), ([3, 40, 300], 200, None), ([1, 2], 2, 5), ([7, 90], 97, 4),
                                                  ([130, 290, 1], 421, 9), ([60, 290], 200, 7), ([1], 1, 1)])
def test_queries_keep_their_places(sb, dtype, H, Hk, d, new, tokens, columns):  # noqa: F811
    """q holds `tokens` of the queries, the table `columns` pages of each request; both of those are what a step without room leaves."""
    kv = [120 + 97 * b + n for b, n in enumerate(new)]
    table, cu, pages = batch(kv, new, 32, 7)
    cache = filled(sb, pages, 32, Hk, d, 4)
    g = torch.Generator().manual_seed(3)
    q = torch.randn(cu[-1], H, d, generator=g).to(dtype)
    columns = columns or len(table[0])
    cut = [row[:columns] + [-1] * (len(row) - columns) for row in table]
    want, want_lse, tol, tol_lse, _ = ref.attention(q, cu, kv, cut, *held_values(cache), 32, True, d ** -0.5, pages)
    out, lse = torch.full((tokens, H, d), 9.0, dtype=dtype, device="cuda"), torch.full((tokens, H), 9.0, device="cuda")
    ws = sb.make_cache_workspace(max(new), H, Hk, d)
    sb.sol_attn_cache_attention(q[:tokens].cuda(), ints(cu), ints(kv), ints(table)[:, :columns], cache, out, max(new), ws, lse=lse)
    assert sb.sol_attn_cache_read_status(ws) == sb.SOL_OK
    close(out, want[:tokens], tol[:tokens], dtype)
    x, w = lse.double().cpu(), want_lse[:tokens]
    assert torch.equal(x.isinf(), w.isinf())
    assert ((x - w).abs()[~w.isinf()] <= tol_lse[:tokens][~w.isinf()]).all()


def test_lengths_at_the_end_of_32_bits(sb):  # noqa: F811
    """Lengths that only the table bounds: places of 2^31 and beyond it, before the first key and behind the last."""
    table, cu, pages = batch([96, 96, 96], [2, 2, 2], 32, 7)
    cache = filled(sb, pages, 32, 1, 64, 4)
    q = torch.randn(6, 2, 64, generator=torch.Generator().manual_seed(3)).bfloat16()
    kv, ends = [2 ** 31 - 1, 50, -2 ** 31], [2, 4, 2 ** 31 - 1]
    out, ws = torch.full((6, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda"), sb.make_cache_workspace(2, 2, 1, 64)
    sb.sol_attn_cache_attention(q.cuda(), ints([0] + ends), ints(kv), ints(table), cache, out, 2, ws)
    want, _, tol, _, _ = ref.attention(q, cu, [98, 50, 0], [row + [-1] for row in table], *held_values(cache), 32, True, 64 ** -0.5, pages)
    close(out, want, tol, torch.bfloat16)
    assert (out[4:] == 0).all()
