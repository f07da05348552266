"""Attention over the cache in the state in which long calls run: blocks with ten steps and more, rings that have turned, several pieces."""
import random

import pytest
import torch

from tests import cache_reference as ref
from tests.test_gpu_cache import batch, filled, ints, sb  # noqa: F401  (sb: a fixture)

pytestmark = pytest.mark.gpu
SMS = 148
FEW, FEW_WIDE, MANY = 4 * SMS, 3 * SMS, SMS                               # blocks: up to 8 rows, up to 48 rows, more
# kind: (requests as (keys, queries), Hq, Hk), 10 or more steps to a block
CALLS = {
    "tokens": ([(70001, 1)], 32, 16),
    "tokens, ragged": ([(60000, 1), (9, 1), (50111, 1), (0, 1), (9000, 1), (127, 1)], 16, 8),
    "drafts": ([(33000, 5), (20007, 3)], 16, 16),
    "drafts, wide": ([(30000, 4), (21000, 1)], 40, 8),
    "chunks": ([(8000, 300)], 40, 40),
    "chunks, ragged": ([(6001, 300), (20, 20), (5000, 130), (3000, 1), (2999, 700)], 32, 16),
}


def values_of(sb, cache):  # noqa: F811
    """What every slot holds, read back (exact in 16 bits; that reading is right is tested by the bytes)."""
    n, dt = cache.pages * cache.page_size, torch.bfloat16
    k, v = (torch.empty(n, cache.heads, cache.d, dtype=dt, device="cuda") for _ in range(2))
    sb.sol_attn_cache_read(cache, torch.arange(n, dtype=torch.int32, device="cuda"), k, v)
    return k.double(), v.double()


def steps_of_a_block(requests, H, Hk):
    """Steps that the block with the fewest has in the kernel for the most rows, from the header comments of the kernels."""
    rows = max(n for _, n in requests) * (H // Hk)
    tile, blocks = (8, FEW) if rows <= 8 else (16, FEW_WIDE) if rows <= 48 else (256, MANY)
    total = 0
    for kv, n in requests:
        r = n * (H // Hk)
        if rows <= 48 or r > 48 or len(requests) == 1:
            total += Hk * sum(max(1, -(-max(1, kv - n + (min((i + 1) * tile, r) - 1) // (H // Hk) + 1) // 128)) for i in range(-(-r // tile)))
    return total // blocks


def check(sb, cache, q, cu, kv, table, causal=True, twice=True, workspace=None):  # noqa: F811
    """Against the definition in 64 bits on the GPU; the same bits twice."""
    k, v = values_of(sb, cache)
    most = max(b - a for a, b in zip(cu, cu[1:]))
    ws = sb.make_cache_workspace(most, q.shape[1], cache.heads, cache.d) if workspace is None else workspace
    args = ints(cu), ints(kv), ints(table)
    runs = []
    for _ in range(2 if twice else 1):
        out, lse = torch.full_like(q, 9.0), torch.full(q.shape[:2], 9.0, device="cuda")
        sb.sol_attn_cache_attention(q, *args, cache, out, most, ws, lse=lse, causal=causal)
        assert sb.sol_attn_cache_read_status(ws) == sb.SOL_OK
        runs.append((out, lse))
    if twice:
        assert torch.equal(runs[0][0], runs[1][0]) and torch.equal(runs[0][1], runs[1][1])
    with torch.device("cuda"):
        want, want_lse, tol, tol_lse, _ = ref.attention(q, cu, kv, table, k, v, cache.page_size, causal, q.shape[2] ** -0.5, cache.pages)
    bound = tol + ref.half_step(q.dtype) * (want.abs() + tol) + (2.0 ** -25 if q.dtype == torch.float16 else 0)
    error = (out.double() - want).abs()
    assert (error <= bound).all(), (error / bound).nan_to_num(0).max().item()          # (a query without keys: both are 0)
    assert torch.equal(lse.isinf(), want_lse.isinf())
    some = ~want_lse.isinf()
    error, bound = (lse.double() - want_lse)[some].abs(), tol_lse[some]
    assert (error <= bound).all(), (error / bound).max().item()
    return out


def growing(sb, pages, page, Hk, d, table, kv, seed):  # noqa: F811
    """A cache whose keys have, in 16 channels, the logarithm of n / (n - position) of their request of n: with queries of 2 there the weights grow
    as 1 / (n - position), up to 2^14, so that maxima are replaced again and again while what was added before still counts."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    cache, n = sb.make_cache(pages, page, Hk, d), pages * page
    k, v = (torch.randn(n, Hk, d, generator=g, device="cuda") for _ in range(2))
    for row, m in zip(table, kv):
        pos = torch.arange(m, device="cuda")
        slots = torch.tensor(row, device="cuda")[pos // page] * page + pos % page
        ramp = torch.log(m / (m - pos).float()) * d ** 0.5 / 32           # (a logit of log(n / (n - position)) with queries of 2)
        k[slots, :, :16] = ramp[:, None, None]
    sb.sol_attn_cache_append(k.bfloat16(), (v + 0.3).bfloat16(), torch.arange(n, dtype=torch.int32, device="cuda"), cache)
    return cache


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind", list(CALLS))
@pytest.mark.parametrize("rising", [False, True], ids=["level", "rising"])
def test_long_calls(sb, kind, d, dtype, causal, rising):  # noqa: F811
    requests, H, Hk = CALLS[kind]
    kv, new = [r[0] for r in requests], [r[1] for r in requests]
    table, cu, pages = batch(kv, new, 128, 6)
    cache = growing(sb, pages, 128, Hk, d, table, kv, 3) if rising else filled(sb, pages, 128, Hk, d, 3)
    q = torch.randn(cu[-1], H, d, generator=torch.Generator().manual_seed(9)) * (0.3 if rising else 1.5)
    if rising:
        q[..., :16] = 2
    assert steps_of_a_block(requests, H, Hk) >= 10
    check(sb, cache, q.to(dtype).cuda(), cu, kv, table, causal)


@pytest.mark.parametrize("d, dtype", [(128, torch.bfloat16), (64, torch.float16)])
@pytest.mark.parametrize("kind", ["tokens", "drafts", "chunks"])
def test_missing_pages_amid_long_pieces(sb, kind, d, dtype):  # noqa: F811
    """Some pages are not there, found by a block at any of its steps while its other warps are at work."""
    requests, H, Hk = CALLS[kind]
    kv, new = [r[0] for r in requests], [r[1] for r in requests]
    table, cu, pages = batch(kv, new, 64, 5)
    rng = random.Random(8)
    for row in table:
        for j in range(0, len(row), 40):
            row[rng.randrange(j, min(j + 40, len(row)))] = rng.choice([-1, pages, 2 ** 31 - 1, -2 ** 31])
    cache = filled(sb, pages, 64, Hk, d, 3)
    q = torch.randn(cu[-1], H, d, generator=torch.Generator().manual_seed(9)).to(dtype).cuda()
    assert steps_of_a_block(requests, H, Hk) >= 10
    check(sb, cache, q, cu, kv, table)


@pytest.mark.parametrize("kind", list(CALLS))
@pytest.mark.parametrize("withheld", [5, 8, 10])
def test_a_wait_that_runs_out_late(sb, kind, withheld):  # noqa: F811
    """The arrival that is left out is that of a step behind the rings' first turn, with copies and products under way."""
    requests, H, Hk = CALLS[kind]
    kv, new = [r[0] for r in requests], [r[1] for r in requests]
    table, cu, pages = batch(kv, new, 64, 5)
    cache = filled(sb, pages, 64, Hk, 128, 3)
    q = torch.randn(cu[-1], H, 128, generator=torch.Generator().manual_seed(9)).bfloat16().cuda()
    ws, out = sb.make_cache_workspace(max(new), H, Hk, 128), torch.empty_like(q)
    assert steps_of_a_block(requests, H, Hk) > withheld // (2 if max(new) > 48 else 1)
    for limit in (200_000, 1):
        sb.sol_attn_debug_set_wait(limit, withheld)
        try:
            sb.sol_attn_cache_attention(q, ints(cu), ints(kv), ints(table), cache, out, max(new), ws)
            torch.cuda.synchronize()
        finally:
            sb.sol_attn_debug_set_wait()
        assert sb.sol_attn_cache_read_status(ws) == sb.SOL_ERR_DEVICE_TIMEOUT
        assert sb.sol_attn_cache_read_status(ws) == sb.SOL_OK
    check(sb, cache, q, cu, kv, table, workspace=ws)
