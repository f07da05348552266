"""The 4-bit cache and the operators around it against their definitions in 64 bits."""
import math
import random

import pytest
import torch

from tests import cache_reference as ref

pytestmark = pytest.mark.gpu
I32 = torch.int32


@pytest.fixture(scope="module")
def sb():
    from paper_2607_24027_b200 import binding
    binding.lib()
    return binding


def ints(x):
    return torch.tensor(x, dtype=I32, device="cuda")


# ------------------------------------------------------------------------------------------------------------------ block tables
def run_tables(sb, old, new, free, count, table, page, max_tokens, positions=True, pad=3):
    B = len(old)
    wide = torch.full((B, len(table[0]) + pad), -7, dtype=I32, device="cuda")
    wide[:, :len(table[0])] = ints(table)
    t = wide[:, :len(table[0])]
    cu, kv, result = torch.full((B + 1,), -9, dtype=I32, device="cuda"), torch.full((B,), -9, dtype=I32, device="cuda"), ints([-9, -9])
    slots, pos = torch.full((max_tokens,), -9, dtype=I32, device="cuda"), torch.full((max_tokens,), -9, dtype=I32, device="cuda")
    sb.sol_attn_block_tables(ints(old), ints(new), ints(free), ints([count]), t, cu, kv, slots, result, page,
                             positions=pos if positions else None)
    assert (wide[:, len(table[0]):] == -7).all()
    return t.tolist(), cu.tolist(), kv.tolist(), slots.tolist(), pos.tolist(), result.tolist()


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("B, longest, room, short", [(1, 1, 0, 0), (1, 300, 0, 0), (7, 90, 40, 0), (7, 90, 0, 3), (300, 40, 10, 0), (700, 9, 0, 20),
                                                     (5, 3000, 100, 2), (257, 1, 0, 0)])
def test_tables(sb, page, B, longest, room, short):
    rng = random.Random(B * page + longest)
    old = [rng.choice([0, 0, page, page - 1, rng.randrange(5 * page), -3]) for _ in range(B)]
    new = [rng.choice([0, 1, longest, rng.randint(0, longest), -1]) for _ in range(B)]
    width = max(1, max(-(-(max(o, 0) + max(n, 0)) // page) for o, n in zip(old, new)))
    pages = list(range(B * width + 9))
    rng.shuffle(pages)
    table = [[pages.pop() if j * page < o else -1 for j in range(width)] for o in old]
    total = sum(max(n, 0) for n in new)
    need = sum(-(-(max(o, 0) + max(n, 0)) // page) - -(-max(o, 0) // page) for o, n in zip(old, new))
    free = pages[:max(0, need - short) + (5 if short == 0 else 0)] or [12345]
    count = max(0, need - short) + (3 if short == 0 else 0)
    cap = total + room
    want = ref.tables(old, new, free, count, table, page, cap)
    got = run_tables(sb, old, new, free, count, table, page, cap)
    assert list(got[0]) == want[0] and list(got[1]) == want[1] and list(got[2]) == want[2]
    assert got[3][:total] == want[3] and got[4][:total] == want[4] and got[5] == want[5]
    assert all(x == -9 for x in got[3][total:] + got[4][total:])          # rows behind the last token


def test_tables_too_narrow_pages_missing_and_too_many_tokens(sb):
    # a table row that is too short, a begun page that is not there, a request that is longer than its table already
    old, new, table = [10, 20, 100], [60, 20, 5], [[3, -1], [4, -1], [5, 6]]
    want = ref.tables(old, new, [1, 2, 7, 8], 4, table, 16, 85)
    got = run_tables(sb, old, new, [1, 2, 7, 8], 4, table, 16, 85)
    assert [list(x) for x in got[:3]] == [list(x) for x in want[:3]] and got[3] == want[3] and got[5] == want[5]
    # more tokens than slots
    old, new, table = [3, 0, 0], [10, 20, 30], [[1, -1, -1], [-1] * 3, [-1] * 3]
    want = ref.tables(old, new, list(range(50, 60)), 10, table, 16, 25)
    got = run_tables(sb, old, new, list(range(50, 60)), 10, table, 16, 25, positions=False)
    assert list(got[0]) == want[0] and got[3] == want[3] and got[5] == want[5] and got[4] == [-9] * 25
    # nothing at all
    got = run_tables(sb, [0], [0], [5], 1, [[-1]], 16, 4)
    assert got[1] == [0, 0] and got[5] == [1, 0] and got[3] == [-9] * 4
    # a count beyond the list, and a negative one
    assert run_tables(sb, [0], [16], [5], 99, [[-1]], 16, 16)[5] == [0, 0]
    assert run_tables(sb, [0], [16], [5], -4, [[-1]], 16, 16)[5] == [0, 16]


# ---------------------------------------------------------------------------------------------------------------- norm and rotation
def rotation(rows, rot, far=0):
    angle = (torch.arange(rows, dtype=torch.float64) + far)[:, None] * 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)
    return angle.cos().float(), angle.sin().float()


def close(got, want, tol, dtype):
    """Within the tolerance before the last rounding plus that rounding."""
    got = got.double().cpu()
    bound = tol + ref.half_step(dtype) * (want.abs() + tol) + (2.0 ** -25 if dtype == torch.float16 else 0)
    bad = (got - want).abs() > bound
    assert not bad.any(), (int(bad.sum()), ((got - want).abs() / bound).max().item())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B, N, Hq, Hk, d, rot, layout", [(1, 1, 1, 1, 64, 64, 1), (1, 33, 40, 8, 128, 128, 1), (2, 517, 5, 3, 128, 96, 0),
                                                         (3, 7, 16, 1, 64, 32, 1), (1, 2100, 2, 2, 64, 48, 0), (2, 65, 24, 24, 128, 16, 1),
                                                         (1, 3, 7, 0, 128, 0, 1), (1, 5, 0, 9, 64, 64, 1)])
def test_norm_rope(sb, dtype, interleaved, B, N, Hq, Hk, d, rot, layout):
    g = torch.Generator().manual_seed(N + d)
    cos, sin = rotation(300, rot, far=100000) if rot else (None, None)
    pos = torch.randint(0, 300, (B, N), generator=g, dtype=I32)
    out_of_range = torch.rand(B, N, generator=g) < 0.1
    pos[out_of_range] = torch.tensor([-1, 300, 2 ** 31 - 1])[torch.randint(0, 3, (int(out_of_range.sum()),), generator=g)].int()
    weights = [1 + 0.3 * torch.randn(d, generator=g) if i == 0 or Hq == 0 else None for i in range(2)]
    call, want = [], []
    for H, w in ((Hq, weights[0]), (Hk, weights[1])):
        if not H:
            call += [None, None]
            want.append(None)
            continue
        x = (torch.randn(B, N, H, d, generator=g) * torch.exp(2 * torch.randn(B, N, H, 1, generator=g))).to(dtype)
        want.append((x, ref.norm_rope(x, w, cos, sin, pos, 1e-5, interleaved)))
        y = x.cuda() if layout == 1 else x.transpose(1, 2).contiguous().cuda()
        call += [y, torch.full_like(y, 7.0)]
    dev = [None if t is None else t.cuda() for t in (cos, sin, pos, *weights)]
    sb.sol_attn_qk_norm_rope(call[0], call[2], call[1], call[3], dev[0], dev[1], positions=dev[2], q_weight=dev[3], k_weight=dev[4],
                             eps=1e-5, interleaved=interleaved, layout=layout)
    for out, w in ((call[1], want[0]), (call[3], want[1])):
        if w is None:
            continue
        out = out if layout == 1 else out.transpose(1, 2)
        keep = ~out_of_range if rot else torch.ones(B, N, dtype=torch.bool)
        close(out.cpu()[keep], w[1][0][keep], w[1][1][keep], dtype)
        assert (out.cpu()[~keep] == 7).all()                             # positions outside the table: left alone


def test_norm_rope_strided_in_place_and_without_positions(sb):
    g = torch.Generator().manual_seed(5)
    B, N, H, d = 2, 19, 6, 128
    fused = torch.randn(B, N, 3 * H, d, generator=g).bfloat16()
    cos, sin = rotation(N - 2, d)                                         # the last two tokens have no row
    dev = fused.cuda()
    q, k = dev[:, :, :H], dev[:, :, H:2 * H]
    sb.sol_attn_qk_norm_rope(q, k, q, k, cos.cuda(), sin.cuda())
    at = torch.arange(N, dtype=I32).expand(B, N)
    for i, x in ((0, q), (H, k)):
        want, tol = ref.norm_rope(fused[:, :, i:i + H], None, cos, sin, at, 1e-6, False)
        close(x.cpu()[:, :N - 2], want[:, :N - 2], tol[:, :N - 2], torch.bfloat16)
        assert torch.equal(x.cpu()[:, N - 2:], fused[:, N - 2:, i:i + H])
    assert torch.equal(dev[:, :, 2 * H:].cpu(), fused[:, :, 2 * H:])
    empty = torch.empty(1, 0, H, d, dtype=torch.bfloat16, device="cuda")
    sb.sol_attn_qk_norm_rope(empty, None, empty, None, None, None)


# ---------------------------------------------------------------------------------------------------------------- writes and reads
def same(a, b):
    """Equal, with NaN where the other has it (fp16 inputs of this spread may overflow, which marks their token)."""
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(0, 1e300, -1e300), b.nan_to_num(0, 1e300, -1e300))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T, H, d, page, k_exp, v_exp", [(1, 1, 64, 16, 0, 0), (5, 3, 128, 16, 2, -3), (33, 8, 128, 64, 0, 1), (130, 2, 64, 32, -4, 0),
                                                         (517, 5, 64, 256, 0, 0), (257, 1, 128, 128, -1, 7),
                                                         (40, 2, 128, 16, 64, -64)])
def test_append_and_read(sb, dtype, T, H, d, page, k_exp, v_exp):
    g = torch.Generator().manual_seed(T * d)
    pages = -(-T // page) + 2
    cache = sb.make_cache(pages, page, H, d, k_exp, v_exp)
    cache.data.fill_(0xa5)
    before = cache.data.clone()
    k = (torch.randn(T, H, d, generator=g) * torch.exp(3 * torch.randn(T, H, d // 16, generator=g)).repeat_interleave(16, -1)).to(dtype)
    v = torch.randn(T, H, d, generator=g).to(dtype)
    k[0, 0], v[T // 2, H - 1, :16] = 0, -0.0
    v[T - 1, 0, 16:32] = torch.arange(16) * 0.125 + 4.5                  # ties: 6 is the largest, the scale is 1
    v[T - 1, 0, 16] = 6.0
    slots = torch.randperm(pages * page, generator=g)[:T].int()
    skipped = torch.rand(T, generator=g) < 0.2
    bad = slots.clone()
    bad[skipped] = torch.tensor([-1, pages * page, 2 ** 31 - 1, -2 ** 31])[torch.randint(0, 4, (int(skipped.sum()),), generator=g)].int()
    wide = torch.full((T, H + 2, 2 * d), 3.0, dtype=dtype, device="cuda")                # strided rows
    wide[:, 1:1 + H, :d], wide[:, 1:1 + H, d:] = k.cuda(), v.cuda()
    sb.sol_attn_cache_append(wide[:, 1:1 + H, :d], wide[:, 1:1 + H, d:], bad.cuda(), cache)
    want = [x.to(dtype).double() for x in ref.appended(k, v, k_exp, v_exp)]
    there = ~skipped
    # the bytes, by the documented layout
    held = ref.decode(cache.data, pages, page, H, d)
    untouched = torch.ones(pages * page, dtype=torch.bool)
    untouched[slots[there].long()] = False
    old = ref.decode(before, pages, page, H, d)
    for x, o, w, exp in zip(held, old, want, (k_exp, v_exp)):
        if dtype == torch.bfloat16:
            assert same(x[slots[there].long()] * 2.0 ** exp, w[there])
        assert same(x[untouched], o[untouched])
    # read back, into strided rows
    out = torch.full((T, H + 2, 2 * d), 5.0, dtype=dtype, device="cuda")
    sb.sol_attn_cache_read(cache, bad.cuda(), out[:, 1:1 + H, :d], out[:, 1:1 + H, d:])
    got = out.cpu().double()
    for i, w in enumerate(want):
        part = got[:, 1:1 + H, i * d:(i + 1) * d]
        assert same(part[there], w[there])
        assert (part[skipped] == 5).all()
    assert (got[:, 0] == 5).all() and (got[:, -1] == 5).all()
    alone = torch.empty(T, H, d, dtype=dtype, device="cuda")
    sb.sol_attn_cache_read(cache, slots.cuda(), None, alone)
    assert same(alone.cpu().double()[there], want[1][there])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_codes_of_every_number(sb, dtype):
    """Every 16-bit pattern against many largest elements, all that are ties among them."""
    every = torch.arange(-2 ** 15, 2 ** 15, dtype=torch.int32).to(torch.int16).view(dtype)
    every = every[torch.isfinite(every) & (every != 0)]
    g = torch.Generator().manual_seed(3)
    rows = []
    for top in (0.0107, 0.09, 0.75, 1.0, 1.3, 6.0, 6.375, 100.0, 2688.0, 60000.0):
        e = every[every.abs().double() <= top]
        e = e[torch.randperm(len(e), generator=g)][:15 * 4000]
        e = e[:len(e) // 15 * 15].view(-1, 15)
        rows.append(torch.cat([torch.full((len(e), 1), top).to(dtype), e], 1))
    x = torch.cat(rows)
    x = x[:len(x) // 8 * 8].view(-1, 1, 128)
    T = len(x)
    cache = sb.make_cache(-(-T // 64), 64, 1, 128)
    slots = torch.arange(T, dtype=I32, device="cuda")
    sb.sol_attn_cache_append(x.cuda(), x.flip(-1).contiguous().cuda(), slots, cache)
    held = ref.decode(cache.data, cache.pages, 64, 1, 128)
    assert torch.equal(held[0][:T], ref.held(x, 0)[2]) and torch.equal(held[1][:T], ref.held(x.flip(-1), 0)[2])


@pytest.mark.parametrize("d", [64, 128])
def test_numbers_that_are_not_finite_mark_their_token(sb, d):
    g = torch.Generator().manual_seed(d)
    k, v = torch.randn(40, 3, d, generator=g).bfloat16(), torch.randn(40, 3, d, generator=g).bfloat16()
    k[3, 1, d - 1], k[7, 0, 5], v[9, 2, 20], v[39, 1, 0] = math.nan, math.inf, -math.inf, math.nan
    cache = sb.make_cache(3, 16, 3, d)
    sb.sol_attn_cache_append(k.cuda(), v.cuda(), torch.arange(40, dtype=I32, device="cuda"), cache)
    out = [torch.empty_like(k, device="cuda") for _ in range(2)]
    sb.sol_attn_cache_read(cache, torch.arange(40, dtype=I32, device="cuda"), *out)
    for got, want in zip(out, ref.appended(k, v, 0, 0)):
        assert torch.equal(got.cpu().double().nan_to_num(12345.0), want.nan_to_num(12345.0))
    assert out[0].isnan().sum() == 4 * 16 and not out[1].isnan().any()


# ---------------------------------------------------------------------------------------------------------------------- attention
def filled(sb, pages, page, Hk, d, seed, k_exp=0, v_exp=0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    cache = sb.make_cache(pages, page, Hk, d, k_exp, v_exp)
    n = pages * page
    k = torch.randn(n, Hk, d, generator=g, device="cuda") * 2.0 ** k_exp
    v = (torch.randn(n, Hk, d, generator=g, device="cuda") + 0.3) * 2.0 ** v_exp
    sb.sol_attn_cache_append(k.to(dtype), v.to(dtype), torch.arange(n, dtype=I32, device="cuda"), cache)
    return cache


def held_values(cache):
    k, v = ref.decode(cache.data, cache.pages, cache.page_size, cache.heads, cache.d)
    return k * 2.0 ** cache.k_exp, v * 2.0 ** cache.v_exp


def batch(kv, new, page, seed, spare=2, width=0):
    """Block tables (list of lists) over shuffled pages, cu_q, number of pages."""
    rng = random.Random(seed)
    counts = [-(-n // page) for n in kv]
    pages = list(range(sum(counts) + spare))
    rng.shuffle(pages)
    columns = max(max(counts), 1) + width
    table, at = [], 0
    for c in counts:
        table.append(pages[at:at + c] + [rng.choice([-1, 10 ** 6, 2 ** 31 - 1]) for _ in range(columns - c)])
        at += c
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    return table, cu, sum(counts) + spare


def check_attention(sb, cache, q, cu, kv, table, causal, scale=0.0, pad=0, max_q=None, lse=True, values=None, workspace=None):
    T, H, d = q.shape
    k, v = held_values(cache) if values is None else values
    want, want_lse, tol, tol_lse, touched = ref.attention(q.cpu(), cu, kv, table, k, v, cache.page_size, causal,
                                                          scale or d ** -0.5, cache.pages)
    out = torch.full((T, H, d), 9.0, dtype=q.dtype, device="cuda")
    got_lse = torch.full((T, H), 9.0, device="cuda") if lse else None
    most = max_q or max(b - a for a, b in zip(cu, cu[1:])) or 1
    ws = sb.make_cache_workspace(most, H, cache.heads, d) if workspace is None else workspace
    sb.sol_attn_cache_attention(q, ints(cu), ints(kv), ints(table), cache, out, most, ws, lse=got_lse, causal=causal, scale=scale)
    assert sb.sol_attn_cache_read_status(ws) == sb.SOL_OK
    poisoned = want.isnan().any(-1)
    assert torch.equal(out.cpu().isnan().any(-1), poisoned)
    fine = touched[:, None] & ~poisoned
    close(out.cpu()[fine], want[fine], tol[fine], q.dtype)
    assert (out.cpu()[~touched] == 9).all()                              # rows of no request: left as they were
    if lse:
        x = got_lse.double().cpu()
        assert torch.equal(x[fine].isinf(), want_lse[fine].isinf())
        some = fine & ~want_lse.isinf()
        assert ((x - want_lse).abs()[some] <= tol_lse[some]).all(), ((x - want_lse).abs()[some] - tol_lse[some]).max()
        assert (x[~touched] == 9).all()
    return out, got_lse


# requests as (keys, queries): lengths around units, steps and pages; queries without keys; keys without queries
STEPS = [(1, 1)], [(0, 1)], [(15, 1), (16, 1), (17, 1), (0, 1), (31, 1), (33, 1)], [(127, 1), (128, 1), (129, 1), (1000, 1), (2, 1)], [(4100, 1)]
CHUNKS = [(3, 3), (2, 5), (40, 7), (0, 4), (64, 0)], [(200, 3), (131, 2), (1, 2)], [(300, 130), (77, 77), (129, 1)], [(515, 260), (60, 33)]


@pytest.mark.parametrize("dtype, page, H, Hk, d", [(torch.bfloat16, 16, 8, 2, 128), (torch.float16, 64, 4, 4, 64), (torch.bfloat16, 32, 16, 1, 64),
                                                   (torch.float16, 128, 5, 1, 128), (torch.bfloat16, 256, 6, 2, 128)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("requests", STEPS + CHUNKS, ids=lambda r: "-".join(f"{a}x{b}" for a, b in r))
def test_attention(sb, dtype, page, H, Hk, d, causal, requests):
    kv, new = [r[0] for r in requests], [r[1] for r in requests]
    table, cu, pages = batch(kv, new, page, len(kv), width=1)
    cache = filled(sb, pages, page, Hk, d, 3, k_exp=1, v_exp=-2, dtype=dtype)
    q = (torch.randn(cu[-1] + 3, H, d, generator=torch.Generator().manual_seed(9)) * 1.5).to(dtype).cuda()
    check_attention(sb, cache, q, cu, kv, table, causal, scale=0.5 * d ** -0.5)


@pytest.mark.parametrize("requests, most", [(333, 2), (700, 60)])
def test_many_requests(sb, requests, most):
    """More than there are threads to look at their lengths at once, for either kernel."""
    rng = random.Random(2)
    kv = [rng.choice([1, 5, 16, 100, 300]) for _ in range(requests)]
    new = [rng.choice([1, 1, 1, 0, 2]) if rng.random() < 0.9 else rng.randint(1, most) for _ in kv]
    table, cu, pages = batch(kv, new, 16, 1)
    cache = filled(sb, pages, 16, 2, 64, 4)
    q = torch.randn(cu[-1], 2, 64, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    check_attention(sb, cache, q, cu, kv, table, True)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("keys, queries, H", [(20000, 64, 1), (20000, 1, 3), (9000, 1, 96), (1300, 7, 40)])
def test_one_item_among_all_blocks(sb, d, keys, queries, H):
    """A single key / value head: every block has a piece of the same item, or of one of two; a token with more heads than a tile of rows."""
    table, cu, pages = batch([keys], [queries], 64, 1)
    cache = filled(sb, pages, 64, 1, d, 4)
    q = torch.randn(queries, H, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    check_attention(sb, cache, q, cu, [keys], table, True)


def test_strides_and_a_larger_hint(sb):
    kv, new = [70, 33], [2, 1]
    table, cu, pages = batch(kv, new, 16, 1)
    cache = filled(sb, pages, 16, 2, 128, 4)
    g = torch.Generator().manual_seed(1)
    wide = torch.randn(3, 3, 8, 128, generator=g).half().cuda()
    q = wide[:, 1, ::2]
    out = torch.full((3, 2, 9, 128), 9.0, dtype=torch.half, device="cuda")
    ws = sb.make_cache_workspace(1, 4, 2, 128)
    plain, _ = check_attention(sb, cache, q.contiguous(), cu, kv, table, True)
    sb.sol_attn_cache_attention(q, ints(cu), ints(kv), ints(table), cache, out[:, 1, 1:9:2], 2, sb.make_cache_workspace(2, 4, 2, 128))
    assert torch.equal(out[:, 1, 1:9:2], plain)
    rest = out.clone()
    rest[:, 1, 1:9:2] = 9
    assert (rest == 9).all()
    # max_q only chooses the kernel: a longer request is computed all the same
    check_attention(sb, cache, q.contiguous(), cu, kv, table, True, max_q=1, workspace=ws)


@pytest.mark.parametrize("new", [1, 40])
def test_pages_that_are_not_there_and_bytes_behind_the_last_key(sb, new):
    kv, new = [100, 50], [new, 1]
    table, cu, pages = batch(kv, new, 16, 1)
    cache = filled(sb, pages, 16, 1, 128, 4)
    table[0][2], table[0][4] = -5, pages                                   # not seen
    raw = cache.data.view(pages, 1, 1, 18 * 128)
    last = raw[table[1][3], 0, 0]                                         # keys 48 and 49 of request 1 and 14 tokens behind
    keep = ref.decode(cache.data, pages, 16, 1, 128)
    k48 = [x[table[1][3] * 16:table[1][3] * 16 + 2].clone() for x in keep]
    scales = last[16 * 128:].clone()
    last[16 * 128:] = 0x7f                                                # NaN scales, then the two keys' own again
    for i in range(2):
        for group in range(8):
            for at in ((i % 8 * 4 + group // 2) * 4 + i // 8 * 2 + group % 2, 128 + group * 16 + i % 8 // 2 * 4 + i // 8 * 2 + i % 2):
                last[16 * 128 + at] = scales[at]
    k, v = held_values(cache)
    for x, w in zip((k, v), k48):
        assert torch.equal(x[table[1][3] * 16:table[1][3] * 16 + 2], w)
    q = torch.randn(cu[-1], 2, 128, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    check_attention(sb, cache, q, cu, kv, table, True)


@pytest.mark.parametrize("new", [1, 3, 90])
def test_numbers_that_are_not_finite_reach_only_who_sees_them(sb, new):
    """Key or value of a token in the causal part: the queries before it are exact."""
    kv = [200, 150]
    table, cu, pages = batch(kv, [new, 1], 16, 1)
    cache = filled(sb, pages, 16, 2, 64, 4)
    bad = [table[0][(200 - 1) // 16] * 16 + 199 % 16]                     # the last token: only the last query sees it
    x = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    y = x.clone()
    y[0, 1, 63] = math.inf                                                # a value, in one of two heads
    sb.sol_attn_cache_append(x, y, ints(bad), cache)
    q = torch.randn(cu[-1], 4, 64, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    out, _ = check_attention(sb, cache, q, cu, kv, table, True)
    assert out.isnan().any(-1).nonzero().tolist() == [[new - 1, 2], [new - 1, 3]]
    # queries that are not finite give NaN, and only they
    q[0, 1, 5], q[new, 2, 0] = math.inf, math.nan
    sb.sol_attn_cache_attention(q, ints(cu), ints(kv), ints(table), cache, out, new, sb.make_cache_workspace(new, 4, 2, 64))
    assert {(0, 1), (new, 2)} | {(new - 1, 2), (new - 1, 3)} == {tuple(x) for x in out.isnan().any(-1).nonzero().tolist()}


@pytest.mark.parametrize("new", [1, 20])
def test_large_and_small_queries_and_logits(sb, new):
    """Rows whose elements span fp16's range and far beyond, logits of hundreds: the scaling per row and the running maximum."""
    kv = [700, 1500]
    table, cu, pages = batch(kv, [new, 1], 32, 1)
    cache = filled(sb, pages, 32, 1, 128, 4)
    g = torch.Generator().manual_seed(1)
    q = torch.randn(cu[-1], 3, 128, generator=g)
    q[:, 1] *= 1e18
    q[:, 2] *= 1e-20
    q[0, 0, :64] *= 2.0 ** -10
    q = q.bfloat16().cuda()
    values = held_values(cache)
    check_attention(sb, cache, q[:, :1].contiguous(), cu, kv, table, True, scale=3.0, values=values)
    check_attention(sb, cache, q[:, 1:2].contiguous(), cu, kv, table, True, scale=1e-18, values=values)
    check_attention(sb, cache, q[:, 2:].contiguous(), cu, kv, table, True, scale=1e20, values=values)


def test_offsets_past_32_bits(sb):
    """A cache of more than 4 GB, whose last pages are used."""
    page, Hk, d = 256, 8, 128
    pages = (2 ** 32 + 2 ** 28) // (Hk * page * 18 * d // 16)
    cache = sb.make_cache(pages, page, Hk, d)
    assert cache.data.numel() > 2 ** 32
    used = [pages - 1, 3, pages - 2]
    g = torch.Generator(device="cuda").manual_seed(1)
    n = 600
    k, v = (torch.randn(n, Hk, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    pos = torch.arange(n)
    slots = (torch.tensor(used)[pos // page] * page + pos % page).int().cuda()
    sb.sol_attn_cache_append(k, v, slots, cache)
    out = [torch.empty_like(k) for _ in range(2)]
    sb.sol_attn_cache_read(cache, slots, *out)
    values = ref.appended(k.cpu(), v.cpu(), 0, 0)
    assert all(torch.equal(a.cpu().double(), b) for a, b in zip(out, values))
    small = sb.make_cache(3, page, Hk, d)                                  # the same tokens at the start of another cache
    for new in (1, 50):
        q = torch.randn(new, Hk, d, generator=g, device="cuda").bfloat16()
        res = []
        for c, rows in ((cache, used), (small, [0, 1, 2])):
            if c is small:
                sb.sol_attn_cache_append(k, v, pos.int().cuda(), small)
            o = torch.empty_like(q)
            sb.sol_attn_cache_attention(q, ints([0, new]), ints([n]), ints([rows]), c, o, new, sb.make_cache_workspace(new, Hk, Hk, d))
            res.append(o)
        assert torch.equal(*res)


@pytest.mark.parametrize("new", [1, 9, 200])
def test_replay_streams_and_repetition(sb, new):
    """A captured call replayed on other contents and lengths, on another stream; the same call twice gives the same bits."""
    kv, H, Hk, d, page = [900, 333, 64], 8, 2, 128, 64
    table, cu, pages = batch([1000] * 3, [new, 1, 1], page, 1)
    caches = [filled(sb, pages, page, Hk, d, s) for s in (4, 5)]
    g = torch.Generator().manual_seed(1)
    qs = [torch.randn(cu[-1], H, d, generator=g).bfloat16().cuda() for _ in range(2)]
    lens = [kv, [1000, 1, 700]]
    ws = sb.make_cache_workspace(new, H, Hk, d)
    out, kv_d, q, cache = torch.empty_like(qs[0]), ints(kv), qs[0].clone(), sb.make_cache(pages, page, Hk, d)
    want = []
    for i in range(2):
        cache.data.copy_(caches[i].data)
        want.append(check_attention(sb, cache, qs[i], cu, lens[i], table, True)[0])
        assert torch.equal(want[-1], check_attention(sb, cache, qs[i], cu, lens[i], table, True)[0])
    cu_d, table_d = ints(cu), ints(table)
    run = lambda: sb.sol_attn_cache_attention(q, cu_d, kv_d, table_d, cache, out, new, ws)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run()
        for i in (1, 0, 1):
            q.copy_(qs[i]), kv_d.copy_(ints(lens[i])), cache.data.copy_(caches[i].data)
            out.fill_(9)
            graph.replay()
            side.synchronize()
            assert torch.equal(out, want[i])
    assert sb.sol_attn_cache_read_status(ws) == sb.SOL_OK


@pytest.mark.parametrize("requests", [[(1000, 1)] * 3, [(600, 5), (600, 1)], [(900, 300), (500, 1)], [(900, 300)]],
                         ids=["single tokens", "few rows", "mixed", "many rows"])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_clean(sb, requests):
    """Each kernel leaves out the arrival for a stage (a test hook): its waits run out, it ends, says so, and leaves nothing behind."""
    kv, new = [r[0] for r in requests], [r[1] for r in requests]
    table, cu, pages = batch(kv, new, 16, 3)
    cache = filled(sb, pages, 16, 2, 128, 4)
    q = torch.randn(cu[-1], 4, 128, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    ws, out = sb.make_cache_workspace(max(new), 4, 2, 128), torch.empty_like(q)
    for withheld in (0, 1, 3):
        sb.sol_attn_debug_set_wait(200_000, withheld)
        try:
            sb.sol_attn_cache_attention(q, ints(cu), ints(kv), ints(table), cache, out, max(new), ws)
            torch.cuda.synchronize()
        finally:
            sb.sol_attn_debug_set_wait()
        # (blocks have a single step here: one stage, or the two tiles of its keys and its values)
        if withheld == 0 or (withheld == 1 and max(new) > 100):
            assert sb.sol_attn_cache_read_status(ws) == sb.SOL_ERR_DEVICE_TIMEOUT
        sb.sol_attn_cache_read_status(ws)
        assert sb.sol_attn_cache_read_status(ws) == sb.SOL_OK                # cleared by being read
        check_attention(sb, cache, q, cu, kv, table, True, workspace=ws)


def test_calls_on_two_streams_and_from_another_one(sb):
    """Two calls at once, each with a workspace of its own; the stream given, not the current one, is used."""
    kv, new = [3000, 700], [1, 80]
    table, cu, pages = batch(kv, new, 64, 3)
    cache = filled(sb, pages, 64, 2, 128, 4)
    g = torch.Generator().manual_seed(1)
    qs = [torch.randn(cu[-1], 8, 128, generator=g).bfloat16().cuda() for _ in range(2)]
    args = ints(cu), ints(kv), ints(table)
    want = [check_attention(sb, cache, q, cu, kv, table, True)[0] for q in qs]
    streams, spaces, outs = [torch.cuda.Stream() for _ in qs], [sb.make_cache_workspace(80, 8, 2, 128) for _ in qs], [torch.empty_like(q) for q in qs]
    torch.cuda.synchronize()
    for _ in range(10):
        for q, st, ws, out in zip(qs, streams, spaces, outs):
            sb.sol_attn_cache_attention(q, *args, cache, out, 80, ws, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("rows", [1, 3, 100])
def test_unaligned_rows_of_32_bytes(sb, rows):
    """Rows on 16-byte boundaries only, for every operator that has a path for 32."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    d, H = 64, 2
    flat = torch.randn(rows * (2 * H * d + 8) + 8, generator=g, device="cuda").bfloat16()
    k = flat[8:].as_strided((rows, H, d), (2 * H * d + 8, d, 1))
    v = flat[8 + H * d:].as_strided((rows, H, d), (2 * H * d + 8, d, 1))
    cache, slots = sb.make_cache(8, 16, H, d), torch.arange(rows, dtype=I32, device="cuda")
    sb.sol_attn_cache_append(k, v, slots, cache)
    room = torch.zeros_like(flat)
    ko, vo = (room[n:].as_strided((rows, H, d), (2 * H * d + 8, d, 1)) for n in (8, 8 + H * d))
    sb.sol_attn_cache_read(cache, slots, ko, vo)
    for got, x in ((ko, k), (vo, v)):
        assert torch.equal(got.cpu().double(), ref.held(x.cpu(), 0)[2])
    table = [list(range(8))]
    check_attention(sb, cache, ko, [0, rows], [rows], table, True, values=held_values(cache))
    sb.sol_attn_qk_norm_rope(ko[None], None, ko[None], None, None, None)
    want, tol = ref.norm_rope(torch.as_tensor(ref.held(k.cpu(), 0)[2])[None], None, None, None, None, 1e-6, False)
    close(ko.cpu()[None], want, tol, torch.bfloat16)


def test_refusals_of_the_binding(sb):
    cache, q = sb.make_cache(4, 16, 2, 64), torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    cu, kv, table, ws = ints([0, 2]), ints([10]), ints([[0]]), sb.make_cache_workspace(2, 4, 2, 64)
    call = lambda **kw: sb.sol_attn_cache_attention(*[kw.get(n, x) for n, x in (("q", q), ("cu", cu), ("kv", kv), ("table", table),  # noqa: E731
                                                                               ("cache", cache), ("out", torch.empty_like(q)))], 2,
                                                    kw.get("ws", ws), lse=kw.get("lse"))
    call()
    for bad in (dict(q=q.float()), dict(q=q[..., ::2]), dict(cu=cu.long()), dict(cu=ints([0, 1, 2])), dict(table=table[0]), dict(kv=kv.cpu()),
                dict(out=torch.empty_like(q).half()), dict(lse=torch.empty(2, 3, device="cuda")), dict(ws=ws.float()),
                dict(cache=sb.make_cache(4, 16, 2, 128))):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(sb.SolAttnError):
        call(ws=ws[:2048])
    with pytest.raises(ValueError):
        sb.sol_attn_cache_append(q, q, ints([1, 2]), cache)               # four heads into a cache of two
    with pytest.raises(ValueError):
        sb.sol_attn_qk_norm_rope(q[None], None, None, None, None, None)
    with pytest.raises(ValueError):
        sb.sol_attn_qk_norm_rope(q[None], q[None].half(), q[None], q[None].half(), None, None)
    with pytest.raises(sb.SolAttnError):
        x = torch.zeros(1, 2, 4, 72, dtype=torch.bfloat16, device="cuda")
        sb.sol_attn_qk_norm_rope(x, None, x, None, None, None)


# ------------------------------------------------------------------------------------------------------------------ all together
@pytest.mark.parametrize("dtype, H, Hk, d, page", [(torch.bfloat16, 8, 2, 128, 16), (torch.float16, 4, 4, 64, 64)])
def test_a_generator(sb, dtype, H, Hk, d, page):
    """Prompts, a chunk and single tokens of three requests, as a program runs them: tables, norm and rotation, writes, attention."""
    g = torch.Generator().manual_seed(1)
    B, width, pages = 3, 8, 30
    cos, sin = rotation(width * page, d)
    cos_d, sin_d = cos.cuda(), sin.cuda()
    weight = 1 + 0.1 * torch.randn(d, generator=g)
    cache, counts = sb.make_cache(pages, page, Hk, d), [ints([pages, 0]), ints([0, 0])]
    table_d, lens = torch.full((B, width), -1, dtype=I32, device="cuda"), torch.zeros(B, dtype=I32, device="cuda")
    free = torch.arange(pages, dtype=I32, device="cuda")
    host_table, host_old, host_count = [[-1] * width] * B, [0] * B, pages
    all_k, all_v = torch.zeros(pages * page, Hk, d, dtype=torch.float64), torch.zeros(pages * page, Hk, d, dtype=torch.float64)
    for step, new in enumerate([[37, 5, 60], [1, 20, 1], [1, 1, 1], [1, 1, 0]]):
        T = sum(new)
        q, k, v = ((torch.randn(T, h, d, generator=g) * 2).to(dtype) for h in (H, Hk, Hk))
        cu, kv, slots, pos = (torch.empty(n, dtype=I32, device="cuda") for n in (B + 1, B, T, T))
        now, then = counts[step % 2], counts[(step + 1) % 2]
        sb.sol_attn_block_tables(lens, ints(new), free, now[:1], table_d, cu, kv, slots, then, page, positions=pos)
        qo, ko = torch.empty_like(q, device="cuda"), torch.empty_like(k, device="cuda")
        sb.sol_attn_qk_norm_rope(q.cuda()[None], k.cuda()[None], qo[None], ko[None], cos_d, sin_d, positions=pos[None], q_weight=weight.cuda(),
                                 k_weight=weight.cuda())
        sb.sol_attn_cache_append(ko, v.cuda(), slots, cache)
        out, ws = torch.empty_like(qo), sb.make_cache_workspace(max(new), H, Hk, d)
        sb.sol_attn_cache_attention(qo, cu, kv, table_d, cache, out, max(new), ws)
        # the same in 64 bits
        host_table, hcu, hkv, hslots, hpos, result = ref.tables(host_old, new, list(range(pages)), host_count, host_table, page, T)
        host_old, host_count = hkv, result[0]
        assert table_d.tolist() == host_table and cu.tolist() == hcu and kv.tolist() == hkv and slots.tolist() == hslots
        assert then.tolist() == result
        at = torch.tensor(hpos, dtype=I32)[None]
        for x, got in ((q, qo), (k, ko)):
            want, tol = ref.norm_rope(x[None], weight, cos, sin, at, 1e-6, False)
            close(got.cpu()[None], want, tol, dtype)
        # (what is written is the rounded result: it may be a rounding away from the reference's)
        all_k[hslots], all_v[hslots] = ref.appended(ko.cpu(), v, 0, 0)
        want, _, tol, _, touched = ref.attention(qo.cpu(), hcu, hkv, host_table, all_k, all_v, page, True, d ** -0.5, pages)
        assert touched.all()
        close(out, want, tol, dtype)
        lens = kv


def test_a_captured_step(sb):
    """A decoding step of all four operators as one graph, replayed step after step with what a program changes between them."""
    B, H, Hk, d, page, width, pages = 5, 8, 2, 128, 16, 6, 40
    g = torch.Generator().manual_seed(3)
    start = [3, 15, 16, 40, 0]
    cos, sin = (x.cuda() for x in rotation(width * page, d))
    free = torch.arange(pages, dtype=I32, device="cuda")

    def fresh():
        s = dict(old=ints(start), new=ints([1] * B), count=ints([pages - 5 * 3]), table=torch.full((B, width), -1, dtype=I32, device="cuda"),
                 cache=filled(sb, pages, page, Hk, d, 6), cu=ints([0] * (B + 1)), kv=ints([0] * B), slots=ints([0] * B), pos=ints([0] * B),
                 result=ints([0, 0]), ws=sb.make_cache_workspace(1, H, Hk, d))
        s["table"][:, :3] = torch.arange(pages - 15, pages, dtype=I32).view(B, 3).cuda()
        s.update({n: torch.zeros(B, h, d, dtype=torch.bfloat16, device="cuda") for n, h in (("q", H), ("k", Hk), ("v", Hk), ("qr", H), ("kr", Hk), ("out", H))})
        return s

    def step(s):
        sb.sol_attn_block_tables(s["old"], s["new"], free, s["count"], s["table"], s["cu"], s["kv"], s["slots"], s["result"], page, positions=s["pos"])
        sb.sol_attn_qk_norm_rope(s["q"][None], s["k"][None], s["qr"][None], s["kr"][None], cos, sin, positions=s["pos"][None])
        sb.sol_attn_cache_append(s["kr"], s["v"], s["slots"], s["cache"])
        sb.sol_attn_cache_attention(s["qr"], s["cu"], s["kv"], s["table"], s["cache"], s["out"], 1, s["ws"])

    plain, graphed = fresh(), fresh()
    step(fresh())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(graphed)
    for _ in range(20):
        x = [torch.randn(B, h, d, generator=g).bfloat16() for h in (H, Hk, Hk)]
        for s in (plain, graphed):
            for n, y in zip(("q", "k", "v"), x):
                s[n].copy_(y)
        step(plain)
        graph.replay()
        for n in ("table", "kv", "slots", "pos", "result", "out"):
            assert torch.equal(plain[n], graphed[n]), n
        assert torch.equal(plain["cache"].data, graphed["cache"].data) and not plain["out"].isnan().any()
        for s in (plain, graphed):                                         # the next step: lengths and the count move on
            s["old"].copy_(s["kv"]), s["count"].copy_(s["result"][:1])
    assert plain["kv"].tolist() == [n + 20 for n in start]
