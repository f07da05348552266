"""Cache operators without a GPU: what the C entry points refuse before anything is launched, sizes, and the byte layout."""
import ctypes
import random

import pytest
import torch

from tests import cache_reference as ref


@pytest.fixture(scope="module")
def sb():
    from paper_2607_24027_b200 import build, binding
    build.build()
    return binding


def P(x):
    return ctypes.c_void_p(x)


def test_cache_and_workspace_sizes(sb):
    assert sb.sol_attn_cache_bytes(3, 16, 2, 128) == 3 * 2 * 18 * 128
    assert sb.sol_attn_cache_bytes(5, 64, 1, 64) == 5 * 4 * 18 * 64
    for bad in ((0, 16, 2, 128), (3, 24, 2, 128), (3, 512, 2, 128), (3, 8, 2, 128), (3, 16, 0, 128), (3, 16, 1025, 128), (3, 16, 2, 96),
                (2 ** 27, 16, 2, 128), (-1, 16, 2, 64)):
        assert sb.sol_attn_cache_bytes(*bad) == 0, bad
    assert sb.sol_attn_cache_bytes(2 ** 27 - 1, 16, 8, 128) == (2 ** 27 - 1) * 8 * 18 * 128      # past 32 bits
    assert sb.sol_attn_cache_workspace_bytes(1, 8, 8, 128) % 1024 == 0
    for bad in ((0, 8, 8, 128), (1, 8, 3, 128), (1, 8, 8, 96), (1, 0, 1, 64), (1, 2048, 8, 64)):
        assert sb.sol_attn_cache_workspace_bytes(*bad) == 0, bad
    with pytest.raises(sb.SolAttnError):
        sb.make_cache(4, 24, 2, 128, device="cpu")


def cache_of(sb, **kw):
    c = dict(data=4096, pages=4, page_size=16, Hk=2, d=128, k_exp=0, v_exp=0)
    c.update(kw)
    return sb._Cache(*(c[n] for n in ("data", "pages", "page_size", "Hk", "d", "k_exp", "v_exp")))


BAD_CACHES = [(dict(data=None), "INVALID"), (dict(data=4104), "INVALID"), (dict(pages=0), "INVALID"), (dict(k_exp=65), "INVALID"),
              (dict(v_exp=-65), "INVALID"), (dict(page_size=48), "SHAPE"), (dict(d=32), "SHAPE"), (dict(Hk=2000), "SHAPE")]


@pytest.mark.parametrize("change, why", BAD_CACHES)
def test_bad_caches_are_refused(sb, change, why):
    want = sb.SOL_ERR_INVALID_ARG if why == "INVALID" else sb.SOL_ERR_UNSUPPORTED_SHAPE
    c, st = cache_of(sb, **change), (ctypes.c_int64 * 2)(256, 128)
    for f in (sb.lib().sol_attn_cache_append, sb.lib().sol_attn_cache_read):
        assert f(ctypes.byref(c), P(4096), P(4096), st, st, P(4096), 4, 0, None) == want
    assert sb.lib().sol_attn_cache_attention(ctypes.byref(attention_args(sb, cache=c))) == want


def test_bad_rows_are_refused(sb):
    st, odd, c = (ctypes.c_int64 * 2)(256, 128), (ctypes.c_int64 * 2)(256, 124), cache_of(sb)
    bad, f = sb.SOL_ERR_INVALID_ARG, sb.lib().sol_attn_cache_append
    assert f(None, P(4096), P(4096), st, st, P(4096), 4, 0, None) == bad
    assert f(ctypes.byref(c), None, P(4096), st, st, P(4096), 4, 0, None) == bad
    assert f(ctypes.byref(c), P(4096), P(4100), st, st, P(4096), 4, 0, None) == bad
    assert f(ctypes.byref(c), P(4096), P(4096), st, odd, P(4096), 4, 0, None) == bad
    assert f(ctypes.byref(c), P(4096), P(4096), st, None, P(4096), 4, 0, None) == bad
    assert f(ctypes.byref(c), P(4096), P(4096), st, st, None, 4, 0, None) == bad
    assert f(ctypes.byref(c), P(4096), P(4096), st, st, P(4098), 4, 0, None) == bad
    assert f(ctypes.byref(c), P(4096), P(4096), st, st, P(4096), -1, 0, None) == bad
    assert f(ctypes.byref(c), P(4096), P(4096), st, st, P(4096), 4, 2, None) == bad
    assert f(ctypes.byref(c), None, None, st, st, None, 0, 0, None) == sb.SOL_OK        # nothing to do
    assert sb.lib().sol_attn_cache_read(ctypes.byref(c), None, None, st, st, P(4096), 4, 0, None) == bad


def attention_args(sb, cache=None, **kw):
    two = ctypes.c_int64 * 2
    a = dict(q=4096, out=4096 * 9, lse=None, q_stride=two(512, 128), out_stride=two(512, 128), table_stride=8, cu_q=4096, kv_lens=4096,
             block_tables=4096, tokens=5, requests=2, max_blocks=8, max_q=4, Hq=4, type=0, causal=1, scale=0.0, workspace=1 << 20,
             workspace_bytes=1 << 30)
    a.update(kw)
    return sb._CacheArgs(cache=cache if cache is not None else cache_of(sb), **a)


BAD_ATTENTION = [(dict(tokens=-1), "INVALID"), (dict(requests=-1), "INVALID"), (dict(max_q=0), "INVALID"), (dict(max_blocks=0), "INVALID"),
                 (dict(type=3), "INVALID"), (dict(scale=float("nan")), "INVALID"), (dict(scale=float("inf")), "INVALID"),
                 (dict(table_stride=7), "INVALID"), (dict(q=None), "INVALID"), (dict(out=4104), "INVALID"), (dict(out=4096), "INVALID"), (dict(cu_q=None), "INVALID"),
                 (dict(kv_lens=4097), "INVALID"), (dict(block_tables=None), "INVALID"), (dict(lse=4097), "INVALID"), (dict(Hq=0), "INVALID"),
                 (dict(Hq=5), "SHAPE"), (dict(Hq=2048), "SHAPE"), (dict(workspace=None), "WORKSPACE"), (dict(workspace=4096 + 16), "WORKSPACE"),
                 (dict(workspace_bytes=4096), "WORKSPACE"), (dict(q_stride=(ctypes.c_int64 * 2)(512, 4)), "INVALID")]


@pytest.mark.parametrize("change, why", BAD_ATTENTION)
def test_bad_attention_is_refused(sb, change, why):
    want = {"INVALID": sb.SOL_ERR_INVALID_ARG, "SHAPE": sb.SOL_ERR_UNSUPPORTED_SHAPE, "WORKSPACE": sb.SOL_ERR_WORKSPACE}[why]
    assert sb.lib().sol_attn_cache_attention(ctypes.byref(attention_args(sb, **change))) == want


def test_attention_of_nothing_is_fine(sb):
    assert sb.lib().sol_attn_cache_attention(None) == sb.SOL_ERR_INVALID_ARG
    assert sb.lib().sol_attn_cache_attention(ctypes.byref(attention_args(sb, tokens=0, q=None, out=None))) == sb.SOL_OK
    assert sb.lib().sol_attn_cache_attention(ctypes.byref(attention_args(sb, requests=0, cu_q=None))) == sb.SOL_OK
    assert sb.lib().sol_attn_cache_read_status(None, None) == sb.SOL_ERR_WORKSPACE


def norm_args(sb, **kw):
    three = ctypes.c_int64 * 3
    a = dict(q=4096, k=8192, q_out=4096, k_out=8192, q_stride=three(4096, 512, 128), k_stride=three(4096, 512, 128),
             q_out_stride=three(4096, 512, 128), k_out_stride=three(4096, 512, 128), cos=4096, sin=4096, batch=1, tokens=3, Hq=4, Hk=4, d=128,
             rot=64, table_rows=10, type=0, eps=1e-6)
    a.update(kw)
    return sb._NormArgs(**a)


BAD_NORM = [(dict(q=None), "INVALID"), (dict(k_out=None), "INVALID"), (dict(batch=-1), "INVALID"), (dict(Hq=0, Hk=0), "INVALID"),
            (dict(type=2), "INVALID"), (dict(eps=-1.0), "INVALID"), (dict(eps=float("nan")), "INVALID"), (dict(cos=None), "INVALID"),
            (dict(table_rows=0), "INVALID"), (dict(rot=-16), "INVALID"), (dict(rot=24), "SHAPE"), (dict(rot=144), "SHAPE"), (dict(d=96), "SHAPE"),
            (dict(Hk=1025), "SHAPE"), (dict(q=4104), "INVALID"), (dict(sin=4100), "INVALID"), (dict(positions=4098), "INVALID"),
            (dict(q_weight=4100), "INVALID"), (dict(batch=70000, tokens=70000), "SHAPE"),
            (dict(k_stride=(ctypes.c_int64 * 3)(0, 512, 100)), "INVALID")]


@pytest.mark.parametrize("change, why", BAD_NORM)
def test_bad_norms_are_refused(sb, change, why):
    want = sb.SOL_ERR_INVALID_ARG if why == "INVALID" else sb.SOL_ERR_UNSUPPORTED_SHAPE
    assert sb.lib().sol_attn_qk_norm_rope(ctypes.byref(norm_args(sb, **change))) == want
    assert sb.lib().sol_attn_qk_norm_rope(None) == sb.SOL_ERR_INVALID_ARG
    assert sb.lib().sol_attn_qk_norm_rope(ctypes.byref(norm_args(sb, tokens=0, q=None))) == sb.SOL_OK


def tables_args(sb, **kw):
    a = dict(old_lens=4096, new_lens=4096, free_pages=4096, free_count=4096, block_tables=4 * 4096, cu_q=5 * 4096, kv_lens=6 * 4096,
             slots=7 * 4096, positions=None, result=8192, table_stride=8, requests=2, max_blocks=8, max_tokens=9, free_capacity=3, page_size=16)
    a.update(kw)
    return sb._TablesArgs(**a)


BAD_TABLES = [(dict(requests=-1), "INVALID"), (dict(max_tokens=-1), "INVALID"), (dict(max_blocks=0), "INVALID"), (dict(free_capacity=-1), "INVALID"),
              (dict(cu_q=None), "INVALID"), (dict(result=None), "INVALID"), (dict(result=4096), "INVALID"), (dict(result=4092), "INVALID"),
              (dict(old_lens=None), "INVALID"), (dict(slots=None), "INVALID"), (dict(free_pages=None), "INVALID"), (dict(table_stride=7), "INVALID"),
              (dict(page_size=24), "SHAPE"), (dict(page_size=8), "SHAPE"), (dict(kv_lens=4097), "INVALID"), (dict(kv_lens=4096), "INVALID"),
              (dict(old_lens=8192), "INVALID"), (dict(slots=4096), "INVALID"), (dict(block_tables=4096), "INVALID")]


@pytest.mark.parametrize("change, why", BAD_TABLES)
def test_bad_tables_are_refused(sb, change, why):
    want = sb.SOL_ERR_INVALID_ARG if why == "INVALID" else sb.SOL_ERR_UNSUPPORTED_SHAPE
    assert sb.lib().sol_attn_block_tables(ctypes.byref(tables_args(sb, **change))) == want
    assert sb.lib().sol_attn_block_tables(None) == sb.SOL_ERR_INVALID_ARG


def test_packed_structures_match_the_header_s(sb):
    """The bytes that the binding packs are the C structures: sizes, and every field where it belongs."""
    for cls, pack in ((sb._Cache, sb._PACK_CACHE), (sb._TablesArgs, sb._PACK_TABLES), (sb._NormArgs, sb._PACK_NORM),
                      (sb._CacheArgs, sb._PACK_ATTENTION)):
        assert ctypes.sizeof(cls) == pack.size, cls

        def leaves(c):
            for name, t in c._fields_:
                if isinstance(t, type) and issubclass(t, ctypes.Structure):
                    yield from leaves(t)
                elif isinstance(t, type) and issubclass(t, ctypes.Array):
                    yield from ((t._type_, x) for x in range(t._length_))
                else:
                    yield t, 0

        def values(obj):
            for name, t in obj._fields_:
                v = getattr(obj, name)
                if isinstance(v, ctypes.Structure):
                    yield from values(v)
                elif isinstance(v, ctypes.Array):
                    yield from v
                else:
                    yield v

        n = len(list(leaves(cls)))
        obj = cls.from_buffer_copy(pack.pack(*range(1, n + 1)))
        assert list(values(obj)) == list(range(1, n + 1)), cls


def test_binding_refuses_what_the_kernels_could_not_know(sb):
    cache = sb.Cache(torch.zeros(10, dtype=torch.uint8), 4, 16, 2, 128)
    with pytest.raises(ValueError):
        cache.c(0)
    with pytest.raises(sb.SolAttnError):
        sb.Cache(torch.zeros(10, dtype=torch.uint8), 4, 24, 2, 128)
    with pytest.raises(ValueError):
        sb._flat(0, torch.int32, "x", torch.zeros(3, dtype=torch.int32), (3,))     # not on a GPU
    with pytest.raises(ValueError):
        sb._type(torch.float32)                                                 # not a 16-bit type
    with pytest.raises(ValueError):
        sb._heads(-1, "x", torch.zeros(3, 2, 64).half().transpose(1, 2), (3, 64, 2), torch.float16)
    assert sb._flat(0, torch.int32, "x", None, (3,)) == 0


@pytest.mark.parametrize("value, code", [(0.25, 0), (0.26, 1), (0.75, 2), (0.74, 1), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (5.1, 7)])
def test_reference_ties_go_to_even(value, code):
    x = torch.zeros(16, dtype=torch.float64)
    x[0], x[1] = 6.0, value
    codes, scale, _ = ref.held(x, 0)
    assert scale.item() == ref.E4M3.index(1.0) and codes[1].item() == code and codes[0].item() == 7


def test_reference_tables():
    table, cu, kv, slots, positions, result = ref.tables([0, 17, 5], [18, 1, 0], [7, 8, 9], 3, [[-1, -1], [4, 5], [6, -1]], 16, 100)
    assert table == [[9, 8], [4, 5], [6, -1]] and cu == [0, 18, 19, 19] and kv == [18, 18, 5]
    assert slots == [9 * 16 + i for i in range(16)] + [8 * 16, 8 * 16 + 1, 5 * 16 + 1]
    assert positions == list(range(18)) + [17] and result == [1, 0]


def test_work_shares_cover_everything():
    """The arithmetic by which the attention kernels deal out their steps and find who had the first piece of an item."""
    rng = random.Random(4)
    for _ in range(2000):
        work, grid = rng.randint(1, 10 ** rng.randint(1, 11)), rng.randint(1, 640)
        blocks = min(grid, work)
        each, extra = work // blocks, work % blocks
        begin = lambda c: c * each + min(c, extra)  # noqa: E731
        c = rng.randrange(blocks)
        lo, hi = begin(c), begin(c + 1)
        assert hi - lo in (each, each + 1) and hi > lo and begin(0) == 0 and begin(blocks) == work
        for w in {lo, hi - 1, rng.randrange(lo, hi)}:
            assert (w // (each + 1) if w < extra * (each + 1) else extra + (w - extra * (each + 1)) // each) == c
